"""Host-side refusals of the adapter calls: bad arguments are answered before anything is launched.  No GPU needed."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2405_01067_b200 import build
    build.build()
    from paper_2405_01067_b200 import binding
    binding.lib()
    return binding


P = ctypes.c_void_p(4096)          # never dereferenced: every call below fails its checks first


def forward(b, **kw):
    a = dict(x=P, W=P, A=P, B=P, scale=None, ids=P, y=P, T=None, N=4, m=16, n=24, r=8, L=2, sA=128, sB=192, dt=b.AB_BF16, ws=P,
             ws_bytes=1 << 30) | kw
    return b.lib().ab_adapter_forward(*a.values(), None)


def backward(b, **kw):
    a = dict(x=P, dY=P, W=P, A=P, B=P, scale=None, ids=P, T=None, dX=P, dA=P, dB=P, N=4, m=16, n=24, r=8, L=2, sA=128, sB=192,
             dt=b.AB_BF16, ws=P, ws_bytes=1 << 30) | kw
    return b.lib().ab_adapter_backward(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(x=None), dict(A=None), dict(B=None), dict(ids=None), dict(N=-1), dict(m=0), dict(n=0), dict(r=0), dict(r=17),
                                dict(L=0), dict(L=-3), dict(sA=127), dict(sB=191), dict(dt=2), dict(x=ctypes.c_void_p(4097)),
                                dict(A=ctypes.c_void_p(4097)), dict(ids=ctypes.c_void_p(4098))])
def test_bad_arguments_of_both(b, kw):
    assert forward(b, **kw) == b.AB_ERR_INVALID_ARG
    assert backward(b, **kw) == b.AB_ERR_INVALID_ARG


def test_bad_arguments_of_one(b):
    assert forward(b, W=None) == b.AB_ERR_INVALID_ARG
    assert forward(b, y=None) == b.AB_ERR_INVALID_ARG
    assert forward(b, T=ctypes.c_void_p(4098)) == b.AB_ERR_INVALID_ARG
    assert backward(b, dY=None) == b.AB_ERR_INVALID_ARG
    assert backward(b, W=None) == b.AB_ERR_INVALID_ARG
    assert backward(b, dA=ctypes.c_void_p(4098)) == b.AB_ERR_INVALID_ARG
    assert forward(b, N=1 << 31) == b.AB_ERR_UNSUPPORTED
    assert backward(b, N=1 << 31) == b.AB_ERR_UNSUPPORTED


def test_workspace_query(b):
    q = b.lib().ab_adapter_workspace_bytes
    assert q(64, 256, 512, 32, 2, b.AB_F32) >= 256
    assert q(0, 256, 512, 32, 2, b.AB_BF16) >= 256
    for bad in ((-1, 256, 512, 32, 2, 0), (64, 0, 512, 32, 2, 0), (64, 256, 512, 0, 2, 0), (64, 256, 512, 32, 0, 0), (64, 256, 512, 32, 2, 7),
                (1 << 31, 256, 512, 32, 2, 0)):
        assert q(*bad) == 0


def test_no_device_means_an_error(b):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    assert forward(b) == b.AB_ERR_CUDA and backward(b) == b.AB_ERR_CUDA


def clip(b, tensors, **kw):
    arr = (b.ab_clip_desc * max(1, len(tensors)))(*tensors)
    a = dict(descs=arr, L=len(tensors), max_norm=1.0, norm=P, dt=b.AB_F32, ws=P, ws_bytes=1 << 20) | kw
    return b.lib().ab_grad_clip(*a.values(), None)


def test_clip_refusals(b):
    good = [(4096, 8192, 10), (4100, 8196, 0)]
    bad = b.AB_ERR_INVALID_ARG
    assert clip(b, []) == bad and clip(b, good, descs=None) == bad and clip(b, good, norm=None) == bad and clip(b, good, dt=3) == bad
    assert clip(b, good, max_norm=-1.0) == bad and clip(b, good, max_norm=float("nan")) == bad
    assert clip(b, [(None, 4096, 3)]) == bad and clip(b, [(4096, 4096, -1)]) == bad and clip(b, [(4097, 8192, 3)]) == bad
    assert clip(b, [(4096, 8194, 3)]) == bad
    assert clip(b, [(4096, 4096, 3), (8192, None, 3)]) == bad          # all are scaled or none is
    assert clip(b, [(4096, 4096, (1 << 40) + 1)]) == b.AB_ERR_UNSUPPORTED
    assert b.lib().ab_grad_clip_workspace_bytes(0) == 0 and b.lib().ab_grad_clip_workspace_bytes(5) >= 256


def test_workspace_of_many_adapters_stays_small(b):
    """The lists behind the gradients are bounded whatever the number of adapters: 2^20 adapters beside 2^20 rows."""
    assert 0 < b.lib().ab_adapter_workspace_bytes(1 << 20, 64, 64, 8, 1 << 20, b.AB_BF16) < 1 << 31


@pytest.mark.parametrize("N,m,n", [(8191, 4096, 4096), (65536, 4096, 4096), (262144, 4096, 4096), (32768, 8192, 28672), (1 << 20, 4096, 4096)])
@pytest.mark.parametrize("bf16", [True, False])
def test_workspace_of_many_rows_stays_small(b, N, m, n, bf16):
    """Beside T, U, their pieces and what the rows' lists take (under 2 KB a row here) there is a bounded part: 64 MB for sizes of the
    tensor-core path, 1 GB for the others.  The results' fp32 slices are not all there at a time."""
    need = b.lib().ab_adapter_workspace_bytes(N, m, n, 16, 8, b.AB_BF16 if bf16 else b.AB_F32)
    assert 0 < need <= 2048 * N + ((64 << 20) if bf16 else (1 << 30)) + 1024
    assert b.lib().ab_adapter_workspace_bytes(N, m + 1, n, 15, 8, b.AB_BF16) <= 2048 * N + (1 << 30) + 1024


def test_workspace_of_sizes_whose_slices_pass_64_bits(b):
    """2^31 - 1 rows of 2^31 - 1 values in eight slices are more than 2^63 bytes: the bounded part stays what it is."""
    most = (1 << 31) - 1
    rows = b.lib().ab_adapter_workspace_bytes(most, 64, 64, 1, 1, b.AB_F32)
    assert rows >= 12 * most
    for dt in (b.AB_F32, b.AB_BF16):
        assert rows <= b.lib().ab_adapter_workspace_bytes(most, most, 10_000, 1, 1, dt) <= rows + 128 * 8 * 4 * most + (2 << 30)
