"""The general path of the adapters with a workspace that holds the shared product's slices of some rows alone: several bands of rows, the last
one shorter, with the bits of one band, whose results test_gpu_adapter.check holds against the oracle."""
import pytest
import torch

from paper_2405_01067_b200 import binding as ab
from test_gpu_adapter import BF16, F32, Case, check

pytestmark = pytest.mark.gpu

# rows' slices take 80 to 260 MB here where all of them are there at a time
CASES = [(F32, 1500, 8200, 1600, 12, "mixed"), (BF16, 1500, 8201, 1601, 7, "mixed"), (F32, 1411, 1600, 8200, 9, "runs"), (BF16, 4100, 8203, 333, 5, "single")]


@pytest.mark.parametrize("dtype,N,m,n,r,kind", CASES)
def test_bands_have_the_bits_of_one(dtype, N, m, n, r, kind):
    c = Case(N, m, n, r, 3, kind, dtype)
    check(c)
    x, dY, W, A, B, ids, s = c.cuda()
    need = ab.ab_adapter_workspace_bytes(x, A, B)
    want = None
    for nbytes in (need, 64 << 20, 48 << 20):
        assert nbytes <= need
        ws = ab.workspace(nbytes, "cuda").fill_(0x7f)
        y, T = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, save_T=True, ws=ws)
        out = (y, T) + ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s, T_saved=T, ws=ws)
        assert ab.workspace_status(ws) == ab.AB_OK
        want = want or out
        assert all(torch.equal(p, q) for p, q in zip(out, want))
    with pytest.raises(ab.AbError):
        ab.ab_adapter_forward(x, W, A, B, ids, scale=s, ws=ab.workspace(1 << 20, "cuda"))


def test_nothing_is_written_behind_a_small_workspace():
    c = Case(1500, 8201, 1601, 7, 3, "mixed", BF16)
    x, dY, W, A, B, ids, s = c.cuda()
    for nbytes in (48 << 20, (48 << 20) + 256 * 7):
        ws = torch.full((nbytes + (1 << 20),), 7, dtype=torch.uint8, device="cuda")
        y, T = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, save_T=True, ws=ws[:nbytes])
        ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s, T_saved=T, ws=ws[:nbytes])
        assert (ws[nbytes:] == 7).all()


def test_sizes_of_the_tensor_cores_at_odd_addresses():
    """Sizes of the tensor-core path ask for 64 MB of slices at most: at addresses that it does not take they go in bands."""
    c = Case(1500, 8208, 1600, 8, 3, "mixed", BF16)
    x, dY, W, A, B, ids, s = c.cuda()
    buf = torch.empty(x.numel() + 1, dtype=BF16, device="cuda")
    x1 = buf[1:].view(x.shape).copy_(x)
    need = ab.ab_adapter_workspace_bytes(x1, A, B)
    assert need < 80 << 20
    small, large = ab.workspace(need, "cuda"), ab.workspace(512 << 20, "cuda")
    outs = []
    for ws in (small, large):
        y, T = ab.ab_adapter_forward(x1, W, A, B, ids, scale=s, save_T=True, ws=ws)
        outs.append((y, T) + ab.ab_adapter_backward(x1, dY, W, A, B, ids, scale=s, T_saved=T, ws=ws))
    assert all(torch.equal(p, q) for p, q in zip(*outs))
    y, T = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, save_T=True)
    # each is within half a step of bf16 (2^-8 of an element) of the same value
    assert ((outs[0][0].double() - y.double()).norm() <= 2 * 2.0 ** -8 * y.double().norm()).item()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_bad_entries_in_any_band(dtype):
    c = Case(1500, 8201, 1601, 7, 3, "mixed", dtype)
    x, _, W, A, B, ids, s = c.cuda()
    ws = ab.workspace(48 << 20, "cuda")
    want, _ = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, ws=ws)
    for at in (0, 700, 1499):
        wrong = ids.clone()
        wrong[at] = 3
        y, _ = ab.ab_adapter_forward(x, W, A, B, wrong, scale=s, ws=ws)
        assert ab.workspace_status(ws) == ab.AB_ERR_INVALID_ARG
        others = torch.arange(1500, device="cuda") != at
        assert torch.equal(y[others], want[others])
