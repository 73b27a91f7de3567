"""How many bits the adapters' products are formed with.  The bounds of test_gpu_adapter.py grow with the lengths of the sums, so that they
hold with fewer bits too; here every row has one value (adapter_pieces.py), or a long sum has one large term."""
import pytest
import torch

from adapter_pieces import GATE, lone_rows
from paper_2405_01067_b200 import binding as ab

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def a_map(kind, N, L):
    i = torch.arange(N)
    return {"one": i * 0 + L - 1, "runs": i * L // N, "alternate": i % L, "none": i * 0 - 1}[kind]


def case(N, m, n, r, L, kind, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)

    def values(*shape):
        return ((1 + torch.rand(*shape, generator=g)) * torch.randn(*shape, generator=g).sign()).to(dtype)
    x, k, xv = lone_rows(N, n, seed + 1, dtype)
    dY, f, dv = lone_rows(N, m, seed + 2, dtype)
    return x, k, xv, dY, f, dv, values(m, n), values(L, m, r), values(L, r, n), 0.5 + torch.rand(L, generator=g), a_map(kind, N, L).int()


ROUTES = [(100, 136, 200, 16, 3), (260, 264, 328, 24, 5), (264, 264, 328, 136, 2), (1200, 1208, 1304, 40, 12), (1200, 1304, 1208, 72, 3)]


@pytest.mark.parametrize("kind", ["one", "runs", "alternate"])
@pytest.mark.parametrize("dtype,shift", [(BF16, 0), (BF16, 1), (F32, 0)])
@pytest.mark.parametrize("N,m,n,r,L", ROUTES)
def test_gradients_have_the_bits_of_t(N, m, n, r, L, dtype, shift, kind):
    """dA of a feature is one row's dY times its T, dB of a feature one row's U times its x.  shift: widths that the tensor-core path does not take."""
    m, n = m + shift, n + shift
    x, k, xv, dY, f, dv, W, A, B, s, ids = case(N, m, n, r, L, kind, dtype)
    dev = [t.cuda() for t in (x, dY, W, A, B, ids, s)]
    _, T = ab.ab_adapter_forward(dev[0], dev[2], dev[3], dev[4], dev[5], scale=dev[6], save_T=True)
    a, i = ids.long(), torch.arange(N)
    want_T = (s.double()[a] * xv)[:, None] * B.double()[a, :, k]
    want_U = (s.double()[a] * dv)[:, None] * A.double()[a, f, :]
    # fp32: the product is rounded (2^-24) before it is scaled (2^-24)
    assert ((T.cpu().double() - want_T).abs() <= 2.0 ** -23 * (1 + 2.0 ** -20) * want_T.abs()).all()
    want_A, want_B = torch.zeros(L, m, r, dtype=torch.float64), torch.zeros(L, r, n, dtype=torch.float64)
    want_A[a, f] = dv[:, None] * want_T
    want_B[a, :, k] = xv[:, None] * want_U
    for saved in (T, None):
        _, dA, dB = ab.ab_adapter_backward(dev[0], dev[1], dev[2], dev[3], dev[4], dev[5], scale=dev[6], T_saved=saved)
        for got, want in ((dA, want_A), (dB, want_B)):
            assert ((got.cpu().double() - want).abs() <= GATE * want.abs()).all()


@pytest.mark.parametrize("N,m,n", [(100, 136, 200), (333, 504, 1000), (1000, 1001, 1003), (128, 256, 512)])
def test_the_shared_product_of_fp32_has_fp32s_bits(N, m, n):
    x, k, xv, dY, f, dv, W, A, B, _, ids = case(N, m, n, 8, 2, "none", F32)
    dev = [t.cuda() for t in (x, dY, W, A, B, ids)]
    y, _ = ab.ab_adapter_forward(dev[0], dev[2], dev[3], dev[4], dev[5])
    dX, _, _ = ab.ab_adapter_backward(dev[0], dev[1], dev[2], dev[3], dev[4], dev[5], want=("dX",))
    for got, want in ((y, xv[:, None] * W.double()[:, k].T), (dX, dv[:, None] * W.double()[f])):
        assert ((got.cpu().double() - want).abs() <= GATE * want.abs()).all()


@pytest.mark.parametrize("kind", ["one", "runs", "alternate"])
@pytest.mark.parametrize("N,m,n,r,L", [(100, 136, 200, 16, 3), (260, 264, 328, 24, 5), (1200, 1208, 1304, 72, 12)])
def test_results_are_rounded_once(N, m, n, r, L, kind):
    """bf16, a shared weight of zeros and one value of r: y is A's value times T, right to half a step and 2^-16 for T."""
    x, k, xv, dY, f, dv, W, A, B, s, ids = case(N, m, n, r, L, kind, BF16)
    W.zero_()
    at = r // 2 + 1
    A[:, :, :at], A[:, :, at + 1:], B[:, :at], B[:, at + 1:] = 0, 0, 0, 0
    dev = [t.cuda() for t in (x, dY, W, A, B, ids, s)]
    y, T = ab.ab_adapter_forward(dev[0], dev[2], dev[3], dev[4], dev[5], scale=dev[6], save_T=True)
    dX, _, _ = ab.ab_adapter_backward(dev[0], dev[1], dev[2], dev[3], dev[4], dev[5], scale=dev[6], T_saved=T, want=("dX",))
    a = ids.long()
    t, u = s.double()[a] * xv * B.double()[a, at, k], s.double()[a] * dv * A.double()[a, f, at]
    for got, want in ((y, t[:, None] * A.double()[a, :, at]), (dX, u[:, None] * B.double()[a, at, :])):
        step = torch.exp2(torch.floor(torch.log2(want.abs())) - 7)
        assert ((got.cpu().double() - want).abs() <= step / 2 + 2.0 ** -16 * want.abs()).all()


# One term of 1 and the rest 2^-29: of a sum that is cut off at 24 bits at every step those beside the 1 are lost (a step adds 2^-25 at most, half
# of what 1 can hold), of one in parts only those of the part with the 1.  All parts here are multiples of 64 2^-29 = 2^-23: adding them
# to the 1 is exact.  What may be lost is what the part has, and a rounding.
SMALL = 2.0 ** -29


@pytest.mark.parametrize("first", [0, 1999, 4095])
@pytest.mark.parametrize("N,kind", [(40, "one"), (300, "runs"), (1300, "runs"), (1300, "alternate")])
def test_long_sums_of_t(N, kind, first):
    """Four slabs of 64 at a time are summed on the tensor cores; a lane's share of a row on the fp32 pipes is smaller."""
    n, L = 4096, 12
    x = torch.ones(N, n, dtype=BF16, device="cuda")
    B = torch.full((L, 8, n), SMALL, dtype=BF16, device="cuda")
    B[:, :, first] = 1
    A, W = torch.zeros(L, 72, 8, dtype=BF16, device="cuda"), torch.zeros(72, n, dtype=BF16, device="cuda")
    _, T = ab.ab_adapter_forward(x, W, A, B, a_map(kind, N, L).int().cuda(), save_T=True)
    assert ((T.double() - (1 + (n - 1) * SMALL)).abs() <= 256 * SMALL + 2.0 ** -23).all()


@pytest.mark.parametrize("first", [0, 2000, 4095])
@pytest.mark.parametrize("r", [16, 136])
@pytest.mark.parametrize("dtype,width", [(BF16, 136), (BF16, 137), (F32, 137)])
def test_long_sums_of_gradients(dtype, width, r, first):
    """Rows in fours of 64 as above; T and U are 1 in every row."""
    N = 4096
    x = torch.zeros(N, width, dtype=dtype, device="cuda")
    dY = torch.zeros(N, width, dtype=dtype, device="cuda")
    A, B = torch.zeros(1, width, r, dtype=dtype, device="cuda"), torch.zeros(1, r, width, dtype=dtype, device="cuda")
    W, ids = torch.zeros(width, width, dtype=dtype, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")
    # dA: x has 1 in its first place, and B there: T = 1
    x[:, 0], B[0, :, 0] = 1, 1
    dY[:], dY[first] = SMALL, 1
    _, dA, _ = ab.ab_adapter_backward(x, dY, W, A, B, ids, want=("dA",))
    want = 1 + (N - 1) * SMALL
    assert ((dA.double() - want).abs() <= 256 * SMALL + 2.0 ** -23).all()
    # dB: dY has 1 in its first place, and A there: U = 1
    x[:], x[first], dY[:] = SMALL, 1, 0
    dY[:, 0], A[0, 0] = 1, 1
    _, _, dB = ab.ab_adapter_backward(x, dY, W, A, B, ids, want=("dB",))
    assert ((dB.double() - want).abs() <= 256 * SMALL + 2.0 ** -23).all()


@pytest.mark.parametrize("first", [0, 2000, 3899])
@pytest.mark.parametrize("N,P", [(300, 264), (1000, 1001)])
def test_long_shared_sums_of_fp32(N, P, first):
    """The reduction of the shared product in slices of at most 768."""
    K = 3900
    W = torch.full((P, K), SMALL, device="cuda")
    W[:, first] = 1
    A, B = torch.zeros(1, P, 8, device="cuda"), torch.zeros(1, 8, K, device="cuda")
    ids = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    want = 1 + (K - 1) * SMALL
    y, _ = ab.ab_adapter_forward(torch.ones(N, K, device="cuda"), W, A, B, ids)
    assert ((y.double() - want).abs() <= 768 * SMALL + 8 * 2.0 ** -24).all()
    At, Bt = torch.zeros(1, K, 8, device="cuda"), torch.zeros(1, 8, P, device="cuda")
    dX, _, _ = ab.ab_adapter_backward(torch.zeros(N, P, device="cuda"), torch.ones(N, K, device="cuda"), W.T.contiguous(), At, Bt, ids, want=("dX",))
    assert ((dX.double() - want).abs() <= 768 * SMALL + 8 * 2.0 ** -24).all()
