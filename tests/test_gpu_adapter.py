"""ab_adapter_forward / ab_adapter_backward against the float64 checker: every type and route, maps of every kind, from one row on.

Tolerances, element by element.  With S the same sum over absolute values, K terms of fp32 lose at most K 2^-23 S (also where a sum is
cut off instead of rounded at every step); T and U are carried on with 16 bits at least (2^-16 of the second product's S); a result
held in bf16 is off by half a step of itself, 2^-8."""
import numpy as np
import pytest
import torch

from oracle import ab_oracle as orc
from paper_2405_01067_b200 import binding as ab

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def make_map(kind, N, L, rng):
    if kind == "none":
        return np.full(N, -1)
    if kind == "one":
        return np.full(N, L - 1)
    if kind == "single":
        return rng.integers(-1, L, N)
    if kind == "alternate":
        return np.arange(N) % (L + 1) - 1
    cuts = np.sort(rng.integers(0, N + 1, max(1, N // 40)))
    ids = rng.integers(-1, L, cuts.size + 1)
    runs = ids[np.searchsorted(cuts, np.arange(N), side="right")]
    if kind == "mixed":
        runs[: N // 3] = rng.integers(-1, L, N // 3)
    return runs


class Case:
    def __init__(self, N, m, n, r, L, kind, dtype, seed=0, scale=True):
        rng = np.random.default_rng([seed, N, m, n, r, L])
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, std=1.0):
            return (torch.randn(*shape, generator=g) * std).to(dtype)
        self.x, self.dY, self.W = normal(N, n), normal(N, m), normal(m, n, std=n ** -0.5)
        self.A, self.B = normal(L, m, r, std=r ** -0.5), normal(L, r, n, std=n ** -0.5)
        self.scale = torch.tensor(rng.uniform(0.5, 2.0, L), dtype=F32) if scale else None
        self.ids = make_map(kind, N, L, rng)
        self.map = torch.tensor(self.ids, dtype=torch.int32)
        self.dtype = dtype

    def cuda(self):
        return [None if t is None else t.cuda() for t in (self.x, self.dY, self.W, self.A, self.B, self.map, self.scale)]

    def host(self, absolute=False):
        f = np.abs if absolute else (lambda v: v)
        x, dY, W, A, B = (f(t.float().numpy().astype(np.float64)) for t in (self.x, self.dY, self.W, self.A, self.B))
        return x, dY, W, A, B, self.ids, None if self.scale is None else self.scale.numpy().astype(np.float64)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def close(got, want, bound, what):
    got = f64(got)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(np.max(np.abs(got - want) / np.maximum(bound, 1e-300))), np.argwhere(bad)[:4].tolist())


def check(c, want=("dX", "dA", "dB"), saved=True):
    x, dY, W, A, B, ids, s = c.host()
    ax, adY, aW, aA, aB, _, _ = c.host(True)
    N, n = x.shape
    m, r, L = W.shape[0], A.shape[2], A.shape[0]
    T_ref, y_ref = orc.adapter_forward(x, W, A, B, ids, s)
    T_abs, y_abs = orc.adapter_forward(ax, aW, aA, aB, ids, s)
    delta_abs = y_abs - ax @ aW.T
    half = 2.0 ** -8 if c.dtype == BF16 else 2.0 ** -24
    step = 2.0 ** -23
    dev = c.cuda()
    ws = ab.workspace(ab.ab_adapter_workspace_bytes(dev[0], dev[3], dev[4]), "cuda")
    ws.fill_(0x7f)                                            # whatever a workspace held before
    y, T = ab.ab_adapter_forward(dev[0], dev[2], dev[3], dev[4], dev[5], scale=dev[6], save_T=True, ws=ws)
    assert ab.workspace_status(ws) == ab.AB_OK
    close(T, T_ref, (n + 4) * step * T_abs, "T")
    y_bound = half * np.abs(y_ref) * (1 + 2 ** -7) + (n + r + 4) * step * y_abs + 2.0 ** -16 * delta_abs
    close(y, y_ref, y_bound, "y")
    y2, _ = ab.ab_adapter_forward(dev[0], dev[2], dev[3], dev[4], dev[5], scale=dev[6])
    close(y2, y_ref, y_bound, "y without T")
    ws.fill_(0x55)
    dX, dA, dB = ab.ab_adapter_backward(dev[0], dev[1], dev[2], dev[3], dev[4], dev[5], scale=dev[6], T_saved=T if saved else None, want=want,
                                        ws=ws)
    assert ab.workspace_status(ws) == ab.AB_OK
    dX_ref, dA_ref, dB_ref = orc.adapter_backward(x, dY, W, A, B, ids, s)
    dX_abs, dA_abs, dB_abs = orc.adapter_backward(ax, adY, aW, aA, aB, ids, s)
    if "dX" in want:
        close(dX, dX_ref, half * np.abs(dX_ref) * (1 + 2 ** -7) + (m + r + 4) * step * dX_abs + 2.0 ** -16 * (dX_abs - adY @ aW), "dX")
    if "dA" in want:
        close(dA, dA_ref, (N + n + 8) * step * dA_abs, "dA")
        assert orc.rel_frob(f64(dA), dA_ref) <= 1e-5
    if "dB" in want:
        close(dB, dB_ref, (N + m + 8) * step * dB_abs, "dB")
        assert orc.rel_frob(f64(dB), dB_ref) <= 1e-5


KINDS = ["none", "one", "single", "alternate", "runs", "mixed"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,m,n,r,L", [(1, 64, 64, 8, 1), (1, 200, 136, 16, 5), (15, 128, 72, 8, 3), (64, 256, 512, 32, 2), (130, 264, 200, 24, 7),
                                       (333, 504, 328, 40, 40), (700, 136, 264, 128, 3)])
def test_sizes_of_eight(N, m, n, r, L, dtype, kind):
    check(Case(N, m, n, r, L, kind, dtype))


@pytest.mark.parametrize("kind", ["single", "runs"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,m,n,r,L", [(1, 1, 1, 1, 1), (2, 3, 5, 2, 4), (77, 33, 65, 7, 3), (257, 101, 77, 12, 6), (129, 90, 131, 70, 2)])
def test_odd_sizes(N, m, n, r, L, dtype, kind):
    check(Case(N, m, n, r, L, kind, dtype))


@pytest.mark.parametrize("r", [8, 16, 24, 48, 56, 64, 72, 80, 88, 120, 128, 136, 192, 200, 248, 256])
def test_ranks(r):
    check(Case(300, 264, 328, r, 3, "mixed", BF16), saved=False)


@pytest.mark.parametrize("N", [2, 8, 16, 17, 31, 32, 33, 63, 65, 127, 128, 129, 191, 255, 256, 257, 513, 1025])
def test_row_counts(N):
    check(Case(N, 136, 200, 16, 4, "mixed", BF16))


@pytest.mark.parametrize("m,n", [(8, 8), (16, 520), (520, 16), (1000, 776), (776, 1000), (64, 2056), (2056, 64)])
def test_widths(m, n):
    check(Case(150, m, n, 8, 5, "runs", BF16))


@pytest.mark.parametrize("L", [1, 2, 31, 64, 200])
def test_many_adapters(L):
    check(Case(260, 72, 88, 16, L, "single", BF16))
    check(Case(260, 72, 88, 16, L, "runs", F32))


@pytest.mark.parametrize("want", [("dX",), ("dA",), ("dB",), ("dX", "dA"), ("dA", "dB"), ("dX", "dB")])
@pytest.mark.parametrize("saved", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_wanted_results(want, saved, dtype):
    check(Case(200, 136, 72, 16, 3, "mixed", dtype), want=want, saved=saved)


def test_without_scale():
    check(Case(90, 64, 128, 8, 3, "runs", BF16, scale=False))


@pytest.mark.parametrize("dtype,m,n,r", [(BF16, 136, 200, 16), (BF16, 133, 199, 15), (F32, 136, 200, 16)])
def test_stacks_with_gaps(dtype, m, n, r):
    """Adapters in slots of a pool that are larger than they are."""
    c = Case(150, m, n, r, 4, "mixed", dtype)
    x, dY, W, A, B, ids, s = c.cuda()
    poolA, poolB = (torch.full((4, k + 40), float("nan"), dtype=dtype, device="cuda") for k in (m * r, r * n))
    poolA[:, : m * r], poolB[:, : r * n] = A.reshape(4, -1), B.reshape(4, -1)
    vA, vB = poolA[:, : m * r].unflatten(1, (m, r)), poolB[:, : r * n].unflatten(1, (r, n))
    y, T = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, save_T=True)
    y2, T2 = ab.ab_adapter_forward(x, W, vA, vB, ids, scale=s, save_T=True)
    g = ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s)
    g2 = ab.ab_adapter_backward(x, dY, W, vA, vB, ids, scale=s)
    assert torch.equal(y, y2) and torch.equal(T, T2) and all(torch.equal(p, q) for p, q in zip(g, g2))


@pytest.mark.parametrize("dtype,m,n,r", [(BF16, 136, 200, 16), (BF16, 132, 200, 16), (F32, 136, 200, 16)])
@pytest.mark.parametrize("kind", ["mixed", "runs", "alternate"])
def test_nothing_leaks_between_rows_or_adapters(dtype, m, n, r, kind):
    """Rows of NaN and infinities, and an adapter of them: every other row and adapter has the bits that it has without them."""
    L = 4
    c = Case(300, m, n, r, L, kind, dtype)
    c.ids[c.ids == 2] = 1
    c.ids[40:45], c.ids[140:200] = 2, 2
    c.map = torch.tensor(c.ids, dtype=torch.int32)
    x, dY, W, A, B, ids, s = c.cuda()
    y, T = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, save_T=True)
    dX, dA, dB = ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s)
    bad = torch.tensor(c.ids == 2)
    x2, dY2, A2, B2 = (t.clone() for t in (x, dY, A, B))
    x2[bad.cuda()] = float("nan")
    dY2[bad.cuda()] = float("inf")
    A2[2], B2[2] = float("inf"), float("nan")
    y2, T2 = ab.ab_adapter_forward(x2, W, A2, B2, ids, scale=s, save_T=True)
    dX2, dA2, dB2 = ab.ab_adapter_backward(x2, dY2, W, A2, B2, ids, scale=s)
    ok, others = ~bad, [0, 1, 3]
    for got, ref in ((y2, y), (T2, T), (dX2, dX)):
        assert torch.equal(got.cpu()[ok], ref.cpu()[ok])
    for got, ref in ((dA2, dA), (dB2, dB)):
        assert torch.equal(got[others], ref[others]) and not torch.isfinite(got[2]).any()
    assert not torch.isfinite(y2.cpu()[bad]).any() and torch.isnan(T2.cpu()[bad]).all()


@pytest.mark.parametrize("dtype,m,n,r", [(BF16, 136, 200, 16), (BF16, 133, 200, 16), (F32, 136, 200, 16)])
def test_entries_that_are_no_adapter(dtype, m, n, r):
    c = Case(200, m, n, r, 3, "mixed", dtype)
    x, dY, W, A, B, ids, s = c.cuda()
    ws = ab.workspace(ab.ab_adapter_workspace_bytes(x, A, B), "cuda")
    for at, value in ((0, 3), (199, -2), (77, 2 ** 31 - 1), (130, -2 ** 31)):
        wrong, right = ids.clone(), ids.clone()
        wrong[at], right[at] = value, -1
        y, _ = ab.ab_adapter_forward(x, W, A, B, wrong, scale=s, ws=ws)
        assert ab.workspace_status(ws) == ab.AB_ERR_INVALID_ARG
        g = ab.ab_adapter_backward(x, dY, W, A, B, wrong, scale=s, ws=ws)
        assert ab.workspace_status(ws) == ab.AB_ERR_INVALID_ARG
        ab.ab_adapter_backward(x, dY, None, A, B, wrong, scale=s, ws=ws, want=("dA",))
        assert ab.workspace_status(ws) == ab.AB_ERR_INVALID_ARG
        y2, _ = ab.ab_adapter_forward(x, W, A, B, right, scale=s, ws=ws)
        assert ab.workspace_status(ws) == ab.AB_OK
        g2 = ab.ab_adapter_backward(x, dY, W, A, B, right, scale=s, ws=ws)
        assert ab.workspace_status(ws) == ab.AB_OK
        assert torch.equal(y, y2) and all(torch.equal(p, q) for p, q in zip(g, g2))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_outputs_are_written_whole_and_alone(dtype):
    """Every element of every output, also of adapters without rows; nothing beside them."""
    c = Case(150, 136, 200, 16, 5, "runs", dtype)
    c.ids[:] = np.where(c.ids == 3, -1, c.ids)
    c.map = torch.tensor(c.ids, dtype=torch.int32)
    x, dY, W, A, B, ids, s = c.cuda()

    def framed(shape, dt):
        k = int(np.prod(shape))
        buf = torch.full((k + 512,), 7.0, dtype=dt, device="cuda")
        return buf, buf[256: 256 + k].view(shape)
    frames = {k: framed(sh, dt) for k, (sh, dt) in {"y": ((150, 136), dtype), "T": ((150, 16), F32), "dX": ((150, 200), dtype),
                                                     "dA": ((5, 136, 16), F32), "dB": ((5, 16, 200), F32)}.items()}
    v = {k: f[1].fill_(float("nan")) for k, f in frames.items()}
    ab.ab_adapter_forward(x, W, A, B, ids, scale=s, y=v["y"], T_save=v["T"])
    ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s, T_saved=v["T"], dX=v["dX"], dA=v["dA"], dB=v["dB"])
    for k, (buf, view) in frames.items():
        assert torch.isfinite(view).all(), k
        assert (buf[:256] == 7).all() and (buf[-256:] == 7).all(), k
    assert (v["dA"][3] == 0).all() and (v["dB"][3] == 0).all()


@pytest.mark.parametrize("shift", [1, 2, 4])
def test_misaligned_pointers(shift):
    """Tensors that start at any element take the general kernels; T of one route serves the other's backward."""
    c = Case(100, 72, 136, 8, 3, "mixed", BF16)
    dev = c.cuda()

    def shifted(t):
        buf = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")
        buf[shift:] = t.reshape(-1)
        return buf[shift:].view(t.shape)
    x, dY, W, A, B, ids, s = dev
    y, T = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, save_T=True)
    y2, T2 = ab.ab_adapter_forward(shifted(x), shifted(W), shifted(A), shifted(B), ids, scale=s, save_T=True)
    g = ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s, T_saved=T2)
    g2 = ab.ab_adapter_backward(shifted(x), shifted(dY), W, A, shifted(B), ids, scale=s, T_saved=T)
    assert orc.rel_frob(f64(y2), f64(y)) <= 2.0 ** -8 and orc.rel_frob(f64(T2), f64(T)) <= 1e-6
    for p, q in zip(g, g2):
        assert orc.rel_frob(f64(q), f64(p)) <= (2.0 ** -8 if p.dtype == BF16 else 2e-5)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_rows(dtype):
    x, dY = torch.empty((0, 64), dtype=dtype, device="cuda"), torch.empty((0, 72), dtype=dtype, device="cuda")
    W, A, B = (torch.ones(s, dtype=dtype, device="cuda") for s in ((72, 64), (2, 72, 8), (2, 8, 64)))
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    y, T = ab.ab_adapter_forward(x, W, A, B, ids, save_T=True)
    dX, dA, dB = ab.ab_adapter_backward(x, dY, W, A, B, ids, T_saved=T, dA=torch.ones((2, 72, 8), device="cuda"))
    assert y.shape == (0, 72) and dX.shape == (0, 64) and (dA == 0).all() and (dB == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,m,n,r,L,kind", [(3, 256, 512, 16, 4, "single"), (600, 264, 200, 24, 5, "mixed")])
def test_two_runs_give_the_same_bits(dtype, N, m, n, r, L, kind):
    x, dY, W, A, B, ids, s = Case(N, m, n, r, L, kind, dtype).cuda()
    first = None
    for _ in range(5):
        y, T = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, save_T=True)
        out = (y, T) + ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s, T_saved=T)
        first = first or out
        assert all(torch.equal(p, q) for p, q in zip(out, first))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_captured_with_another_map(dtype):
    """A captured forward and backward, replayed on other rows and another map (a padded batch)."""
    c, d = Case(200, 136, 200, 16, 4, "runs", dtype), Case(200, 136, 200, 16, 4, "single", dtype, seed=9)
    x, dY, W, A, B, ids, s = c.cuda()
    ws = ab.workspace(ab.ab_adapter_workspace_bytes(x, A, B), "cuda")

    def call():
        y, T = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, save_T=True, ws=ws)
        return (y, T) + ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s, T_saved=T, ws=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    x.copy_(d.x), dY.copy_(d.dY), ids.copy_(d.map)
    ids[150:] = -1
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in out]
    assert all(torch.equal(p, q) for p, q in zip(got, call()))


def test_two_streams_at_once():
    cases = [Case(400, 264, 328, 16, 4, "mixed", BF16, seed=k) for k in range(2)]
    devs = [c.cuda() for c in cases]
    want = [ab.ab_adapter_forward(d[0], d[2], d[3], d[4], d[5], scale=d[6])[0] for d in devs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in devs]
    outs, wss = [], [ab.workspace(ab.ab_adapter_workspace_bytes(d[0], d[3], d[4]), "cuda") for d in devs]
    for _ in range(20):
        for d, st, ws in zip(devs, streams, wss):
            outs.append(ab.ab_adapter_forward(d[0], d[2], d[3], d[4], d[5], scale=d[6], ws=ws, stream=st)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i % 2]) for i, o in enumerate(outs))


def test_gradients_against_differences():
    """fp32 differences of the library's own forward along random directions: f(p + h) - f(p - h) over 2h of a bilinear map."""
    c = Case(60, 48, 40, 8, 3, "mixed", F32)
    x, dY, W, A, B, ids, s = c.cuda()
    dX, dA, dB = ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s)

    def loss(x_, A_, B_):
        return float((ab.ab_adapter_forward(x_, W, A_, B_, ids, scale=s)[0].double() * dY.double()).sum())
    g = torch.Generator(device="cuda").manual_seed(5)
    for which, grad in ((0, dX), (1, dA), (2, dB)):
        p = [x, A, B]
        v = torch.randn(p[which].shape, device="cuda", generator=g)
        hi, lo = list(p), list(p)
        hi[which], lo[which] = p[which] + v / 4, p[which] - v / 4
        diff = 2 * (loss(*hi) - loss(*lo))
        want = float((grad.double() * v.double()).sum())
        # 2880 outputs of magnitude about 3, each off by at most 2^-23 (n + r + 4) S with S about 20: their sum with dY is off by
        # less than sqrt(2880) 20 52 2^-23 = 7e-3 (independent errors), times the 2 above
        assert abs(diff - want) <= 2e-2, (which, diff, want)


def test_refusals():
    c = Case(10, 16, 24, 8, 2, "runs", BF16)
    x, dY, W, A, B, ids, s = c.cuda()
    for bad in (dict(W=W[:, :16].contiguous()), dict(A=A.float()), dict(B=B[:1]), dict(row_adapter=ids.long()), dict(row_adapter=ids[:5]),
                dict(scale=s[:1].contiguous()), dict(scale=s.double()), dict(x=x.cpu()), dict(y=torch.empty((10, 17), dtype=BF16, device="cuda")),
                dict(T_save=torch.empty((10, 8), dtype=BF16, device="cuda")), dict(x=x.t()), dict(A=A.transpose(1, 2))):
        args = dict(x=x, W=W, A=A, B=B, row_adapter=ids, scale=s) | bad
        with pytest.raises((ValueError, TypeError)):
            ab.ab_adapter_forward(**args)
    with pytest.raises(ValueError):
        ab.ab_adapter_backward(x, dY[:, :8].contiguous(), W, A, B, ids)
    with pytest.raises(ab.AbError):
        ab.ab_adapter_forward(x, W, A, B, ids, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))


# Rows beyond the kernel for few: 32 to 256 rows a tile, CTAs by themselves and in pairs, one tile a CTA and several
WIDE = [(1025, 136, 200, 16, 3), (1300, 264, 328, 64, 5), (3000, 1000, 200, 24, 9), (1100, 2000, 136, 72, 4), (2500, 136, 72, 8, 2),
        (9000, 520, 392, 40, 6), (20000, 264, 328, 136, 3)]


@pytest.mark.parametrize("kind", ["one", "runs", "mixed", "alternate"])
@pytest.mark.parametrize("N,m,n,r,L", WIDE)
def test_many_rows(N, m, n, r, L, kind):
    check(Case(N, m, n, r, L, kind, BF16))


@pytest.mark.parametrize("kind", ["runs", "mixed"])
@pytest.mark.parametrize("N,m,n,r,L", [(1300, 264, 328, 64, 4), (9000, 520, 392, 40, 4)])
def test_nothing_leaks_between_many_rows(N, m, n, r, L, kind):
    c = Case(N, m, n, r, L, kind, BF16)
    c.ids[c.ids == 2] = 1
    c.ids[400:405], c.ids[700:901] = 2, 2
    c.map = torch.tensor(c.ids, dtype=torch.int32)
    x, dY, W, A, B, ids, s = c.cuda()
    y, T = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, save_T=True)
    dX, dA, dB = ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s)
    bad = torch.tensor(c.ids == 2)
    x2, dY2, A2, B2 = (t.clone() for t in (x, dY, A, B))
    x2[bad.cuda()], dY2[bad.cuda()] = float("nan"), float("inf")
    A2[2], B2[2] = float("inf"), float("nan")
    y2, T2 = ab.ab_adapter_forward(x2, W, A2, B2, ids, scale=s, save_T=True)
    dX2, dA2, dB2 = ab.ab_adapter_backward(x2, dY2, W, A2, B2, ids, scale=s)
    ok, others = ~bad, [0, 1, 3]
    for got, ref in ((y2, y), (T2, T), (dX2, dX)):
        assert torch.equal(got.cpu()[ok], ref.cpu()[ok])
    for got, ref in ((dA2, dA), (dB2, dB)):
        assert torch.equal(got[others], ref[others]) and not torch.isfinite(got[2]).any()


def test_bad_entries_among_many_rows():
    c = Case(3000, 1000, 200, 24, 3, "mixed", BF16)
    x, dY, W, A, B, ids, s = c.cuda()
    ws = ab.workspace(ab.ab_adapter_workspace_bytes(x, A, B), "cuda")
    for at, value in ((0, 3), (2999, -2), (1777, 2 ** 31 - 1)):
        wrong, right = ids.clone(), ids.clone()
        wrong[at], right[at] = value, -1
        y, _ = ab.ab_adapter_forward(x, W, A, B, wrong, scale=s, ws=ws)
        assert ab.workspace_status(ws) == ab.AB_ERR_INVALID_ARG
        y2, _ = ab.ab_adapter_forward(x, W, A, B, right, scale=s, ws=ws)
        assert ab.workspace_status(ws) == ab.AB_OK and torch.equal(y, y2)


@pytest.mark.parametrize("dtype,N,m,n,r,L,kind", [(BF16, 1500, 72, 100, 4, 1, "one"), (F32, 700, 65, 130, 5, 2, "mixed"), (BF16, 2000, 40, 33, 12, 3, "runs"),
                                                  (F32, 3000, 100, 60, 3, 1, "single"), (BF16, 127, 232, 160, 128, 25, "runs"),
                                                  (BF16, 120, 216, 264, 200, 30, "single"), (F32, 300, 40, 1600, 8, 4, "mixed")])
def test_few_tiles_many_rows(dtype, N, m, n, r, L, kind):
    """Gradients whose rows are cut into slices, shared products whose reduction is, many adapters of high rank among few rows."""
    check(Case(N, m, n, r, L, kind, dtype))


def test_rank_above_a_size_is_refused_on_the_device():
    """A rank above one of the sizes (200 of a 136 x 264 projection) is no rank that the projection can have."""
    c = Case(120, 136, 264, 200, 30, "single", BF16)
    with pytest.raises(ab.AbError):
        check(c)


def test_more_adapters_than_lists_hold():
    """Beyond 2^24 entries of the slab lists the gradients go by the general kernels, whose results are the same sums."""
    N, L, m, n, r = 64 * 900 - 5, 20000, 16, 24, 8
    g = torch.Generator(device="cuda").manual_seed(5)
    x, dY = (torch.randn(N, k, device="cuda", generator=g).bfloat16() for k in (n, m))
    W = (torch.randn(m, n, device="cuda", generator=g) / n ** 0.5).bfloat16()
    A = torch.randn(L, m, r, device="cuda", generator=g).bfloat16()
    B = torch.randn(L, r, n, device="cuda", generator=g).bfloat16()
    ids = torch.randint(-1, L, (N,), device="cuda", generator=g, dtype=torch.int32)
    y, T = ab.ab_adapter_forward(x, W, A, B, ids, save_T=True)
    dX, dA, dB = ab.ab_adapter_backward(x, dY, W, A, B, ids, T_saved=T)
    has, a = (ids >= 0).double()[:, None], ids.clamp(min=0).long()
    xd, yd, Ad, Bd = x.double(), dY.double(), A.double()[a], B.double()[a]
    t = has * torch.einsum("irn,in->ir", Bd, xd)
    u = has * torch.einsum("imr,im->ir", Ad, yd)
    want_y = xd @ W.double().T + torch.einsum("imr,ir->im", Ad, t)
    want_dX = yd @ W.double() + torch.einsum("irn,ir->in", Bd, u)
    want_dA = torch.zeros(L, m, r, device="cuda", dtype=torch.float64).index_add_(0, a, yd[:, :, None] * t[:, None, :])
    want_dB = torch.zeros(L, r, n, device="cuda", dtype=torch.float64).index_add_(0, a, u[:, :, None] * xd[:, None, :])
    # y, dX: half a step of bf16; dA, dB: sums of up to 24 products of 8 to 24 terms in fp32 (24 + 24 roundings of 2^-24)
    for got, want, tol in ((y, want_y, 2.0 ** -8), (dX, want_dX, 2.0 ** -8), (dA, want_dA, 48 * 2.0 ** -24), (dB, want_dB, 48 * 2.0 ** -24)):
        assert float((got.double() - want).norm() / want.norm()) < tol


def test_a_stream_of_the_caller_keeps_its_workspace():
    """A workspace that the call allocates is not handed out again while a side stream still uses it."""
    c = Case(700, 264, 512, 24, 5, "mixed", BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    x, _, W, A, B, ids, scale = c.cuda()
    want, _ = ab.ab_adapter_forward(x, W, A, B, ids, scale)
    torch.cuda.synchronize()
    y = torch.empty_like(want)
    for _ in range(20):
        ab.ab_adapter_forward(x, W, A, B, ids, scale, y=y, stream=side)
        junk = [torch.full((1 << 16,), 255, dtype=torch.uint8, device="cuda") for _ in range(40)]
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        del junk
