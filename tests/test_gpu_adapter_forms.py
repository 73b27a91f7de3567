"""Every form in which the tensor-core path of the adapters makes its results (few rows; 32 to 256 rows a tile, CTAs by themselves and in
pairs), in both directions, with ranks of one slab and of several, and what else was only looked at with few rows: the same bits in every
run, captured calls, two streams at once, results by themselves.  Tolerances as in test_gpu_adapter.py."""
import pytest
import torch

from paper_2405_01067_b200 import binding as ab
from test_gpu_adapter import BF16, F32, Case, check

pytestmark = pytest.mark.gpu

# (rows, m, n): the form of y, the form of dX on 148 SMs
FORMS = {(100, 200, 136): (0, 0), (1030, 136, 200): (32, 32), (2500, 136, 2000): (65, 257), (2500, 2000, 136): (257, 65), (1500, 1000, 1000): (129, 129),
         (6000, 776, 200): (257, 129), (6000, 200, 776): (129, 257), (2500, 136, 72): (64, 32), (5000, 392, 136): (256, 128)}


def form(N, P, K):
    return ab.lib().ab_selftest_adapter_form(N, P, K)


def test_the_sizes_have_the_forms_that_they_stand_for():
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the rule depends on the count of SMs")
    assert {k: (form(k[0], k[1], k[2]), form(k[0], k[2], k[1])) for k in FORMS} == FORMS
    assert {f for v in FORMS.values() for f in v} == {0, 32, 64, 65, 128, 129, 256, 257}


@pytest.mark.parametrize("kind", ["one", "runs", "mixed", "alternate"])
@pytest.mark.parametrize("r", [16, 72, 136])
@pytest.mark.parametrize("N,m,n", FORMS)
def test_forms(N, m, n, r, kind):
    check(Case(N, m, n, min(r, m, n), 5, kind, BF16))


LARGE = [(1500, 1000, 1000, 24, 5, "mixed"), (2500, 136, 2000, 72, 3, "runs"), (6000, 776, 200, 16, 9, "alternate"), (2100, 200, 136, 136, 4, "single")]


def both(dev, ws=None, stream=None, T=None):
    x, dY, W, A, B, ids, s = dev
    y, T = ab.ab_adapter_forward(x, W, A, B, ids, scale=s, save_T=True, ws=ws, stream=stream)
    return (y, T) + ab.ab_adapter_backward(x, dY, W, A, B, ids, scale=s, T_saved=T, ws=ws, stream=stream)


@pytest.mark.parametrize("N,m,n,r,L,kind", LARGE)
def test_many_rows_have_the_same_bits_in_every_run(N, m, n, r, L, kind):
    dev = Case(N, m, n, r, L, kind, BF16).cuda()
    first = both(dev)
    for _ in range(4):
        assert all(torch.equal(p, q) for p, q in zip(both(dev), first))


@pytest.mark.parametrize("N,m,n,r,L,kind", LARGE)
def test_many_rows_captured_with_another_map(N, m, n, r, L, kind):
    c, d = Case(N, m, n, r, L, kind, BF16), Case(N, m, n, r, L, "runs" if kind != "runs" else "single", BF16, seed=9)
    dev = c.cuda()
    ws = ab.workspace(ab.ab_adapter_workspace_bytes(dev[0], dev[3], dev[4]), "cuda")
    both(dev, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(dev, ws)
    dev[0].copy_(d.x), dev[1].copy_(d.dY), dev[5].copy_(d.map)
    dev[5][N - N // 4:] = -1
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in out]
    assert all(torch.equal(p, q) for p, q in zip(got, both(dev, ws)))


@pytest.mark.parametrize("sizes", [(LARGE[0], LARGE[1]), (LARGE[2], LARGE[3])])
def test_many_rows_on_two_streams_at_once(sizes):
    devs = [Case(*s, BF16, seed=k).cuda() for k, s in enumerate(sizes)]
    want = [both(d) for d in devs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in devs]
    wss = [ab.workspace(ab.ab_adapter_workspace_bytes(d[0], d[3], d[4]), "cuda") for d in devs]
    outs = []
    for _ in range(10):
        for d, st, ws in zip(devs, streams, wss):
            outs.append(both(d, ws, st))
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for i, o in enumerate(outs) for p, q in zip(o, want[i % 2]))


@pytest.mark.parametrize("want", [("dX",), ("dA",), ("dB",), ("dX", "dA"), ("dA", "dB"), ("dX", "dB")])
@pytest.mark.parametrize("saved", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_wanted_results_of_many_rows(want, saved, dtype):
    check(Case(1500, 264, 328, 24, 12, "mixed", dtype), want=want, saved=saved)


@pytest.mark.parametrize("N,kind", [(90, "single"), (300, "mixed"), (1300, "runs")])
@pytest.mark.parametrize("r", [264, 320])
def test_ranks_above_those_of_the_tensor_cores(N, r, kind):
    check(Case(N, 328, 400, r, 3, kind, BF16))
