"""Calls on a stream of the caller's: what a call makes itself (workspaces, results) is not handed to anybody else while that stream still
has the call to run, is no block that the current stream still works on, and stays while the current stream still reads it.

The caller's stream is held up by a kernel that waits some time, so that what is looked at is looked at before the call has run; ranges
of memory are compared, and what a wrong range would do to the results."""
import math

import pytest
import torch

from oracle import ab_oracle as orc
from paper_2405_01067_b200 import binding as ab

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
HOLD = 1_000_000_000                    # cycles: half a second


def normal(*shape, seed=0, dtype=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def ranges(tensors):
    return [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors]


def apart(a, b):
    return all(x1 <= y0 or y1 <= x0 for x0, x1 in a for y0, y1 in b)


def results_of(out):
    flat = []
    for o in out if isinstance(out, (tuple, list)) else [out]:
        flat += results_of(o) if isinstance(o, (tuple, list)) else [] if o is None else [o]
    return flat


def clip(norm_only=False):
    grads = [normal(50_001, seed=k) for k in range(3)]
    outs = [torch.empty_like(g) for g in grads]

    def call(stream=None):
        out, norm = ab.ab_grad_clip(ab.ClipPlan(grads, out=None if norm_only else outs, norm_only=norm_only), 2.0, stream=stream)
        return norm if out is None else ([o.clone() for o in out] if stream is None else out, norm)
    call.made = 1                       # results that the call makes, at the end
    return call


def adapters(back, dtype, N, m, n):
    x, dY, W = normal(N, n, seed=1, dtype=dtype), normal(N, m, seed=2, dtype=dtype), normal(m, n, seed=3, dtype=dtype)
    A, B = normal(3, m, 16, seed=4, dtype=dtype), normal(3, 16, n, seed=5, dtype=dtype)
    ids = (torch.arange(N, device="cuda", dtype=torch.int32) * 7 // N) % 4 - 1

    def call(stream=None):
        if back:
            return ab.ab_adapter_backward(x, dY, W, A, B, ids, stream=stream)
        return ab.ab_adapter_forward(x, W, A, B, ids, stream=stream, save_T=True)
    call.made = 3 if back else 2
    return call


def layer(back, dtype):
    x, dY, A, B = (normal(*s, seed=k, dtype=dtype) for k, s in enumerate([(1000, 200), (1000, 264), (264, 16), (16, 200)]))

    def call(stream=None):
        if back:
            return ab.ab_layer_backward(x, dY, A, B, stream=stream)
        return ab.ab_layer_forward(x, A, B, stream=stream, save_T=True)
    call.made = 3 if back else 2
    return call


def conv(back):
    x, dY, A, B = (normal(*s, seed=k, dtype=BF16) for k, s in enumerate([(3, 9, 10, 16), (3, 9, 10, 24), (24, 16), (16, 144)]))

    def call(stream=None):
        if back:
            return ab.ab_conv3x3_backward(x, dY, A, B, stream=stream)
        return ab.ab_conv3x3_forward(x, A, B, stream=stream, save_T=True)
    call.made = 3 if back else 2
    return call


def dense(back, dtype):
    x, dY, W = (normal(*s, seed=k, dtype=dtype) for k, s in enumerate([(900, 200), (900, 264), (264, 200)]))

    def call(stream=None):
        return ab.ab_dense_backward(x, dY, W, stream=stream) if back else ab.ab_dense_forward(x, W, stream=stream)
    call.made = 2 if back else 1
    return call


def sync(which):
    A, B = normal(3, 200, 16), normal(3, 16, 264, seed=1)
    W = (A[0] @ B[0]).contiguous()
    call = {"average": lambda stream=None: ab.ab_group_average(A, stream=stream), "recombine": lambda stream=None: ab.ab_recombine(A[0], B[0], stream=stream),
            "mean": lambda stream=None: ab.ab_recombine_mean(A, B, stream=stream), "split": lambda stream=None: ab.ab_svd_split(W, 16, 0.05, stream=stream)}[which]
    call.made = {"average": 1, "recombine": 1, "mean": 3, "split": 5}[which]
    call.scratch = which in ("recombine", "split")
    return call


CALLS = {"clip": clip, "clip_norm": lambda: clip(True),
         "adapter_forward": lambda: adapters(False, BF16, 1500, 264, 200), "adapter_backward": lambda: adapters(True, BF16, 1500, 264, 200),
         "layer_forward": lambda: layer(False, BF16), "layer_backward": lambda: layer(True, BF16), "layer_backward_fp32": lambda: layer(True, F32),
         "conv_forward": lambda: conv(False), "conv_backward": lambda: conv(True), "dense_forward": lambda: dense(False, BF16),
         "dense_backward": lambda: dense(True, BF16), "dense_backward_fp32": lambda: dense(True, F32), "average": lambda: sync("average"),
         "recombine": lambda: sync("recombine"), "recombine_mean": lambda: sync("mean"), "split": lambda: sync("split"),
         "adapter_forward_few": lambda: adapters(False, BF16, 5, 72, 88), "adapter_backward_fp32": lambda: adapters(True, F32, 300, 101, 77)}


@pytest.fixture(autouse=True)
def loaded():
    """The first launch of a kernel loads it, which may wait for the device: what holds a stream up and what fills are launched before."""
    torch.cuda._sleep(1)
    torch.full((1000,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()


@pytest.fixture
def scratch(monkeypatch):
    """The workspaces that calls make, as ranges."""
    seen, real = [], ab.workspace

    def workspace(nbytes, device):
        t = real(nbytes, device)
        seen.extend(ranges([t]))
        return t
    monkeypatch.setattr(ab, "workspace", workspace)
    return seen


@pytest.mark.parametrize("name", CALLS)
def test_what_a_call_makes_stays_while_its_stream_has_it_to_run(name, scratch):
    call = CALLS[name]()
    want = [t.clone() for t in results_of(call())]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for keep in (True, False):
        scratch.clear()
        with torch.cuda.stream(side):
            torch.cuda._sleep(HOLD)
        out = results_of(call(stream=side))
        made = ranges(out[len(out) - call.made:]) + scratch
        assert scratch or not getattr(call, "scratch", True)
        if not keep:
            out = None
        # as many blocks of every size as the call made, and more, all of them filled
        junk = [torch.full((b - a,), 255, dtype=torch.uint8, device="cuda") for a, b in made for _ in range(3)]
        assert not side.query(), "held up for too short a time to see anything"
        assert apart(ranges(junk), made)
        torch.cuda.synchronize()
        if keep:
            assert all(torch.equal(p, q) for p, q in zip(out, want))
        del out, junk


@pytest.mark.parametrize("name", CALLS)
def test_no_block_that_the_current_stream_still_writes(name, scratch):
    call = CALLS[name]()
    first = results_of(call())
    want = [t.clone() for t in first]
    sizes = [b - a for a, b in ranges(first[len(first) - call.made:]) + scratch]
    torch.cuda.synchronize()
    del first
    side = torch.cuda.Stream()
    scratch.clear()
    torch.cuda._sleep(HOLD)
    late = [torch.full((s,), 255, dtype=torch.uint8, device="cuda") for s in sizes for _ in range(3)]
    theirs = ranges(late)
    del late                            # blocks that the current stream may hand out again, and still has to fill
    out = results_of(call(stream=side))
    made = ranges(out[len(out) - call.made:]) + scratch
    assert not torch.cuda.current_stream().query()
    assert apart(theirs, made)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, want))


@pytest.mark.parametrize("name", CALLS)
def test_results_stay_while_the_current_stream_reads_them(name):
    call = CALLS[name]()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = results_of(call(stream=side))
    out = out[len(out) - call.made:]
    made = ranges(out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(HOLD)
    copies = [t.clone() for t in out]
    del out
    with torch.cuda.stream(side):
        junk = [torch.full((b - a,), 255, dtype=torch.uint8, device="cuda") for a, b in made for _ in range(3)]
    assert not torch.cuda.current_stream().query()
    assert apart(ranges(junk), made)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(copies, [t for t in results_of(call())][-call.made:]))


def test_a_norm_behind_a_current_stream_that_is_late():
    grads = [normal(70_001, seed=k) for k in range(2)]
    want = orc.grad_clip([g.double().cpu().numpy() for g in grads], 2.0)[1]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(HOLD)
    _, norm = ab.ab_grad_clip(ab.ClipPlan(grads), 2.0, stream=side)
    side.synchronize()
    assert not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    # four squares at a time in fp32, half of their error in the root, one rounding
    assert abs(float(norm) - want) <= (2.0 ** -23 + 2.0 ** -24) * want


def test_a_norm_that_is_kept_stays():
    """One plan, another norm a call: what an earlier call returned does not change."""
    g = normal(10_000)
    plan = ab.ClipPlan([g], norm_only=True)
    norms = []
    for _ in range(4):
        norms.append(ab.ab_grad_clip(plan, 1.0)[1])
        g.mul_(2.0)
    first = float(norms[0])
    # doubling is exact, and so are the sums' and the root's
    assert first > 0 and [float(n) for n in norms] == [first, 2 * first, 4 * first, 8 * first] and plan.norm is norms[-1]


def test_one_plan_on_two_streams_and_in_two_graphs():
    a = [normal(300_001, seed=k) for k in range(4)]
    plan = ab.ClipPlan(a, norm_only=True)
    want = ab.ab_grad_clip(plan, 1.0)[1].clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    norms = [ab.ab_grad_clip(plan, 1.0, stream=streams[i % 2])[1] for i in range(40)]
    torch.cuda.synchronize()
    assert math.isfinite(float(want)) and all(torch.equal(n, want) for n in norms)
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(ab.ab_grad_clip(plan, 1.0)[1])
    assert outs[0].data_ptr() != outs[1].data_ptr()
    for _ in range(20):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs)


def test_norms_of_many_calls_are_all_their_own():
    g = normal(1000)
    plan = ab.ClipPlan([g], norm_only=True)
    norms = [ab.ab_grad_clip(plan, 1.0)[1] for _ in range(200)]
    assert len({n.data_ptr() for n in norms}) == 200 and len({float(n) for n in norms}) == 1


@pytest.mark.parametrize("name", CALLS)
def test_captured_on_a_branch(name):
    """A call on a stream that joins a capture and leaves it again: what it makes is the graph's."""
    call = CALLS[name]()
    want = [t.clone() for t in results_of(call())]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        out = results_of(call(stream=side))
        torch.cuda.current_stream().wait_stream(side)
    for t in out:
        t.fill_(3)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, want))
