"""ab_grad_clip against the float64 checker.  Tolerances: the norm is a sum in 64 bits of squares of which four at a time are added in
fp32 (2^-22 of the sum, half of that of its root), rounded to fp32 (2^-24); an output is off by c's and its own rounding."""
import math

import numpy as np
import pytest
import torch

from oracle import ab_oracle as orc
from paper_2405_01067_b200 import binding as ab

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def run_and_check(grads, max_norm, out=None):
    before = [f64(g) for g in grads]
    want, norm = orc.grad_clip(before, max_norm)
    outs, got = ab.ab_grad_clip(ab.ClipPlan(grads, out=out), max_norm)
    rel = 2.0 ** -23 + 2.0 ** -24
    assert abs(float(got) - norm) <= rel * norm
    eps = 2.0 ** -8 if grads[0].dtype == BF16 else 2.0 ** -24
    for o, w in zip(outs, want):
        assert o.dtype == grads[0].dtype
        assert (np.abs(f64(o) - w) <= (eps + 2.0 ** -23 + rel) * np.abs(w) * (1 + 2.0 ** -7) + 1e-45).all()
    if out is not None:
        for g, b in zip(grads, before):
            assert np.array_equal(f64(g), b)
    return outs


def tensors(counts, dtype, seed=0, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(c, device="cuda", generator=g) * std * 10.0 ** (i % 3)).to(dtype) for i, c in enumerate(counts)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("counts", [[1], [7], [8192], [8191, 8193], [1, 0, 3, 100000], [16384] * 3, [2_500_003], list(range(1, 170)), [37] * 1001,
                                    [5000] * 2300])
def test_sizes(counts, dtype, in_place):
    grads = tensors(counts, dtype)
    out = None if in_place else [torch.full_like(g, float("nan")) for g in grads]
    run_and_check(grads, 0.37 * math.sqrt(sum(counts)), out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift_g,shift_o", [(1, 1), (3, 3), (1, 2), (0, 3), (7, 7), (5, 0)])
def test_tensors_that_start_anywhere(dtype, shift_g, shift_o):
    n = 40_001
    arena = tensors([3 * n + 64], dtype)[0]
    out = torch.full_like(arena, 7.0)
    grads = [arena[shift_g + k * (n + 9): shift_g + k * (n + 9) + n] for k in range(3)]
    outs = [out[shift_o + k * (n + 9): shift_o + k * (n + 9) + n] for k in range(3)]
    run_and_check(grads, 1.5, outs)
    covered = torch.zeros(out.numel(), dtype=torch.bool)
    for k in range(3):
        covered[shift_o + k * (n + 9): shift_o + k * (n + 9) + n] = True
    assert (out.cpu()[~covered] == 7).all()
    run_and_check(grads, 1.5)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_below_the_limit_nothing_changes(dtype):
    grads = tensors([1000, 33], dtype)
    before = [g.clone() for g in grads]
    for max_norm in (1e9, float("inf")):
        outs, _ = ab.ab_grad_clip(ab.ClipPlan(grads), max_norm)
        assert all(torch.equal(a, b) for a, b in zip(outs, before))
        copies = [torch.full_like(g, 3.0) for g in grads]
        ab.ab_grad_clip(ab.ClipPlan(grads, out=copies), max_norm)
        assert all(torch.equal(a, b) for a, b in zip(copies, before))
    ab.ab_grad_clip(ab.ClipPlan(grads), 0.0)
    assert all((g == 0).all() for g in grads)


@pytest.mark.parametrize("value", [3e38, 1e30, 1e20, 1e-20, 1e-30, 1e-42])
def test_values_whose_squares_leave_fp32(value):
    g = torch.full((5001,), value, device="cuda")
    g[::2] *= -1
    _, norm = ab.ab_grad_clip(ab.ClipPlan([g], norm_only=True), 1.0)
    want = abs(float(g[0].double())) * math.sqrt(5001)
    if want < 3.4e38:
        assert abs(float(norm) - want) <= 2.0 ** -22 * want + 1e-45
    else:
        assert float(norm) == math.inf
    out = torch.empty_like(g)
    ab.ab_grad_clip(ab.ClipPlan([g], out=[out]), value / 4)
    got = f64(out)
    scale = (float(np.float32(value / 4))) / want            # also where the norm itself is no fp32 number
    assert (np.abs(got - f64(g) * scale) <= 2.0 ** -21 * np.abs(f64(g) * scale) + 2e-45).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("at", [0, 8000, 12344])
def test_a_norm_that_is_not_finite_scales_nothing(dtype, value, at):
    grads = tensors([12345, 77], dtype)
    grads[0][at] = value
    before = [g.clone() for g in grads]
    outs, norm = ab.ab_grad_clip(ab.ClipPlan(grads), 1e-3)
    assert not math.isfinite(float(norm))
    assert all(torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0)) for a, b in zip(outs, before))


def test_zeros():
    grads = [torch.zeros(100, device="cuda"), torch.zeros(0, device="cuda")]
    outs, norm = ab.ab_grad_clip(ab.ClipPlan(grads), 1.0)
    assert float(norm) == 0 and (outs[0] == 0).all()


def test_norm_alone():
    grads = tensors([5000, 1, 70_001], F32)
    before = [g.clone() for g in grads]
    out, norm = ab.ab_grad_clip(ab.ClipPlan(grads, norm_only=True), 1e-6)
    assert out is None and all(torch.equal(a, b) for a, b in zip(grads, before))
    assert abs(float(norm) - orc.grad_clip([f64(g) for g in grads], 1.0)[1]) <= 2.0 ** -22 * float(norm)


def test_two_runs_and_a_replay_give_the_same_bits():
    grads = tensors([100_003] * 60, F32)
    outs = [torch.empty_like(g) for g in grads]
    plan = ab.ClipPlan(grads, out=outs)
    norms = set()
    for _ in range(5):
        norms.add(float(ab.ab_grad_clip(plan, 1.0)[1]))
    assert len(norms) == 1
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ab.ab_grad_clip(plan, 1.0)
    for g in grads:
        g.mul_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    got = [o.clone() for o in outs] + [plan.norm.clone()]
    ab.ab_grad_clip(plan, 1.0)
    assert all(torch.equal(a, b) for a, b in zip(got, outs + [plan.norm]))


def test_on_a_stream():
    grads = tensors([200_000] * 4, F32)
    want = orc.grad_clip([f64(g) for g in grads], 2.0)[0]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    ab.ab_grad_clip(ab.ClipPlan(grads), 2.0, stream=st)
    st.synchronize()
    assert all(orc.rel_frob(f64(g), w) <= 1e-6 for g, w in zip(grads, want))


def test_a_step_of_training_with_adapters():
    """Backward of many adapters, clipping of their gradients, AdamW on every factor, the next forward on the updated bf16 copies."""
    rng = np.random.default_rng(0)
    N, m, n, r, L = 300, 72, 136, 8, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dY = (torch.randn(s, device="cuda", generator=g).to(BF16) for s in ((N, n), (N, m)))
    W = (torch.randn(m, n, device="cuda", generator=g) / 12).to(BF16)
    A, B = torch.randn(L, m, r, device="cuda", generator=g), torch.randn(L, r, n, device="cuda", generator=g) / 12
    ids = torch.tensor(rng.integers(-1, L, N), dtype=torch.int32, device="cuda")
    A16, B16 = A.to(BF16), B.to(BF16)
    y, T = ab.ab_adapter_forward(x, W, A16, B16, ids, save_T=True)
    dX, dA, dB = ab.ab_adapter_backward(x, dY, W, A16, B16, ids, T_saved=T)
    ref = orc.adapter_backward(f64(x), f64(dY), f64(W), f64(A16), f64(B16), ids.cpu().numpy())
    clipped, norm_ref = orc.grad_clip(ref[1:], 0.5)
    _, norm = ab.ab_grad_clip(ab.ClipPlan([dA, dB]), 0.5)
    assert abs(float(norm) - norm_ref) <= 1e-4 * norm_ref
    A_ref, B_ref = f64(A), f64(B)
    for p, p16, grad, want, p_ref in ((A, A16, dA, clipped[0], A_ref), (B, B16, dB, clipped[1], B_ref)):
        mom, var = torch.zeros_like(p), torch.zeros_like(p)
        ab.ab_adamw_step(p, grad, mom, var, 1e-2, 1, eps=1e-3, param_bf16=p16)
        new, _, _ = orc.adamw_step(p_ref, want, np.zeros_like(want), np.zeros_like(want), 1e-2, 1, 0.9, 0.999, 1e-3, 1e-2)
        # the step is 1e-2 g / (|g| + 1e-3): its slope in g is at most 10, and g is off by at most 1e-4 of values below 0.5
        assert np.abs(f64(p) - new).max() <= 10 * 0.5e-4 + 1e-6
        assert torch.equal(p16, p.to(BF16))
    y2, _ = ab.ab_adapter_forward(x, W, A16, B16, ids)
    y2_ref = orc.adapter_forward(f64(x), f64(W), f64(A16), f64(B16), ids.cpu().numpy())[1]
    assert orc.rel_frob(f64(y2), y2_ref) <= 2.0 ** -8


def test_refusals():
    g = torch.ones(8, device="cuda")
    for bad in (lambda: ab.ClipPlan([]), lambda: ab.ClipPlan([g, g.bfloat16()]), lambda: ab.ClipPlan([g], out=[g[:4]]), lambda: ab.ClipPlan([g.cpu()]),
                lambda: ab.ClipPlan([g[::2]]), lambda: ab.ClipPlan([g, g], out=[g])):
        with pytest.raises((ValueError, TypeError)):
            bad()
    plan = ab.ClipPlan([g])
    for bad in (-1.0, float("nan")):
        with pytest.raises(ab.AbError):
            ab.ab_grad_clip(plan, bad)
