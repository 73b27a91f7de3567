"""ab_grad_clip where max_norm / norm is no full fp32 number: gradients near the type's largest value, or a tiny limit.

Tolerance: the squares of these values are added in 64 bits, so that the factor is right to about 2^-50; what is left is the product's
rounding to fp32 (2^-24, or half of the smallest subnormal, 2^-150) and the result's own (bf16: 2^-8, or 2^-134)."""
import math

import numpy as np
import pytest
import torch

from paper_2405_01067_b200 import binding as ab

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("count,value,max_norm", [(5001, 3e38, 1.0), (5001, 3e38, 1e-3), (40_000, 3e38, 1e-6), (5001, 3e38, 1e-30), (100_003, 1e30, 1e-12),
                                                  (5001, 1e38, 2.0), (1, 3e38, 1e-40)])
def test_factors_below_fp32(count, value, max_norm, shift, dtype):
    g = torch.Generator(device="cuda").manual_seed(count)
    arena = torch.empty(count + shift, dtype=dtype, device="cuda")
    grad = arena[shift:]
    # magnitudes from the largest down by five orders, either sign
    grad.copy_(value * 10.0 ** (-5 * torch.rand(count, device="cuda", generator=g)) * torch.randn(count, device="cuda", generator=g).sign())
    grad[0] = value
    x = grad.float().cpu().numpy().astype(np.float64)
    norm = math.sqrt(float((x * x).sum()))
    want = x * (float(np.float32(max_norm)) / norm)
    for out in (torch.full_like(grad, float("nan")), grad):
        ab.ab_grad_clip(ab.ClipPlan([grad], out=[out]), max_norm)
        got = out.float().cpu().numpy().astype(np.float64)
        step, least = (2.0 ** -24, 2.0 ** -150) if dtype == F32 else (2.0 ** -8 + 2.0 ** -23, 2.0 ** -134 + 2.0 ** -149)
        assert (np.abs(got - want) <= step * np.abs(want) * (1 + 2.0 ** -20) + least * (1 + 2.0 ** -20)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_list_of_gradients(dtype):
    """Without a plan: other tensors every step, as a backward pass leaves them that found none."""
    for step in range(3):
        g = torch.Generator(device="cuda").manual_seed(step)
        grads = [torch.randn(k, device="cuda", generator=g).to(dtype) for k in (1000, 77, 5)]
        copies = [t.clone() for t in grads]
        out, norm = ab.ab_grad_clip(grads if step else iter(grads), 1.0)
        want, norm2 = ab.ab_grad_clip(ab.ClipPlan(copies), 1.0)
        assert torch.equal(norm, norm2) and len(out) == 3
        assert all(p is q and torch.equal(p, w) for p, q, w in zip(out, grads, want))
    for bad in ([], [torch.ones(3)], [torch.ones(3, device="cuda"), torch.ones(3, device="cuda", dtype=torch.float64)]):
        with pytest.raises((ValueError, TypeError)):
            ab.ab_grad_clip(bad, 1.0)
