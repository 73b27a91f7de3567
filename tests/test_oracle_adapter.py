"""Pins of the checker's adapters and gradient clipping: row loops written from the definition, finite differences, the library's
clipping.  CPU only."""
import numpy as np
import torch

from oracle import ab_oracle as orc


def _case(seed, N=13, m=7, n=9, r=3, L=4):
    rng = np.random.default_rng(seed)
    ids = rng.integers(-1, L, N)
    return (rng.standard_normal((N, n)), rng.standard_normal((m, n)), rng.standard_normal((L, m, r)), rng.standard_normal((L, r, n)),
            ids, rng.uniform(0.5, 2.0, L))


def test_forward_row_by_row():
    x, W, A, B, ids, s = _case(0)
    T, y = orc.adapter_forward(x, W, A, B, ids, s)
    for i, a in enumerate(ids):
        want = W @ x[i]
        if a >= 0:
            want = (W + s[a] * A[a] @ B[a]) @ x[i]
        assert np.allclose(y[i], want, rtol=1e-12, atol=1e-12)
        assert np.allclose(T[i], s[a] * (B[a] @ x[i]) if a >= 0 else 0.0, rtol=1e-12, atol=1e-12)


def test_gradients_against_differences():
    x, W, A, B, ids, s = _case(1)
    dY = np.random.default_rng(2).standard_normal((x.shape[0], W.shape[0]))
    grads = orc.adapter_backward(x, dY, W, A, B, ids, s)
    for which, g in zip((0, 2, 3), grads):
        args = [x, W, A, B]
        for flat in range(0, g.size, 5):
            at = np.unravel_index(flat, g.shape)
            hi, lo = [a.copy() for a in args], [a.copy() for a in args]
            hi[which][at] += 1e-5
            lo[which][at] -= 1e-5
            diff = ((orc.adapter_forward(*hi, ids, s)[1] - orc.adapter_forward(*lo, ids, s)[1]) * dY).sum() / 2e-5
            assert abs(diff - g[at]) <= 1e-7 * (1.0 + abs(g[at])), (which, at)      # a bilinear map: only rounding is left


def test_clip_against_the_library():
    rng = np.random.default_rng(3)
    grads = [rng.standard_normal(k) * 10.0 ** (k % 3) for k in (1, 5, 200, 33)]
    for max_norm in (0.5, 1e4):
        ps = [torch.nn.Parameter(torch.zeros(g.size, dtype=torch.float64)) for g in grads]
        for p, g in zip(ps, grads):
            p.grad = torch.tensor(g)
        norm = float(torch.nn.utils.clip_grad_norm_(ps, max_norm))
        out, got = orc.grad_clip(grads, max_norm)
        assert abs(got - norm) <= 1e-12 * norm
        for o, p in zip(out, ps):
            assert np.allclose(o, p.grad.numpy(), rtol=2e-6 / norm + 1e-12, atol=0)      # the library divides by norm + 1e-6


def test_clip_leaves_what_is_not_finite():
    out, norm = orc.grad_clip([np.array([1.0, np.inf]), np.array([2.0])], 0.1)
    assert norm == np.inf and out[1][0] == 2.0
