"""The gates of test_gpu_adapter_precision.py tell what they are for: products of three pieces, or of six terms, pass, those of fewer do not.
No GPU needed."""
import torch

from adapter_pieces import GATE, lone_rows, pieces


def values(n, seed):
    g = torch.Generator().manual_seed(seed)
    return (1 + torch.rand(n, generator=g)) * torch.randn(n, generator=g).sign()


def share_outside(got, want, gate=GATE):
    return float((((got - want).abs() > gate * want.abs())).double().mean())


def test_three_pieces_pass_and_two_do_not():
    t, d = values(20_000, 1), values(20_000, 2).bfloat16().double()
    want = d * t.double()
    assert share_outside((d * pieces(t, 3)).float().double(), want) == 0
    assert share_outside((d * pieces(t, 2)).float().double(), want) > 0.5


def test_six_terms_pass_and_three_do_not():
    a, b = values(20_000, 3), values(20_000, 4)
    want = a.double() * b.double()
    p = [pieces(a, k + 1) - (pieces(a, k) if k else 0) for k in range(3)]
    q = [pieces(b, k + 1) - (pieces(b, k) if k else 0) for k in range(3)]
    three = p[0] * q[0] + p[0] * q[1] + p[1] * q[0]
    six = three + p[1] * q[1] + p[0] * q[2] + p[2] * q[0]
    assert share_outside(six.float().double(), want) == 0
    assert share_outside(three.float().double(), want) > 0.5


def test_half_a_step_passes_with_two_pieces_and_not_with_one():
    """A bf16 result: half a step of it, and 2^-16 of it for T."""
    t, a = values(20_000, 5), values(20_000, 6).bfloat16().double()
    want = a * t.double()
    step = torch.exp2(torch.floor(torch.log2(want.abs())) - 7)
    for count, ok in ((1, False), (2, True), (3, True)):
        got = (a * pieces(t, count)).bfloat16().double()
        outside = float(((got - want).abs() > step / 2 + 2.0 ** -16 * want.abs()).double().mean())
        assert outside == 0 if ok else outside > 0.2


def test_rows_have_one_value_each():
    x, at, value = lone_rows(50, 64, 7, torch.bfloat16)
    assert ((x != 0).sum(1) == 1).all() and len(set(at.tolist())) == 50 and torch.equal(x.double().sum(1), value)
