"""Inputs of the adapters whose results show how many bits a product was formed with: one value a row, so that nothing is summed and only
roundings and what was cut off are left; and long sums of small values beside one large one."""
import torch

# Of an element: T is rounded once (2^-24); its three pieces add up to it, their products with a bf16 value are exact, and at most three
# additions round or cut the sum (2^-23 each).  Of an fp32 product in six bf16 terms: the three that are left out have at most 2 2^-24 + 2^-32, and three
# additions.  What two pieces of T, or three terms of a product, leave out reaches 2^-16.
GATE = 4 * 2.0 ** -23


def lone_rows(N, width, seed, dtype):
    """N rows, each with one value: (rows, positions, values)."""
    g = torch.Generator().manual_seed(seed)
    at = torch.randperm(width, generator=g)[:N]
    value = (1 + torch.rand(N, generator=g)) * torch.randn(N, generator=g).sign()
    value = value.to(dtype)
    x = torch.zeros(N, width, dtype=dtype)
    x[torch.arange(N), at] = value
    return x, at, value.double()


def pieces(t, count):
    """The sum of the first `count` bf16 pieces of fp32 values, as doubles."""
    rest, total = t.double(), torch.zeros(t.shape, dtype=torch.float64)
    for _ in range(count):
        p = rest.float().bfloat16().double()
        total += p
        rest = rest - p
    return total
