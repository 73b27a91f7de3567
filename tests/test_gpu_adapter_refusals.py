"""Workspaces that an adapter call cannot use are refused on the host: nothing is launched with them."""
import pytest
import torch

from paper_2405_01067_b200 import binding as ab

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_workspaces_elsewhere_are_refused(dtype):
    x, dY, W = (torch.ones(s, dtype=dtype, device="cuda") for s in ((10, 24), (10, 16), (16, 24)))
    A, B = (torch.ones(s, dtype=dtype, device="cuda") for s in ((2, 16, 8), (2, 8, 24)))
    ids = torch.zeros(10, dtype=torch.int32, device="cuda")
    need = ab.ab_adapter_workspace_bytes(x, A, B)
    on_host = torch.empty(need, dtype=torch.uint8)
    pinned = torch.empty(need, dtype=torch.uint8, pin_memory=True)
    one_byte = torch.empty(1, dtype=torch.uint8, device="cuda").expand(need)
    spaced = torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]
    for ws in (on_host, pinned, one_byte, spaced):
        with pytest.raises(ValueError):
            ab.ab_adapter_forward(x, W, A, B, ids, ws=ws)
        with pytest.raises(ValueError):
            ab.ab_adapter_backward(x, dY, W, A, B, ids, ws=ws)
    shifted = torch.empty(need + 512, dtype=torch.uint8, device="cuda")[1:]
    with pytest.raises(ab.AbError):
        ab.ab_adapter_forward(x, W, A, B, ids, ws=shifted)
    y, _ = ab.ab_adapter_forward(x, W, A, B, ids, ws=torch.empty(need, dtype=torch.uint8, device="cuda"))
    # 24 + 8 times 24, exact in bf16
    assert (y == 216).all()
