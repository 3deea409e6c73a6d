"""What a PackedSublayer keeps and reports."""
import pytest
import torch

from paper_2603_06619_b200 import nat
from paper_2603_06619_b200.body import PackedSublayer

pytestmark = pytest.mark.gpu


def _sublayer(cap=64, B=2, dtype=torch.bfloat16, **kw):
    return PackedSublayer(cap, B, 64, 2, 1, 64, dtype, **kw)


def _cu(*bounds):
    return torch.tensor(bounds, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("captured", [False, True])
def test_status_keeps_what_either_direction_found(captured, dtype):
    sub = _sublayer(dtype=dtype)
    qkv = torch.randn(64, 4, 64, device="cuda").to(dtype)
    dout = torch.randn(64, 2, 64, device="cuda").to(dtype)
    forward, backward = _cu(0, 30, 64), _cu(0, 30, 64)   # bounds of their own, to go wrong one by one

    def step():
        sub.attend(qkv, forward)
        sub.attend_backward(qkv, backward, dout)

    step()
    if captured:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        step = g.replay
    step()
    assert sub.status() == 0
    for of in (forward, backward):
        of[2] = 4000                                     # more rows than there are
        step()
        assert sub.status() == nat.NAT_DEV_CAPACITY
        of[2] = 64
        step()
        assert sub.status() == 0                         # of the last calls, not of all
