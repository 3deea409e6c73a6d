"""Packed attention in workspaces that were made for other batches: right results, and nothing written past the end."""
import pytest
import torch

from paper_2603_06619_b200 import nat
from test_body_workspace import accepted
from test_gpu_body import DT, Attn

pytestmark = pytest.mark.gpu


def least(p, B, cap):
    """The smallest size that both directions accept."""
    lo, hi = 0, nat.nat_attn_workspace_bytes(p, B, cap)
    while hi - lo > 1:
        mid = (lo + hi) // 2
        lo, hi = (lo, mid) if all(accepted(p, B, cap, mid, b) for b in (False, True)) else (mid, hi)
    return hi


def guarded(a, nbytes):
    buf = torch.full((nbytes + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    a.ws = buf[:nbytes]
    return buf[nbytes:]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,heads", [([2100], (4, 1, 128)), ([1500, 3, 700], (2, 2, 64)), ([0, 1029, 0, 1], (7, 1, 96)),
                                           ([700, 40], (8, 2, 128)), ([1], (1, 1, 8)), ([3] * 1100, (2, 1, 64))])
def test_least_workspace(lengths, heads, dtype):
    a = Attn(lengths, *heads, DT[dtype], seed=31)
    need = least(a.params, a.B, a.cap)
    guard = guarded(a, need)
    a.check()
    assert (guard == 0xA5).all()
    guard = guarded(a, nat.nat_attn_workspace_bytes(a.params, a.B, a.cap))
    a.check()
    assert (guard == 0xA5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_batches_in_the_workspace_of_a_large_one(dtype):
    """One buffer, sized once for the largest batch, for batches of any shape below it."""
    heads = (4, 2, 64)
    p = nat.attn_params(*heads, DT[dtype])
    ws = nat.alloc_workspace(nat.nat_attn_workspace_bytes(p, 64, 74000), "cuda")
    for lengths in ([2100], [1900, 200], [5] * 60, [1], [300, 0, 700]):
        a = Attn(lengths, *heads, DT[dtype], seed=32)
        a.ws = ws
        a.check()
