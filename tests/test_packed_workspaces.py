"""Workspaces of the operators around the packed attention: one that was made for a large batch serves every smaller one (no GPU
needed)."""
import pytest
import torch

from paper_2603_06619_b200 import nat

F32, BF16 = torch.float32, torch.bfloat16


def _around(marks, top):
    caps = {0, 1, 7, 64, 1000, top}
    for m in marks:
        caps.update(range(max(m - 70, 0), m + 70))
    c = 1
    while c < top:
        caps.update((c, c + 1))
        c += c // 7 + 1
    return sorted(caps)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E", [1, 4, 7, 64, 65, 128, 1024])
@pytest.mark.parametrize("n_in,n_out", [(64, 64), (2048, 768), (1024, 1024), (8, 16), (264, 72), (4096, 136)])
def test_experts_workspace_grows_with_cap(n_in, n_out, E, dtype):
    """Over the capacities at which tiles of other sizes are taken, whatever those are for each type."""
    p = nat.experts_params(E, n_in, n_out, dtype)
    marks = [k * E for k in (32, 48, 49, 64, 96, 97, 128, 256)] + [128 * k for k in (1, 9, 10, 37, 74, 148)]
    sizes = [nat.nat_experts_workspace_bytes(p, c) for c in _around(marks, 2_000_000)]
    assert sizes[0] > 0 and sizes == sorted(sizes)


def test_a_smaller_call_is_not_refused():
    """Pairs of capacities on both sides of a change of tiles."""
    for E, large, small in ((64, 3147, 2120), (128, 6280, 6215), (1024, 50176, 50175), (128, 12416, 12415)):
        p = nat.experts_params(E, 2048, 768, BF16)
        assert nat.nat_experts_workspace_bytes(p, small) <= nat.nat_experts_workspace_bytes(p, large)
