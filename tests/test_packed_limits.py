"""The largest capacities of the operators around the packed attention (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2603_06619_b200 import nat

A = 4096                           # a fake device address: nothing is dereferenced


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E", [1, 64, 65, 1024])
def test_experts_rows_whose_tiles_would_leave_32_bits_are_refused(E, dtype):
    """A tile has up to 256 rows: with an expert of 2^31 - 256 rows or more, the number of the row behind its last tile has no place
    in 32 bits.  Up to 1024 rows below 2^31 there is room for a tile and what the loads are ahead."""
    p = nat.experts_params(E, 8, 8, dtype)
    lib = nat.load()
    most = 2 ** 31 - 1024
    for cap in (most + 1, 2 ** 31 - 256, 2 ** 31 - 1):
        assert nat.nat_experts_workspace_bytes(p, cap) == 0
        assert lib.nat_experts_fwd(ctypes.byref(p), A, cap, A, A, A, A, 1 << 40, None) == -1
        assert lib.nat_experts_bwd(ctypes.byref(p), A, cap, A, A, A, A, A, A, 1 << 40, None) == -1
    assert nat.nat_experts_workspace_bytes(p, most) > 0
    assert most + 2 * 256 + 4 * 64 < 2 ** 31
