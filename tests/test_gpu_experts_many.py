"""Expert products around and above 64 experts, beyond which a kernel in front lists the tiles: parity and tolerances are those
of ``test_gpu_experts.py``."""
import pytest
import torch

from paper_2603_06619_b200 import nat
from test_gpu_experts import Experts

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E", [60, 64, 65, 130])
def test_one_workspace_for_batches_of_every_size(E, dtype):
    """One that was made for the largest batch, with other bytes behind it, serves the smaller ones."""
    batches = [Experts([k] * E, 72, 136, dtype, seed=k, spare=k) for k in (100, 60, 49, 48, 20, 1, 0)]
    need = nat.nat_experts_workspace_bytes(batches[0].params, batches[0].cap)
    buf = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    for e in batches:
        e.ws = buf[:need]
        e.check()
    assert (buf[need:] == 0xA5).all()
