"""A sublayer on packed prefixes, as a trainer runs it, against the same chain in float64."""
import pytest
import torch

import body_parity

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ckpt8", [False, True])
@pytest.mark.parametrize("gate", ["none", "channel", "row"])
def test_sublayer_on_packed_prefixes(gate, ckpt8, dtype):
    body_parity.run_sublayer([33, 1, 70, 128, 5, 200], dtype, gate=gate, ckpt8=ckpt8, seed=1)


def test_sublayer_with_other_head_layouts_and_empty_responses():
    body_parity.run_sublayer([0, 90, 0, 301, 2, 0], torch.bfloat16, d=384, Hq=6, Hkv=2, D=64, seed=2)
    body_parity.run_sublayer([150, 150], torch.bfloat16, d=256, Hq=2, Hkv=2, D=128, gate="row", seed=3)


def test_sublayer_without_rows_reports_nothing():
    import paper_2603_06619_b200.body as body
    spoil = torch.full((1 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    del spoil  # the allocator's next blocks may hold these bytes
    sub = body.PackedSublayer(0, 0, 64, 2, 1, 64, torch.bfloat16)
    assert sub.status() == 0
    sub.attend(torch.empty(1, 4, 64, dtype=torch.bfloat16, device="cuda"),
               torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert sub.status() == 0
