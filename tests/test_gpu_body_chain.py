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
