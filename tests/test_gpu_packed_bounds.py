"""Rows that no sequence owns: with positions of their own as with those of the sequences, the head norms leave them alone, in
front of the first sequence and behind the last, and out of the weights' gradients."""
import pytest
import torch

from paper_2603_06619_b200 import nat
from paper_2603_06619_b200.body import PackedSublayer

pytestmark = pytest.mark.gpu


def _batch(dtype, cap, Hq, Hkv, D, bounds, seed):
    """NaN outside the sequences; their tokens' positions, and others outside."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    cu = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    qkv, dqk = rand(cap, Hq + 2 * Hkv, D).to(dtype), rand(cap, Hq + Hkv, D).to(dtype)
    positions = torch.full((cap,), 5, dtype=torch.int32, device="cuda")
    for lo, hi in zip(bounds[:-1], bounds[1:]):
        positions[lo:hi] = torch.arange(hi - lo)
    for t in (qkv, dqk):
        t[:bounds[0]], t[bounds[-1]:] = float("nan"), float("nan")
    return cu, qkv, dqk, positions, 1 + 0.1 * rand(D), nat.rope_freqs(D, 1e4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bounds", [[7, 20, 33], [0, 0, 33], [40, 40, 40], [3, 50, 50], [49, 49, 50]])
def test_a_sublayers_rows_are_those_of_its_sequences(bounds, dtype):
    """The same positions, given and from the bounds: the same bits."""
    cap, Hq, Hkv, D = 50, 4, 2, 64
    cu, qkv, dqk, positions, w, freq = _batch(dtype, cap, Hq, Hkv, D, bounds, 8)
    got = []
    for at in (None, positions):
        sub = PackedSublayer(cap, len(bounds) - 1, 128, Hq, Hkv, D, dtype)
        qk = sub.rotate(qkv, cu, w, w, freq, positions=at, qk=torch.full_like(dqk, 7.0))
        dqkv = sub.rotate_backward(qkv, cu, w, w, freq, torch.full_like(qkv, 7.0), positions=at, dqk=dqk)
        got.append((qk, dqkv, sub.dw_q, sub.dw_k))
        for t in (qk, dqkv):
            assert (t[:bounds[0]] == 7).all() and (t[bounds[-1]:] == 7).all()
        assert sub.dw_q.isfinite().all() and sub.dw_k.isfinite().all()
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_gradients_of_a_sublayer_that_begins_above_row_zero():
    """Attention leaves the rows in front of the first sequence out of its gradients: whatever the buffers held there has no part
    in what the sublayer's gradients are."""
    cap, Hq, Hkv, D, bounds = 96, 4, 2, 64, [17, 47, 88]
    cu, qkv, _, positions, w, freq = _batch(torch.float32, cap, Hq, Hkv, D, bounds, 9)
    dout = torch.randn(cap, Hq, D, device="cuda")
    got = []
    for at, held in ((None, 0.0), (positions, 1e6)):
        sub = PackedSublayer(cap, 2, 128, Hq, Hkv, D, torch.float32)
        for t in (sub.qk, sub.dqk, sub.dqkv):
            t.fill_(held)
        qk = sub.rotate(qkv, cu, w, w, freq, positions=at)
        sub.attend(qkv, cu, qk)
        dqkv = sub.attend_backward(qkv, cu, dout, qk=qk)
        sub.rotate_backward(qkv, cu, w, w, freq, dqkv, positions=at)
        assert sub.status() == 0 and (dqkv[:17] == held).all() and (dqkv[88:] == held).all()
        got.append((dqkv[17:88], sub.dw_q, sub.dw_k))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_sublayer_without_sequences_has_no_rows():
    cu, qkv, dqk, positions, w, freq = _batch(torch.float32, 20, 2, 1, 64, [4], 10)
    sub = PackedSublayer(20, 0, 128, 2, 1, 64, torch.float32)
    qk = sub.rotate(qkv, cu, w, w, freq, positions=positions, qk=torch.full_like(dqk, 7.0))
    dqkv = sub.rotate_backward(qkv, cu, w, w, freq, torch.full_like(qkv, 7.0), positions=positions, dqk=dqk)
    assert (qk == 7).all() and (dqkv == 7).all() and (sub.dw_q == 0).all() and (sub.dw_k == 0).all()
