"""Expert products around and above 64 experts, beyond which a kernel in front lists the tiles: parity and tolerances are those
of ``test_gpu_experts.py``."""
import numpy as np
import pytest
import torch

from oracle import nat_packed as op
from paper_2603_06619_b200 import nat
from test_gpu_experts import Experts, _close, _np

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


def _loads(E, seed, most):
    """Some experts without rows, some with a few, some with many."""
    r = np.random.default_rng(seed)
    return np.where(r.random(E) < 0.2, 0, np.rint(np.exp(r.uniform(0.0, np.log(most), E)))).astype(int)


# by their average rows: tiles of 64, 128 and 256
@pytest.mark.parametrize("E,most", [(65, 60), (200, 90), (65, 400), (100, 350), (65, 2000), (130, 1300)])
@pytest.mark.parametrize("sizes", [(72, 136), (264, 520), (24, 1000)])
def test_parity_in_tiles_of_every_size(sizes, E, most):
    Experts(_loads(E, E + most, most), *sizes, BF16, seed=most, first=9, strides=(8, 24)).check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("most", [30, 200, 1500])
def test_accumulation(most, dtype):
    Experts(_loads(90, most, most), 136, 72, dtype, seed=1, accumulate=True).check()


@pytest.mark.parametrize("accumulate", [False, True])
def test_rows_cut_into_parts(accumulate):
    """Few tiles of the weights' gradient for 66 experts with a thousand rows each, some with none."""
    loads = [1500, 0, 2100] * 22
    e = Experts(loads, 40, 24, BF16, seed=2, accumulate=accumulate)
    # room for the sums of two parts at least
    assert nat.nat_experts_workspace_bytes(e.params, e.cap) > 2 * 4 * e.dw.numel()
    e.check()


def test_all_rows_with_one_expert_and_none_at_all():
    for at in (0, 37, 79):
        loads = [0] * 80
        loads[at] = 3001
        Experts(loads, 136, 264, BF16, seed=3).check()
    Experts([0] * 80, 136, 264, BF16, seed=4, spare=50).check()


@pytest.mark.parametrize("k", [20, 70, 150])
def test_offsets_beyond_the_rows_and_out_of_order(k):
    E = 80
    e, good = (Experts([k] * E, 64, 72, BF16, seed=5, spare=0) for _ in range(2))
    good.fwd()
    good.bwd()
    e.offs[E] = 10 ** 9                               # the rows there are
    e.fwd()
    assert nat.nat_poll_status(e.ws) == nat.NAT_DEV_CAPACITY and torch.equal(e.y, good.y)
    e.bwd()
    assert nat.nat_poll_status(e.ws) == nat.NAT_DEV_CAPACITY
    assert torch.equal(e.dx, good.dx) and torch.equal(e.dw, good.dw)
    for at, bad in ((0, -1), (70, 5), (E, -7), (3, 10 ** 9)):
        e.offs.copy_(good.offs)
        e.offs[at] = bad
        for t in (e.y, e.dx, e.dw):
            t.fill_(7.0)
        e.fwd()
        assert nat.nat_poll_status(e.ws) == nat.NAT_DEV_CAPACITY
        e.bwd()
        assert nat.nat_poll_status(e.ws) == nat.NAT_DEV_CAPACITY
        assert all((t == 7).all() for t in (e.y, e.dx, e.dw))
    e.offs.copy_(good.offs)                           # the workspace keeps nothing of that
    e.fwd()
    assert nat.nat_poll_status(e.ws) == 0 and torch.equal(e.y, good.y)


def test_replay_with_other_loads():
    E, rows = 80, 8000
    loads = [np.diff(np.concatenate([[0], np.sort(np.random.default_rng(s).integers(0, rows + 1, E - 1)), [rows]])) for s in range(3)]
    e = Experts(loads[0], 200, 264, BF16, seed=6)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        e.fwd()
        e.bwd()
    x, w, dy = _np(e.x[:rows]), _np(e.w), _np(e.dy[:rows])
    for turn in (0, 1, 2, 0):
        offs = np.concatenate([[0], np.cumsum(loads[turn])])
        e.offs.copy_(torch.from_numpy(offs))
        e.ws.random_(0, 255)
        for t in (e.y, e.dx, e.dw):
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (e.y, e.dx, e.dw)]
        e.fwd()
        e.bwd()
        assert all(torch.equal(a, b) for a, b in zip(got, (e.y, e.dx, e.dw)))
        ref, mag = op.experts_fwd(x, w, offs)
        _close("y", e.y[:rows], ref, 2.0 ** -8 * np.abs(ref) + 216 * 2.0 ** -23 * mag)
        b = op.experts_bwd(x, w, dy, offs)
        _close("dx", e.dx[:rows], b["dx"], 2.0 ** -8 * np.abs(b["dx"]) + 280 * 2.0 ** -23 * b["mag_dx"])
        _close("dw", e.dw, b["dw"], (loads[turn].max() + 16) * 2.0 ** -23 * b["mag_dw"])


@pytest.mark.parametrize("k", [20, 70, 150])
def test_infinities_and_nan_stay_in_their_row_and_expert(k):
    E = 70
    a, b = (Experts([k] * E, 72, 136, BF16, seed=7) for _ in range(2))
    row = 30 * k + k - 1                              # the last of expert 30
    b.x[row, 5], b.dy[row, 7] = float("nan"), float("inf")
    b.w[64], b.w[31] = float("nan"), float("inf")
    for e in (a, b):
        e.fwd()
        e.bwd()
    keep = torch.ones(a.cap, dtype=torch.bool, device="cuda")
    keep[row], keep[64 * k:65 * k], keep[31 * k:32 * k] = False, False, False
    assert torch.equal(a.y[keep], b.y[keep]) and torch.equal(a.dx[keep], b.dx[keep])
    assert not torch.isfinite(b.y[row]).any() and not torch.isfinite(b.dx[row]).any()
    same = [e for e in range(E) if e != 30]
    assert torch.equal(a.dw[same], b.dw[same])
    assert not torch.isfinite(b.dw[30][:, 5]).any() and not torch.isfinite(b.dw[30][7]).any()
