"""What the embedding, head norms and expert products allow and a training step seldom does: seeded draws over their
shapes, workspaces with guard bytes behind them, the same token named twice, counts below zero, workspaces that calls of
several sizes and streams take in turn.  Parity and tolerances are those of the operators' own tests."""
import random

import numpy as np
import pytest
import torch

from paper_2603_06619_b200 import nat
from test_gpu_embed import Embed
from test_gpu_experts import Experts
from test_gpu_qknorm import Heads

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("seed", range(24))
def test_random_embeddings(seed):
    r = random.Random(seed)
    d = 8 * r.choice([r.randint(1, 40), r.randint(40, 300)])
    V = r.choice([1, 2, r.randint(3, 60), r.randint(60, 3000), r.randint(3000, 140000 if d < 200 else 9000)])
    n = r.choice([0, 1, r.randint(2, 130), r.randint(130, 2100), r.randint(2100, 9000), r.randint(9000, 30000)])
    n = min(n, 6_000_000 // d)
    Embed(n, V, d, r.choice([F32, BF16]), seed=seed, spare=r.choice([0, 1, 150]), scale=r.choice([1.0, 0.0, 22.6]),
          picked=r.random() < 0.5, accumulate=r.random() < 0.4).check()


@pytest.mark.parametrize("seed", range(24))
def test_random_heads(seed):
    r = random.Random(seed)
    D = 8 * r.randint(1, 16)
    Hkv = r.choice([1, 2, 3, 8])
    lengths = [r.choice([0, 1, r.randint(2, 40), r.randint(40, 600)]) for _ in range(r.choice([1, 4, 40]))]
    lengths[0] = max(lengths[0], 1)
    Heads(lengths, Hkv * r.choice([1, 2, 5, 8]), Hkv, D, r.choice([F32, BF16]), R=16 * r.randint(0, D // 16),
          interleaved=r.random() < 0.5, norm=r.random() < 0.7, first=r.choice([None, None, 0, 70000, -9]), seed=seed,
          spare=r.choice([0, 1, 90]), count=r.random() < 0.3).check()


def _guarded(op, need, guard=4096):
    """Exactly the bytes that were asked for, and others behind them."""
    buf = torch.full((need + guard,), 0xA5, dtype=torch.uint8, device="cuda")
    op.ws = buf[:need]
    return buf[need:]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("what", ["few", "some", "many"])
def test_workspaces_are_not_left(what, dtype):
    k = {"few": 1, "some": 40, "many": 700}[what]
    e = Embed(7 * k, 3 * k + 2, 72, dtype, seed=1, spare=0, ids=np.arange(7 * k) // 5 % 3)
    h = Heads([3 * k, k], 3, 1, 72, dtype, R=64, seed=2, spare=0)
    x = Experts([k, 0, 9 * k, 5], 72, 136, dtype, seed=3, spare=0)
    lone = Experts([25 * k], 72, 136, dtype, seed=4, spare=0)   # its weights' gradient is cut into parts
    guards = [_guarded(e, nat.nat_embed_workspace_bytes(e.params, e.cap)),
              _guarded(h, nat.nat_qknorm_workspace_bytes(h.params, h.cap))]
    guards += [_guarded(o, nat.nat_experts_workspace_bytes(o.params, o.cap)) for o in (x, lone)]
    for op in (e, h, x, lone):
        op.check()
    assert all((g == 0xA5).all() for g in guards)


def test_a_token_named_twice_counts_twice():
    e = Embed(600, 40, 64, F32, seed=5, picked=True)
    e.sel[1:600:2] = e.sel[0:600:2]          # pairs of rows of the same token
    e.of_rows = e.ids[e.sel[:600].long()].cpu().numpy()
    e.check()
    e.sel[:] = e.sel[7].clone()              # all rows of one token
    e.of_rows = e.ids[e.sel[:600].long()].cpu().numpy()
    e.check()


def test_counts_below_zero_are_none():
    e = Embed(300, 20, 64, BF16, seed=6)
    e.n_rows.fill_(-3)
    e.fwd()
    e.bwd()
    assert (e.x == 7).all() and (e.dtable == 0).all() and nat.nat_poll_status(e.ws) == 0
    h = Heads([200, 100], 2, 1, 64, BF16, seed=7, first=0)
    h.n_rows.fill_(-1)
    h.fwd()
    h.bwd()
    assert (h.out == 7).all() and (h.dqkv == 7).all() and (h.dw_q == 0).all() and (h.dw_k == 0).all()


def test_one_workspace_for_calls_of_several_kinds_and_sizes():
    """Nothing that a call finds in its workspace tells."""
    ops = [Embed(9000, 70, 64, F32, seed=8), Embed(200, 5000, 64, BF16, seed=9), Experts([700, 0, 2], 136, 72, BF16, seed=10),
           Experts([70, 3, 0, 9], 136, 72, F32, seed=11), Heads([50, 700], 4, 2, 64, BF16, seed=12),
           Experts([30] * 9, 72, 136, BF16, seed=13), Experts([9000], 72, 136, BF16, seed=14)]
    size = max(op.ws.numel() for op in ops)
    shared = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    for op in ops:
        op.ws = shared
    for op in ops + ops[::-1]:
        if op.params.__class__ is not nat.QknormParams and op.params.accumulate:
            continue
        op.check()


def test_two_captured_calls_share_a_workspace():
    """One after the other, in either order: nothing has to survive between calls."""
    a, b = Experts([300, 20, 0, 77], 136, 264, BF16, seed=15), Embed(3000, 100, 64, BF16, seed=16)
    b.ws = a.ws = torch.empty(max(a.ws.numel(), b.ws.numel()), dtype=torch.uint8, device="cuda")
    want = []
    for op, outs in ((a, ("y", "dx", "dw")), (b, ("x", "dtable"))):
        op.fwd()
        op.bwd()
        want.append([getattr(op, o).clone() for o in outs])
    torch.cuda.synchronize()
    graphs = []
    for op in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            op.fwd()
            op.bwd()
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for t in (a.y, a.dx, a.dw, b.x, b.dtable):
            t.fill_(3.0)
        b.ws.random_(0, 255)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for op, outs, ref in ((a, ("y", "dx", "dw"), want[0]), (b, ("x", "dtable"), want[1])):
            for o, w in zip(outs, ref):
                got, rows = getattr(op, o), slice(None)
                if o in ("y", "dx"):
                    rows = slice(a.lo, a.hi)
                elif o == "x":
                    rows = slice(0, b.n)
                assert torch.equal(got[rows], w[rows]), o


def test_calls_on_a_stream_of_their_own_wait_for_nothing_else():
    """Inputs made on the stream of the call, while another stream is at work."""
    e, x = Embed(4000, 200, 128, BF16, seed=17), Experts([500, 0, 90], 136, 264, BF16, seed=18)
    side, busy = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(busy):
        torch.cuda._sleep(20_000_000)
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000)
        e.dx[:e.n].mul_(2.0)
        x.x[:x.hi].mul_(0.5)
        e.check()
        x.check()
    torch.cuda.synchronize()
