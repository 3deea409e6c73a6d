"""The body from ids to expert products on packed prefixes, against the same chain in float64; captured and replayed; and
one table's gradient from both its ends."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import packed_parity
from paper_2603_06619_b200 import nat
from paper_2603_06619_b200.body import PackedEmbedding, PackedExperts, PackedSublayer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("R,interleaved", [(None, False), (16, False), (None, True)])
def test_body_on_packed_prefixes(R, interleaved, norm, dtype):
    packed_parity.run_body([33, 1, 70, 128, 5, 200], dtype, R=R, interleaved=interleaved, norm=norm, seed=1)


def test_body_with_other_layouts_and_empty_responses():
    packed_parity.run_body([0, 90, 0, 301, 2, 0], torch.bfloat16, d=384, Hq=6, Hkv=2, D=64, E=7, n_out=136, seed=2)
    packed_parity.run_body([150, 150], torch.bfloat16, d=256, Hq=2, Hkv=2, D=128, E=1, n_out=256, seed=3)


def test_a_table_tied_to_the_loss_takes_both_gradients():
    """dW of the loss and, added to it, the embedding's: the same as apart."""
    V, d, n = 300, 64, 90
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda").to(torch.int32)
    dx, dW = torch.randn(n, d, generator=g, device="cuda"), torch.randn(V, d, generator=g, device="cuda")
    apart = PackedEmbedding(n, V, d, torch.float32).gradient(ids, dx, torch.empty(V, d, device="cuda"))
    both = PackedEmbedding(n, V, d, torch.float32, accumulate=True).gradient(ids, dx, dW.clone())
    assert torch.equal(both, dW + apart)


def test_one_step_captured_beside_an_eager_one():
    """Everything between ids and the gradients in one graph, replayed with other prefixes: an eager step's bits."""
    B, cap, d, Hq, Hkv, D, V, E, n_out = 3, 400, 128, 4, 2, 32, 97, 4, 64
    dt = torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    table, w_qkv, w_e = rand(V, d).to(dt), (0.1 * rand(d, (Hq + 2 * Hkv) * D)).to(dt), (0.1 * rand(E, n_out, Hq * D)).to(dt)
    ids, dz = torch.randint(0, V, (cap,), generator=g, device="cuda").to(torch.int32), rand(cap, n_out).to(dt)
    w, freq = 1 + 0.1 * rand(D), nat.rope_freqs(D, 1e4)
    cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    n_rows = torch.zeros(1, dtype=torch.int32, device="cuda")
    e_offs = torch.zeros(E + 1, dtype=torch.int32, device="cuda")

    def parts():
        return (PackedEmbedding(cap, V, d, dt), PackedSublayer(cap, B, d, Hq, Hkv, D, dt), PackedExperts(cap, E, Hq * D, n_out, dt),
                {k: torch.zeros(*s, device="cuda").to(t) for k, s, t in (
                    ("x", (cap, d), dt), ("z", (cap, n_out), dt), ("do", (cap, Hq * D), dt), ("dw", (E, n_out, Hq * D), torch.float32),
                    ("dt", (V, d), torch.float32))})

    def step(emb, sub, exp, t):
        emb.lookup(table, ids, t["x"], n_rows=n_rows)
        qkv = (t["x"] @ w_qkv).view(cap, Hq + 2 * Hkv, D)
        qk = sub.rotate(qkv, cu, w, w, freq)
        o = sub.attend(qkv, cu, qk).view(cap, Hq * D)
        exp.forward(o, w_e, e_offs, t["z"])
        exp.backward(o, w_e, e_offs, dz, t["do"], t["dw"])
        dqkv = sub.attend_backward(qkv, cu, t["do"].view(cap, Hq, D), qk=qk)
        sub.rotate_backward(qkv, cu, w, w, freq, dqkv)
        emb.gradient(ids, dqkv.view(cap, -1) @ w_qkv.t(), t["dt"], n_rows=n_rows)

    def batch(bounds, loads):
        cu.copy_(torch.tensor([0] + bounds, dtype=torch.int32))
        n_rows.fill_(bounds[-1])
        e_offs.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(loads)]).astype(np.int32)))

    def results(sub, t, n):
        return [t["x"][:n], t["z"][:n], t["do"][:n], t["dw"], t["dt"], sub.dqkv[:n], sub.dw_q, sub.dw_k]

    batch([100, 130, 390], [90, 0, 200, 100])
    a, b = parts(), parts()
    step(*a)
    step(*b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*b)
    for bounds, loads in (([100, 130, 390], [90, 0, 200, 100]), ([1, 1, 7], [0, 0, 0, 7]), ([200, 300, 400], [100, 100, 100, 100])):
        batch(bounds, loads)
        for t in (a[3], b[3]):
            for v in t.values():
                v.zero_()
        step(*a)
        graph.replay()
        torch.cuda.synchronize()
        n = bounds[-1]
        for x, y in zip(results(a[1], a[3], n), results(b[1], b[3], n)):
            assert torch.equal(x, y)
        assert all(p.status() == 0 for p in (*a[:3], *b[:3]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_positions_that_are_given_leave_the_rows_behind_the_last_sequence_alone(dtype):
    """The same positions, given and from the bounds, with NaN rows behind: the same bits."""
    B, n, cap, Hq, Hkv, D = 2, 33, 50, 4, 2, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    cu = torch.tensor([0, 20, n], dtype=torch.int32, device="cuda")
    qkv, dqk = rand(cap, Hq + 2 * Hkv, D).to(dtype), rand(cap, Hq + Hkv, D).to(dtype)
    qkv[n:], dqk[n:] = float("nan"), float("nan")
    positions = torch.full((cap,), 5, dtype=torch.int32, device="cuda")
    positions[:20], positions[20:n] = torch.arange(20), torch.arange(n - 20)
    w, freq = 1 + 0.1 * rand(D), nat.rope_freqs(D, 1e4)
    got = []
    for at in (None, positions):
        sub = PackedSublayer(cap, B, 128, Hq, Hkv, D, dtype)
        qk = sub.rotate(qkv, cu, w, w, freq, positions=at, qk=torch.full_like(dqk, 7.0))
        dqkv = sub.rotate_backward(qkv, cu, w, w, freq, torch.full_like(qkv, 7.0), positions=at, dqk=dqk)
        got.append((qk, dqkv, sub.dw_q, sub.dw_k))
        assert (qk[n:] == 7).all() and (dqkv[n:] == 7).all() and sub.dw_q.isfinite().all() and sub.dw_k.isfinite().all()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


FIRST_CALLS = """
import sys
sys.path.insert(0, {root!r})
sys.path.insert(0, {root!r} + "/tests")
import torch
from test_gpu_embed import Embed
from test_gpu_experts import Experts
from test_gpu_qknorm import Heads
dt = torch.{dtype}
ops = [Embed(7000, 300, 128, dt, seed=1), Embed(4000, 90, 64, dt, seed=2), Heads([90, 41], 4, 2, 64, dt, seed=3),
       Experts([300, 0, 41], 136, 264, dt, seed=4), Experts([9, 0, 4, 1], 136, 264, dt, seed=5),
       Experts([5000, 4000], 72, 136, dt, seed=6)]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    for op in ops:
        op.fwd()
        op.bwd()
graph.replay()
torch.cuda.synchronize()
names = {{Embed: ("x", "dtable"), Heads: ("out", "dqkv", "dw_q", "dw_k"), Experts: ("y", "dx", "dw")}}
got = [[getattr(op, k).clone() for k in names[type(op)]] for op in ops]
for op, first in zip(ops, got):
    op.fwd()
    op.bwd()
    assert all(torch.equal(a, getattr(op, k)) for a, k in zip(first, names[type(op)])), type(op)
print("same bits")
"""


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_first_calls_of_a_process_inside_a_capture(dtype):
    """Whatever a first call sets up needs no call before the capture."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS.format(root=root, dtype=dtype)], capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and "same bits" in r.stdout, r.stdout + r.stderr
