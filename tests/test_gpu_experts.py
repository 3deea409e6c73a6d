"""GPU parity of the products grouped by expert against the float64 forms in ``oracle/nat_packed.py``.

Tolerances, by arithmetic: a sum of K products in 32 bits is off by at most (K + 16) steps of 2^-23 of the sum of the terms'
magnitudes (twice half a step, since tensor cores may cut off what they add; products of bfloat16 are exact in 32
bits), and y and dx by half a step of their type, u = 2^-8 in bfloat16 relative to the value.
"""
import random

import numpy as np
import pytest
import torch

from oracle import nat_packed as op
from paper_2603_06619_b200 import nat

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _np(t):
    return t.detach().double().cpu().numpy()


class Experts:
    """Rows before, between the last expert's and the capacity hold NaN; outputs are poisoned."""

    def __init__(self, loads, n_in, n_out, dtype, seed=0, first=0, spare=5, strides=(0, 0), accumulate=False):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.E, self.n_in, self.n_out, self.dtype = len(loads), n_in, n_out, dtype
        self.offs_h = (first + np.concatenate([[0], np.cumsum(loads)])).astype(np.int32)
        self.lo, self.hi = int(self.offs_h[0]), int(self.offs_h[-1])
        self.cap = self.hi + spare
        self.offs = torch.from_numpy(self.offs_h).cuda()
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        rows = max(self.cap, 1)

        def wide(width, more, fill):
            t = torch.full((rows, width + more), 7.0, device="cuda").to(dtype)
            if fill:
                t.copy_(rand(rows, width + more))
                t[:self.lo] = float("nan")
                t[self.hi:] = float("nan")
            return t[:, :width]

        self.x, self.dy = wide(n_in, strides[0], True), wide(n_out, strides[1], True)
        self.y, self.dx = wide(n_out, strides[1], False), wide(n_in, strides[0], False)
        self.w = (rand(self.E, n_out, n_in) / n_in ** 0.5).to(dtype)
        self.old = rand(self.E, n_out, n_in)
        self.dw = self.old.clone() if accumulate else torch.full_like(self.old, 7.0)
        self.params = nat.experts_params(self.E, n_in, n_out, dtype, accumulate=accumulate)
        self.ws = nat.alloc_workspace(nat.nat_experts_workspace_bytes(self.params, self.cap), "cuda")
        self.ws.random_(0, 255)

    def fwd(self):
        nat.nat_experts_fwd(self.params, self.offs, self.cap, self.x, self.w, self.y, self.ws)

    def bwd(self, dx=True, dw=True):
        nat.nat_experts_bwd(self.params, self.offs, self.cap, self.x, self.w, self.dy, self.dx if dx else None,
                            self.dw if dw else None, self.ws)

    def check(self):
        u = 2.0 ** -8 if self.dtype == torch.bfloat16 else 0.0
        lo, hi = self.lo, self.hi
        offs = self.offs_h - lo
        x, w, dy = _np(self.x[lo:hi]), _np(self.w), _np(self.dy[lo:hi])
        self.fwd()
        assert nat.nat_poll_status(self.ws) == 0
        ref, mag = op.experts_fwd(x, w, offs)
        _close("y", self.y[lo:hi], ref, u * np.abs(ref) + (self.n_in + 16) * 2.0 ** -23 * mag)
        self.bwd()
        assert nat.nat_poll_status(self.ws) == 0
        b = op.experts_bwd(x, w, dy, offs)
        _close("dx", self.dx[lo:hi], b["dx"], u * np.abs(b["dx"]) + (self.n_out + 16) * 2.0 ** -23 * b["mag_dx"])
        terms = np.diff(self.offs_h)[:, None, None]
        tol = (terms + 16) * 2.0 ** -23 * b["mag_dw"]
        if self.params.accumulate:
            b["dw"] = b["dw"] + _np(self.old)
            tol = tol + 2.0 ** -23 * np.abs(_np(self.old))
        _close("dw", self.dw, b["dw"], tol)
        for t in (self.y, self.dx):
            assert (t[:lo] == 7).all() and (t[hi:] == 7).all()
            more = t.as_strided((t.shape[0], t.stride(0)), (t.stride(0), 1))[:, t.shape[1]:]
            assert (more == 7).all()


def _close(name, got, ref, tol):
    got = _np(got)
    assert got.shape == ref.shape
    assert np.isfinite(got).all(), name
    over = np.abs(got - ref) - 1.001 * tol - 1e-37
    assert (over <= 0).all(), (name, float(over.max()), float(np.abs(got - ref).max()), np.argwhere(over > 0)[:4].tolist())


LOADS = {"one_row": [1], "few": [0, 3, 0, 1, 0], "edges": [63, 64, 65, 0, 127, 128, 129], "tiles": [255, 256, 257, 1, 511, 513],
         "many": [7, 0, 31, 2, 90, 1, 0, 16] * 6, "long": [1500, 0, 40], "none": [0, 0]}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [(8, 8), (64, 128), (136, 72), (264, 520), (1000, 24), (24, 1000)])
@pytest.mark.parametrize("loads", list(LOADS))
def test_experts_parity(loads, sizes, dtype):
    Experts(LOADS[loads], *sizes, DT[dtype], seed=len(loads)).check()


@pytest.mark.parametrize("loads", [[16, 17, 32, 33, 48, 95, 96, 97, 127, 128, 129, 160, 161, 224, 225, 255, 384, 385, 640],
                                   [0] * 20 + [700] + [1, 15, 63, 64, 65, 0, 0, 31, 130] + [0] * 20],
                         ids=["last_tiles", "lopsided"])
@pytest.mark.parametrize("sizes", [(72, 264), (328, 136), (512, 512)])
def test_experts_last_tiles_of_every_length(loads, sizes):
    """Tiles with few rows lie the other way round; and one expert with many rows among many with few."""
    Experts(loads, *sizes, torch.bfloat16, seed=21, strides=(8, 16)).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_experts_strides_rows_in_front_and_accumulation(dtype):
    Experts([40, 300, 0, 5], 136, 200, DT[dtype], seed=1, first=13, strides=(24, 8)).check()
    Experts([40, 300, 0, 5], 136, 200, DT[dtype], seed=2, accumulate=True).check()
    Experts([300], 64, 64, DT[dtype], seed=3, spare=0, accumulate=True, strides=(0, 64)).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("loads", [[9000], [5000, 0, 70, 4000], [0, 0, 20000]])
def test_experts_rows_cut_into_parts(loads, accumulate, dtype):
    """Few tiles of the weights' gradient and many rows."""
    e = Experts(loads, 72, 136, DT[dtype], seed=4, accumulate=accumulate)
    small = nat.experts_params(len(loads), 72, 136, DT[dtype])
    assert nat.nat_experts_workspace_bytes(small, e.cap) > nat.nat_experts_workspace_bytes(small, 600) + 2 * e.dw.numel() * 4
    e.check()


@pytest.mark.parametrize("accumulate", [False, True])
def test_experts_sums_longer_than_an_accumulator_takes(accumulate):
    """Tiles enough that the rows are not cut into parts; sums of thousands of rows are added up in pieces, in order."""
    e = Experts([7000, 10, 6300, 0, 1, 200, 0, 12500], 520, 2056, torch.bfloat16, seed=12, accumulate=accumulate)
    assert nat.nat_experts_workspace_bytes(e.params, e.cap) < 1 << 20
    e.check()
    first = e.dw.clone()
    for _ in range(3):
        e.dw.copy_(e.old)
        e.bwd(dx=False)
        assert torch.equal(first, e.dw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_experts_either_gradient_alone(dtype):
    a, b = (Experts([90, 200, 3], 72, 136, DT[dtype], seed=5) for _ in range(2))
    a.bwd()
    x, b.x = b.x, None                                # not read for dx
    b.bwd(dw=False)
    assert torch.equal(a.dx, b.dx) and (b.dw == 7).all()
    b.dx.fill_(7.0)
    b.x, b.w = x, None                                # not read for dw
    b.bwd(dx=False)
    assert torch.equal(a.dw, b.dw) and (b.dx == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_experts_infinities_and_nan_stay_in_their_row_and_expert(dtype):
    loads = [70, 0, 33, 130, 64]
    a, b = (Experts(loads, 72, 136, DT[dtype], seed=6) for _ in range(2))
    row = 80                                          # of expert 2
    b.x[row, 5], b.dy[row, 7] = float("nan"), float("inf")
    b.w[4] = float("nan")
    b.w[1] = float("inf")
    for e in (a, b):
        e.fwd()
        e.bwd()
    keep = torch.ones(a.cap, dtype=torch.bool, device="cuda")
    keep[row] = False
    keep[a.offs_h[4]:a.offs_h[5]] = False
    assert torch.equal(a.y[keep], b.y[keep]) and torch.equal(a.dx[keep], b.dx[keep])
    assert not torch.isfinite(b.y[row]).any() and not torch.isfinite(b.dx[row]).any()
    for e in (0, 1, 3, 4):
        assert torch.equal(a.dw[e], b.dw[e]), e
    assert not torch.isfinite(b.dw[2][:, 5]).any() and not torch.isfinite(b.dw[2][7]).any()


def test_experts_offsets_beyond_the_rows_and_out_of_order():
    for dtype in (torch.float32, torch.bfloat16):
        e = Experts([50, 100, 60], 64, 72, dtype, seed=7, spare=0)
        good = Experts([50, 100, 60], 64, 72, dtype, seed=7, spare=0)
        good.fwd()
        good.bwd()
        e.offs[3] = 5000                              # the rows there are
        e.fwd()
        assert nat.nat_poll_status(e.ws) == nat.NAT_DEV_CAPACITY
        assert torch.equal(e.y, good.y)
        e.bwd()
        assert nat.nat_poll_status(e.ws) == nat.NAT_DEV_CAPACITY
        assert torch.equal(e.dx, good.dx) and torch.equal(e.dw, good.dw)
        for bad in ([0, 150, 50, 210], [-4, 50, 150, 210], [0, 50, 150, -1]):
            e.offs.copy_(torch.tensor(bad))
            for t in (e.y, e.dx, e.dw):
                t.fill_(7.0)
            e.fwd()
            assert nat.nat_poll_status(e.ws) == nat.NAT_DEV_CAPACITY
            e.bwd()
            assert nat.nat_poll_status(e.ws) == nat.NAT_DEV_CAPACITY
            assert all((t == 7).all() for t in (e.y, e.dx, e.dw))
        # offsets in order again: the workspace keeps nothing of that
        e.offs.copy_(good.offs)
        e.fwd()
        assert nat.nat_poll_status(e.ws) == 0 and torch.equal(e.y, good.y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_experts_repeat_bit_for_bit_and_replay_with_other_loads(dtype):
    a = Experts([300, 0, 41, 700], 200, 264, DT[dtype], seed=8)
    b = Experts([0, 1000, 1, 40], 200, 264, DT[dtype], seed=8)
    want = []
    for e in (a, b):
        e.fwd()
        e.bwd()
        want.append([t.clone() for t in (e.y, e.dx, e.dw)])
    a.ws.random_(0, 255)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        a.fwd()
        a.bwd()
    for turn in range(4):
        a.offs.copy_(torch.from_numpy((a, b)[turn % 2].offs_h))
        for t in (a.y, a.dx, a.dw):
            t.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        if turn % 2 == 0:
            assert all(torch.equal(x, y) for x, y in zip(want[0], (a.y, a.dx, a.dw)))
        else:                                         # the same rows dealt otherwise
            ref, mag = op.experts_fwd(_np(a.x[:1041]), _np(a.w), b.offs_h)
            u = 2.0 ** -8 if dtype == "bf16" else 0.0
            _close("y", a.y[:1041], ref, u * np.abs(ref) + 216 * 2.0 ** -23 * mag)
            r = op.experts_bwd(_np(a.x[:1041]), _np(a.w), _np(a.dy[:1041]), b.offs_h)
            _close("dw", a.dw, r["dw"], 1016 * 2.0 ** -23 * r["mag_dw"])


def test_experts_two_calls_at_once():
    a = Experts([500, 80, 1200], 264, 200, torch.bfloat16, seed=9)
    b = Experts([40, 900, 0, 333], 136, 520, torch.bfloat16, seed=10)
    want = []
    for e in (a, b):
        e.fwd()
        e.bwd()
        want += [t.clone() for t in (e.y, e.dx, e.dw)]
        for t in (e.y, e.dx, e.dw):
            t.fill_(7.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, e in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            e.fwd()
            e.bwd()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, (a.y, a.dx, a.dw, b.y, b.dx, b.dw)))


def test_experts_many_experts():
    loads = np.random.default_rng(0).integers(0, 5, 1024)
    Experts(loads, 24, 16, torch.bfloat16, seed=11).check()
    Experts(loads, 24, 16, torch.float32, seed=11).check()


def test_experts_past_32_bits():
    """Rows whose elements lie more than 2^31 behind the first: the last expert's against a short call."""
    n, n_in, n_out, E = 600100, 4096, 64, 3
    x = torch.empty(n, n_in, dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 1 << 31
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    w = torch.randn(E, n_out, n_in, device="cuda").to(torch.bfloat16)
    p = nat.experts_params(E, n_in, n_out, torch.bfloat16)
    offs = torch.tensor([0, 1000, n - 100, n], dtype=torch.int32, device="cuda")
    y, dw = torch.empty(n, n_out, dtype=torch.bfloat16, device="cuda"), torch.empty(E, n_out, n_in, device="cuda")
    ws = nat.alloc_workspace(nat.nat_experts_workspace_bytes(p, n), "cuda")
    nat.nat_experts_fwd(p, offs, n, x, w, y, ws)
    short = torch.tensor([0, 0, 0, 100], dtype=torch.int32, device="cuda")
    y1, dw1 = torch.empty(100, n_out, dtype=torch.bfloat16, device="cuda"), torch.empty_like(dw)
    nat.nat_experts_fwd(p, short, 100, x[-100:], w, y1, ws)
    assert torch.equal(y[-100:], y1)
    dx, dx1 = torch.empty_like(x), torch.empty(100, n_in, dtype=torch.bfloat16, device="cuda")
    nat.nat_experts_bwd(p, offs, n, x, w, y, dx, dw, ws)
    assert nat.nat_poll_status(ws) == 0
    nat.nat_experts_bwd(p, short, 100, x[-100:], w, y1, dx1, dw1, ws)
    assert torch.equal(dx[-100:], dx1)
    ref = y1.double().t() @ x[-100:].double()
    mag = y1.double().abs().t() @ x[-100:].double().abs()
    assert ((dw[2].double() - ref).abs() <= 116 * 2.0 ** -23 * mag).all()


@pytest.mark.parametrize("seed", range(30))
def test_random_experts(seed):
    r = random.Random(seed)
    E = r.choice([1, 2, 3, 7, 20])
    n_in, n_out = (8 * r.choice([r.randint(1, 20), r.randint(20, 80)]) for _ in range(2))
    loads = [r.choice([0, 1, r.randint(2, 60), r.randint(60, 700), 256, 512]) for _ in range(E)]
    Experts(loads, n_in, n_out, r.choice([torch.float32, torch.bfloat16, torch.bfloat16]), seed=seed, first=r.choice([0, 0, 9]),
            spare=r.choice([0, 1, 200]), strides=(8 * r.randint(0, 3), 8 * r.randint(0, 3)),
            accumulate=r.random() < 0.4).check()
