"""GPU parity of the heads' norms with the rotation against the float64 forms in ``oracle/nat_packed.py``.

Tolerances, by arithmetic, with u = half a step of the type where it is narrower than 32 bits and D the head's size:
  rstd      the mean of D squares, D + 2 roundings of 2^-24 halved by the root, and rsqrtf's two steps of 2^-23
  sin, cos  the reduced angle rounded in 32 bits, pi 2^-25, and two steps of 2^-23 of sincospif: 2^-21 of the circle
  forward   e = (D + 8) 2^-24 + 2^-20 of |n_a| + |n_b|, and u |out|
  dx        the same of each of its parts, rstd in them twice: (2 D + 32) 2^-24 + 2^-19, and u |dx|
  dw        N terms added in 32 bits: (N + 64) 2^-24 more
"""
import numpy as np
import pytest
import torch

from oracle import nat_packed as op
from paper_2603_06619_b200 import nat

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _np(t):
    return t.detach().double().cpu().numpy()


class Heads:
    """A packed batch with NaN rows behind the last sequence and poisoned outputs."""

    def __init__(self, lengths, Hq, Hkv, D, dtype, R=None, interleaved=False, norm=True, first=None, seed=0, spare=5,
                 theta=1e4, eps=1e-6, count=False):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        R = D if R is None else R
        self.Hq, self.Hkv, self.D, self.R, self.dtype, self.inter, self.eps = Hq, Hkv, D, R, dtype, interleaved, eps
        self.cu_h = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        self.B, self.n = len(lengths), int(self.cu_h[-1])
        self.cap = self.n + spare
        self.cu = torch.from_numpy(self.cu_h).cuda()
        self.pos = np.arange(self.n) - np.repeat(self.cu_h[:-1], lengths)
        self.positions = None
        if first is not None:
            self.pos = self.pos + first
            self.positions = torch.full((max(self.cap, 1),), 99, dtype=torch.int32, device="cuda")
            self.positions[:self.n] = torch.from_numpy(self.pos).cuda().to(torch.int32)
        self.n_rows = torch.tensor([self.n], dtype=torch.int32, device="cuda") if count or first is not None else None
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        rows = max(self.cap, 1)
        qkv = rand(rows, Hq + 2 * Hkv, D) * torch.exp(rand(rows, Hq + 2 * Hkv, 1))
        qkv[self.n:] = float("nan")
        self.qkv = qkv.to(dtype)
        self.q, self.k, self.v = self.qkv.split([Hq, Hkv, Hkv], dim=1)
        self.out = torch.full((rows, Hq + Hkv, D), 7.0, dtype=dtype, device="cuda")
        self.q_out, self.k_out = self.out.split([Hq, Hkv], dim=1)
        self.dout = rand(rows, Hq + Hkv, D).to(dtype)
        self.dout[self.n:] = float("nan")
        self.dq_out, self.dk_out = self.dout.split([Hq, Hkv], dim=1)
        self.dqkv = torch.full_like(self.qkv, 7.0)
        self.dq, self.dk, self.dv = self.dqkv.split([Hq, Hkv, Hkv], dim=1)
        self.w_q, self.w_k = (1 + 0.3 * rand(D), 1 + 0.3 * rand(D)) if norm else (None, None)
        self.dw_q, self.dw_k = (torch.full((D,), 7.0, device="cuda") for _ in range(2)) if norm else (None, None)
        self.freq = nat.rope_freqs(R, theta) if R else None
        self.params = nat.qknorm_params(Hq, Hkv, D, dtype, rot_dim=R, interleaved=interleaved, eps=eps)
        self.ws = None
        if norm:
            self.ws = nat.alloc_workspace(nat.nat_qknorm_workspace_bytes(self.params, self.cap), "cuda")
            self.ws.random_(0, 255)

    def where(self):
        return self.B, (None if self.positions is not None else self.cu), self.positions, self.n_rows, self.cap

    def fwd(self):
        nat.nat_qknorm_fwd(self.params, *self.where(), self.q, self.k, self.w_q, self.w_k, self.freq, self.q_out, self.k_out)

    def bwd(self):
        q, k = (self.q, self.k) if self.w_q is not None else (None, None)
        nat.nat_qknorm_bwd(self.params, *self.where(), q, k, self.w_q, self.w_k, self.freq, self.dq_out, self.dk_out,
                           self.dq, self.dk, self.dw_q, self.dw_k, self.ws)

    def check(self):
        n, D = self.n, self.D
        u = 2.0 ** -8 if self.dtype == torch.bfloat16 else 0.0
        freq = np.zeros(0) if self.freq is None else _np(self.freq)
        self.fwd()
        self.bwd()
        for name in ("q", "k"):
            x, w, dout = _np(getattr(self, name)[:n]), getattr(self, "w_" + name), _np(getattr(self, "d%s_out" % name)[:n])
            w = None if w is None else _np(w)
            ref, mag = op.qknorm_fwd(x, w, self.pos, freq, self.eps, self.inter)
            _close(name, getattr(self, name + "_out")[:n], ref, u * np.abs(ref) + ((D + 8) * 2.0 ** -24 + 2.0 ** -20) * mag)
            b = op.qknorm_bwd(x, w, self.pos, freq, self.eps, self.inter, dout)
            e = (2 * D + 32) * 2.0 ** -24 + 2.0 ** -19
            _close("d" + name, getattr(self, "d" + name)[:n], b["dx"], u * np.abs(b["dx"]) + 1.01 * e * b["mag_dx"])
            if w is not None:
                terms = n * x.shape[1]
                _close("dw_" + name, getattr(self, "dw_" + name), b["dw"],
                       (e + (terms + 64) * 2.0 ** -24) * b["mag_dw"])
        for t in (self.out, self.dqkv):
            assert (t[n:] == 7).all()
        assert (self.dv == 7).all()


def _close(name, got, ref, tol):
    got = _np(got)
    assert got.shape == ref.shape
    assert np.isfinite(got).all(), name
    over = np.abs(got - ref) - 1.001 * tol - 1e-37
    assert (over <= 0).all(), (name, float(over.max()), float(np.abs(got - ref).max()), np.argwhere(over > 0)[:4].tolist())


LENGTHS = {"one": [1], "empty": [0, 3, 0, 0, 29, 1, 0], "many": [3, 1, 17, 40, 9, 0, 31] * 8, "long": [2500, 1, 900]}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (32, 8, 128), (1, 1, 8), (3, 1, 96), (5, 5, 80), (2, 1, 16), (7, 1, 32),
                                   (6, 2, 112)])
@pytest.mark.parametrize("lengths", list(LENGTHS))
def test_qknorm_parity(lengths, heads, dtype):
    R = heads[2] // 16 * 16
    Heads(LENGTHS[lengths], *heads, DT[dtype], R=R, seed=len(lengths), count=lengths == "many").check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", [(128, 128), (128, 64), (128, 16), (128, 0), (72, 64), (120, 32), (64, 48), (8, 0),
                                 (24, 16), (104, 96), (40, 0)])
def test_qknorm_parts_that_turn(D, R, interleaved, norm, dtype):
    Heads([5, 0, 70], 5, 2, D, DT[dtype], R=R, interleaved=interleaved, norm=norm, seed=D + R).check()


@pytest.mark.parametrize("first", [0, 3, 100000, 2 ** 31 - 200, -1000])
@pytest.mark.parametrize("interleaved", [False, True])
def test_qknorm_positions_of_their_own(interleaved, first):
    """Far positions too: the angle of 2^31 steps is reduced in 64 bits."""
    Heads([90, 20, 51], 4, 2, 64, torch.float32, interleaved=interleaved, first=first, seed=1).check()


def test_qknorm_rows_of_zeros_and_of_one_loud_element():
    h = Heads([40], 4, 2, 64, torch.float32, seed=2)
    h.q[3] = 0
    h.k[5] = 0
    h.k[6, 0, 7] = 1e12
    h.q[7] *= 1e-12
    h.check()


def test_qknorm_a_row_leaves_the_others_alone():
    a, b = (Heads([100, 33], 4, 2, 128, torch.bfloat16, seed=3) for _ in range(2))
    b.q[17, 1], b.k[40, 0], b.dk_out[41, 1] = float("nan"), float("inf"), float("nan")
    for h in (a, b):
        h.fwd()
        h.bwd()
    for t, where in (("q_out", (17, 1)), ("k_out", (40, 0)), ("dq", (17, 1))):
        x, y = getattr(a, t)[:133].clone(), getattr(b, t)[:133].clone()
        assert not torch.isfinite(y[where]).any()
        x[where], y[where] = 0, 0
        assert torch.equal(x, y), t
    x, y = a.dk[:133].clone(), b.dk[:133].clone()
    for where in ((40, 0), (41, 1)):
        x[where], y[where] = 0, 0
    assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("R", [64, 32])
def test_qknorm_in_place(R, norm, dtype):
    """Outputs on the inputs that they may lie on: the same bits as apart from them."""
    def make():
        return Heads([60, 201], 4, 2, 64, DT[dtype], R=R, norm=norm, seed=4)

    a = make()
    a.fwd()
    a.bwd()
    b = make()
    b.q_out, b.k_out = b.q, b.k                       # forward on its inputs
    b.fwd()
    assert torch.equal(a.q_out[:261], b.q[:261]) and torch.equal(a.k_out[:261], b.k[:261])
    assert torch.equal(a.v[:261], b.v[:261])
    c = make()
    c.dqkv.copy_(torch.cat([c.dout, c.v], dim=1))     # backward on its gradients, which have the inputs' strides
    c.dq_out, c.dk_out = c.dq, c.dk
    c.bwd()
    assert torch.equal(a.dq[:261], c.dq[:261]) and torch.equal(a.dk[:261], c.dk[:261])
    if norm:
        assert torch.equal(a.dw_q, c.dw_q) and torch.equal(a.dw_k, c.dw_k)
        d = make()                                    # and on q and k themselves
        d.dq, d.dk = d.q, d.k
        d.bwd()
        assert torch.equal(a.dq[:261], d.q[:261]) and torch.equal(a.dk[:261], d.k[:261])


def test_qknorm_repeats_bit_for_bit_and_replays_with_other_lengths():
    h = Heads([700, 90, 1210], 8, 2, 128, torch.bfloat16, seed=5, spare=50)
    h.fwd()
    h.bwd()
    outs = lambda: [t.clone() for t in (h.out, h.dqkv, h.dw_q, h.dw_k)]  # noqa: E731
    first = outs()
    h.ws.random_(0, 255)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        h.fwd()
        h.bwd()
    for t in (h.out, h.dqkv, h.dw_q):
        t.fill_(7.0)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, outs()))
    # other sequences at replay
    other = Heads([11, 1000, 2], 8, 2, 128, torch.bfloat16, seed=5, spare=50 + 2000 - 1013)
    other.cap = h.cap
    other.fwd()
    other.bwd()
    h.cu.copy_(other.cu)
    for name in ("qkv", "dout"):
        getattr(h, name).copy_(getattr(other, name)[:h.cap])
    for t in (h.out, h.dqkv):
        t.fill_(7.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(h.out, other.out[:h.cap]) and torch.equal(h.dqkv, other.dqkv[:h.cap])
    assert torch.equal(h.dw_q, other.dw_q) and torch.equal(h.dw_k, other.dw_k)


def test_qknorm_without_rows():
    h = Heads([0, 0], 4, 2, 64, torch.bfloat16, seed=6, spare=4)
    h.check()
    assert (h.dw_q == 0).all() and (h.dw_k == 0).all()
    p = h.params
    nat.nat_qknorm_bwd(p, 0, None, None, None, 0, h.q, h.k, h.w_q, h.w_k, h.freq, h.dq_out, h.dk_out, h.dq, h.dk, h.dw_q,
                       h.dw_k, h.ws)
    assert (h.dw_q == 0).all() and (h.dq == 7).all()


def test_qknorm_rows_in_front_of_the_first_sequence():
    h = Heads([30, 50], 4, 2, 64, torch.float32, seed=7)
    whole = Heads([30, 50], 4, 2, 64, torch.float32, seed=7)
    whole.fwd()
    h.cu.copy_(torch.tensor([30, 30, 80]))
    h.fwd()
    h.bwd()
    assert (h.out[:30] == 7).all() and (h.dqkv[:30] == 7).all() and (h.out[80:] == 7).all()
    assert torch.equal(h.out[30:80], whole.out[30:80])


def test_qknorm_fewer_rows_than_the_sequences_hold():
    h = Heads([30, 50], 4, 2, 64, torch.float32, seed=7, count=True)
    h.n_rows.fill_(41)
    h.fwd()
    h.bwd()
    assert (h.out[41:] == 7).all() and (h.dqkv[41:] == 7).all()
    short = Heads([30, 50], 4, 2, 64, torch.float32, seed=7, count=True)
    short.fwd()
    assert torch.equal(h.out[:41], short.out[:41])


def test_qknorm_past_32_bits():
    """Rows whose elements lie more than 2^31 behind the first: the last ones against a short call."""
    Hq, Hkv, D, n = 32, 8, 128, 370000
    qkv = torch.empty(n, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    assert qkv.numel() > 1 << 31
    qkv.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    w, f = torch.ones(D, device="cuda"), nat.rope_freqs(D)
    p = nat.qknorm_params(Hq, Hkv, D, torch.bfloat16)
    cu = torch.tensor([0, n - 70, n], dtype=torch.int32, device="cuda")
    q, k, _ = qkv.split([Hq, Hkv, Hkv], dim=1)
    tail = qkv[-70:].clone()
    tq, tk, _ = tail.split([Hq, Hkv, Hkv], dim=1)
    nat.nat_qknorm_fwd(p, 2, cu, None, None, n, q, k, w, w, f, q, k)
    nat.nat_qknorm_fwd(p, 1, torch.tensor([0, 70], dtype=torch.int32, device="cuda"), None, None, 70, tq, tk, w, w, f, tq, tk)
    assert torch.equal(qkv[-70:], tail)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_qknorm_rows_of_16_byte_alignment(dtype):
    """Rows that begin 16 bytes past a 32-byte boundary: the same bits as on one."""
    a, b = (Heads([50, 9], 4, 2, 64, DT[dtype], seed=8) for _ in range(2))
    off = 16 // b.qkv.element_size()
    for name in ("qkv", "out", "dout", "dqkv"):
        t = getattr(b, name)
        buf = torch.empty(t.numel() + off, dtype=t.dtype, device="cuda")
        setattr(b, name, buf[off:].view(t.shape).copy_(t))
    b.q, b.k, b.v = b.qkv.split([4, 2, 2], dim=1)
    b.q_out, b.k_out = b.out.split([4, 2], dim=1)
    b.dq_out, b.dk_out = b.dout.split([4, 2], dim=1)
    b.dq, b.dk, b.dv = b.dqkv.split([4, 2, 2], dim=1)
    for h in (a, b):
        h.fwd()
        h.bwd()
    for name in ("out", "dqkv", "dw_q", "dw_k"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


def test_qknorm_gradient_against_differences():
    """The kernel's gradient against differences of the float64 forward along random directions."""
    h = Heads([40, 23], 4, 2, 64, torch.float32, seed=9, spare=0)
    h.fwd()
    h.bwd()
    r = np.random.default_rng(0)
    freq = _np(h.freq)
    for name in ("q", "k"):
        x, w, G = _np(getattr(h, name)), _np(getattr(h, "w_" + name)), _np(getattr(h, "d%s_out" % name))
        f = lambda x, w: (G * op.qknorm_fwd(x, w, h.pos, freq, h.eps, False)[0]).sum()  # noqa: E731
        for got, at in ((_np(getattr(h, "d" + name)), 0), (_np(getattr(h, "dw_" + name)), 1)):
            step = r.normal(size=got.shape)
            lo, hi = [x, w], [x, w]
            lo[at], hi[at] = lo[at] - 1e-6 * step, hi[at] + 1e-6 * step
            want = (f(*hi) - f(*lo)) / 2e-6
            # 32-bit arithmetic moves no element by more than 2^-15 of the norms; the differences' own error is below
            assert abs((got * step).sum() - want) <= 2.0 ** -15 * np.linalg.norm(got) * np.linalg.norm(step), name
