"""GPU parity of the transformer body's operators against the float64 forms in ``oracle/nat_body.py``.

Tolerances, by arithmetic.  Every product and sum of the kernels is in 32 bits; what is rounded to
bfloat16 is off by at most half a step, u = finfo.eps / 2 relative to the value (2^-8).
  attention out     u |out| for the stored value and u sum_j P_ij |v_j| for P before the second
                    product (0 and 0 in float32);
  dq, dk, dv        u |value| and u times the sum of the magnitudes of the terms (dS or P rounded);
                    dP - delta cancels, so dS also carries the rounding of its parts, which
                    the oracle's magnitudes hold at 2^-12 of them (see abs_dq there);
  32-bit parts      a score is a sum of D products: its error e_S <= (D + 4) 2^-23 max|scale q||k|
                    moves P by the factor 1 + e_S, a sum over T keys adds (T + 16) 2^-23;
                    the softmax's exponential adds 2^-21 (two ulps of the function, one of its
                    argument for arguments up to 2^2 of a unit, the rest is in e_S).
  resnorm           u |value| plus (d + 32) 2^-24 of the magnitudes that are added.
  ckpt8             bit for bit.
"""
import ctypes

import numpy as np
import pytest
import torch

from oracle import nat_body as ob
from paper_2603_06619_b200 import nat

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _np(t):
    return t.detach().double().cpu().numpy()


def _half(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------------- attention
class Attn:
    """A packed batch with NaN rows behind the last sequence and poisoned outputs."""

    def __init__(self, lengths, Hq, Hkv, D, dtype, seed=0, spare=5, fused=True, sharp=2.0, scale=None):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.cu_h = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        self.B, self.n, self.Hq, self.Hkv, self.D = len(lengths), int(self.cu_h[-1]), Hq, Hkv, D
        self.cap, self.dtype = self.n + spare, dtype
        self.cu = torch.from_numpy(self.cu_h).cuda()
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        qkv = rand(self.cap, Hq + 2 * Hkv, D)
        qkv[:, :Hq] *= sharp
        qkv[self.n:] = float("nan")
        qkv = qkv.to(dtype)
        if fused:
            self.q, self.k, self.v = qkv.split([Hq, Hkv, Hkv], dim=1)
        else:
            self.q, self.k, self.v = (t.contiguous() for t in qkv.split([Hq, Hkv, Hkv], dim=1))
        self.dout = rand(self.cap, Hq, D).to(dtype)
        self.dout[self.n:] = float("nan")
        self.out = torch.full((self.cap, Hq, D), 7.0, dtype=dtype, device="cuda")
        self.lse = torch.full((self.cap, Hq), 7.0, device="cuda")
        self.dq, self.dk, self.dv = (torch.full_like(t, 7.0) if not fused else None for t in (self.q, self.k, self.v))
        if fused:
            d = torch.full_like(qkv, 7.0)
            self.dq, self.dk, self.dv = d.split([Hq, Hkv, Hkv], dim=1)
        self.params = nat.attn_params(Hq, Hkv, D, dtype, scale=scale)
        self.ws = nat.alloc_workspace(nat.nat_attn_workspace_bytes(self.params, self.B, self.cap), "cuda")

    def fwd(self):
        nat.nat_attn_fwd(self.params, self.B, self.cu, self.cap, self.q, self.k, self.v, self.out,
                         self.lse, self.ws)

    def bwd(self):
        nat.nat_attn_bwd(self.params, self.B, self.cu, self.cap, self.q, self.k, self.v, self.out,
                         self.lse, self.dout, self.dq, self.dk, self.dv, self.ws)

    def factors(self):
        """(u, e): the rounding to the type, and the relative error of P in 32 bits."""
        n = max(self.n, 1)
        qk = abs(self.params.scale) * float(self.q[:n].float().norm(dim=2).max()) * float(self.k[:n].float().norm(dim=2).max())
        longest = int(np.diff(self.cu_h).max(initial=0))
        e = ((self.D + 4) * qk + longest + 16) * 2.0 ** -23 + 2.0 ** -21
        return (_half(self.dtype) if self.dtype == torch.bfloat16 else 2.0 ** -24), e

    def check(self, back=True):
        u, e = self.factors()
        n, up = self.n, (u if self.dtype == torch.bfloat16 else 0.0)
        q, k, v = (_np(t[:n]) for t in (self.q, self.k, self.v))
        self.fwd()
        assert nat.nat_poll_status(self.ws) == 0
        out, lse, mag = ob.attn_fwd(q, k, v, self.cu_h, self.params.scale)
        _close("out", self.out[:n], out, u * np.abs(out) + (up + 2 * e) * 1.01 * mag)
        _close("lse", self.lse[:n], lse, 2 * e + 2.0 ** -22 * np.abs(lse))
        assert (self.out[n:] == 7).all() and (self.lse[n:] == 7).all()
        if not back:
            return
        self.bwd()
        assert nat.nat_poll_status(self.ws) == 0
        # the gradient's definition takes the stored out and lse
        ref = ob.attn_bwd(q, k, v, _np(self.out[:n]), _np(self.lse[:n]), _np(self.dout[:n]), self.cu_h,
                          self.params.scale)
        e2 = e + 2.0 ** -22 * float(np.abs(lse).max(initial=0))
        for name in ("dq", "dk", "dv"):
            # abs_* weighs the parts of dP - delta by 2^-12, so 2 e2 of them is 2^13 e2 of it
            tol = u * np.abs(ref[name]) + (up + 2 * e2) * 1.01 * ref["abs_" + name]
            if name != "dv":
                tol = tol + 2.0 ** 12 * 2 * (self.D + 16) * 2.0 ** -24 * ref["abs_" + name]
            _close(name, getattr(self, name)[:n], ref[name], tol)
            assert (getattr(self, name)[n:] == 7).all()


def _close(name, got, ref, tol):
    got = _np(got)
    assert got.shape == ref.shape
    assert np.isfinite(got).all(), name
    over = np.abs(got - ref) - (tol + 1e-30)
    assert (over <= 0).all(), (name, float(over.max()), float(np.abs(got - ref).max()), np.argwhere(over > 0)[:4].tolist())


LENGTHS = {
    "one": [1], "two": [2], "ragged": [0, 5, 0, 1, 33, 128, 129, 0], "tiles": [127, 128, 257, 64],
    "long": [700], "many": [3, 1, 17, 40, 9, 64, 31, 32] * 5,
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (2, 2, 128), (8, 1, 64), (3, 1, 96), (5, 1, 80), (14, 2, 32),
                                   (1, 1, 8), (12, 2, 128), (8, 2, 128), (20, 1, 64)])
@pytest.mark.parametrize("lengths", list(LENGTHS))
def test_attn_parity(lengths, heads, dtype):
    Attn(LENGTHS[lengths], *heads, DT[dtype], seed=len(lengths)).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attn_contiguous_tensors_and_sharp_rows(dtype):
    # separate tensors; scores of tens of units, so that rows attend to few keys and the running
    # maximum moves late in a row
    Attn([300, 77], 4, 2, 64, DT[dtype], seed=3, fused=False, sharp=24.0).check()
    Attn([200], 2, 1, 128, DT[dtype], seed=4, scale=-0.2).check()
    Attn([200], 2, 1, 128, DT[dtype], seed=4, scale=0.0).check()


def test_attn_growing_scores():
    """Keys that grow along the sequence: every tile raises the running maximum by far."""
    a = Attn([900], 4, 2, 64, torch.bfloat16, seed=5)
    ramp = torch.linspace(0.05, 6.0, a.cap, device="cuda")[:, None, None]
    a.k.copy_((a.k[:1].float().abs() * ramp).to(torch.bfloat16))
    a.q.copy_(a.q.abs())
    a.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attn_other_sequences_do_not_leak(dtype):
    """Infinities and NaN in one sequence stay in it."""
    lengths = [70, 50, 200, 3]
    a, b = (Attn(lengths, 4, 2, 64, DT[dtype], seed=6) for _ in range(2))
    lo, hi = 120, 320
    for t in (b.q, b.k, b.v, b.dout):
        t[lo:hi:2] = float("nan")
        t[lo + 1:hi:2] = float("inf")
    for s in (a, b):
        s.fwd()
        s.bwd()
    keep = torch.ones(a.n, dtype=torch.bool, device="cuda")
    keep[lo:hi] = False
    for name in ("out", "lse", "dq", "dk", "dv"):
        x, y = getattr(a, name)[:a.n][keep], getattr(b, name)[:a.n][keep]
        assert torch.equal(x, y), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attn_repeats_bit_for_bit_and_shares_nothing(dtype):
    a = Attn([513, 40, 260], 8, 2, 128, DT[dtype], seed=7)
    b = Attn([90, 333], 8, 2, 128, DT[dtype], seed=8)
    first = None
    for turn in range(3):
        a.fwd()
        a.bwd()
        got = [t[:a.n].clone() for t in (a.out, a.lse, a.dq, a.dk, a.dv)]
        first = first or got
        assert all(torch.equal(x, y) for x, y in zip(first, got))
        b.fwd()                          # another batch in between, in the same workspace size class
        b.bwd()
        a.ws.random_(0, 255)             # the workspace carries nothing over
    # two calls at once, on streams of their own
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, x in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            x.fwd()
            x.bwd()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y[:a.n]) for x, y in zip(first, (a.out, a.lse, a.dq, a.dk, a.dv)))


def test_attn_captured_and_replayed_with_other_lengths():
    """A captured call reads cu_seqlens from the device at replay."""
    a = Attn([100, 30, 170], 4, 2, 64, torch.bfloat16, seed=9, spare=40)
    a.fwd()
    a.bwd()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.fwd()
        a.bwd()
    for cu in ([0, 5, 290, 300], [0, 0, 0, 1], [0, 300, 300, 300]):
        a.cu.copy_(torch.tensor(cu, dtype=torch.int32))
        for t in (a.out, a.lse, a.dq, a.dk, a.dv):
            t.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (a.out, a.lse, a.dq, a.dk, a.dv)]
        for t in (a.out, a.lse, a.dq, a.dk, a.dv):
            t.fill_(7.0)
        a.fwd()
        a.bwd()
        assert all(torch.equal(x, y) for x, y in zip(got, (a.out, a.lse, a.dq, a.dk, a.dv)))
        assert (got[0][cu[-1]:] == 7).all() and (got[0][:cu[-1]] != 7).any()
        assert torch.isfinite(got[0]).all() and torch.isfinite(got[2]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attn_rows_beyond_the_capacity(dtype):
    a = Attn([60, 90], 4, 2, 64, DT[dtype], seed=10, spare=0)
    b = Attn([60, 90], 4, 2, 64, DT[dtype], seed=10, spare=0)
    b.cu = torch.tensor([0, 60, 4000], dtype=torch.int32, device="cuda")
    a.fwd()
    a.bwd()
    b.fwd()
    assert nat.nat_poll_status(b.ws) == nat.NAT_DEV_CAPACITY
    b.bwd()
    assert nat.nat_poll_status(b.ws) == nat.NAT_DEV_CAPACITY
    for name in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


@pytest.mark.parametrize("cap", [150, 3000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attn_bounds_that_do_not_ascend(dtype, cap):
    a = Attn([60, 90], 4, 2, 64, DT[dtype], seed=10, spare=cap - 150)
    a.fwd()
    for cu in ([0, 90, 60], [-5, 20, 40], [5, 2 ** 31 - 1, 40]):
        a.cu.copy_(torch.tensor(cu, dtype=torch.int32))
        for t in (a.out, a.dq, a.dk, a.dv):
            t.fill_(7.0)
        a.fwd()
        assert nat.nat_poll_status(a.ws) == nat.NAT_DEV_CAPACITY
        a.bwd()
        assert nat.nat_poll_status(a.ws) == nat.NAT_DEV_CAPACITY
        for t in (a.out, a.dq, a.dk, a.dv):
            assert (t == 7).all()


@pytest.mark.parametrize("heads", [(4, 1, 128), (2, 2, 64), (7, 1, 96), (1, 1, 128)])
@pytest.mark.parametrize("lengths", [[2100], [1500, 3, 700], [0, 1029, 0, 1]])
def test_attn_long_rows_of_few_heads(lengths, heads):
    """Few tiles with many steps: cut into pieces, whose partial results are joined."""
    a = Attn(lengths, *heads, torch.bfloat16, seed=12)
    a.check()
    got = [t[:a.n].clone() for t in (a.out, a.lse, a.dq, a.dk, a.dv)]
    a.ws.random_(0, 255)
    for _ in range(3):
        a.fwd()
        a.bwd()
        assert all(torch.equal(x, y[:a.n]) for x, y in zip(got, (a.out, a.lse, a.dq, a.dk, a.dv)))


def test_attn_long_rows_with_growing_scores():
    a = Attn([1900], 4, 2, 64, torch.bfloat16, seed=13)
    ramp = torch.linspace(0.05, 6.0, a.cap, device="cuda")[:, None, None]
    a.k.copy_((a.k[:1].float().abs() * ramp).to(torch.bfloat16))
    a.q.copy_(a.q.abs())
    a.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attn_offsets_past_32_bits(dtype):
    """Token strides so wide that the last rows lie more than 2^31 elements behind the first."""
    n, wide = 1100, 1 << 21
    a = Attn([500, 600], 2, 1, 64, DT[dtype], seed=11, spare=0)
    buf = torch.empty(n * wide, dtype=DT[dtype], device="cuda")
    far = buf.view(n, wide)
    assert n * wide > 1 << 31
    b = Attn([500, 600], 2, 1, 64, DT[dtype], seed=11, spare=0)
    at = 0
    for name, heads in (("q", 2), ("k", 1), ("v", 1), ("dq", 2), ("dk", 1), ("dv", 1), ("out", 2), ("dout", 2)):
        view = far[:, at:at + heads * 64].unflatten(1, (heads, 64))
        at += heads * 64
        view.copy_(getattr(a, name))
        setattr(b, name, view)
    for s in (a, b):
        s.fwd()
        s.bwd()
    for name in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


def test_attn_binding_refuses_wrong_layouts():
    a = Attn([8], 4, 2, 64, torch.bfloat16)
    with pytest.raises(nat.NatError, match="not contiguous"):
        nat.nat_attn_fwd(a.params, 1, a.cu, a.cap, a.q.transpose(1, 2).contiguous().transpose(1, 2), a.k, a.v,
                         a.out, a.lse, a.ws)
    with pytest.raises(nat.NatError, match="counterpart"):
        nat.nat_attn_bwd(a.params, 1, a.cu, a.cap, a.q, a.k, a.v, a.out, a.lse, a.dout,
                         a.dq.contiguous(), a.dk, a.dv, a.ws)
    with pytest.raises(nat.NatError, match="shape"):
        nat.nat_attn_fwd(a.params, 1, a.cu, a.cap + 1, a.q, a.k, a.v, a.out, a.lse, a.ws)
    with pytest.raises(nat.NatError, match="workspace too small"):
        nat.nat_attn_fwd(a.params, 1, a.cu, a.cap, a.q, a.k, a.v, a.out, a.lse, a.ws[:256])


# --------------------------------------------------------------------- residual join
class Join:
    def __init__(self, n, d, dtype, gate="none", parts="all", ckpt=False, seed=0, spare=3, eps=1e-6, alpha=0.8):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.n, self.d, self.cap, self.dtype, self.gate_mode, self.ckpt = n, d, n + spare, dtype, gate, ckpt
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        row = lambda s=1.0: (rand(self.cap, d) * s).to(dtype)  # noqa: E731
        hole = lambda: torch.full((self.cap, d), 7.0, dtype=dtype, device="cuda")  # noqa: E731
        vec = lambda m: torch.full((m,), 7.0, device="cuda")  # noqa: E731
        self.x, self.y = row(), None if parts == "no_y" else row(3.0)
        self.w_post = None if parts in ("no_post", "no_y", "only_add") else 1 + 0.3 * rand(d)
        self.w_pre = None if parts in ("no_pre", "only_add") else 1 + 0.3 * rand(d)
        self.gate = None if gate == "none" else rand(d if gate == "channel" else self.cap)
        self.dr = None if parts == "no_dr" else row()
        self.dh = None if self.w_pre is None else row()
        for t in (self.x, self.y, self.dr, self.dh):
            if t is not None:
                t[n:] = float("nan")
        self.r, self.dx = hole(), hole()
        self.h = None if self.w_pre is None else hole()
        self.dy = None if self.y is None else hole()
        self.rstd_y, self.rstd_r = vec(self.cap), vec(self.cap)
        self.dw_post = None if self.w_post is None else vec(d)
        self.dw_pre = None if self.w_pre is None else vec(d)
        self.dgate = None if self.gate is None else torch.full_like(self.gate, 7.0)
        pair = lambda: (torch.full((self.cap, d), 7, dtype=torch.int8, device="cuda"),  # noqa: E731
                        torch.full((self.cap, -(-d // 128)), 7.0, device="cuda"))
        self.y8 = pair() if ckpt and self.y is not None else None
        self.r8 = pair() if ckpt else None
        self.n_rows = torch.tensor([n], dtype=torch.int32, device="cuda")
        self.eps, self.alpha = eps, alpha
        self.params = nat.resnorm_params(d, dtype, eps=eps, alpha=alpha, gate=gate)
        self.ws = nat.alloc_workspace(nat.nat_resnorm_workspace_bytes(self.params, self.cap), "cuda")

    def fwd(self):
        nat.nat_resnorm_fwd(self.params, self.x, self.y, self.w_post, self.gate, self.w_pre, self.n_rows,
                            self.cap, self.r, self.h, self.rstd_y, self.rstd_r, y8=self.y8, r8=self.r8)

    def bwd(self):
        y, r = (None, None) if self.ckpt else (self.y, self.r)
        nat.nat_resnorm_bwd(self.params, y, r, self.w_post, self.gate, self.w_pre, self.rstd_y, self.rstd_r,
                            self.n_rows, self.cap, self.dr, self.dh, self.dx, self.dy, self.dw_post,
                            self.dgate, self.dw_pre, self.ws, y8=self.y8, r8=self.r8)

    def check(self):
        n, u, w = self.n, _half(self.dtype), (self.d + 32) * 2.0 ** -24
        cut = lambda t: None if t is None else _np(t[:n])  # noqa: E731
        full = lambda t: None if t is None else _np(t)  # noqa: E731
        gate = cut(self.gate) if self.gate_mode == "row" else full(self.gate)
        self.fwd()
        ref = ob.resnorm_fwd(cut(self.x), cut(self.y), full(self.w_post), gate, full(self.w_pre), self.eps,
                             self.alpha, self.gate_mode)
        mag = np.abs(self.alpha * cut(self.x)) + np.abs(ref["r"] - self.alpha * cut(self.x))
        _close("r", self.r[:n], ref["r"], u * np.abs(ref["r"]) + w * mag)
        for name in ("rstd_y", "rstd_r"):
            if name in ref:
                _close(name, getattr(self, name)[:n], ref[name], 2 * w * ref[name])
                assert (getattr(self, name)[n:] == 7).all()
        if "h" in ref:
            unit = np.abs(ref["rstd_r"][:, None] * full(self.w_pre))
            _close("h", self.h[:n], ref["h"], u * np.abs(ref["h"]) + w * (3 * np.abs(ref["h"]) + mag * unit))
            assert (self.h[n:] == 7).all()
        assert (self.r[n:] == 7).all()
        y, r = cut(self.y), cut(self.r)
        if self.ckpt:
            for of, pair in ((self.y, self.y8), (self.r, self.r8)):
                if of is None:
                    continue
                codes, scales = ob.ckpt8_store(of[:n].float().cpu().numpy())
                assert np.array_equal(pair[0][:n].cpu().numpy(), codes)
                assert np.array_equal(pair[1][:n].cpu().numpy(), scales)
                assert (pair[0][n:] == 7).all() and (pair[1][n:] == 7).all()
            y = None if self.y is None else ob.ckpt8_load(*(t[:n].cpu().numpy() for t in self.y8)).astype(np.float64)
            r = ob.ckpt8_load(*(t[:n].cpu().numpy() for t in self.r8)).astype(np.float64)
        self.bwd()
        ref = ob.resnorm_bwd(y, r, full(self.w_post), gate, full(self.w_pre), cut(self.rstd_y), cut(self.rstd_r),
                             cut(self.dr), cut(self.dh), self.alpha, self.gate_mode)
        # magnitudes of what is added: |dr| + rstd_r (|u| + |rhat| mean |u rhat|), and so on
        A = np.abs(cut(self.dr)) if self.dr is not None else np.zeros((n, self.d))
        if self.w_pre is not None:
            rr = cut(self.rstd_r)[:, None]
            U, R = np.abs(cut(self.dh) * full(self.w_pre)), np.abs(r * rr)
            A = A + rr * (U + R * (U * R).mean(axis=1, keepdims=True))
            _close("dw_pre", self.dw_pre, ref["dw_pre"], (n + 64) * 2.0 ** -24 * (np.abs(cut(self.dh)) * R).sum(axis=0))
        _close("dx", self.dx[:n], ref["dx"], u * np.abs(ref["dx"]) + 4 * w * abs(self.alpha) * A)
        assert (self.dx[n:] == 7).all()
        if y is not None:
            Y = np.abs(y if self.w_post is None else y * cut(self.rstd_y)[:, None])
            W = 1.0 if self.w_post is None else np.abs(full(self.w_post))
            G = np.abs(ob._gate(gate, self.gate_mode))
            if self.w_post is None:
                B = G * A
            else:
                B = cut(self.rstd_y)[:, None] * (G * A * W + Y * (G * A * W * Y).mean(axis=1, keepdims=True))
                _close("dw_post", self.dw_post, ref["dw_post"], ((n + 64) * 2.0 ** -24 + 4 * w) * (G * A * Y).sum(axis=0))
            _close("dy", self.dy[:n], ref["dy"], u * np.abs(ref["dy"]) + 8 * w * B)
            assert (self.dy[n:] == 7).all()
            if self.gate_mode == "channel":
                _close("dgate", self.dgate, ref["dgate"], ((n + 64) * 2.0 ** -24 + 4 * w) * (A * Y * W).sum(axis=0))
            elif self.gate_mode == "row":
                _close("dgate", self.dgate[:n], ref["dgate"], 8 * w * (A * Y * W).sum(axis=1))
                assert (self.dgate[n:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("n,d", [(1, 8), (3, 64), (7, 200), (33, 264), (290, 512), (5, 1024), (19, 1000),
                                 (40, 2048), (9, 4096), (3, 5000), (2, 8192), (1500, 128)])
@pytest.mark.parametrize("gate", ["none", "channel", "row"])
def test_resnorm_parity(n, d, gate, ckpt, dtype):
    Join(n, d, DT[dtype], gate=gate, ckpt=ckpt, seed=n + d).check()


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("parts", ["no_post", "no_pre", "no_y", "only_add", "no_dr"])
def test_resnorm_parts_left_out(parts, ckpt):
    for gate in ("none", "channel", "row"):
        if parts == "no_y" and gate != "none":
            continue
        Join(21, 320, torch.bfloat16, gate=gate, parts=parts, ckpt=ckpt, seed=4).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("n,d", [(1, 64), (1003, 40), (2, 72), (517, 128), (6, 136), (77, 256), (9001, 64), (5, 16)])
def test_resnorm_rows_that_share_a_warp(n, d, ckpt, dtype):
    gate = ("none", "channel", "row")[n % 3]
    Join(n, d, DT[dtype], gate=gate, ckpt=ckpt, seed=n + d).check()


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256, 512])
def test_resnorm_a_row_leaves_its_neighbours_alone(d, ckpt):
    """A row's results do not depend on what the rows beside it hold, infinities and NaN among it."""
    outs = lambda j: [t for t in (j.r, j.h, j.dx, j.dy, j.rstd_y, j.rstd_r, j.dgate)]  # noqa: E731
    for n, bad in ((7, 2), (6, 5), (301, 300), (301, 0)):
        runs = []
        for value in (None, float("nan"), float("inf")):
            j = Join(n, d, torch.bfloat16, gate="row", ckpt=ckpt, seed=9)
            j.n_rows.fill_(n)
            if value is not None:
                j.x[bad], j.dr[bad] = value, value
                j.y[bad, 3] = value
            j.fwd()
            j.bwd()
            runs.append(outs(j))
        keep = [i for i in range(n) if i != bad]
        for run in runs[1:]:
            assert all(torch.equal(a[keep], b[keep]) for a, b in zip(runs[0], run))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("n,d", [(3001, 64), (700, 200), (2000, 512), (1500, 1024), (300, 8192)])
def test_resnorm_in_place(n, d, ckpt, dtype):
    """Outputs on the inputs that they may lie on: the same bits as apart from them."""
    def run(lay):
        j = Join(n, d, DT[dtype], gate="channel", ckpt=ckpt, seed=2)
        if lay == "r on x, h on y":
            j.r, j.h = j.x, j.y.clone() if not ckpt else j.y
        elif lay == "h on x":
            j.h = j.x
        if lay == "r on x, h on y" and not ckpt:
            kept, j.y = j.y, j.h  # the forward's y is overwritten by h, the backward reads the copy
            j.fwd()
            j.y = kept
        else:
            j.fwd()
        if lay == "dx on dr, dy on dh":
            j.dx, j.dy = j.dr, j.dh
        elif lay == "dx on dh, dy on dr":
            j.dx, j.dy = j.dh, j.dr
        elif lay == "dx on r, dy on y" and not ckpt:
            j.dx, j.dy = j.r.clone(), j.y
            j.r = j.dx
        out = [t[:n].clone() for t in (j.h,)]
        r = j.r[:n].clone()
        j.bwd()
        return out + [r] + [t[:n].clone() for t in (j.dx, j.dy, j.rstd_y, j.rstd_r)] + [j.dw_post, j.dw_pre, j.dgate]

    apart = run("")
    for lay in ("r on x, h on y", "h on x", "dx on dr, dy on dh", "dx on dh, dy on dr", "dx on r, dy on y"):
        assert all(torch.equal(a, b) for a, b in zip(apart, run(lay))), lay


def test_resnorm_no_rows_and_zero_rows():
    j = Join(0, 256, torch.bfloat16, gate="channel", spare=4)
    j.fwd()
    j.bwd()
    for t in (j.r, j.h, j.dx, j.dy):
        assert (t == 7).all()
    for t in (j.dw_post, j.dw_pre, j.dgate):
        assert (t == 0).all()
    # rows of zeros: finite through eps
    j = Join(5, 256, torch.float32, gate="channel", spare=0)
    j.x.zero_()
    j.y.zero_()
    j.check()


def test_resnorm_repeats_bit_for_bit_and_replays():
    j = Join(3001, 1024, torch.bfloat16, gate="row", ckpt=True, seed=6)
    outs = lambda: [t.clone() for t in (j.r, j.h, j.dx, j.dy, j.dw_post, j.dw_pre, j.dgate, j.y8[0], j.r8[0])]  # noqa: E731
    j.fwd()
    j.bwd()
    first = outs()
    j.ws.random_(0, 255)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        j.fwd()
        j.bwd()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs()))
    # fewer rows at replay: the rest stay as they were
    j.n_rows.fill_(1000)
    for t in (j.r, j.dx):
        t.fill_(7.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(j.r[:1000], first[0][:1000]) and (j.r[1000:] == 7).all()
    assert torch.equal(j.dx[:1000], first[2][:1000]) and (j.dx[1000:] == 7).all()


# ------------------------------------------------------------------------ checkpoints
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1, 8), (2, 128), (37, 136), (5, 64), (300, 264), (3, 4096), (4, 20000), (20011, 64)])
def test_ckpt8_bit_for_bit(n, d, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    cap = n + 3
    x = (torch.randn(cap, d, generator=g, device="cuda") * torch.exp(torch.randn(cap, 1, generator=g, device="cuda") * 8)).to(DT[dtype])
    if n > 2:
        x[0] = 0
        x[1, :d // 2] = float("inf")
        x[2, d - 1] = float("nan")
        x[2, 0] = 1e-38
    codes = torch.full((cap, d), 7, dtype=torch.int8, device="cuda")
    scales = torch.full((cap, -(-d // 128)), 7.0, device="cuda")
    back = torch.full((cap, d), 7.0, dtype=DT[dtype], device="cuda")
    n_rows = torch.tensor([n], dtype=torch.int32, device="cuda")
    nat.nat_ckpt8_store(x, n_rows, cap, codes, scales)
    nat.nat_ckpt8_load(codes, scales, n_rows, cap, back)
    c, s = ob.ckpt8_store(x[:n].float().cpu().numpy())
    assert np.array_equal(codes[:n].cpu().numpy(), c)
    assert np.array_equal(scales[:n].cpu().numpy(), s, equal_nan=True)
    want = torch.from_numpy(ob.ckpt8_load(c, s)).to(DT[dtype])
    assert torch.equal(back[:n].cpu().nan_to_num(nan=-5.0), want.nan_to_num(nan=-5.0))
    assert (codes[n:] == 7).all() and (scales[n:] == 7).all() and (back[n:] == 7).all()
    # all rows where no count is given
    nat.nat_ckpt8_store(x[:n].contiguous(), None, n, codes, scales)
    assert np.array_equal(codes[:n].cpu().numpy(), c)


def test_row_operators_past_32_bits():
    """Rows whose elements lie more than 2^31 behind the first: the last ones against a short call."""
    d, n = 8192, 262300
    assert n * d > 1 << 31
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    codes = torch.empty(n, d, dtype=torch.int8, device="cuda")
    scales = torch.empty(n, 64, device="cuda")
    nat.nat_ckpt8_store(x, None, n, codes, scales)
    tail = [t[-100:].contiguous() for t in (x, codes, scales)]
    c, s = torch.empty_like(tail[1]), torch.empty_like(tail[2])
    nat.nat_ckpt8_store(tail[0], None, 100, c, s)
    assert torch.equal(c, tail[1]) and torch.equal(s, tail[2])
    back, b = torch.empty_like(x), torch.empty_like(tail[0])
    nat.nat_ckpt8_load(codes, scales, None, n, back)
    nat.nat_ckpt8_load(c, s, None, 100, b)
    assert torch.equal(back[-100:], b)
    p = nat.resnorm_params(d, torch.bfloat16)
    w = torch.ones(d, device="cuda")
    h, h1, r1 = codes.view(-1)[:0], torch.empty_like(b), torch.empty_like(b)
    del codes
    h = torch.empty_like(x)
    ry, rr = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    nat.nat_resnorm_fwd(p, x, x, w, None, w, None, n, back, h, ry, rr)
    nat.nat_resnorm_fwd(p, tail[0], tail[0], w, None, w, None, 100, r1, h1, ry[:100], rr[:100])
    assert torch.equal(back[-100:], r1) and torch.equal(h[-100:], h1)


def test_attn_float32_confines_infinities_to_the_tokens_that_see_them():
    a, b = (Attn([150], 4, 2, 64, torch.float32, seed=21) for _ in range(2))
    t = 70
    for x in (b.k, b.v):
        x[t] = float("inf")
    for s in (a, b):
        s.fwd()
    assert torch.equal(a.out[:t], b.out[:t]) and torch.equal(a.lse[:t], b.lse[:t])
    assert not torch.isfinite(b.out[t:150]).any()
    # a query's infinity reaches the keys that it sees, and no others
    a, b = (Attn([150], 4, 2, 64, torch.float32, seed=21) for _ in range(2))
    for s in (a, b):
        s.fwd()
    b.dout[t] = float("inf")
    for s in (a, b):
        s.bwd()
    for name in ("dk", "dv"):
        assert torch.equal(getattr(a, name)[t + 1:150], getattr(b, name)[t + 1:150]), name
    assert torch.equal(a.dq[:t], b.dq[:t]) and torch.equal(a.dq[t + 1:150], b.dq[t + 1:150])


def test_attn_bfloat16_infinities_reach_less_than_128_tokens():
    a, b = (Attn([900], 4, 2, 64, torch.bfloat16, seed=22) for _ in range(2))
    t = 500
    b.v[t] = float("inf")
    b.k[t] = float("nan")
    for s in (a, b):
        s.fwd()
        s.bwd()
    keep = t - 127
    assert torch.equal(a.out[:keep], b.out[:keep]) and torch.equal(a.lse[:t], b.lse[:t])
    assert torch.equal(a.dq[:keep], b.dq[:keep])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attn_gradient_against_differences(dtype):
    """The kernel's gradient against differences of the float64 forward along random directions (the
    kernel's inputs are exact in float64; the differences' own error is below 1e-6 of the norms)."""
    a = Attn([90, 41], 4, 2, 64, DT[dtype], seed=23, spare=0)
    a.fwd()
    a.bwd()
    q, k, v, w = (_np(t) for t in (a.q, a.k, a.v, a.dout))
    g = np.random.default_rng(0)
    f = lambda q, k, v: float((w * ob.attn_fwd(q, k, v, a.cu_h, a.params.scale)[0]).sum())  # noqa: E731
    for name, which in (("dq", 0), ("dk", 1), ("dv", 2)):
        got = _np(getattr(a, name))
        step = g.normal(size=got.shape)
        lo, hi = [q, k, v], [q, k, v]
        lo[which], hi[which] = lo[which] - 1e-5 * step, hi[which] + 1e-5 * step
        want = (f(*hi) - f(*lo)) / 2e-5
        # a rounding of u of every element moves the sum by at most u times the norms' product; bfloat16
        # rounds out (which delta reads), P, dS and the result: 4 u of the gradient's largest scale
        u = _half(DT[dtype]) if dtype == "bf16" else 2.0 ** -16
        scale = np.linalg.norm(got) * np.linalg.norm(step)
        assert abs((got * step).sum() - want) <= 4 * u * scale + 1e-6 * scale, name


@pytest.mark.parametrize("d", [64, 200, 1024])
def test_row_operators_on_rows_of_16_byte_alignment(d):
    """float32 rows that begin 16 bytes past a 32-byte boundary: the same bits as on one."""
    n = 257

    def shifted(t):
        buf = torch.empty(t.numel() + 4, dtype=t.dtype, device="cuda")
        assert buf.data_ptr() % 32 == 0
        return buf[4:].view(t.shape).copy_(t)

    a, b = (Join(n, d, torch.float32, gate="channel", ckpt=True, seed=5) for _ in range(2))
    for name in ("x", "y", "dr", "dh", "r", "h", "dx", "dy"):
        setattr(b, name, shifted(getattr(b, name)))
    for j in (a, b):
        j.fwd()
        j.bwd()
    for name in ("r", "h", "dx", "dy", "dw_post", "dw_pre", "dgate"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    codes, scales = (torch.empty_like(t[:n]) for t in a.y8)
    nat.nat_ckpt8_store(b.y[:n], None, n, codes, scales)
    assert torch.equal(codes, a.y8[0][:n]) and torch.equal(scales, a.y8[1][:n])
    back, far = torch.empty(n, d, device="cuda"), shifted(torch.zeros(n, d, device="cuda"))
    nat.nat_ckpt8_load(codes, scales, None, n, back)
    nat.nat_ckpt8_load(codes, scales, None, n, far)
    assert torch.equal(back, far)
