"""Calls that the documentation allows and that lie at its edges."""
import numpy as np
import pytest
import torch

from oracle import nat_body as ob
from paper_2603_06619_b200 import nat
from test_gpu_body import DT, Attn, Join, _close, _np
from test_gpu_body_gradients import check_gradients

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,spare", [(1, 1), (3, 70), (3, 3000), (1500, 40)])
def test_attention_of_empty_sequences_alone(B, spare, dtype):
    a = Attn([0] * B, 4, 2, 64, DT[dtype], spare=spare)
    a.fwd()
    assert nat.nat_poll_status(a.ws) == 0
    a.bwd()
    assert nat.nat_poll_status(a.ws) == 0
    for t in (a.out, a.lse, a.dq, a.dk, a.dv):
        assert (t == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("first,lengths,heads", [(5, [70, 0, 33], (4, 2, 64)), (129, [1900], (2, 2, 64)), (3, [1] * 1200, (2, 1, 32))])
def test_attention_of_sequences_that_begin_later(first, lengths, heads, dtype):
    """cu_seqlens from above zero: the rows in front of the first sequence are left alone like those behind the last."""
    a, b = Attn([first] + lengths, *heads, DT[dtype], seed=71), Attn([first] + lengths, *heads, DT[dtype], seed=71)
    b.B, b.cu = len(lengths), b.cu[1:].contiguous()
    for x in ("q", "k", "v", "dout"):
        getattr(b, x)[:first] = float("nan")
    b.ws = nat.alloc_workspace(nat.nat_attn_workspace_bytes(b.params, b.B, b.cap), "cuda")
    a.check()
    check_gradients(a)
    b.fwd()
    b.bwd()
    assert nat.nat_poll_status(b.ws) == 0
    for name in ("out", "lse", "dq", "dk", "dv"):
        x, y = getattr(a, name), getattr(b, name)
        assert (y[:first] == 7).all() and (y[b.n:] == 7).all(), name
        assert torch.isfinite(y).all()
        if len(lengths) > 1 or dtype == "f32":   # (one more sequence may cut the rows into other pieces)
            assert torch.equal(x[first:], y[first:]), name
        else:
            assert (x[first:].float() - y[first:].float()).abs().max() <= 0.02 * x[first:b.n].float().abs().max(), name


@pytest.mark.parametrize("scale", [-0.2, 0.0, 1e-3])
def test_attention_in_pieces_with_other_scales(scale):
    a = Attn([2100], 4, 1, 64, torch.bfloat16, seed=72, scale=scale)
    a.check()
    if scale:
        check_gradients(a)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", [[300, 40], [1700]])
@pytest.mark.parametrize("size", [1e2, 1e4, 1e6, 1e8, 1e9, 1e10, 1e20, 1e30])
def test_attention_of_large_scores(size, lengths, dtype):
    """A score's error is relative to it, and moves P by as much: out is still a mean of the values, within the
    bound that this gives."""
    a = Attn(lengths, 2, 2, 64, DT[dtype], seed=73)
    a.q.mul_(size ** 0.5)
    a.k.mul_(size ** 0.5)
    a.fwd()
    q, k, v = (_np(t[:a.n]) for t in (a.q, a.k, a.v))
    out, lse, mag = ob.attn_fwd(q, k, v, a.cu_h, a.params.scale)
    u, e = a.factors()
    # a weight moves by exp(2 e) - 1 at most, and no mean of the values leaves their range
    move = np.minimum((np.exp(min(2 * e, 50.0)) - 1 + (u if dtype == "bf16" else 0.0)) * 1.01 * mag, 2 * np.abs(v).max())
    _close("out", a.out[:a.n], out, u * np.abs(out) + move)
    _close("lse", a.lse[:a.n], lse, 2 * e + 2.0 ** -22 * np.abs(lse))
    # rows that one key owns by far are that key's value, whatever the size
    S = np.stack([a.params.scale * q[: lengths[0], h] @ k[: lengths[0], h].T for h in range(2)], axis=1)
    S[np.triu_indices(lengths[0], 1)[0], :, np.triu_indices(lengths[0], 1)[1]] = -np.inf
    order = np.sort(S, axis=2)
    clear = (order[:, :, -1] - order[:, :, -2] > 60 + 4 * e)
    top = S.argmax(axis=2)
    for t, h in np.argwhere(clear)[:200]:
        assert np.abs(_np(a.out[t, h]) - v[top[t, h], h]).max() <= 4 * u * np.abs(v[top[t, h], h]).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["none", "channel", "row"])
@pytest.mark.parametrize("n,d", [(7, 64), (5, 128), (3, 256), (4, 512), (3, 4096)])
@pytest.mark.parametrize("x,y,w,alpha", [(1e-30, 1e-18, 1e-6, 1.0), (1e-18, 1e-18, 1e-6, 1.0), (1e-22, 1.0, 1e-20, 1e10), (0.0, 1e-10, 1e-12, 0.5),
                                         (1e-21, 0.0, 1.0, 1e15), (1e18, 1.0, 1.0, 1e-18)])
def test_join_of_rows_far_from_one(x, y, w, alpha, n, d, gate, dtype):
    """r is of a size that its norm in 32 bits can take, made of parts whose squares are not.  (y and r themselves
    have to be: the header says so.)"""
    j = Join(n, d, DT[dtype], gate=gate, seed=81, eps=0.0 if y else 1e-30, alpha=alpha)
    j.x.mul_(x)
    j.y.mul_(y)
    j.w_post.mul_(w)
    j.fwd()
    cut = lambda t: _np(t[:n])  # noqa: E731
    g = None if gate == "none" else cut(j.gate) if gate == "row" else _np(j.gate)
    ref = ob.resnorm_fwd(cut(j.x), cut(j.y), _np(j.w_post), g, _np(j.w_pre), j.eps, alpha, gate)
    u, e = torch.finfo(DT[dtype]).eps / 2, (d + 32) * 2.0 ** -24
    mag = np.abs(alpha * cut(j.x)) + np.abs(ref["r"] - alpha * cut(j.x))
    _close("rstd_r", j.rstd_r[:n], ref["rstd_r"], 2 * e * ref["rstd_r"] * (1 + 8 * (mag ** 2).sum(axis=1) / (ref["r"] ** 2).sum(axis=1)))
    unit = np.abs(ref["rstd_r"][:, None] * _np(j.w_pre))
    ratio = np.sqrt((mag ** 2).sum(axis=1) / (ref["r"] ** 2).sum(axis=1))[:, None]
    _close("h", j.h[:n], ref["h"], u * np.abs(ref["h"]) + e * ((3 + 16 * ratio ** 2) * np.abs(ref["h"]) + 3 * mag * unit))
