"""Attention's gradients within the bounds of ``body_bounds``: against the formula, and against differences."""
import numpy as np
import pytest
import torch

import body_bounds
from oracle import nat_body as ob
from test_gpu_body import DT, Attn, _half, _np

pytestmark = pytest.mark.gpu


def _reference(a):
    q, k, v = (_np(t[:a.n]) for t in (a.q, a.k, a.v))
    out, lse, do = _np(a.out[:a.n]), _np(a.lse[:a.n]), _np(a.dout[:a.n])
    return ob.attn_bwd(q, k, v, out, lse, do, a.cu_h, a.params.scale), (q, k, lse, a.cu_h, a.params.scale,
                                                                       a.dtype == torch.bfloat16)


def check_gradients(a):
    a.fwd()
    a.bwd()
    ref, where = _reference(a)
    for name in ("dq", "dk", "dv"):
        err = np.abs(_np(getattr(a, name)[:a.n]) - ref[name])
        over = err - body_bounds.element(name, ref, *where) - 1e-30
        assert (over <= 0).all(), (name, float(over.max()), np.argwhere(over > 0)[:4].tolist())
        if a.n >= 64:   # enough elements for sums of squares
            assert np.linalg.norm(err) <= body_bounds.norm(name, ref, *where), (
                name, np.linalg.norm(err) / np.linalg.norm(ref[name]), body_bounds.norm(name, ref, *where) / np.linalg.norm(ref[name]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (2, 2, 128), (8, 1, 64), (3, 1, 96), (14, 2, 32), (12, 2, 128), (1, 1, 8)])
@pytest.mark.parametrize("lengths", [[700], [127, 128, 257, 64], [0, 5, 0, 1, 33, 128, 129, 0], [2], [1]])
def test_gradients_against_the_formula(lengths, heads, dtype):
    check_gradients(Attn(lengths, *heads, DT[dtype], seed=41))


@pytest.mark.parametrize("heads", [(4, 1, 128), (2, 2, 64)])
def test_gradients_of_tiles_in_pieces(heads):
    check_gradients(Attn([1500, 3, 700], *heads, torch.bfloat16, seed=42))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_gradient_along_itself_against_differences(D, dtype):
    """The slope of the float64 forward along the gradient's own direction is the gradient's norm, so an error of the
    whole gradient by a factor shows in full.  The stored out, rounded, moves delta of row i by up to
    u sum |dout| |out|, at random within it: by rms u / sqrt(3) (sum dout^2 out^2)^1/2; that moves dq_i by as much of
    scale sum_j P_ij k_j, and dk_j by as much of scale P_ij q_i, whose squares over all j add up to
    |q_i|^2 sum_j P_ij^2, with sum_j P_ij^2 = exp(lse of twice the scores - 2 lse)."""
    a = Attn([90, 41], 4, 2, D, DT[dtype], seed=43, spare=0)
    a.fwd()
    a.bwd()
    ref, where = _reference(a)
    q, k, v, w, out = (_np(t) for t in (a.q, a.k, a.v, a.dout, a.out))
    scale, u = a.params.scale, _half(DT[dtype])
    f = lambda q, k, v: float((w * ob.attn_fwd(q, k, v, a.cu_h, scale)[0]).sum())  # noqa: E731
    delta = u / np.sqrt(3) * np.sqrt((w * w * out * out).sum(axis=2))
    seen, lse, _ = ob.attn_fwd(q, k, k, a.cu_h, scale)
    squares = np.exp(ob.attn_fwd(2 * q, k, k, a.cu_h, scale)[1] - 2 * lse)
    moved = {"dq": scale * np.sqrt((delta ** 2 * (seen ** 2).sum(axis=2)).sum()),
             "dk": scale * np.sqrt((delta ** 2 * (q ** 2).sum(axis=2) * squares).sum()), "dv": 0.0}
    for which, name in enumerate(("dq", "dk", "dv")):
        got = _np(getattr(a, name))
        step = got / np.linalg.norm(got)
        lo, hi = [q, k, v], [q, k, v]
        lo[which], hi[which] = lo[which] - 1e-4 * step, hi[which] + 1e-4 * step
        slope = (f(*hi) - f(*lo)) / 2e-4
        bound = body_bounds.norm(name, ref, *where) + 1.25 * moved[name]
        # the differences' own error: 1e-8 of the third derivative, a few units of the norm
        assert abs(np.linalg.norm(got) - slope) <= bound + 1e-6 * slope, (name, np.linalg.norm(got), slope, bound)
        assert bound < 0.008 * slope, (name, bound / slope)
