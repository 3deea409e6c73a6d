"""Sums over many rows: no row without a part in them and none with two, and no larger error than the order of the sums explains.
Bounds: ``packed_bounds.py``."""
import numpy as np
import pytest
import torch

import packed_bounds
from oracle import nat_packed as op
from test_gpu_experts import Experts
from test_gpu_qknorm import Heads

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _np(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads", [(32, 8, 128), (16, 4, 64), (1, 1, 8), (3, 1, 96), (2, 1, 32)])
@pytest.mark.parametrize("lengths", [[2500, 1, 900], [7000], [3, 1, 17, 40, 9, 0, 31] * 8, [1]], ids=["long", "one", "many", "token"])
def test_head_norms_weights(lengths, heads, interleaved, dtype):
    h = Heads(lengths, *heads, dtype, R=heads[2] // 16 * 16, interleaved=interleaved, seed=sum(lengths))
    h.bwd()
    freq = np.zeros(0) if h.freq is None else _np(h.freq)
    for name in ("q", "k"):
        x, G = _np(getattr(h, name)[:h.n]), _np(getattr(h, "d%s_out" % name)[:h.n])
        xhat = x * (np.mean(x * x, axis=2, keepdims=True) + h.eps) ** -0.5
        ref = (op.rotate(G, h.pos, freq, interleaved, back=True) * xhat).sum(axis=(0, 1))
        tol = packed_bounds.heads(op.spread(G, 2 * len(freq), interleaved) * np.abs(xhat))
        off = np.abs(_np(getattr(h, "dw_" + name)) - ref)
        assert (off <= tol).all(), (name, float((off / tol).max()))


LOADS = {"one": [20000], "tails": [12500, 0, 9001, 1, 63, 64, 65, 511, 512, 513, 1023, 1025],
         "even": [512, 1024, 2048, 4096], "many": [k * 37 % 1500 for k in range(70)]}
SIZES = [(72, 136), (520, 264), (8, 16), (256, 512)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("loads", list(LOADS))
def test_experts_count_every_row_once(loads, sizes, accumulate, dtype):
    """Whole numbers: every product and sum is exact below 2^24, and y and dx are those numbers rounded once."""
    e = Experts(LOADS[loads], *sizes, dtype, seed=1, first=3, accumulate=accumulate)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    for t in (e.x, e.dy):
        t[e.lo:e.hi] = torch.randint(-3, 4, (e.hi - e.lo, t.shape[1]), generator=g, device="cuda").to(dtype)
    e.w.copy_(torch.randint(-3, 4, e.w.shape, generator=g, device="cuda"))
    e.old.copy_(torch.randint(-50, 50, e.old.shape, generator=g, device="cuda"))
    if accumulate:
        e.dw.copy_(e.old)
    e.fwd()
    e.bwd()
    for i in range(e.E):
        rows = slice(int(e.offs_h[i]), int(e.offs_h[i + 1]))
        x, dy, w = e.x[rows].double(), e.dy[rows].double(), e.w[i].double()
        assert torch.equal(e.y[rows], (x @ w.t()).to(dtype)), i
        assert torch.equal(e.dx[rows], (dy @ w).to(dtype)), i
        dw = dy.t() @ x + (e.old[i].double() if accumulate else 0.0)
        assert dw.abs().max() < 2 ** 24 and torch.equal(e.dw[i].double(), dw), i


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("loads", ["one", "tails"])
def test_experts_long_sums(loads, sizes, dtype):
    e = Experts(LOADS[loads], *sizes, dtype, seed=3)
    e.bwd(dx=False)
    for i, n in enumerate(LOADS[loads]):
        if n >= 500:
            rows = slice(int(e.offs_h[i]), int(e.offs_h[i + 1]))
            ref = e.dy[rows].double().t() @ e.x[rows].double()
            off = float((e.dw[i].double() - ref).norm() / ref.norm())
            assert off <= packed_bounds.experts(n, dtype == BF16), (i, n, off)
