"""Long contractions of the expert products, in a bound that follows how they are added up.

On the tensor cores an accumulator of a long contraction takes 1024 terms at most, for which the parity tests' bound holds,
(terms + 16) steps of 2^-23; what the S = terms / 1024 accumulators hold is added in 32 bits, rounded to nearest: S 2^-24 more.
With terms of one sign, where what the accumulators cut off adds up, whole sums are off by several times that.  y and dx are
rounded to bfloat16 once, by half a step of their place: what is left of the difference is the sum's.
"""
import numpy as np
import pytest
import torch

from paper_2603_06619_b200 import nat
from test_gpu_experts import Experts

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
SEGMENT = 1024


def _sum_bound(terms):
    return (min(terms, SEGMENT) + 16) * 2.0 ** -23 + -(-terms // SEGMENT) * 2.0 ** -24


def _beyond_rounding(got, ref):
    """How far bfloat16 values are from `ref` beyond half a step, relative to it."""
    half = 2.0 ** (np.floor(np.log2(np.abs(ref))) - 8)
    return (np.abs(got.double().cpu().numpy() - ref) - half) / np.abs(ref)


@pytest.mark.parametrize("loads", [[7, 40, 0, 100], [200, 0, 33, 300]], ids=["turned", "mixed"])
@pytest.mark.parametrize("terms", [65536 + 8, 262144])
def test_long_contractions_round_once(terms, loads):
    n, narrow = sum(loads), 24
    g = torch.Generator(device="cuda")
    g.manual_seed(terms)
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    offs_h = np.concatenate([[0], np.cumsum(loads)]).astype(np.int32)
    offs = torch.from_numpy(offs_h).cuda()
    E = len(loads)

    def call(x, w, backward):
        p = nat.experts_params(E, w.shape[2], w.shape[1], BF16)
        ws = nat.alloc_workspace(nat.nat_experts_workspace_bytes(p, n), "cuda")
        out = torch.empty(n, w.shape[2] if backward else w.shape[1], dtype=BF16, device="cuda")
        if backward:
            nat.nat_experts_bwd(p, offs, n, None, w, x, out, None, ws)
        else:
            nat.nat_experts_fwd(p, offs, n, x, w, out, ws)
        assert nat.nat_poll_status(ws) == 0
        return out

    x = rand(n, terms)
    for backward in (False, True):
        w = rand(E, terms, narrow) if backward else rand(E, narrow, terms)
        out = call(x, w, backward)
        for e in range(E):
            lo, hi = offs_h[e], offs_h[e + 1]
            if hi > lo:
                m = w[e] if backward else w[e].t()
                ref = (x[lo:hi].double() @ m.double()).cpu().numpy()
                over = _beyond_rounding(out[lo:hi], ref)
                assert over.max() <= _sum_bound(terms), (backward, e, float(over.max()), _sum_bound(terms), float((over > _sum_bound(terms)).mean()))


@pytest.mark.parametrize("sizes", [(4104, 40), (4160, 264), (5128, 24), (8200, 136), (20000, 8)])
@pytest.mark.parametrize("loads", [[7, 40, 0, 100], [200, 0, 33, 300, 257], [600, 1, 1023], [k * 37 % 90 for k in range(70)],
                                   [k * 37 % 190 for k in range(70)], [k * 37 % 600 for k in range(70)]],
                         ids=["turned", "mixed", "whole", "many_few", "many_some", "many"])
def test_long_contractions_count_every_term_once(loads, sizes):
    """Whole numbers, whose sums are exact: y and dx are those, rounded once; forward and, the other way round, backward."""
    for n_in, n_out in (sizes, sizes[::-1]):
        e = Experts(loads, n_in, n_out, BF16, seed=1, first=2, strides=(8, 16))
        g = torch.Generator(device="cuda")
        g.manual_seed(2)
        for t in (e.x, e.dy):
            t[e.lo:e.hi] = torch.randint(-3, 4, (e.hi - e.lo, t.shape[1]), generator=g, device="cuda").to(BF16)
        e.w.copy_(torch.randint(-3, 4, e.w.shape, generator=g, device="cuda"))
        e.fwd()
        e.bwd(dw=False)
        for i in range(e.E):
            rows = slice(int(e.offs_h[i]), int(e.offs_h[i + 1]))
            assert torch.equal(e.y[rows], (e.x[rows].double() @ e.w[i].double().t()).to(BF16)), i
            assert torch.equal(e.dx[rows], (e.dy[rows].double() @ e.w[i].double()).to(BF16)), i
        for t in (e.y, e.dx):
            assert (t[:e.lo] == 7).all() and (t[e.hi:] == 7).all()


def test_infinities_and_nan_stay_in_their_row_in_long_contractions():
    loads = [70, 0, 333, 20]
    a, b = (Experts(loads, 6000, 136, BF16, seed=6) for _ in range(2))
    b.x[80, 5000], b.x[402, 3] = float("nan"), float("inf")
    b.w[3] = float("nan")
    for e in (a, b):
        e.fwd()
    keep = torch.ones(a.cap, dtype=torch.bool, device="cuda")
    keep[80], keep[402], keep[403:423] = False, False, False
    assert torch.equal(a.y[keep], b.y[keep])
    assert not torch.isfinite(b.y[80]).any() and not torch.isfinite(b.y[402]).any() and b.y[403:423].isnan().all()
