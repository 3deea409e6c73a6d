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
