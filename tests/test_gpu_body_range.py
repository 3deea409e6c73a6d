"""Packed attention at the far ends of its range: long sequences, many heads to a key head, more than 2^17 rows, and a
capacity far above the rows.  Long sequences are compared in rows drawn from them, in float64."""
import numpy as np
import pytest
import torch

import body_bounds
from paper_2603_06619_b200 import nat
from test_gpu_body import DT, Attn, _np
from test_gpu_body_gradients import check_gradients

pytestmark = pytest.mark.gpu


def _sampled(a, tokens):
    """(reference, magnitudes) of the forward and of all gradients of these tokens, a dict of [tokens, heads, D]."""
    scale, g, D = a.params.scale, a.Hq // a.Hkv, a.D
    wide = lambda t: t[:a.n].double()  # noqa: E731
    q, k, v, out, lse, do = (wide(t) for t in (a.q, a.k, a.v, a.out, a.lse, a.dout))
    zeros = lambda heads: torch.zeros(len(tokens), heads, D, dtype=torch.float64, device="cuda")  # noqa: E731
    r = {x: zeros(a.Hkv if x[-2:] in ("dk", "dv") else a.Hq) for y in ("dq", "dk", "dv")
         for x in [y] + [m + y for m in ("terms_", "parts_", "squares_")]}
    r.update(out=zeros(a.Hq), absolute=zeros(a.Hq), lse=torch.zeros(len(tokens), a.Hq, dtype=torch.float64, device="cuda"))
    for n, t in enumerate(tokens):
        i = int(np.searchsorted(a.cu_h, t, side="right")) - 1
        lo, hi = int(a.cu_h[i]), int(a.cu_h[i + 1])
        for h in range(a.Hq):
            kh = h // g
            K, V = k[lo:t + 1, kh], v[lo:t + 1, kh]
            S = scale * (K @ q[t, h])
            r["lse"][n, h] = torch.logsumexp(S, 0)
            P = torch.exp(S - r["lse"][n, h])
            r["out"][n, h], r["absolute"][n, h] = P @ V, P @ V.abs()
            P = torch.exp(S - lse[t, h])
            dS = P * (V @ do[t, h] - do[t, h] @ out[t, h])
            parts = P * (V.abs() @ do[t, h].abs() + do[t, h].abs() @ out[t, h].abs())
            for m, w, e in (("", dS, 0), ("terms_", dS.abs(), 1), ("parts_", parts, 1), ("squares_", dS * dS, 2)):
                r[m + "dq"][n, h] = scale ** max(e, 1) * (w @ (K.abs() ** e if e else K))
            # as a key: the queries from it on
            Q, G = q[t:hi, h], do[t:hi, h]
            P = torch.exp(scale * (Q @ k[t, kh]) - lse[t:hi, h])
            delta, size = (G * out[t:hi, h]).sum(1), (G * out[t:hi, h]).abs().sum(1)
            dS, parts = P * (G @ v[t, kh] - delta), P * (G.abs() @ v[t, kh].abs() + size)
            for m, w, e in (("", dS, 0), ("terms_", dS.abs(), 1), ("parts_", parts, 1), ("squares_", dS * dS, 2)):
                r[m + "dk"][n, kh] += scale ** max(e, 1) * (w @ (Q.abs() ** e if e else Q))
            r["dv"][n, kh] += P @ G
            r["terms_dv"][n, kh] += P @ G.abs()
            r["squares_dv"][n, kh] += (P * P) @ (G * G)
    return {x: t.cpu().numpy() for x, t in r.items()}


def check_sampled(a, count=24, seed=0):
    a.fwd()
    a.bwd()
    assert nat.nat_poll_status(a.ws) == 0
    g = np.random.default_rng(seed)
    edges = [t for lo, hi in zip(a.cu_h[:-1], a.cu_h[1:]) if hi > lo for t in (lo, hi - 1, min(lo + 127, hi - 1), min(lo + 128, hi - 1))]
    tokens = np.array(sorted({int(t) for t in edges[:24]} | {int(t) for t in g.integers(0, a.n, count)}))
    r = _sampled(a, tokens)
    at = torch.from_numpy(tokens).cuda()
    q, k, lse = (_np(t[:a.n]) for t in (a.q, a.k, a.lse))
    where = (q, k, lse, a.cu_h, a.params.scale, a.dtype == torch.bfloat16)
    u, e = a.factors()
    second = u if a.dtype == torch.bfloat16 else 0.0
    for name, tol in (("out", u * np.abs(r["out"]) + (second + 2 * e) * 1.01 * r["absolute"]),
                      ("lse", 2 * e + 2.0 ** -22 * np.abs(r["lse"]))):
        over = np.abs(_np(getattr(a, name)[at]) - r[name]) - tol
        assert (over <= 0).all(), (name, float(over.max()))
    for name in ("dq", "dk", "dv"):
        err = np.abs(_np(getattr(a, name)[at]) - r[name])
        over = err - body_bounds.element(name, r, *where) - 1e-30
        assert (over <= 0).all(), (name, float(over.max()))
        assert np.linalg.norm(err) <= body_bounds.norm(name, r, *where), name
    for name in ("out", "lse", "dq", "dk", "dv"):
        t = getattr(a, name)
        assert (t[a.n:] == 7).all() and torch.isfinite(t[:a.n]).all(), name


@pytest.mark.parametrize("lengths,heads,dtype", [
    ([9000], (2, 1, 64), "bf16"),                       # in pieces
    ([12000, 1, 9000], (4, 2, 128), "bf16"),
    ([33000], (8, 2, 96), "bf16"),
    ([5000, 300], (2, 1, 128), "f32"),
    ([20000], (8, 1, 64), "bf16"),                      # the keys' plan: 1250 steps in 1024 buckets
    ([135000], (2, 1, 64), "bf16"),                     # all plans: more steps than buckets
    ([3600] * 39 + [0, 1], (2, 2, 64), "bf16"),         # 140,401 rows
])
def test_long_sequences(lengths, heads, dtype):
    check_sampled(Attn(lengths, *heads, DT[dtype], seed=51))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(64, 1, 64), (43, 1, 40), (128, 2, 32), (33, 1, 128)])
def test_many_heads_to_a_key_head(heads, dtype):
    a = Attn([129, 1, 0, 300], *heads, DT[dtype], seed=52)
    a.check()
    check_gradients(a)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,heads,cap", [([2100], (2, 2, 64), 30000), ([2100], (4, 1, 128), 9000), ([1500, 3, 700], (1, 1, 128), 30000),
                                               ([70, 5], (8, 2, 64), 50000), ([300, 20, 9], (2, 1, 96), 1200)])
def test_capacity_far_above_the_rows(lengths, heads, cap, dtype):
    a = Attn(lengths, *heads, DT[dtype], seed=53, spare=cap - sum(lengths))
    a.check()
    check_gradients(a)
