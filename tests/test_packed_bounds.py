"""The bounds on sums over many rows pass what is right and refuse what they are there to refuse (no GPU needed)."""
import numpy as np
import pytest

import packed_bounds
from oracle import nat_packed as op


def _terms(lengths, H, D, seed):
    """(terms of dw, their magnitudes) [tokens, heads, D] of a batch of head norms."""
    r = np.random.default_rng(seed)
    n = sum(lengths)
    x, G = r.normal(size=(n, H, D)), r.normal(size=(n, H, D))
    pos = np.concatenate([np.arange(t) for t in lengths])
    f = 1e4 ** (-2.0 * np.arange(D // 2) / D)
    g, mg = op.rotate(G, pos, f, False, back=True), op.spread(G, D, False)
    xhat = x * (np.mean(x * x, axis=2, keepdims=True) + 1e-6) ** -0.5
    return g * xhat, mg * np.abs(xhat)


@pytest.mark.parametrize("lengths,H,D", [([2500, 1, 900], 32, 128), ([300, 41], 4, 64), ([1], 1, 8)])
def test_heads(lengths, H, D):
    terms, mag = _terms(lengths, H, D, 0)
    dw, tol = terms.sum(axis=(0, 1)), packed_bounds.heads(mag)
    # added up in 32 bits, one by one
    plain = np.add.accumulate(terms.astype(np.float32).reshape(-1, D), axis=0, dtype=np.float32)[-1]
    assert (np.abs(plain - dw) <= tol).all()
    fails = lambda off: (np.abs(off) > tol).any()  # noqa: E731
    assert fails(dw) and fails(0.01 * dw)                               # no gradient, one per cent
    for t in {0, len(terms) // 2, len(terms) - 1}:                      # a token without a part, or with two
        assert fails(terms[t].sum(axis=0))
        assert fails(terms[t, H - 1])                                   # one head of it
    if len(lengths) > 1:
        assert fails(terms[sum(lengths[:-1]):].sum(axis=(0, 1)))        # the last sequence


def _cut(x):
    """To 24 bits, toward zero."""
    m, e = np.frexp(x)
    return np.ldexp(np.trunc(m * 2.0 ** 24) * 2.0 ** -24, e)


def _on_tensor_cores(terms, segment):
    """Sums over the first axis, 16 terms a step, cut off; every `segment` terms to a register of 32 bits."""
    total = np.zeros(terms.shape[1], dtype=np.float32)
    for lo in range(0, len(terms), segment):
        s = np.zeros(terms.shape[1])
        for i in range(lo, min(lo + segment, len(terms)), 16):
            s = _cut(s + terms[i:min(i + 16, lo + segment)].sum(axis=0))
        total = total + s.astype(np.float32)
    return total.astype(np.float64)


def test_experts():
    r = np.random.default_rng(1)
    for n in (700, 12500, 20000):
        terms = r.normal(size=(n, 500)) * r.normal(size=(n, 500))
        dw = terms.sum(axis=0)
        err = lambda got: np.linalg.norm(got - dw) / np.linalg.norm(dw)  # noqa: E731
        bf16, f32 = packed_bounds.experts(n, True), packed_bounds.experts(n, False)
        assert err(_on_tensor_cores(terms, 512)) <= bf16
        if n > 10000:
            assert err(_on_tensor_cores(terms, n)) > bf16               # one accumulator for all
        plain = np.add.accumulate(terms.astype(np.float32), axis=0, dtype=np.float32)[-1]
        assert err(plain) <= f32
        for row in (0, n // 2, n - 1):                                  # a row without a part
            assert err(dw - terms[row]) > max(bf16, f32)
