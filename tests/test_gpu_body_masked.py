"""Infinities and NaN behind the causal mask: attention's results that do not see them are those of the clean inputs,
within the same bounds of the float64 form."""
import numpy as np
import pytest
import torch

import body_bounds
from oracle import nat_body as ob
from test_gpu_body import DT, Attn, _np

pytestmark = pytest.mark.gpu

CASES = [([300, 77], (4, 2, 64)), ([130], (1, 1, 8)), ([500, 3], (3, 1, 96)), ([700], (8, 1, 64)), ([5, 260, 1], (5, 1, 80)),
         ([2100], (2, 2, 64)), ([2100], (4, 1, 128))]   # the last two in pieces
VALUES = {"nan": float("nan"), "inf": float("inf"), "both": (float("inf"), float("-inf"))}


class Pair:
    """A batch, its clean results in float64 with their bounds, and the same batch to be spoilt."""

    def __init__(self, lengths, heads, dtype):
        self.a, self.b = (Attn(lengths, *heads, dtype, seed=61) for _ in range(2))
        a = self.a
        a.fwd()
        a.bwd()
        q, k, v = (_np(t[:a.n]) for t in (a.q, a.k, a.v))
        u, e = a.factors()
        up = u if a.dtype == torch.bfloat16 else 0.0
        out, lse, mag = ob.attn_fwd(q, k, v, a.cu_h, a.params.scale)
        self.ref = ob.attn_bwd(q, k, v, _np(a.out[:a.n]), _np(a.lse[:a.n]), _np(a.dout[:a.n]), a.cu_h, a.params.scale)
        where = (q, k, _np(a.lse[:a.n]), a.cu_h, a.params.scale, a.dtype == torch.bfloat16)
        self.tol = {x: body_bounds.element(x, self.ref, *where) + 1e-30 for x in ("dq", "dk", "dv")}
        self.ref.update(out=out, lse=lse)
        self.tol.update(out=u * np.abs(out) + (up + 2 * e) * 1.01 * mag, lse=2 * e + 2.0 ** -22 * np.abs(lse))
        sizes = np.diff(a.cu_h)
        self.lo, self.hi = (int(x[np.argmax(sizes)]) for x in (a.cu_h[:-1], a.cu_h[1:]))

    def spoil(self, name, tokens, columns, value):
        a, b = self.a, self.b
        for x in ("q", "k", "v", "dout", "out", "lse"):
            getattr(b, x).copy_(getattr(a, x))
        values = value if isinstance(value, tuple) else (value,)
        t = getattr(b, name)
        for i, token in enumerate(tokens):
            t[token, :, columns] = values[i % len(values)]

    def right(self, name, rows, columns=slice(None)):
        """The spoilt batch's result is the clean one in these rows and columns."""
        got, ref, tol = (x[rows] if name == "lse" else x[rows][..., columns]
                         for x in (_np(getattr(self.b, name)[:self.a.n]), self.ref[name], self.tol[name]))
        assert np.isfinite(got).all(), (name, np.argwhere(~np.isfinite(got))[:4].tolist())
        over = np.abs(got - ref) - tol
        assert (over <= 0).all(), (name, float(over.max()))


def _tokens(p):
    n = p.hi - p.lo
    return [[t] for t in sorted({0, 1, 31, 62, 63, 64, 127, 128, 129, n // 2, n - 2, n - 1}) if 0 <= t < n] + [
        list(range(n // 3, n, 41)), list(range(n - 1))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("value", list(VALUES))
def test_results_that_do_not_see_them(case, value, dtype):
    p = Pair(*CASES[case], DT[dtype])
    a, b, D = p.a, p.b, p.a.D
    rows = np.arange(a.n)
    inside = (rows >= p.lo) & (rows < p.hi)
    column, rest = [min(5, D - 1)], [c for c in range(D) if c != min(5, D - 1)]
    for tokens in _tokens(p):
        bad = [p.lo + t for t in tokens]
        first, last = bad[0], bad[-1]
        before, behind, others = rows[(rows < first) | ~inside], rows[(rows > last) | ~inside], np.setdiff1d(rows, bad)
        # forward: v in one column, then in all
        p.spoil("v", bad, column, VALUES[value])
        b.fwd()
        p.right("out", before)
        p.right("out", rows, rest)
        p.right("lse", rows)
        assert not torch.isfinite(b.out[first:p.hi][:, :, column]).any()
        p.spoil("v", bad, slice(None), VALUES[value])
        b.fwd()
        p.right("out", before)
        # k: the rows before its token
        p.spoil("k", bad, column, VALUES[value])
        b.fwd()
        p.right("out", before)
        p.right("lse", before)
        # backward, from the clean out and lse
        p.spoil("k", bad, column, VALUES[value])
        b.bwd()
        p.right("dq", before)
        p.right("dk", others)
        p.right("dv", others)
        p.spoil("v", bad, column, VALUES[value])
        b.bwd()
        p.right("dq", before)
        p.right("dk", others)
        p.right("dv", rows)
        for name in ("q", "dout"):
            p.spoil(name, bad, column, VALUES[value])
            b.bwd()
            p.right("dq", others)
            p.right("dk", behind)
            p.right("dv", behind)
        p.right("dv", rows, rest)


def test_everything_infinite_ends_soon():
    """A batch that has diverged: no row is added up again whose own tokens explain its infinities."""
    a = Attn([3000, 2000], 8, 2, 128, torch.bfloat16, seed=62)
    times = []
    for value in (None, float("nan"), float("inf")):
        if value is not None:
            for t in (a.v, a.dout):
                t.fill_(value)
        for _ in range(2):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            a.fwd()
            a.bwd()
            end.record()
            end.synchronize()
        times.append(begin.elapsed_time(end))
    assert max(times[1:]) < 100 * times[0], times


@pytest.mark.parametrize("lengths,heads", [([300], (4, 2, 64)), ([2100], (2, 2, 64))])
@pytest.mark.parametrize("size", [1e5, 1e9])
def test_rows_of_large_scores_that_do_not_see_them(size, lengths, heads):
    """Where one key owns a row by far the row is that key's value, spoilt neighbours or not."""
    a, b = (Attn(lengths, *heads, torch.bfloat16, seed=63) for _ in range(2))
    for x in (a, b):
        x.q.mul_(size ** 0.5)
        x.k.mul_(size ** 0.5)
    a.fwd()
    for t in (1, 100, 250, lengths[0] - 5):
        b.v.copy_(a.v)
        b.v[t, :, 7] = float("nan")
        b.fwd()
        # P is rounded to bfloat16 in both, and the result once more: two half steps of each
        u = 2.0 ** -8
        S = a.params.scale * torch.einsum("ihd,jhd->hij", a.q[:t].double(), a.k[:t].double().repeat_interleave(heads[0] // heads[1], 1))
        S.masked_fill_(torch.ones(t, t, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
        top = S.topk(min(2, t), dim=2).values
        clear = (top[:, :, 0] - top[:, :, -1] > 1e-4 * size).t() if t > 1 else torch.ones(1, heads[0], dtype=torch.bool, device="cuda")
        clear[0] = True
        x, y = a.out[:t].double(), b.out[:t].double()
        assert torch.isfinite(y).all()
        assert ((x - y).abs() <= 4 * u * x.abs())[clear].all()
