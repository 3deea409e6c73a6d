"""Pins of the float64 forms in ``oracle/nat_packed.py``: closed forms, identities and finite differences."""
import numpy as np
import pytest

from oracle import nat_packed as op


def _rng(seed):
    return np.random.default_rng(seed)


def test_embedding_and_its_gradient_are_adjoint():
    r = _rng(0)
    V, d, ids = 11, 8, np.array([3, 3, 0, 10, 3, 7, -1, 11, 0])
    table, dx = r.normal(size=(V, d)), r.normal(size=(len(ids), d))
    x = op.embed_fwd(table, ids, 0.5)
    ok = (ids >= 0) & (ids < V)
    assert np.isnan(x[~ok]).all() and np.array_equal(x[ok], 0.5 * table[ids[ok]])
    g, mag, count = op.embed_bwd(dx, ids, V, 0.5)
    assert np.isclose((x[ok] * dx[ok]).sum(), (table * g).sum(), rtol=1e-13)
    assert count.sum() == ok.sum() and count[3] == 3 and (mag >= np.abs(g) - 1e-15).all()
    assert (g[count == 0] == 0).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [0, 8, 16])
def test_rotation(interleaved, R):
    r = _rng(1)
    x, pos = r.normal(size=(5, 3, 16)), np.array([0, 1, 7, 100000, 3])
    f = 0.3 ** np.arange(R // 2)
    y = op.rotate(x, pos, f, interleaved)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., R:], x[..., R:])
    assert np.allclose((y * y).sum(2), (x * x).sum(2), rtol=1e-12)
    assert np.allclose(op.rotate(y, pos, f, interleaved, back=True), x, atol=1e-12)
    # products of a query and a key depend on the distance of their positions alone
    q, k = r.normal(size=(1, 1, 16)), r.normal(size=(1, 1, 16))
    dot = lambda p, s: (op.rotate(q, [p], f, interleaved) * op.rotate(k, [s], f, interleaved)).sum()  # noqa: E731
    assert np.isclose(dot(9, 4), dot(105, 100), rtol=1e-11)
    if R:
        one = op.rotate(np.eye(16)[None, :1], [1], f, interleaved)[0, 0]
        at = 1 if interleaved else R // 2
        assert np.isclose(one[0], np.cos(f[0])) and np.isclose(one[at], np.sin(f[0]))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_qknorm_gradient_against_differences(norm, interleaved):
    r = _rng(2)
    x, G, pos, f = r.normal(size=(4, 2, 16)), r.normal(size=(4, 2, 16)), np.array([0, 5, 2, 33]), 0.5 ** np.arange(4)
    w = 1 + 0.1 * r.normal(size=16) if norm else None
    fwd = lambda x, w: (G * op.qknorm_fwd(x, w, pos, f, 1e-6, interleaved)[0]).sum()  # noqa: E731
    b = op.qknorm_bwd(x, w, pos, f, 1e-6, interleaved, G)
    h = 1e-6
    step = r.normal(size=x.shape)
    assert np.isclose((b["dx"] * step).sum(), (fwd(x + h * step, w) - fwd(x - h * step, w)) / (2 * h), rtol=1e-7)
    if norm:
        step = r.normal(size=16)
        assert np.isclose((b["dw"] * step).sum(), (fwd(x, w + h * step) - fwd(x, w - h * step)) / (2 * h), rtol=1e-7)
        # a normed row does not grow with its input: its gradient has no part along it (eps aside)
        assert np.abs((b["dx"] * x).sum(2)).max() < 1e-4
        assert (b["mag_dw"] >= np.abs(b["dw"]) - 1e-12).all()
    assert (b["mag_dx"] >= np.abs(b["dx"]) - 1e-12).all()


def test_experts_against_whole_products_and_differences():
    r = _rng(3)
    x, w, dy = r.normal(size=(9, 5)), r.normal(size=(3, 4, 5)), r.normal(size=(9, 4))
    y, _ = op.experts_fwd(x, w, [0, 2, 2, 9])
    assert np.allclose(y[:2], x[:2] @ w[0].T) and np.allclose(y[2:], x[2:] @ w[2].T)
    b = op.experts_bwd(x, w, dy, [0, 2, 2, 9])
    assert (b["dw"][1] == 0).all()
    # linear in either argument
    assert np.isclose((b["dx"] * x).sum(), (y * dy).sum()) and np.isclose((b["dw"] * w).sum(), (y * dy).sum())
    # rows outside all experts have no part
    y, _ = op.experts_fwd(x, w, [1, 2, 2, 7])
    assert (y[0] == 0).all() and (y[7:] == 0).all()
