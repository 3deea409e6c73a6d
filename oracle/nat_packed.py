"""Plain float64 numpy form of what stands around the packed attention and the joins of blocks.

The embedding of packed tokens, the heads' norms with the rotation by position, and products of rows that are grouped
by expert; forward and backward, straight from the formulas in ``include/nat.h``.  Shares nothing with the CUDA path.
Beside each result stands the sum of the magnitudes of its terms ("mag" names), by which rounding errors are measured.
"""
import numpy as np


def embed_fwd(table, ids, scale):
    """Rows of the table; NaN for ids outside it."""
    table = np.asarray(table, dtype=np.float64)
    out = np.full((len(ids), table.shape[1]), np.nan)
    for k, v in enumerate(ids):
        if 0 <= v < table.shape[0]:
            out[k] = scale * table[v]
    return out


def embed_bwd(dx, ids, V, scale):
    """(dtable, mag, tokens a row)."""
    dx = np.asarray(dx, dtype=np.float64)
    out, mag, count = np.zeros((V, dx.shape[1])), np.zeros((V, dx.shape[1])), np.zeros(V, dtype=np.int64)
    for k, v in enumerate(ids):
        if 0 <= v < V:
            out[v] += scale * dx[k]
            mag[v] += abs(scale) * np.abs(dx[k])
            count[v] += 1
    return out, mag, count


def _pairs(D, R, interleaved):
    i = np.arange(R // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)


def rotate(x, pos, inv_freq, interleaved, back=False):
    """x [n, H, D] turned by the angle pos inv_freq (back: by minus that)."""
    a, b = _pairs(x.shape[2], 2 * len(inv_freq), interleaved)
    t = np.multiply.outer(np.asarray(pos, dtype=np.float64), np.asarray(inv_freq, dtype=np.float64))[:, None, :]
    c, s = np.cos(t), np.sin(-t if back else t)
    out = x.copy()
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., b] * c + x[..., a] * s
    return out


def spread(x, R, interleaved):
    """|x_a| + |x_b| in both places of each pair."""
    a, b = _pairs(x.shape[2], R, interleaved)
    out = np.abs(x)
    both = out[..., a] + out[..., b]
    out[..., a], out[..., b] = both, both
    return out


def qknorm_fwd(x, w, pos, inv_freq, eps, interleaved):
    """(out, mag)."""
    n = x if w is None else x * (np.mean(x * x, axis=2, keepdims=True) + eps) ** -0.5 * w
    return rotate(n, pos, inv_freq, interleaved), spread(n, 2 * len(inv_freq), interleaved)


def qknorm_bwd(x, w, pos, inv_freq, eps, interleaved, dout):
    """dict of dx, mag_dx and, with a norm, dw, mag_dw."""
    g = rotate(dout, pos, inv_freq, interleaved, back=True)
    mg = spread(dout, 2 * len(inv_freq), interleaved)
    if w is None:
        return {"dx": g, "mag_dx": mg}
    rstd = (np.mean(x * x, axis=2, keepdims=True) + eps) ** -0.5
    xhat = x * rstd
    u, mu = g * w, mg * np.abs(w)
    mean = lambda t: t.mean(axis=2, keepdims=True)  # noqa: E731
    return {"dx": rstd * (u - xhat * mean(u * xhat)), "mag_dx": rstd * (mu + np.abs(xhat) * mean(mu * np.abs(xhat))),
            "dw": (g * xhat).sum(axis=(0, 1)), "mag_dw": (mg * np.abs(xhat)).sum(axis=(0, 1))}


def experts_fwd(x, w, offsets):
    """(y, mag): rows offsets[e] .. offsets[e + 1] times expert e's weights [n_out, n_in]."""
    y, mag = (np.zeros((x.shape[0], w.shape[1])) for _ in range(2))
    for e, (lo, hi) in enumerate(zip(offsets[:-1], offsets[1:])):
        y[lo:hi] = x[lo:hi] @ w[e].T
        mag[lo:hi] = np.abs(x[lo:hi]) @ np.abs(w[e]).T
    return y, mag


def experts_bwd(x, w, dy, offsets):
    """dict of dx, dw and their mag."""
    dx, mdx = np.zeros_like(x), np.zeros_like(x)
    dw, mdw = np.zeros_like(w), np.zeros_like(w)
    for e, (lo, hi) in enumerate(zip(offsets[:-1], offsets[1:])):
        dx[lo:hi], mdx[lo:hi] = dy[lo:hi] @ w[e], np.abs(dy[lo:hi]) @ np.abs(w[e])
        dw[e], mdw[e] = dy[lo:hi].T @ x[lo:hi], np.abs(dy[lo:hi]).T @ np.abs(x[lo:hi])
    return {"dx": dx, "mag_dx": mdx, "dw": dw, "mag_dw": mdw}
