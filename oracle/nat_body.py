"""Plain float64 numpy form of the operators of the packed transformer body.

Causal attention over packed sequences with grouped heads, the residual join with its norms, and
8-bit activation checkpoints; forward and backward, straight from the formulas in ``include/nat.h``.
Shares nothing with the CUDA path.
"""
import numpy as np

GROUP8 = 128


def _spans(cu, cap):
    return [(int(min(lo, cap)), int(min(hi, cap))) for lo, hi in zip(cu[:-1], cu[1:])]


def attn_scores(q, k, i_head, scale, lo, hi):
    """(S, seen) of one sequence and query head; entries above the diagonal are not seen."""
    Hq, Hkv = q.shape[1], k.shape[1]
    S = scale * np.matmul(q[lo:hi, i_head], k[lo:hi, i_head // (Hq // Hkv)].T)
    return S, np.tril(np.ones(S.shape, dtype=bool))


def attn_fwd(q, k, v, cu, scale):
    """(out, lse, absolute) with absolute = sum_j P_ij |v_j|, the scale of the rounding errors."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n, Hq, D = q.shape
    g = Hq // k.shape[1]
    out, absolute = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    lse = np.zeros((n, Hq))
    for lo, hi in _spans(cu, n):
        if hi <= lo:
            continue
        for h in range(Hq):
            S, seen = attn_scores(q, k, h, scale, lo, hi)
            S = np.where(seen, S, -np.inf)
            top = S.max(axis=1, keepdims=True)
            e = np.exp(S - top)
            lse[lo:hi, h] = top[:, 0] + np.log(e.sum(axis=1))
            P = e / e.sum(axis=1, keepdims=True)
            out[lo:hi, h] = P @ v[lo:hi, h // g]
            absolute[lo:hi, h] = P @ np.abs(v[lo:hi, h // g])
    return out, lse, absolute


def attn_bwd(q, k, v, out, lse, dout, cu, scale):
    """dict of dq, dk, dv and, under "abs_" names, the sums of the magnitudes of their terms.

    What rounding errors are measured by, each kind by itself: "terms_", the sums of |dS| |k| (or |q|, or P |dout|);
    "parts_", the same with what dP and delta are summed from in place of |dS|; "squares_", the sums of the
    terms' squares."""
    q, k, v, out, lse, dout = (np.asarray(x, dtype=np.float64) for x in (q, k, v, out, lse, dout))
    n, Hq, D = q.shape
    g = Hq // k.shape[1]
    kinds = ("", "abs_", "terms_", "parts_", "squares_")
    r = {m + x: np.zeros_like(y) for m in kinds for x, y in (("dq", q), ("dk", k), ("dv", v))}
    for lo, hi in _spans(cu, n):
        if hi <= lo:
            continue
        for h in range(Hq):
            kh = h // g
            S, seen = attn_scores(q, k, h, scale, lo, hi)
            P = np.where(seen, np.exp(np.where(seen, S - lse[lo:hi, h, None], 0.0)), 0.0)
            do, V = dout[lo:hi, h], v[lo:hi, kh]
            delta = (do * out[lo:hi, h]).sum(axis=1, keepdims=True)
            dS = P * (do @ V.T - delta)
            # what dP and delta are summed from: their own rounding is relative to this
            aS = P * (np.abs(do) @ np.abs(V).T + (np.abs(do) * np.abs(out[lo:hi, h])).sum(axis=1, keepdims=True))
            r["dq"][lo:hi, h] = scale * dS @ k[lo:hi, kh]
            r["dk"][lo:hi, kh] += scale * dS.T @ q[lo:hi, h]
            r["dv"][lo:hi, kh] += P.T @ do
            mag = np.abs(dS) + 2.0 ** -12 * aS
            r["abs_dq"][lo:hi, h] = abs(scale) * mag @ np.abs(k[lo:hi, kh])
            r["abs_dk"][lo:hi, kh] += abs(scale) * mag.T @ np.abs(q[lo:hi, h])
            r["abs_dv"][lo:hi, kh] += P.T @ np.abs(do)
            for kind, w, e in (("terms_", np.abs(dS), 1), ("parts_", aS, 1), ("squares_", dS * dS, 2)):
                r[kind + "dq"][lo:hi, h] = abs(scale) ** e * w @ np.abs(k[lo:hi, kh]) ** e
                r[kind + "dk"][lo:hi, kh] += abs(scale) ** e * w.T @ np.abs(q[lo:hi, h]) ** e
            r["terms_dv"][lo:hi, kh] += P.T @ np.abs(do)
            r["squares_dv"][lo:hi, kh] += (P * P).T @ (do * do)
    return r


def resnorm_fwd(x, y, w_post, gate, w_pre, eps, alpha, gate_mode):
    """dict r, h, rstd_y, rstd_r; `gate_mode` "none", "channel" or "row"; None leaves a part out."""
    x = np.asarray(x, dtype=np.float64)
    res = {}
    r = alpha * x
    if y is not None:
        n = np.asarray(y, dtype=np.float64)
        if w_post is not None:
            res["rstd_y"] = 1.0 / np.sqrt((n * n).mean(axis=1) + eps)
            n = n * res["rstd_y"][:, None] * np.asarray(w_post, dtype=np.float64)
        r = r + _gate(gate, gate_mode) * n
    res["r"] = r
    if w_pre is not None:
        res["rstd_r"] = 1.0 / np.sqrt((r * r).mean(axis=1) + eps)
        res["h"] = r * res["rstd_r"][:, None] * np.asarray(w_pre, dtype=np.float64)
    return res


def _gate(gate, mode):
    if mode == "none":
        return 1.0
    gate = np.asarray(gate, dtype=np.float64)
    return gate[None, :] if mode == "channel" else gate[:, None]


def resnorm_bwd(y, r, w_post, gate, w_pre, rstd_y, rstd_r, dr, dh, alpha, gate_mode):
    """dict dx, dy, dw_post, dgate, dw_pre (those that apply)."""
    res = {}
    f = lambda t: None if t is None else np.asarray(t, dtype=np.float64)  # noqa: E731
    y, r, w_post, w_pre, rstd_y, rstd_r, dr, dh = map(f, (y, r, w_post, w_pre, rstd_y, rstd_r, dr, dh))
    total = np.zeros_like(dh if dr is None else dr) if dr is None else dr
    if w_pre is not None:
        rhat = r * rstd_r[:, None]
        u = dh * w_pre
        total = total + rstd_r[:, None] * (u - rhat * (u * rhat).mean(axis=1, keepdims=True))
        res["dw_pre"] = (dh * rhat).sum(axis=0)
    res["dx"] = alpha * total
    if y is not None:
        yhat = y if w_post is None else y * rstd_y[:, None]
        n = yhat if w_post is None else yhat * w_post
        dn = _gate(gate, gate_mode) * total
        if gate_mode != "none":
            res["dgate"] = (total * n).sum(axis=0 if gate_mode == "channel" else 1)
        if w_post is None:
            res["dy"] = dn
        else:
            v = dn * w_post
            res["dw_post"] = (dn * yhat).sum(axis=0)
            res["dy"] = rstd_y[:, None] * (v - yhat * (v * yhat).mean(axis=1, keepdims=True))
    return res


def ckpt8_store(x):
    """(codes int8, scales float32): the float32 operations of the definition, each rounded once."""
    x = np.asarray(x, dtype=np.float32)
    n, d = x.shape
    groups = (d + GROUP8 - 1) // GROUP8
    codes, scales = np.zeros((n, d), dtype=np.int8), np.zeros((n, groups), dtype=np.float32)
    for i in range(groups):
        part = x[:, i * GROUP8:(i + 1) * GROUP8]
        top = np.abs(part).max(axis=1)              # a NaN wins
        fine = np.isfinite(top)
        kept = fine & (top >= np.float32(2.0 ** -120))
        # the reciprocal of the mantissa, so that it is rounded to 24 bits for every top
        mant, expo = np.frexp(np.where(kept, top, np.float32(1.0)))
        inv = np.ldexp(np.float32(1.0) / mant * np.float32(127.0), -expo)
        with np.errstate(invalid="ignore", over="ignore"):
            q = np.rint(np.where(kept[:, None], part, np.float32(0.0)) * inv[:, None])
        codes[:, i * GROUP8:(i + 1) * GROUP8] = q.astype(np.int8)
        scales[:, i] = np.where(kept, np.where(fine, top, 0) / np.float32(127.0),
                                np.where(fine, np.float32(0.0), np.float32(np.nan)))
    return codes, scales


def ckpt8_load(codes, scales):
    """float32 values, before the rounding to the rows' type."""
    d = codes.shape[1]
    return codes.astype(np.float32) * np.repeat(scales, GROUP8, axis=1)[:, :d]
