"""The body's operators as a trainer runs them: a prefix-cut batch is selected, compacted and packed, one
attention sublayer runs forward and backward on the packed prefixes, and everything is compared with the
same chain in float64.  Shared by the GPU tests and the smoke check.

Bounds on relative Frobenius errors, fixed by the number of roundings on the way: a rounding to
bfloat16 moves a tensor by at most 2^-8 of its norm; the forward chain to h has seven of them (the
packed rows, qkv, P, out, y, r, h), the backward chain to dqkv eight more (dr', dy, dout, dS and P, the
products' results, and what it reads: y, r, out), each amplified by at most the projections' and norms'
gain, which for these inputs (orthonormal projections, weights near 1) is near one: 15 2^-8 = 0.06.
An 8-bit checkpoint adds half of a 127th of a group's top, under four times its rms: 0.016 each.  In float32 the
same count with 2^-24, times the length of the sums (1024 terms), stays under 1e-3.
"""
import numpy as np
import torch

from oracle import nat_body as ob
from paper_2603_06619_b200 import nat
from paper_2603_06619_b200.body import PackedSublayer

BOUND = {torch.bfloat16: 0.06, torch.float32: 1e-3}


def _np(t):
    return t.detach().double().cpu().numpy()


def _err(got, ref):
    return float(np.linalg.norm(_np(got) - ref) / max(np.linalg.norm(ref), 1e-30))


def run_sublayer(lengths, dtype, d=128, Hq=4, Hkv=2, D=32, gate="channel", ckpt8=True, min_cut=4, seed=0):
    """Returns {name: relative error}; asserts the bounds and the untouched rows."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    cu_h = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    B, n_tot = len(lengths), int(cu_h[-1])
    cu = torch.from_numpy(cu_h).cuda()
    # the batch: prefix cutting, compaction, and the packed rows of the residual stream and the
    # normed input
    mask = torch.empty(n_tot, dtype=torch.uint8, device="cuda")
    pi = torch.empty(n_tot, device="cuda")
    cut = torch.empty(B, dtype=torch.int32, device="cuda")
    idx, resp = (torch.empty(n_tot, dtype=torch.int32, device="cuda") for _ in range(2))
    offs = torch.empty(B + 1, dtype=torch.int32, device="cuda")
    n_sel = torch.empty(1, dtype=torch.int32, device="cuda")
    nat.nat_select(nat.select_params("rpc", min_cut=min_cut, seed=seed), B, cu, n_tot, mask, pi, cut)
    nat.nat_compact_prefix(B, cu, n_tot, cut, idx, resp, offs, n_sel, n_tot)
    x_all, h_all = rand(n_tot, d).to(dtype), rand(n_tot, d).to(dtype)
    x, h = (torch.full_like(x_all, float("nan")) for _ in range(2))
    nat.nat_gather_rows(x_all, idx, n_sel, n_tot, x)
    nat.nat_gather_rows(h_all, idx, n_sel, n_tot, h)

    heads = Hq + 2 * Hkv
    ortho = lambda a, b: torch.linalg.qr(rand(max(a, b), min(a, b)))[0].reshape(max(a, b), min(a, b))  # noqa: E731
    w_qkv = ortho(d, heads * D)
    w_qkv = (w_qkv if w_qkv.shape == (d, heads * D) else w_qkv.t()).contiguous().to(dtype)
    w_o = ortho(Hq * D, d)
    w_o = (w_o if w_o.shape == (Hq * D, d) else w_o.t()).contiguous().to(dtype)
    w_post, w_pre = 1 + 0.1 * rand(d), 1 + 0.1 * rand(d)
    gates = {"none": None, "channel": 0.5 + 0.1 * rand(d), "row": torch.sigmoid(rand(n_tot))}
    sub = PackedSublayer(n_tot, B, d, Hq, Hkv, D, dtype, gate=gate, alpha=0.9, ckpt8=ckpt8)
    for t in (sub.r, sub.h, sub.dx, sub.dy, sub.dqkv):
        t.fill_(7.0)

    # forward; the rows behind the prefixes hold NaN all the way
    qkv = (h @ w_qkv).view(n_tot, heads, D)
    out = sub.attend(qkv, offs)
    y = out.view(n_tot, Hq * D) @ w_o
    r, h_next = sub.join(x, y, w_post, gates[gate], w_pre, n_sel)
    # backward
    dr, dh = rand(n_tot, d).to(dtype), rand(n_tot, d).to(dtype)
    dx, dy = sub.join_backward(dr, dh, w_post, gates[gate], w_pre, n_sel, y=y)
    dout = (dy @ w_o.t()).view(n_tot, Hq, D)
    dqkv = sub.attend_backward(qkv, offs, dout)
    assert sub.status() == 0
    n = int(n_sel.item())
    assert n == int(mask.sum().item())
    for t in (sub.r, sub.h, sub.dx, sub.dy, sub.dqkv):
        assert (t[n:] == 7).all()

    # the same in float64
    po = offs.cpu().numpy()
    H, X = _np(h[:n]), _np(x[:n])
    QKV = (H @ _np(w_qkv)).reshape(n, heads, D)
    Q, K, V = QKV[:, :Hq], QKV[:, Hq:Hq + Hkv], QKV[:, Hq + Hkv:]
    O, L, _ = ob.attn_fwd(Q, K, V, po, D ** -0.5)
    Y = O.reshape(n, Hq * D) @ _np(w_o)
    G = None if gate == "none" else _np(gates[gate])[: n if gate == "row" else d]
    f = ob.resnorm_fwd(X, Y, _np(w_post), G, _np(w_pre), 1e-6, 0.9, gate)
    b = ob.resnorm_bwd(Y, f["r"], _np(w_post), G, _np(w_pre), f["rstd_y"], f["rstd_r"], _np(dr[:n]), _np(dh[:n]),
                       0.9, gate)
    DO = (b["dy"] @ _np(w_o).T).reshape(n, Hq, D)
    a = ob.attn_bwd(Q, K, V, O, L, DO, po, D ** -0.5)
    err = {"r": _err(r[:n], f["r"]), "h": _err(h_next[:n], f["h"]), "dx": _err(dx[:n], b["dx"]),
           "dy": _err(dy[:n], b["dy"]), "dw_post": _err(sub.dw_post, b["dw_post"]),
           "dw_pre": _err(sub.dw_pre, b["dw_pre"]),
           "dqkv": _err(dqkv[:n], np.concatenate([a["dq"], a["dk"], a["dv"]], axis=1))}
    if gate != "none":
        err["dgate"] = _err(sub.dgate[: n if gate == "row" else d], b["dgate"])
    backward = ("dx", "dy", "dw_post", "dw_pre", "dqkv", "dgate")
    for name, e in err.items():
        bound = BOUND[dtype] + (0.032 if ckpt8 and name in backward else 0.0)
        assert e <= bound, (name, e, bound, err)
    return err
