"""The body from token ids to expert products as a trainer runs it, forward and backward, on packed prefixes: embedding,
projection, head norms with rotation, attention, join, a product grouped by expert; compared with the same chain in
float64.  Shared by the GPU tests and the smoke check.

Bounds on relative Frobenius errors, fixed by the number of roundings on the way: a rounding to bfloat16 moves a tensor by
at most 2^-8 of its norm; forward there are nine (x, qkv, q and k turned, P, out, y, r, h, z), backward nine more (dh,
dr', dy, dout, dS and P, the turned gradients, dq and dk, dx), each amplified by at most the projections' and norms' gain,
which is near one for these inputs (orthonormal projections, weights near 1): 18 2^-8 = 0.07.  In float32 the same
count with 2^-24, times the length of the sums (1024 terms), stays under 1.1e-3.
"""
import numpy as np
import torch

from oracle import nat_body as ob
from oracle import nat_packed as op
from paper_2603_06619_b200 import nat
from paper_2603_06619_b200.body import PackedEmbedding, PackedExperts, PackedSublayer

BOUND = {torch.bfloat16: 0.07, torch.float32: 1.1e-3}


def _np(t):
    return t.detach().double().cpu().numpy()


def _err(got, ref):
    return float(np.linalg.norm(_np(got) - ref) / max(np.linalg.norm(ref), 1e-30))


def run_body(lengths, dtype, d=128, Hq=4, Hkv=2, D=32, V=211, E=3, n_out=64, R=None, interleaved=False, norm=True, seed=0):
    """Returns {name: relative error}; asserts the bounds and the untouched rows."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    cu_h = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    B, n_tot = len(lengths), int(cu_h[-1])
    cu = torch.from_numpy(cu_h).cuda()
    # the batch's prefixes
    mask = torch.empty(n_tot, dtype=torch.uint8, device="cuda")
    pi = torch.empty(n_tot, device="cuda")
    cut = torch.empty(B, dtype=torch.int32, device="cuda")
    idx, resp = (torch.empty(n_tot, dtype=torch.int32, device="cuda") for _ in range(2))
    offs = torch.empty(B + 1, dtype=torch.int32, device="cuda")
    n_sel = torch.empty(1, dtype=torch.int32, device="cuda")
    nat.nat_select(nat.select_params("rpc", min_cut=4, seed=seed), B, cu, n_tot, mask, pi, cut)
    nat.nat_compact_prefix(B, cu, n_tot, cut, idx, resp, offs, n_sel, n_tot)
    n = int(n_sel.item())

    heads = Hq + 2 * Hkv
    ortho = lambda a, b: torch.linalg.qr(rand(max(a, b), min(a, b)))[0].reshape(max(a, b), min(a, b))  # noqa: E731
    shaped = lambda m, a, b: (m if m.shape == (a, b) else m.t()).contiguous().to(dtype)  # noqa: E731
    w_qkv, w_o = shaped(ortho(d, heads * D), d, heads * D), shaped(ortho(Hq * D, d), Hq * D, d)
    w_e = torch.stack([shaped(ortho(n_out, d), n_out, d) for _ in range(E)])
    table = rand(V, d).to(dtype)
    ids = (torch.rand(n_tot, generator=g, device="cuda") ** 2 * V).to(torch.int32)
    w_post, w_pre, w_q, w_k = 1 + 0.1 * rand(d), 1 + 0.1 * rand(d), 1 + 0.1 * rand(D), 1 + 0.1 * rand(D)
    if not norm:
        w_q = w_k = None
    freq = nat.rope_freqs(D if R is None else R, 1e4)

    emb = PackedEmbedding(n_tot, V, d, dtype, scale=0.5)
    sub = PackedSublayer(n_tot, B, d, Hq, Hkv, D, dtype, alpha=0.9, ckpt8=False, rot_dim=R, interleaved=interleaved)
    exp = PackedExperts(n_tot, E, d, n_out, dtype)
    blank = lambda *s: torch.full(s, 7.0, device="cuda").to(dtype)  # noqa: E731
    for t in (sub.r, sub.h, sub.dx, sub.dy, sub.dqkv, sub.qk, sub.dqk):
        t.fill_(7.0)
    # the experts' rows: any routing will do
    of = torch.full((n_tot,), E, device="cuda")
    of[:n] = torch.randint(0, E, (n,), generator=g, device="cuda")
    order = of.argsort(stable=True).to(torch.int32)
    e_offs = torch.searchsorted(of[order.long()], torch.arange(E + 1, device="cuda")).to(torch.int32)

    # forward
    x = emb.lookup(table, ids, blank(n_tot, d), sel_idx=idx, n_rows=n_sel)
    qkv = (x @ w_qkv).view(n_tot, heads, D)
    qk = sub.rotate(qkv, offs, w_q, w_k, freq)
    y = sub.attend(qkv, offs, qk).view(n_tot, Hq * D) @ w_o
    r, h = sub.join(x, y, w_post, None, w_pre, n_sel)
    h_e, z_e, z = blank(n_tot, d), blank(n_tot, n_out), blank(n_tot, n_out)
    nat.nat_gather_rows(h, order, n_sel, n_tot, h_e)
    exp.forward(h_e, w_e, e_offs, z_e)
    nat.nat_scatter_rows(z_e, order, n_sel, n_tot, n_tot, z)
    # backward
    dr, dz = rand(n_tot, d).to(dtype), rand(n_tot, n_out).to(dtype)
    dz_e, dh_e, dh = blank(n_tot, n_out), blank(n_tot, d), blank(n_tot, d)
    dw_e = torch.full((E, n_out, d), 7.0, device="cuda")
    nat.nat_gather_rows(dz, order, n_sel, n_tot, dz_e)
    exp.backward(h_e, w_e, e_offs, dz_e, dh_e, dw_e)
    nat.nat_scatter_rows(dh_e, order, n_sel, n_tot, n_tot, dh)
    dx, dy = sub.join_backward(dr, dh, w_post, None, w_pre, n_sel, y=y)
    dout = (dy @ w_o.t()).view(n_tot, Hq, D)
    dqkv = sub.attend_backward(qkv, offs, dout, qk=qk)
    sub.rotate_backward(qkv, offs, w_q, w_k, freq, dqkv)
    dx_all = dx + dqkv.view(n_tot, heads * D) @ w_qkv.t()
    dtable = emb.gradient(ids, dx_all, torch.full((V, d), 7.0, device="cuda"), sel_idx=idx, n_rows=n_sel)
    assert sub.status() == 0 and emb.status() == 0 and exp.status() == 0
    for t in (sub.r, sub.h, sub.dx, sub.dy, sub.dqkv, sub.qk, sub.dqk, x, z_e, dh_e):
        assert (t[n:] == 7).all()

    # the same in float64
    po, rows = offs.cpu().numpy(), idx[:n].long()
    pos = np.arange(n) - np.repeat(po[:-1], np.diff(po))
    id_rows, O = ids[rows].cpu().numpy(), order[:n].long().cpu().numpy()
    Wq, Wo, We, F, eo = _np(w_qkv), _np(w_o), _np(w_e), _np(freq), e_offs.cpu().numpy()
    X = op.embed_fwd(_np(table), id_rows, 0.5)
    QKV = (X @ Wq).reshape(n, heads, D)
    Q, K, Vv = QKV[:, :Hq], QKV[:, Hq:Hq + Hkv], QKV[:, Hq + Hkv:]
    wq, wk = (None, None) if not norm else (_np(w_q), _np(w_k))
    Qt, Kt = op.qknorm_fwd(Q, wq, pos, F, 1e-6, interleaved)[0], op.qknorm_fwd(K, wk, pos, F, 1e-6, interleaved)[0]
    A, L, _ = ob.attn_fwd(Qt, Kt, Vv, po, D ** -0.5)
    Y = A.reshape(n, Hq * D) @ Wo
    f = ob.resnorm_fwd(X, Y, _np(w_post), None, _np(w_pre), 1e-6, 0.9, "none")
    Z = np.zeros((n, n_out))
    Z[O] = op.experts_fwd(f["h"][O], We, eo)[0]
    eb = op.experts_bwd(f["h"][O], We, _np(dz)[:n][O], eo)
    DH = np.zeros((n, d))
    DH[O] = eb["dx"]
    b = ob.resnorm_bwd(Y, f["r"], _np(w_post), None, _np(w_pre), f["rstd_y"], f["rstd_r"], _np(dr[:n]), DH, 0.9, "none")
    ab = ob.attn_bwd(Qt, Kt, Vv, A, L, (b["dy"] @ Wo.T).reshape(n, Hq, D), po, D ** -0.5)
    bq = op.qknorm_bwd(Q, wq, pos, F, 1e-6, interleaved, ab["dq"])
    bk = op.qknorm_bwd(K, wk, pos, F, 1e-6, interleaved, ab["dk"])
    DQKV = np.concatenate([bq["dx"], bk["dx"], ab["dv"]], axis=1)
    DX = b["dx"] + DQKV.reshape(n, heads * D) @ Wq.T
    err = {"x": _err(x[:n], X), "qk": _err(qk[:n], np.concatenate([Qt, Kt], axis=1)), "r": _err(r[:n], f["r"]),
           "z": _err(z[:n], Z), "dw_e": _err(dw_e, eb["dw"]), "dqkv": _err(dqkv[:n], DQKV),
           "dtable": _err(dtable, op.embed_bwd(DX, id_rows, V, 0.5)[0])}
    if norm:
        err.update(dw_q=_err(sub.dw_q, bq["dw"]), dw_k=_err(sub.dw_k, bk["dw"]))
    for name, e in err.items():
        assert e <= BOUND[dtype], (name, e, BOUND[dtype], err)
    return err
