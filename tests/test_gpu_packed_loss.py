"""A policy whose table is both its embedding and the loss's output projection, with a product grouped by expert between: from token
ids to the loss on packed prefixes, and back to one table gradient from both its ends.  Against float64.

Bounds on relative Frobenius errors: the loss's own 1e-2 on its gradients (see ``parity.py``) and, beside it, the roundings to
bfloat16 on the way (x, z, dHidden, dx: four of 2^-8; the coefficients exp(logp - old) follow the logits, whose rows carry two
of them, with deviations near one: two more); in float32 nothing of the kind.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import nat_packed as op
from paper_2603_06619_b200 import nat
from paper_2603_06619_b200.body import PackedEmbedding, PackedExperts
from paper_2603_06619_b200.step import NatStep

pytestmark = pytest.mark.gpu


def _np(t):
    return t.detach().double().cpu().numpy()


def _err(got, ref):
    return float(np.linalg.norm(_np(got) - ref) / np.linalg.norm(ref))


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_from_ids_to_the_loss_and_back(dtype, fused):
    P, G, d, V, E = 3, 4, 128, 500, 5
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    lengths = [40, 1, 77, 9, 130, 25, 64, 3, 51, 18, 90, 33]
    cu_h = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    cu, n_tot, B = torch.from_numpy(cu_h).cuda(), int(cu_h[-1]), P * G
    ids, targets = (torch.randint(0, V, (n_tot,), generator=g, device="cuda").to(torch.int32) for _ in range(2))
    table = (0.3 * rand(V, d)).to(dtype)
    w_e = torch.stack([torch.linalg.qr(rand(d, d))[0] for _ in range(E)]).to(dtype)

    st = NatStep(P, G, d, V, dtype, n_tot, hidden_is_compact=True)
    st.grpo_adv(rand(B))
    st.select(cu, "rpc", min_cut=4, seed=5)
    st.compact(cu)
    n = int(st.n_sel.item())
    look = PackedEmbedding(n_tot, V, d, dtype, scale=2.0)
    back = PackedEmbedding(n_tot, V, d, dtype, scale=2.0, accumulate=True)
    exp = PackedExperts(n_tot, E, d, d, dtype)
    of = torch.full((n_tot,), E, device="cuda")
    of[:n] = torch.randint(0, E, (n,), generator=g, device="cuda")
    order = of.argsort(stable=True).to(torch.int32)
    offs = torch.searchsorted(of[order.long()], torch.arange(E + 1, device="cuda")).to(torch.int32)
    blank = lambda *s: torch.full(s, 7.0, device="cuda").to(dtype)  # noqa: E731

    # the same in float64, whose log-probabilities, a little off, are the old policy's: no ratio is near a clip
    rows, O, eo = st.sel_idx[:n].long().cpu().numpy(), order[:n].long().cpu().numpy(), offs.cpu().numpy()
    of_rows = _np(ids).astype(int)[rows]
    W, We = _np(table), _np(w_e)
    X = op.embed_fwd(W, of_rows, 2.0)
    Z = np.zeros((n, d))
    Z[O] = op.experts_fwd(X[O], We, eo)[0]
    where = (_np(st.adv), _np(st.pi), cu_h, rows, _np(st.sel_resp[:n]).astype(int))
    old = np.zeros(n_tot)
    first = oracle.policy_loss_fwd(Z, W, _np(targets).astype(int), old, *where, hidden_is_compact=True)
    old[rows] = first["logp"] + np.random.default_rng(0).uniform(-0.05, 0.05, n)
    old_logp = torch.from_numpy(old).float().cuda()
    ref = oracle.policy_loss_bwd(Z, W, _np(targets).astype(int), _np(old_logp), *where, hidden_is_compact=True)
    eb = op.experts_bwd(X[O], We, ref["dH"][O], eo)
    DX = np.zeros((n, d))
    DX[O] = eb["dx"]
    DT = ref["dW"] + op.embed_bwd(DX, of_rows, V, 2.0)[0]

    x = look.lookup(table, ids, blank(n_tot, d), sel_idx=st.sel_idx, n_rows=st.n_sel)
    x_e, z_e, z, dz_e, dx_e, dx = (blank(n_tot, d) for _ in range(6))
    nat.nat_gather_rows(x, order, st.n_sel, n_tot, x_e)
    exp.forward(x_e, w_e, offs, z_e)
    nat.nat_scatter_rows(z_e, order, st.n_sel, n_tot, n_tot, z)
    if fused:
        st.loss_fwd_bwd(z, table, targets, old_logp, cu)
    else:
        st.loss_fwd(z, table, targets, old_logp, cu)
        st.loss_bwd(z, table, targets, old_logp, cu)
    nat.nat_gather_rows(st.dH, order, st.n_sel, n_tot, dz_e)
    dw_e = torch.full((E, d, d), 7.0, device="cuda")
    exp.backward(x_e, w_e, offs, dz_e, dx_e, dw_e)
    nat.nat_scatter_rows(dx_e, order, st.n_sel, n_tot, n_tot, dx)
    back.gradient(ids, dx, st.dW, sel_idx=st.sel_idx, n_rows=st.n_sel)
    assert st.status() & ~nat.NAT_DEV_FALLBACK == 0 and look.status() == 0 and back.status() == 0 and exp.status() == 0

    bound = 1e-2 + (6 * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    err = {"z": _err(z[:n], Z), "dH": _err(st.dH[:n], ref["dH"]), "dw_e": _err(dw_e, eb["dw"]), "dtable": _err(st.dW, DT)}
    assert all(e <= bound for e in err.values()), err
    # neither end's part is missing
    assert np.linalg.norm(DT - ref["dW"]) > 10 * bound * np.linalg.norm(DT) and np.linalg.norm(ref["dW"]) > 10 * bound * np.linalg.norm(DT)
    assert abs(float(st.loss.item()) - ref["loss"]) <= bound * float(np.sum(ref["w"] * np.abs(ref["L"])))
