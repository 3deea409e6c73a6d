"""The bounds on attention's gradients refuse what they are there to refuse (no GPU needed)."""
import numpy as np
import pytest
import torch

import body_bounds
from oracle import nat_body as ob


def _bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


def _f32(x):
    return x.astype(np.float32).astype(np.float64)


@pytest.fixture(scope="module", params=[32, 64, 96, 128])
def setting(request):
    D, r, cu = request.param, np.random.default_rng(1), np.array([0, 300, 420])
    n, Hq, Hkv, scale = 420, 4, 2, request.param ** -0.5
    q, k, v, do = 2 * r.normal(size=(n, Hq, D)), r.normal(size=(n, Hkv, D)), r.normal(size=(n, Hkv, D)), r.normal(size=(n, Hq, D))
    return [_f32(x) for x in (q, k, v, do)] + [cu, scale]


def _outside(name, got, ref, *where):
    over = np.abs(got - ref[name]) > body_bounds.element(name, ref, *where)
    far = np.linalg.norm(got - ref[name]) > body_bounds.norm(name, ref, *where)
    return over.any(), far


@pytest.mark.parametrize("bf16", [False, True])
def test_bounds_refuse_one_per_cent(setting, bf16):
    q, k, v, do, cu, scale = setting
    if bf16:
        q, k, v, do = (_bf16(x) for x in (q, k, v, do))
    out, lse, _ = ob.attn_fwd(q, k, v, cu, scale)
    out, lse = (_bf16 if bf16 else _f32)(out), _f32(lse)
    ref = ob.attn_bwd(q, k, v, out, lse, do, cu, scale)
    off = ob.attn_bwd(q, k, v, 1.01 * out, lse, do, cu, scale)      # delta off by 1 %
    for name in ("dq", "dk", "dv"):
        where = (q, k, lse, cu, scale, bf16)
        # what is right passes, rounded as the kernels round
        assert _outside(name, (_bf16 if bf16 else _f32)(ref[name]), ref, *where) == (False, False)
        over, far = _outside(name, 1.01 * ref[name], ref, *where)
        assert far and (over or bf16)
        if name != "dv" and not bf16:
            assert all(_outside(name, off[name], ref, *where))


def test_float32_bounds_refuse_inputs_rounded_to_bfloat16(setting):
    q, k, v, do, cu, scale = setting
    out, lse, _ = ob.attn_fwd(q, k, v, cu, scale)
    ref = ob.attn_bwd(q, k, v, _f32(out), _f32(lse), do, cu, scale)
    rounded = ob.attn_bwd(*(_bf16(x) for x in (q, k, v)), _f32(out), _f32(lse), _bf16(do), cu, scale)
    for name in ("dq", "dk", "dv"):
        assert all(_outside(name, rounded[name], ref, q, k, _f32(lse), cu, scale, False)), name


def test_bfloat16_norms_are_near_what_rounding_leaves(setting):
    """dS and P rounded to bfloat16 and the result once more, nothing else: inside the norm's bound, and above half
    of it, so the bound is not an idle one."""
    q, k, v, do, cu, scale = setting
    q, k, v, do = (_bf16(x) for x in (q, k, v, do))
    out, lse, _ = ob.attn_fwd(q, k, v, cu, scale)
    out, lse = _bf16(out), _f32(lse)
    ref = ob.attn_bwd(q, k, v, out, lse, do, cu, scale)
    got = {x: np.zeros_like(ref[x]) for x in ("dq", "dk", "dv")}
    for lo, hi in zip(cu[:-1], cu[1:]):
        for h in range(q.shape[1]):
            kh = h // 2
            S, seen = ob.attn_scores(q, k, h, scale, lo, hi)
            P = np.where(seen, np.exp(np.where(seen, S - lse[lo:hi, h, None], 0)), 0)
            dS = P * (do[lo:hi, h] @ v[lo:hi, kh].T - (do[lo:hi, h] * out[lo:hi, h]).sum(axis=1, keepdims=True))
            got["dq"][lo:hi, h] = scale * _bf16(dS) @ k[lo:hi, kh]
            got["dk"][lo:hi, kh] += scale * _bf16(dS).T @ q[lo:hi, h]
            got["dv"][lo:hi, kh] += _bf16(P).T @ do[lo:hi, h]
    for name in got:
        where = (q, k, lse, cu, scale, True)
        err = np.linalg.norm(_bf16(got[name]) - ref[name])
        assert 0.4 * body_bounds.norm(name, ref, *where) < err < body_bounds.norm(name, ref, *where), name
        assert (np.abs(_bf16(got[name]) - ref[name]) <= body_bounds.element(name, ref, *where)).all()
