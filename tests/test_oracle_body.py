"""Pins of the float64 forms of the transformer body's operators: closed forms and differences."""
import numpy as np
import pytest

from oracle import nat_body as ob


def _attn_inputs(seed, lengths, Hq, Hkv, D):
    r = np.random.default_rng(seed)
    cu = np.concatenate([[0], np.cumsum(lengths)])
    n = int(cu[-1])
    return r, cu, r.normal(size=(n, Hq, D)), r.normal(size=(n, Hkv, D)), r.normal(size=(n, Hkv, D))


def test_attn_closed_forms():
    r, cu, q, k, v = _attn_inputs(0, [3, 0, 1, 5], 4, 2, 8)
    out, lse, _ = ob.attn_fwd(q, k, v, cu, 0.3)
    # the first token of a sequence attends to itself alone
    for lo in (0, 3, 4):
        assert np.allclose(out[lo], np.repeat(v[lo], 2, axis=0))
        assert np.allclose(lse[lo], 0.3 * (q[lo] * np.repeat(k[lo], 2, axis=0)).sum(-1))
    # equal keys: the running mean of the values
    out, lse, _ = ob.attn_fwd(q, np.zeros_like(k), v, cu, 0.3)
    assert np.allclose(out[4:9, 0], np.cumsum(v[4:9, 0], axis=0) / np.arange(1, 6)[:, None])
    assert np.allclose(lse[4:9], np.log(np.arange(1, 6))[:, None])


def test_attn_gradient_against_differences():
    r, cu, q, k, v = _attn_inputs(1, [4, 0, 1, 6], 4, 2, 8)
    w = r.normal(size=q.shape)
    f = lambda q, k, v: float((w * ob.attn_fwd(q, k, v, cu, 0.4)[0]).sum())  # noqa: E731
    out, lse, _ = ob.attn_fwd(q, k, v, cu, 0.4)
    got = ob.attn_bwd(q, k, v, out, lse, w, cu, 0.4)
    for name, which in (("dq", 0), ("dk", 1), ("dv", 2)):
        for _ in range(3):
            step = r.normal(size=(q, k, v)[which].shape)
            lo, hi = [q, k, v], [q, k, v]
            lo[which], hi[which] = lo[which] - 1e-5 * step, hi[which] + 1e-5 * step
            assert (f(*hi) - f(*lo)) / 2e-5 == pytest.approx(float((got[name] * step).sum()), rel=1e-6, abs=1e-7)


@pytest.mark.parametrize("gate_mode", ["none", "channel", "row"])
@pytest.mark.parametrize("parts", ["all", "no_post", "no_pre", "no_y"])
def test_resnorm_gradient_against_differences(gate_mode, parts):
    if parts == "no_y" and gate_mode != "none":
        return
    r = np.random.default_rng(2)
    n, d, eps, alpha = 5, 24, 1e-3, 0.7
    a = dict(x=r.normal(size=(n, d)), y=None if parts == "no_y" else r.normal(size=(n, d)),
             w_post=None if parts in ("no_post", "no_y") else r.normal(size=d),
             gate=None if gate_mode == "none" else r.normal(size=d if gate_mode == "channel" else n),
             w_pre=None if parts == "no_pre" else r.normal(size=d))
    cr, ch = r.normal(size=(n, d)), r.normal(size=(n, d))

    def f(**kw):
        o = ob.resnorm_fwd(**kw, eps=eps, alpha=alpha, gate_mode=gate_mode)
        return float((cr * o["r"]).sum() + ((ch * o["h"]).sum() if "h" in o else 0.0))

    o = ob.resnorm_fwd(**a, eps=eps, alpha=alpha, gate_mode=gate_mode)
    got = ob.resnorm_bwd(a["y"], o["r"], a["w_post"], a["gate"], a["w_pre"], o.get("rstd_y"),
                         o.get("rstd_r"), cr, ch, alpha, gate_mode)
    for name in ("x", "y", "w_post", "gate", "w_pre"):
        if a[name] is None:
            continue
        key = "d" + name
        step = r.normal(size=a[name].shape)
        hi, lo = dict(a), dict(a)
        hi[name], lo[name] = a[name] + 1e-5 * step, a[name] - 1e-5 * step
        assert (f(**hi) - f(**lo)) / 2e-5 == pytest.approx(float((got[key] * step).sum()), rel=1e-6, abs=1e-7)


def test_ckpt8_grid_and_special_groups():
    r = np.random.default_rng(3)
    x = r.normal(size=(9, 200)).astype(np.float32)
    x[1], x[2, :128], x[3, 5], x[4, 150] = 0.0, 1e-38, np.inf, np.nan
    codes, scales = ob.ckpt8_store(x)
    back = ob.ckpt8_load(codes, scales)
    assert scales.shape == (9, 2) and codes.dtype == np.int8
    assert (back[1] == 0).all() and (back[2, :128] == 0).all() and (scales[2, 1] > 0)
    assert np.isnan(back[3, :128]).all() and np.isfinite(back[3, 128:]).all()
    assert np.isnan(back[4, 128:]).all() and np.isfinite(back[4, :128]).all()
    fine = np.isfinite(back)
    step = np.repeat(scales, 128, axis=1)[:, :200]
    assert (np.abs(back - x)[fine] <= 0.5001 * step[fine] + 1e-37).all()
    assert np.abs(codes).max() == 127
