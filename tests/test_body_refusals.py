"""What the transformer body's entry points refuse, before any device work (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2603_06619_b200 import nat

A, ODD = 4096, 4096 + 8            # fake device addresses: nothing is dereferenced


def _attn(lib, p, back=False, B=2, cap=64, ptrs=None, ws=A, ws_bytes=1 << 30):
    ptrs = [A] * (9 if back else 5) if ptrs is None else ptrs
    fn = lib.nat_attn_bwd if back else lib.nat_attn_fwd
    return fn(ctypes.byref(p) if p is not None else None, B, A, cap, *ptrs, ws, ws_bytes, None)


def test_attn_refusals():
    lib = nat.load()
    ok = lambda **kw: _with(nat.attn_params(8, 2, 64, torch.bfloat16), **kw)  # noqa: E731
    assert lib.nat_attn_workspace_bytes(ctypes.byref(ok()), 2, 64) > 0
    bad = [(dict(n_heads=7), -1), (dict(n_heads=0), -1), (dict(head_dim=0), -1),
           (dict(head_dim=12), -2), (dict(head_dim=136), -2), (dict(dtype=9), -2),
           (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
           (dict(q_stride=504), -1), (dict(k_stride=120), -1), (dict(o_stride=516), -2),
           (dict(v_stride=-128), -1), (dict(q_stride=1 << 31), -2),
           (dict(n_heads=130, q_stride=8320, o_stride=8320), -2)]
    for kw, status in bad:
        assert lib.nat_attn_workspace_bytes(ctypes.byref(ok(**kw)), 2, 64) == 0, kw
        for back in (False, True):
            assert _attn(lib, ok(**kw), back) == status, kw
    for back in (False, True):
        assert _attn(lib, None, back) == -1
        assert _attn(lib, ok(), back, B=-1) == -1
        assert _attn(lib, ok(), back, cap=-1) == -1
        assert _attn(lib, ok(), back, cap=1 << 31) == -1
        assert _attn(lib, ok(), back, ws_bytes=256) == -3
        assert _attn(lib, ok(), back, ws=A + 16) == -1
        assert _attn(lib, ok(), back, ws=None) == -3
        n = 9 if back else 5
        for i in range(n):
            ptrs = [A] * n
            ptrs[i] = None
            assert _attn(lib, ok(), back, ptrs=ptrs) == -1
            if i != (4 if back else 4):          # lse needs no more than its type's alignment
                ptrs[i] = ODD
                assert _attn(lib, ok(), back, ptrs=ptrs) == -1
        # nothing to do: no pointer is looked at
        assert _attn(lib, ok(), back, B=0, ptrs=[None] * n) == 0
        assert _attn(lib, ok(), back, cap=0, ptrs=[None] * n) == 0


def _with(p, **kw):
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _fwd(lib, p, cap=8, n_rows=None, ckpt=(None,) * 4, **kw):
    a = dict(x=A, y=A, w_post=A, gate=None, w_pre=A, r=A, h=A, ry=A, rr=A)
    a.update(kw)
    return lib.nat_resnorm_fwd(ctypes.byref(p) if p is not None else None, a["x"], a["y"], a["w_post"],
                               a["gate"], a["w_pre"], n_rows, cap, a["r"], a["h"], a["ry"], a["rr"],
                               *ckpt, None)


def _bwd(lib, p, cap=8, ckpt=(None,) * 4, ws=A, nbytes=1 << 30, **kw):
    a = dict(y=A, r=A, w_post=A, gate=None, w_pre=A, ry=A, rr=A, dr=A, dh=A, dx=A, dy=A, dw_post=A,
             dgate=None, dw_pre=A)
    a.update(kw)
    return lib.nat_resnorm_bwd(ctypes.byref(p), a["y"], a["r"], *ckpt, a["w_post"], a["gate"],
                               a["w_pre"], a["ry"], a["rr"], None, cap, a["dr"], a["dh"], a["dx"],
                               a["dy"], a["dw_post"], a["dgate"], a["dw_pre"], ws, nbytes, None)


def test_resnorm_refusals():
    lib = nat.load()
    ok = lambda **kw: _with(nat.resnorm_params(64, torch.bfloat16), **kw)  # noqa: E731
    for kw, status in [(dict(d=0), -1), (dict(d=12), -2), (dict(d=8200), -2), (dict(dtype=5), -2),
                       (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
                       (dict(alpha=float("inf")), -1), (dict(gate_mode=3), -1)]:
        assert _fwd(lib, ok(**kw)) == status and _bwd(lib, ok(**kw)) == status, kw
        assert lib.nat_resnorm_workspace_bytes(ctypes.byref(ok(**kw)), 8) == 0
    assert _fwd(lib, None) == -1 and _fwd(lib, ok(), cap=-1) == -1 and _fwd(lib, ok(), cap=1 << 31) == -1
    assert _fwd(lib, ok(), cap=0, x=None, r=None) == 0
    for name in ("x", "r", "h", "ry", "rr"):
        assert _fwd(lib, ok(), **{name: None}) == -1, name
    for name in ("x", "y", "w_post", "w_pre", "r", "h"):
        assert _fwd(lib, ok(), **{name: ODD}) == -1, name
    assert _fwd(lib, ok(), y=None) == -1                               # w_post without y
    assert _fwd(lib, ok(), gate=A) == -1 and _fwd(lib, ok(gate_mode=1)) == -1
    assert _fwd(lib, ok(gate_mode=1), gate=ODD) == -1
    assert _fwd(lib, ok(), ckpt=(A, A, A, None)) == -1
    assert _fwd(lib, ok(), ckpt=(A, A, None, None)) == -1
    assert _fwd(lib, ok(), ckpt=(A, A, ODD, A)) == -1
    for name in ("y", "r", "ry", "rr", "dh", "dx", "dy", "dw_post", "dw_pre"):
        assert _bwd(lib, ok(), **{name: None}) == -1, name
    for name in ("y", "r", "dr", "dh", "dx", "dy", "w_post", "w_pre"):
        assert _bwd(lib, ok(), **{name: ODD}) == -1, name
    assert _bwd(lib, ok(), ckpt=(A, A, A, A)) == -1                     # rows and checkpoints
    assert _bwd(lib, ok(), r=None, ckpt=(None, None, A, A)) == -1       # one of each
    assert _bwd(lib, ok(), y=None, r=None, ckpt=(A, None, A, A)) == -1
    assert _bwd(lib, ok(), w_pre=None, dw_pre=None, dr=None) == -1
    assert _bwd(lib, ok(gate_mode=2), gate=A) == -1                     # dgate missing
    assert _bwd(lib, ok(), nbytes=64) == -3 and _bwd(lib, ok(), ws=A + 4) == -1


def test_ckpt8_refusals():
    lib = nat.load()
    s = lambda dt=0, d=64, src=A, cap=8, c=A, sc=A: lib.nat_ckpt8_store(dt, d, src, None, cap, c, sc, None)  # noqa: E731
    ld = lambda dt=0, d=64, dst=A, cap=8, c=A, sc=A: lib.nat_ckpt8_load(dt, d, c, sc, None, cap, dst, None)  # noqa: E731
    for f, x in ((s, "src"), (ld, "dst")):
        assert f(dt=7) == -2 and f(d=0) == -1 and f(d=20) == -2 and f(cap=-1) == -1
        assert f(d=(1 << 20) + 8) == -2 and f(cap=1 << 31) == -1
        assert f(**{x: None}) == -1 and f(c=None) == -1 and f(sc=None) == -1
        assert f(**{x: ODD}) == -1 and f(c=ODD) == -1 and f(sc=A + 2) == -1
        assert f(cap=0, c=None) == 0


def test_binding_refuses_host_tensors_and_wrong_types():
    p = nat.attn_params(2, 1, 8, torch.float32)
    t = torch.zeros(4, 2, 8)
    with pytest.raises(nat.NatError, match="not on the current CUDA device|expected"):
        nat.nat_attn_fwd(p, 1, torch.zeros(2, dtype=torch.int32), 4, t, t[:, :1], t[:, :1], t,
                         torch.zeros(4, 2), torch.zeros(4096, dtype=torch.uint8))
    with pytest.raises(nat.NatError, match="expected torch.float32"):
        nat.nat_attn_fwd(p, 1, torch.zeros(2, dtype=torch.int32), 4, t.double(), t[:, :1], t[:, :1],
                         t, torch.zeros(4, 2), torch.zeros(4096, dtype=torch.uint8))
    with pytest.raises(nat.NatError):
        nat.nat_ckpt8_store(torch.zeros(4, 8), None, 4, torch.zeros(4, 8, dtype=torch.int8),
                            torch.zeros(4, 1))
