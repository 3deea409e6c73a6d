"""What the entry points around the packed attention refuse, before any device work (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2603_06619_b200 import nat

A, ODD = 4096, 4096 + 8            # fake device addresses: nothing is dereferenced


def _with(p, **kw):
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _ref(p):
    return None if p is None else ctypes.byref(p)


# -------------------------------------------------------------------------- embedding
def _embed_fwd(p, cap=8, **kw):
    a = dict(dict(table=A, ids=A, sel=None, n=None, x=A), **kw)
    return nat.load().nat_embed_fwd(_ref(p), a["table"], a["ids"], a["sel"], a["n"], cap, a["x"], None)


def _embed_bwd(p, cap=8, ws=A, nbytes=1 << 30, **kw):
    a = dict(dict(ids=A, sel=None, n=None, dx=A, dtable=A), **kw)
    return nat.load().nat_embed_bwd(_ref(p), a["ids"], a["sel"], a["n"], cap, a["dx"], a["dtable"], ws, nbytes, None)


def test_embed_refusals():
    ok = lambda **kw: _with(nat.embed_params(100, 64, torch.bfloat16), **kw)  # noqa: E731
    assert nat.nat_embed_workspace_bytes(ok(), 8) > 0
    for kw, status in [(dict(d=0), -1), (dict(d=-8), -1), (dict(V=0), -1), (dict(d=12), -2), (dict(d=65544), -2),
                       (dict(V=(1 << 30) + 1), -2), (dict(dtype=7), -2), (dict(scale=float("nan")), -1),
                       (dict(scale=float("inf")), -1)]:
        assert _embed_fwd(ok(**kw)) == status and _embed_bwd(ok(**kw)) == status, kw
        assert nat.nat_embed_workspace_bytes(ok(**kw), 8) == 0
    for f in (_embed_fwd, _embed_bwd):
        assert f(None) == -1 and f(ok(), cap=-1) == -1 and f(ok(), cap=1 << 31) == -1
        assert f(ok(), ids=None) == -1
        for name in ("ids", "sel", "n"):
            assert f(ok(), **{name: A + 2}) == -1, name
    for name in ("table", "x"):
        assert _embed_fwd(ok(), **{name: None}) == -1 and _embed_fwd(ok(), **{name: ODD}) == -1, name
    for name in ("dx", "dtable"):
        assert _embed_bwd(ok(), **{name: None}) == -1 and _embed_bwd(ok(), **{name: ODD}) == -1, name
    assert _embed_fwd(ok(), cap=0, table=None, ids=None, x=None) == 0
    assert _embed_bwd(ok(), cap=0, dtable=None) == -1
    need = nat.nat_embed_workspace_bytes(ok(), 8)
    assert _embed_bwd(ok(), nbytes=need - 1) == -3 and _embed_bwd(ok(), ws=None) == -3
    assert _embed_bwd(ok(), ws=A + 16) == -1


def test_embed_workspace_grows_with_cap():
    sizes = [nat.nat_embed_workspace_bytes(nat.embed_params(151936, 4096, torch.bfloat16), c)
             for c in (0, 1, 63, 64, 65, 127, 128, 129, 4096, 4097, 166001, 1 << 24)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    # pairs twice, their counts, and two pieces of a row for every 64 tokens
    n, d = 166001, 4096
    assert sizes[10] <= 16 * n + 4 * 512 * (n // 1024 + 2) + 2 * 4 * d * (n // 64 + 1) + 8 * 256


# ------------------------------------------------------------------------- head norms
def _qk_fwd(p, cap=8, B=2, cu=A, pos=None, n=None, w=(A, A), freq=A, **kw):
    a = dict(dict(q=A, k=A, qo=A, ko=A), **kw)
    return nat.load().nat_qknorm_fwd(_ref(p), B, cu, pos, n, cap, a["q"], a["k"], *w, freq, a["qo"], a["ko"], None)


def _qk_bwd(p, cap=8, B=2, cu=A, pos=None, n=None, w=(A, A), freq=A, ws=A, nbytes=1 << 30, **kw):
    a = dict(dict(q=A, k=A, dqo=A, dko=A, dq=A, dk=A, dwq=A, dwk=A), **kw)
    return nat.load().nat_qknorm_bwd(_ref(p), B, cu, pos, n, cap, a["q"], a["k"], *w, freq, a["dqo"], a["dko"], a["dq"],
                                     a["dk"], a["dwq"], a["dwk"], ws, nbytes, None)


def test_qknorm_refusals():
    ok = lambda **kw: _with(nat.qknorm_params(4, 2, 64, torch.bfloat16), **kw)  # noqa: E731
    assert nat.nat_qknorm_workspace_bytes(ok(), 8) > 0
    for kw, status in [(dict(n_heads=0), -1), (dict(n_kv_heads=0), -1), (dict(head_dim=0), -1), (dict(rot_dim=-16), -1),
                       (dict(head_dim=60), -2), (dict(head_dim=136), -2), (dict(rot_dim=80), -1), (dict(rot_dim=24), -2),
                       (dict(rot_dim=8), -2), (dict(interleaved=2), -1), (dict(dtype=3), -2), (dict(eps=-1e-6), -1),
                       (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(q_stride=248), -1),
                       (dict(k_stride=120), -1), (dict(q_out_stride=260), -2), (dict(k_out_stride=1 << 31), -2),
                       (dict(q_stride=-256), -1)]:
        assert _qk_fwd(ok(**kw)) == status and _qk_bwd(ok(**kw)) == status, kw
        assert nat.nat_qknorm_workspace_bytes(ok(**kw), 8) == 0
    for f in (_qk_fwd, _qk_bwd):
        assert f(None) == -1 and f(ok(), cap=-1) == -1 and f(ok(), cap=1 << 31) == -1
        assert f(ok(), cu=None) == -1 and f(ok(), B=0) == -1 and f(ok(), B=-1) == -1
        assert f(ok(), w=(A, None)) == -1 and f(ok(), w=(None, A)) == -1
        assert f(ok(), freq=None) == -1 and f(ok(), freq=A + 4) == -1
        for kw in (dict(cu=A + 2), dict(pos=A + 1), dict(n=A + 2), dict(w=(A + 2, A)), dict(w=(A, A + 1))):
            assert f(ok(), **kw) == -1, kw
    for name in ("q", "k", "qo", "ko"):
        assert _qk_fwd(ok(), **{name: None}) == -1 and _qk_fwd(ok(), **{name: ODD}) == -1, name
    for name in ("q", "k", "dqo", "dko", "dq", "dk"):
        assert _qk_bwd(ok(), **{name: None}) == -1 and _qk_bwd(ok(), **{name: ODD}) == -1, name
    for name in ("dwq", "dwk"):
        assert _qk_bwd(ok(), **{name: None}) == -1 and _qk_bwd(ok(), **{name: A + 2}) == -1, name
    need = nat.nat_qknorm_workspace_bytes(ok(), 8)
    assert _qk_bwd(ok(), nbytes=need - 1) == -3 and _qk_bwd(ok(), ws=None) == -3 and _qk_bwd(ok(), ws=A + 16) == -1
    assert _qk_fwd(ok(), cap=0, q=None, k=None, qo=None, ko=None, cu=None, freq=None) == 0
    assert _qk_bwd(ok(), cap=0, w=(None, None), dq=None, cu=None, ws=None) == 0


def test_qknorm_workspace_grows_with_cap():
    sizes = [nat.nat_qknorm_workspace_bytes(nat.qknorm_params(4, 2, 128, torch.bfloat16), c) for c in (0, 1, 9, 4096, 10 ** 6)]
    # sums of the weights' gradients: less than a hundredth of the rows, which are 1536 bytes each
    assert sizes == sorted(sizes) and 0 < sizes[-1] < 15.36 * 10 ** 6


# ---------------------------------------------------------------------------- experts
def _ex_fwd(p, cap=8, ws=A, nbytes=1 << 30, **kw):
    a = dict(dict(offs=A, x=A, w=A, y=A), **kw)
    return nat.load().nat_experts_fwd(_ref(p), a["offs"], cap, a["x"], a["w"], a["y"], ws, nbytes, None)


def _ex_bwd(p, cap=8, ws=A, nbytes=1 << 30, **kw):
    a = dict(dict(offs=A, x=A, w=A, dy=A, dx=A, dw=A), **kw)
    return nat.load().nat_experts_bwd(_ref(p), a["offs"], cap, a["x"], a["w"], a["dy"], a["dx"], a["dw"], ws, nbytes, None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_experts_refusals(dtype):
    ok = lambda **kw: _with(nat.experts_params(4, 64, 128, dtype), **kw)  # noqa: E731
    assert nat.nat_experts_workspace_bytes(ok(), 8) > 0
    for kw, status in [(dict(n_experts=0), -1), (dict(n_in=0), -1), (dict(n_out=-8), -1), (dict(n_in=60), -2),
                       (dict(n_out=132), -2), (dict(n_experts=1025), -2), (dict(dtype=4), -2), (dict(x_stride=56), -1),
                       (dict(y_stride=120), -1), (dict(x_stride=68), -2), (dict(y_stride=1 << 31), -2),
                       (dict(n_in=(1 << 20) + 8, x_stride=1 << 21), -2), (dict(n_out=(1 << 20) + 8, y_stride=1 << 21), -2),
                       (dict(n_in=1 << 20, n_out=4096, x_stride=1 << 20, y_stride=4096), -2)]:
        assert _ex_fwd(ok(**kw)) == status and _ex_bwd(ok(**kw)) == status, kw
        assert nat.nat_experts_workspace_bytes(ok(**kw), 8) == 0
    need = nat.nat_experts_workspace_bytes(ok(), 8)
    for f, names in ((_ex_fwd, ("x", "w", "y")), (_ex_bwd, ("x", "w", "dy"))):
        assert f(None) == -1 and f(ok(), cap=-1) == -1 and f(ok(), cap=1 << 31) == -1
        assert f(ok(), offs=None) == -1 and f(ok(), offs=A + 2) == -1
        for name in names:
            assert f(ok(), **{name: None}) == -1 and f(ok(), **{name: ODD}) == -1, name
        assert f(ok(), nbytes=need - 1) == -3 and f(ok(), ws=None) == -3 and f(ok(), ws=A + 16) == -1
    assert _ex_bwd(ok(), dx=None, dw=None) == -1
    assert _ex_bwd(ok(), dx=ODD) == -1 and _ex_bwd(ok(), dw=ODD) == -1


def test_experts_workspace_holds_to_its_bound():
    for E, n_in, n_out in ((1, 8, 8), (1, 256, 512), (4, 256, 256), (64, 2048, 1536), (1024, 24, 16)):
        for dtype in (torch.float32, torch.bfloat16):
            for cap in (0, 1, 5000, 300013):
                n = nat.nat_experts_workspace_bytes(nat.experts_params(E, n_in, n_out, dtype), cap)
                assert 0 < n <= 40e6 + 16 * (cap // 64 + 2 * E) + 4 * 256


def test_binding_refuses_host_tensors_types_shapes_and_strides():
    t = torch.zeros(4, 64)
    i = torch.zeros(4, dtype=torch.int32)
    p = nat.embed_params(4, 64, torch.float32)
    with pytest.raises(nat.NatError, match="not on the current CUDA device|expected"):
        nat.nat_embed_fwd(p, t, i, None, None, 4, t)
    with pytest.raises(nat.NatError, match="expected torch.float32"):
        nat.nat_embed_fwd(p, t.bfloat16(), i, None, None, 4, t)
    h = torch.zeros(4, 2, 64)
    e = nat.experts_params(2, 64, 64, torch.float32)
    with pytest.raises(nat.NatError, match="not on the current CUDA device|expected"):
        nat.nat_experts_fwd(e, i, 4, t, t.view(1, 4, 64), t, torch.zeros(4096, dtype=torch.uint8))
    with pytest.raises(nat.NatError, match="expected torch.float32"):
        nat.nat_experts_bwd(e, i, 4, t.bfloat16(), t, t, t, None, torch.zeros(4096, dtype=torch.uint8))
    q = nat.qknorm_params(2, 2, 64, torch.float32)
    with pytest.raises(nat.NatError, match="expected torch.float32"):
        nat.nat_qknorm_fwd(q, 1, i, None, None, 4, h.bfloat16(), h, None, None, None, h, h)
