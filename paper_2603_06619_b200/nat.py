"""Python binding of the NAT C-ABI library (ctypes; argument marshalling only).

Every function here has the name and the meaning of the C entry point it
calls (see include/nat.h).  torch tensors supply device memory and the current
CUDA stream; all arithmetic runs in the library's kernels.  There is no CPU
fallback: loading fails loudly when the shared library is missing.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnat_b200.so")

NAT_SEL_URS, NAT_SEL_RPC, NAT_SEL_DET = 0, 1, 2
NAT_F32, NAT_BF16 = 0, 1
NAT_GATE_NONE, NAT_GATE_CHANNEL, NAT_GATE_ROW = 0, 1, 2
NAT_DEV_TIMEOUT, NAT_DEV_CAPACITY, NAT_DEV_FALLBACK, NAT_DEV_BAD_TARGET = 1, 2, 4, 8

SYMBOLS = (
    "nat_status_string", "nat_last_error", "nat_version", "nat_grpo_adv", "nat_select",
    "nat_compact_workspace_bytes", "nat_compact", "nat_policy_loss_workspace_bytes",
    "nat_policy_loss_fwd", "nat_policy_loss_bwd", "nat_compact_static",
    "nat_compact_static_max_tokens", "nat_policy_loss_fwd_bwd", "nat_trace_begin",
    "nat_trace_end", "nat_select_survival", "nat_gather_rows", "nat_scatter_rows",
    "nat_poll_status", "nat_compact_prefix", "nat_select_cutlaw",
    "nat_select_cutlaw_workspace_bytes", "nat_attn_workspace_bytes", "nat_attn_fwd",
    "nat_attn_bwd", "nat_resnorm_workspace_bytes", "nat_resnorm_fwd", "nat_resnorm_bwd",
    "nat_ckpt8_store", "nat_ckpt8_load", "nat_embed_workspace_bytes", "nat_embed_fwd", "nat_embed_bwd",
    "nat_qknorm_workspace_bytes", "nat_qknorm_fwd", "nat_qknorm_bwd", "nat_experts_workspace_bytes", "nat_experts_fwd",
    "nat_experts_bwd",
)
TRACE_KINDS = ("fwd", "dz", "dh", "dw", "e")


class NatError(RuntimeError):
    pass


class SelectParams(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("min_cut", ctypes.c_int32), ("p", ctypes.c_double),
                ("beta", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64),
                ("resp_base", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class LossParams(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("B", ctypes.c_int32), ("clip_lo", ctypes.c_float), ("clip_hi", ctypes.c_float),
                ("hidden_is_compact", ctypes.c_int32), ("accumulate_dW", ctypes.c_int32),
                ("kl_beta", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("ref_logp", ctypes.c_void_p)]


class AttnParams(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("reserved", ctypes.c_int32), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("o_stride", ctypes.c_int64)]


class ResnormParams(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("dtype", ctypes.c_int32), ("gate_mode", ctypes.c_int32),
                ("eps", ctypes.c_float), ("alpha", ctypes.c_float), ("reserved", ctypes.c_int32)]


class EmbedParams(ctypes.Structure):
    _fields_ = [("V", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("accumulate", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class QknormParams(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("eps", ctypes.c_float), ("reserved", ctypes.c_int32), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("q_out_stride", ctypes.c_int64), ("k_out_stride", ctypes.c_int64)]


class ExpertsParams(ctypes.Structure):
    _fields_ = [("n_experts", ctypes.c_int32), ("n_in", ctypes.c_int32), ("n_out", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("accumulate", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("x_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64)]


_lib = None


def load():
    """dlopen the library (built in-tree by ``build.build()``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise NatError(f"{LIB_PATH} is missing: run `python -m paper_2603_06619_b200.build` "
                       "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.nat_status_string.restype = ctypes.c_char_p
    lib.nat_status_string.argtypes = [ctypes.c_int]
    lib.nat_last_error.restype = ctypes.c_char_p
    lib.nat_version.restype = ctypes.c_int
    lib.nat_grpo_adv.argtypes = [i32, i32, vp, f32, vp, vp]
    lib.nat_select.argtypes = [ctypes.POINTER(SelectParams), i32, vp, i64, vp, vp, vp, vp]
    lib.nat_select_survival.argtypes = [i32, vp, i64, vp, ctypes.c_uint64, ctypes.c_uint64, i32,
                                        vp, vp, vp]
    lib.nat_select_survival.restype = ctypes.c_int
    lib.nat_select_cutlaw_workspace_bytes.restype = ctypes.c_size_t
    lib.nat_select_cutlaw_workspace_bytes.argtypes = [i32, i64]
    lib.nat_select_cutlaw.argtypes = [i32, vp, i64, vp, ctypes.c_uint64, ctypes.c_uint64, i32, vp,
                                      vp, vp, vp, ctypes.c_size_t, vp]
    lib.nat_select_cutlaw.restype = ctypes.c_int
    lib.nat_compact_prefix.argtypes = [i32, vp, i64, vp, vp, vp, vp, vp, i64, vp]
    lib.nat_compact_prefix.restype = ctypes.c_int
    lib.nat_poll_status.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_uint32)]
    lib.nat_poll_status.restype = ctypes.c_int
    lib.nat_gather_rows.argtypes = [vp, i64, vp, vp, i64, vp, vp]
    lib.nat_gather_rows.restype = ctypes.c_int
    lib.nat_scatter_rows.argtypes = [vp, i64, vp, vp, i64, i64, vp, vp]
    lib.nat_scatter_rows.restype = ctypes.c_int
    lib.nat_compact_workspace_bytes.restype = ctypes.c_size_t
    lib.nat_compact_workspace_bytes.argtypes = [i64]
    lib.nat_compact.argtypes = [i32, vp, i64, vp, vp, vp, vp, vp, i64, vp, ctypes.c_size_t, vp]
    lib.nat_compact_static_max_tokens.restype = ctypes.c_int64
    lib.nat_compact_static.argtypes = [i32, vp, i64, vp, vp, vp, vp, vp, i64, vp]
    lib.nat_compact_static.restype = ctypes.c_int
    lib.nat_policy_loss_workspace_bytes.restype = ctypes.c_size_t
    lib.nat_policy_loss_workspace_bytes.argtypes = [ctypes.POINTER(LossParams), i64]
    lib.nat_policy_loss_fwd.argtypes = [ctypes.POINTER(LossParams)] + [vp] * 10 + [i64] + \
        [vp] * 4 + [ctypes.c_size_t, vp]
    lib.nat_policy_loss_bwd.argtypes = [ctypes.POINTER(LossParams)] + [vp] * 10 + [i64] + \
        [vp] * 6 + [ctypes.c_size_t, vp]
    lib.nat_policy_loss_fwd_bwd.argtypes = [ctypes.POINTER(LossParams)] + [vp] * 10 + [i64] + \
        [vp] * 7 + [ctypes.c_size_t, vp]
    lib.nat_trace_begin.restype = ctypes.c_int
    lib.nat_trace_end.restype = ctypes.c_int
    lib.nat_trace_end.argtypes = [vp, vp]
    lib.nat_attn_workspace_bytes.restype = ctypes.c_size_t
    lib.nat_attn_workspace_bytes.argtypes = [ctypes.POINTER(AttnParams), i32, i64]
    lib.nat_attn_fwd.argtypes = [ctypes.POINTER(AttnParams), i32, vp, i64] + [vp] * 6 + \
        [ctypes.c_size_t, vp]
    lib.nat_attn_bwd.argtypes = [ctypes.POINTER(AttnParams), i32, vp, i64] + [vp] * 10 + \
        [ctypes.c_size_t, vp]
    lib.nat_resnorm_workspace_bytes.restype = ctypes.c_size_t
    lib.nat_resnorm_workspace_bytes.argtypes = [ctypes.POINTER(ResnormParams), i64]
    lib.nat_resnorm_fwd.argtypes = [ctypes.POINTER(ResnormParams)] + [vp] * 6 + [i64] + [vp] * 9
    lib.nat_resnorm_bwd.argtypes = [ctypes.POINTER(ResnormParams)] + [vp] * 12 + [i64] + \
        [vp] * 8 + [ctypes.c_size_t, vp]
    lib.nat_ckpt8_store.argtypes = [i32, i64, vp, vp, i64, vp, vp, vp]
    lib.nat_ckpt8_load.argtypes = [i32, i64, vp, vp, vp, i64, vp, vp]
    lib.nat_embed_workspace_bytes.restype = ctypes.c_size_t
    lib.nat_embed_workspace_bytes.argtypes = [ctypes.POINTER(EmbedParams), i64]
    lib.nat_embed_fwd.argtypes = [ctypes.POINTER(EmbedParams)] + [vp] * 4 + [i64, vp, vp]
    lib.nat_embed_bwd.argtypes = [ctypes.POINTER(EmbedParams)] + [vp] * 3 + [i64] + [vp] * 3 + [ctypes.c_size_t, vp]
    lib.nat_qknorm_workspace_bytes.restype = ctypes.c_size_t
    lib.nat_qknorm_workspace_bytes.argtypes = [ctypes.POINTER(QknormParams), i64]
    lib.nat_qknorm_fwd.argtypes = [ctypes.POINTER(QknormParams), i32] + [vp] * 3 + [i64] + [vp] * 8
    lib.nat_qknorm_bwd.argtypes = [ctypes.POINTER(QknormParams), i32] + [vp] * 3 + [i64] + [vp] * 12 + \
        [ctypes.c_size_t, vp]
    lib.nat_experts_workspace_bytes.restype = ctypes.c_size_t
    lib.nat_experts_workspace_bytes.argtypes = [ctypes.POINTER(ExpertsParams), i64]
    lib.nat_experts_fwd.argtypes = [ctypes.POINTER(ExpertsParams), vp, i64] + [vp] * 4 + [ctypes.c_size_t, vp]
    lib.nat_experts_bwd.argtypes = [ctypes.POINTER(ExpertsParams), vp, i64] + [vp] * 6 + [ctypes.c_size_t, vp]
    for name in ("nat_attn_fwd", "nat_attn_bwd", "nat_resnorm_fwd", "nat_resnorm_bwd",
                 "nat_ckpt8_store", "nat_ckpt8_load", "nat_embed_fwd", "nat_embed_bwd", "nat_qknorm_fwd",
                 "nat_qknorm_bwd", "nat_experts_fwd", "nat_experts_bwd"):
        getattr(lib, name).restype = ctypes.c_int
    for name in ("nat_grpo_adv", "nat_select", "nat_compact", "nat_policy_loss_fwd",
                 "nat_policy_loss_bwd", "nat_policy_loss_fwd_bwd"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _check(status):
    if status != 0:
        lib = load()
        raise NatError(f"{lib.nat_status_string(status).decode()}: {lib.nat_last_error().decode()}")


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensors passed to the library must be contiguous"
    return t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def nat_grpo_adv(P, G, rewards, eps, adv):
    _check(load().nat_grpo_adv(P, G, _ptr(rewards), eps, _ptr(adv), _stream()))


def select_params(mode, p=1.0, min_cut=1, beta=1.0, seed=0, offset=0, resp_base=0):
    mode = {"urs": NAT_SEL_URS, "rpc": NAT_SEL_RPC, "det": NAT_SEL_DET}.get(mode, mode)
    return SelectParams(mode=mode, min_cut=min_cut, p=p, beta=beta, seed=seed, offset=offset,
                        resp_base=resp_base, reserved=0)


def nat_select(params, B, cu_seqlens, n_tot, mask, pi, cut_len):
    _check(load().nat_select(ctypes.byref(params), B, _ptr(cu_seqlens), n_tot, _ptr(mask),
                             _ptr(pi), _ptr(cut_len), _stream()))


def nat_select_survival(B, cu_seqlens, n_tot, surv, seed, offset, mask, cut_len, resp_base=0):
    _check(load().nat_select_survival(B, _ptr(cu_seqlens), n_tot, _ptr(surv), seed, offset,
                                      resp_base, _ptr(mask), _ptr(cut_len), _stream()))


def nat_select_cutlaw_workspace_bytes(B, n_tot):
    return load().nat_select_cutlaw_workspace_bytes(B, n_tot)


def nat_select_cutlaw(B, cu_seqlens, n_tot, q, seed, offset, mask, pi, cut_len, workspace,
                      resp_base=0):
    _check(load().nat_select_cutlaw(B, _ptr(cu_seqlens), n_tot, _ptr(q), seed, offset, resp_base,
                                    _ptr(mask), _ptr(pi), _ptr(cut_len), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream()))


def _row_bytes(t):
    return t.stride(0) * t.element_size() if t.dim() > 1 else t.element_size()


def nat_gather_rows(src, sel_idx, n_sel, cap, dst):
    _check(load().nat_gather_rows(_ptr(src), _row_bytes(src), _ptr(sel_idx), _ptr(n_sel), cap,
                                  _ptr(dst), _stream()))


def nat_scatter_rows(src, sel_idx, n_sel, cap, n_tot, dst):
    _check(load().nat_scatter_rows(_ptr(src), _row_bytes(src), _ptr(sel_idx), _ptr(n_sel), cap,
                                   n_tot, _ptr(dst), _stream()))


def nat_compact_workspace_bytes(n_tot):
    return load().nat_compact_workspace_bytes(n_tot)


def nat_compact(B, cu_seqlens, n_tot, mask, sel_idx, sel_resp, sel_offsets, n_sel, cap, workspace):
    _check(load().nat_compact(B, _ptr(cu_seqlens), n_tot, _ptr(mask), _ptr(sel_idx),
                              _ptr(sel_resp), _ptr(sel_offsets), _ptr(n_sel), cap,
                              _ptr(workspace), workspace.numel() * workspace.element_size(),
                              _stream()))


def nat_compact_prefix(B, cu_seqlens, n_tot, cut_len, sel_idx, sel_resp, sel_offsets, n_sel, cap):
    _check(load().nat_compact_prefix(B, _ptr(cu_seqlens), n_tot, _ptr(cut_len), _ptr(sel_idx),
                                     _ptr(sel_resp), _ptr(sel_offsets), _ptr(n_sel), cap,
                                     _stream()))


def nat_compact_static_max_tokens():
    return load().nat_compact_static_max_tokens()


def nat_compact_static(B, cu_seqlens, n_tot, mask, sel_idx, sel_resp, sel_offsets, n_sel, cap):
    """nat_compact for callers that may not allocate: the scratch is a fixed array
    inside the library (shared by all calls on the GPU, so do not overlap calls)."""
    _check(load().nat_compact_static(B, _ptr(cu_seqlens), n_tot, _ptr(mask), _ptr(sel_idx),
                                     _ptr(sel_resp), _ptr(sel_offsets), _ptr(n_sel), cap,
                                     _stream()))


def loss_params(d, V, dtype, B, clip_lo=0.2, clip_hi=0.2, hidden_is_compact=False,
                accumulate_dW=False, kl_beta=0.0, ref_logp=None):
    """ref_logp (float32 device tensor [n_tot]) must outlive the calls that use the params."""
    dtype = {torch.float32: NAT_F32, torch.bfloat16: NAT_BF16}.get(dtype, dtype)
    return LossParams(d=d, V=V, dtype=dtype, B=B, clip_lo=clip_lo, clip_hi=clip_hi,
                      hidden_is_compact=int(hidden_is_compact), accumulate_dW=int(accumulate_dW),
                      kl_beta=kl_beta, reserved=0, ref_logp=_ptr(ref_logp))


def nat_policy_loss_workspace_bytes(params, n_sel_cap):
    return load().nat_policy_loss_workspace_bytes(ctypes.byref(params), n_sel_cap)


def nat_policy_loss_fwd(params, hidden, W, targets, old_logp, adv, pi, cu_seqlens, sel_idx,
                        sel_resp, n_sel, n_sel_cap, loss, logp, lse, workspace):
    _check(load().nat_policy_loss_fwd(
        ctypes.byref(params), _ptr(hidden), _ptr(W), _ptr(targets), _ptr(old_logp), _ptr(adv),
        _ptr(pi), _ptr(cu_seqlens), _ptr(sel_idx), _ptr(sel_resp), _ptr(n_sel), n_sel_cap,
        _ptr(loss), _ptr(logp), _ptr(lse), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream()))


def nat_policy_loss_bwd(params, hidden, W, targets, old_logp, adv, pi, cu_seqlens, sel_idx,
                        sel_resp, n_sel, n_sel_cap, logp, lse, dloss, dHidden, dW, workspace):
    _check(load().nat_policy_loss_bwd(
        ctypes.byref(params), _ptr(hidden), _ptr(W), _ptr(targets), _ptr(old_logp), _ptr(adv),
        _ptr(pi), _ptr(cu_seqlens), _ptr(sel_idx), _ptr(sel_resp), _ptr(n_sel), n_sel_cap,
        _ptr(logp), _ptr(lse), _ptr(dloss), _ptr(dHidden), _ptr(dW), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream()))


def nat_policy_loss_fwd_bwd(params, hidden, W, targets, old_logp, adv, pi, cu_seqlens, sel_idx,
                            sel_resp, n_sel, n_sel_cap, dloss, loss, logp, lse, dHidden, dW,
                            workspace):
    _check(load().nat_policy_loss_fwd_bwd(
        ctypes.byref(params), _ptr(hidden), _ptr(W), _ptr(targets), _ptr(old_logp), _ptr(adv),
        _ptr(pi), _ptr(cu_seqlens), _ptr(sel_idx), _ptr(sel_resp), _ptr(n_sel), n_sel_cap,
        _ptr(dloss), _ptr(loss), _ptr(logp), _ptr(lse), _ptr(dHidden), _ptr(dW), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream()))


# -- the transformer body on packed sequences ------------------------------------------
_DTYPES = {torch.float32: NAT_F32, torch.bfloat16: NAT_BF16}
GROUP8 = 128                 # columns that share a scale in an 8-bit checkpoint


# a torch that was built without CUDA has neither: its tensors are refused as being on no device
_get_device = getattr(torch._C, "_cuda_getDevice", lambda: None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _device():
    try:
        return _get_device()
    except RuntimeError:
        return None                # no CUDA device: no tensor is on it


def _bad(what, t, dtype, shape, device):
    if t.dtype != dtype:
        raise NatError(f"{what}: expected {dtype}, got {t.dtype}")
    if t.get_device() != device:
        raise NatError(f"{what}: on {t.device}, not on the current CUDA device")
    if t.dim() != len(shape) or t.shape[0] < shape[0] or tuple(t.shape[1:]) != tuple(shape[1:]):
        raise NatError(f"{what}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    raise NatError(f"{what}: not contiguous")


def _rows(what, t, dtype, shape, device):
    """Pointer of a contiguous tensor on `device` of that type and shape (leading size: at
    least); None stays None."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == device and t.is_contiguous():
        s = t.shape
        if s == shape or (len(s) == len(shape) and s[0] >= shape[0] and s[1:] == shape[1:]):
            return t.data_ptr()
    _bad(what, t, dtype, shape, device)


def _heads(what, t, dtype, shape, device):
    """(pointer, token stride or None) of [tokens, heads, head_dim] with a stride of its own."""
    if t.dtype is dtype and t.get_device() == device:
        s = t.shape
        if s == shape or (len(s) == 3 and s[0] >= shape[0] and s[1:] == shape[1:]):
            token, head, one = t.stride()
            if one == 1 and (head == shape[2] or shape[1] == 1):
                return t.data_ptr(), token if shape[0] > 1 or s[0] > 1 else None
    _bad(what, t, dtype, shape, device)


def _workspace(t, device):
    if t.get_device() != device or not t.is_contiguous():
        raise NatError("workspace: must be contiguous, on the current CUDA device")
    return t.data_ptr(), t.numel() * t.element_size()


def attn_params(n_heads, n_kv_heads, head_dim, dtype, scale=None):
    """Head layout of the packed causal attention; ``scale`` defaults to head_dim^-1/2.  The
    strides are those of contiguous tensors; nat_attn_fwd / nat_attn_bwd set them from theirs."""
    q, kv = n_heads * head_dim, n_kv_heads * head_dim
    return AttnParams(n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim,
                      dtype=_DTYPES.get(dtype, dtype),
                      scale=head_dim ** -0.5 if scale is None else scale, reserved=0, q_stride=q,
                      k_stride=kv, v_stride=kv, o_stride=q)


def nat_attn_workspace_bytes(params, B, cap):
    return load().nat_attn_workspace_bytes(ctypes.byref(params), B, cap)


def _attn_call(params, B, cu_seqlens, cap, tensors, lse):
    """(pointers, params with the tensors' strides, cu_seqlens, lse, device) of a call; `tensors`
    holds (name, tensor, stride field, head count)."""
    device = _device()
    dtype = torch.float32 if params.dtype == NAT_F32 else torch.bfloat16
    p = AttnParams.from_buffer_copy(params)
    strides, ptrs, D = {}, [], params.head_dim
    for name, t, field, heads in tensors:
        ptr, stride = _heads(name, t, dtype, (cap, heads, D), device)
        ptrs.append(ptr)
        if stride is not None and strides.setdefault(field, stride) != stride:
            raise NatError(f"{name}: token stride {stride}, its counterpart has {strides[field]}")
    for field, stride in strides.items():
        setattr(p, field, stride)
    return (ptrs, p, _rows("cu_seqlens", cu_seqlens, torch.int32, (B + 1,), device),
            _rows("lse", lse, torch.float32, (cap, params.n_heads), device), device)


def nat_attn_fwd(params, B, cu_seqlens, cap, q, k, v, out, lse, workspace):
    h, kv = params.n_heads, params.n_kv_heads
    (q, k, v, out), p, cu, lse, device = _attn_call(
        params, B, cu_seqlens, cap, (("q", q, "q_stride", h), ("k", k, "k_stride", kv),
                                     ("v", v, "v_stride", kv), ("out", out, "o_stride", h)), lse)
    ws, nbytes = _workspace(workspace, device)
    _check(load().nat_attn_fwd(ctypes.byref(p), B, cu, cap, q, k, v, out, lse, ws, nbytes,
                               _raw_stream(device)))


def nat_attn_bwd(params, B, cu_seqlens, cap, q, k, v, out, lse, dout, dq, dk, dv, workspace):
    """dq, dk, dv have the token strides of q, k, v, and dout that of out."""
    h, kv = params.n_heads, params.n_kv_heads
    (q, k, v, out, dout, dq, dk, dv), p, cu, lse, device = _attn_call(
        params, B, cu_seqlens, cap, (
            ("q", q, "q_stride", h), ("k", k, "k_stride", kv), ("v", v, "v_stride", kv),
            ("out", out, "o_stride", h), ("dout", dout, "o_stride", h), ("dq", dq, "q_stride", h),
            ("dk", dk, "k_stride", kv), ("dv", dv, "v_stride", kv)), lse)
    ws, nbytes = _workspace(workspace, device)
    _check(load().nat_attn_bwd(ctypes.byref(p), B, cu, cap, q, k, v, out, lse, dout, dq, dk, dv, ws,
                               nbytes, _raw_stream(device)))


def resnorm_params(d, dtype, eps=1e-6, alpha=1.0, gate="none"):
    """``gate``: "none", "channel" (a factor for each column) or "row" (one for each row)."""
    gate = {"none": NAT_GATE_NONE, "channel": NAT_GATE_CHANNEL, "row": NAT_GATE_ROW}.get(gate, gate)
    return ResnormParams(d=d, dtype=_DTYPES.get(dtype, dtype), gate_mode=gate, eps=eps, alpha=alpha,
                         reserved=0)


def nat_resnorm_workspace_bytes(params, cap):
    return load().nat_resnorm_workspace_bytes(ctypes.byref(params), cap)


def _pair8(what, pair, cap, d, device):
    if pair is None:
        return None, None
    return (_rows(what, pair[0], torch.int8, (cap, d), device),
            _rows(what, pair[1], torch.float32, (cap, (d + GROUP8 - 1) // GROUP8), device))


def nat_resnorm_fwd(params, x, y, w_post, gate, w_pre, n_rows, cap, r, h, rstd_y, rstd_r, y8=None,
                    r8=None):
    """y8, r8: None, or (codes, scales) of the 8-bit checkpoints to leave."""
    dev, d, f32 = _device(), params.d, torch.float32
    dt = f32 if params.dtype == NAT_F32 else torch.bfloat16
    rows, vec, per_row = (cap, d), (d,), (cap,)
    _check(load().nat_resnorm_fwd(
        ctypes.byref(params), _rows("x", x, dt, rows, dev), _rows("y", y, dt, rows, dev),
        _rows("w_post", w_post, f32, vec, dev),
        _rows("gate", gate, f32, per_row if params.gate_mode == NAT_GATE_ROW else vec, dev),
        _rows("w_pre", w_pre, f32, vec, dev), _rows("n_rows", n_rows, torch.int32, (1,), dev), cap,
        _rows("r", r, dt, rows, dev), _rows("h", h, dt, rows, dev),
        _rows("rstd_y", rstd_y, f32, per_row, dev), _rows("rstd_r", rstd_r, f32, per_row, dev),
        *_pair8("y8", y8, cap, d, dev), *_pair8("r8", r8, cap, d, dev), _raw_stream(dev)))


def nat_resnorm_bwd(params, y, r, w_post, gate, w_pre, rstd_y, rstd_r, n_rows, cap, dr, dh, dx, dy,
                    dw_post, dgate, dw_pre, workspace, y8=None, r8=None):
    """y and r as rows, or None with y8 and r8 = (codes, scales)."""
    dev, d, f32 = _device(), params.d, torch.float32
    dt = f32 if params.dtype == NAT_F32 else torch.bfloat16
    rows, vec, per_row = (cap, d), (d,), (cap,)
    of_gate = per_row if params.gate_mode == NAT_GATE_ROW else vec
    ws, nbytes = _workspace(workspace, dev)
    _check(load().nat_resnorm_bwd(
        ctypes.byref(params), _rows("y", y, dt, rows, dev), _rows("r", r, dt, rows, dev),
        *_pair8("y8", y8, cap, d, dev), *_pair8("r8", r8, cap, d, dev),
        _rows("w_post", w_post, f32, vec, dev), _rows("gate", gate, f32, of_gate, dev),
        _rows("w_pre", w_pre, f32, vec, dev), _rows("rstd_y", rstd_y, f32, per_row, dev),
        _rows("rstd_r", rstd_r, f32, per_row, dev), _rows("n_rows", n_rows, torch.int32, (1,), dev),
        cap, _rows("dr", dr, dt, rows, dev), _rows("dh", dh, dt, rows, dev),
        _rows("dx", dx, dt, rows, dev), _rows("dy", dy, dt, rows, dev),
        _rows("dw_post", dw_post, f32, vec, dev), _rows("dgate", dgate, f32, of_gate, dev),
        _rows("dw_pre", dw_pre, f32, vec, dev), ws, nbytes, _raw_stream(dev)))


def nat_ckpt8_store(src, n_rows, cap, codes, scales):
    """8-bit checkpoint of rows [0, n_rows) (a device scalar; None: cap) of src [cap, d]."""
    dev, d = _device(), src.shape[-1]
    c, sc = _pair8("codes", (codes, scales), cap, d, dev)
    _check(load().nat_ckpt8_store(_DTYPES.get(src.dtype, -1), d,
                                  _rows("src", src, src.dtype, (cap, d), dev),
                                  _rows("n_rows", n_rows, torch.int32, (1,), dev), cap, c, sc,
                                  _raw_stream(dev)))


def nat_ckpt8_load(codes, scales, n_rows, cap, dst):
    dev, d = _device(), dst.shape[-1]
    c, sc = _pair8("codes", (codes, scales), cap, d, dev)
    _check(load().nat_ckpt8_load(_DTYPES.get(dst.dtype, -1), d, c, sc,
                                 _rows("n_rows", n_rows, torch.int32, (1,), dev), cap,
                                 _rows("dst", dst, dst.dtype, (cap, d), dev), _raw_stream(dev)))


def embed_params(V, d, dtype, scale=1.0, accumulate=False):
    """``accumulate``: the gradient is added to the table's instead of overwriting it."""
    return EmbedParams(V=V, d=d, dtype=_DTYPES.get(dtype, dtype), scale=scale, accumulate=int(accumulate), reserved=0)


def nat_embed_workspace_bytes(params, cap):
    return load().nat_embed_workspace_bytes(ctypes.byref(params), cap)


def _ids(ids, sel_idx, cap, device):
    # through indices, ids may be of any length; that they lie within it is the caller's contract
    return (_rows("ids", ids, torch.int32, (0 if sel_idx is not None else cap,), device),
            _rows("sel_idx", sel_idx, torch.int32, (cap,), device))


def nat_embed_fwd(params, table, ids, sel_idx, n_rows, cap, x):
    """Row k < n_rows (a device scalar; None: cap) of x from the table's row ids[sel_idx[k]] (sel_idx None: ids[k])."""
    dev = _device()
    dt = torch.float32 if params.dtype == NAT_F32 else torch.bfloat16
    _check(load().nat_embed_fwd(
        ctypes.byref(params), _rows("table", table, dt, (params.V, params.d), dev), *_ids(ids, sel_idx, cap, dev),
        _rows("n_rows", n_rows, torch.int32, (1,), dev), cap, _rows("x", x, dt, (cap, params.d), dev), _raw_stream(dev)))


def nat_embed_bwd(params, ids, sel_idx, n_rows, cap, dx, dtable, workspace):
    dev = _device()
    dt = torch.float32 if params.dtype == NAT_F32 else torch.bfloat16
    ws, nbytes = _workspace(workspace, dev)
    _check(load().nat_embed_bwd(
        ctypes.byref(params), *_ids(ids, sel_idx, cap, dev), _rows("n_rows", n_rows, torch.int32, (1,), dev), cap,
        _rows("dx", dx, dt, (cap, params.d), dev), _rows("dtable", dtable, torch.float32, (params.V, params.d), dev),
        ws, nbytes, _raw_stream(dev)))


def rope_freqs(rot_dim, theta=1e6, device="cuda"):
    """The usual law of the angles a position: theta^(-2 i / rot_dim), i < rot_dim / 2, in float64."""
    return theta ** (-2.0 * torch.arange(rot_dim // 2, dtype=torch.float64, device=device) / rot_dim)


def qknorm_params(n_heads, n_kv_heads, head_dim, dtype, rot_dim=None, interleaved=False, eps=1e-6):
    """``rot_dim``: the elements of a head that turn, from its first on (None: all).  The strides are those of
    contiguous tensors; nat_qknorm_fwd / nat_qknorm_bwd set them from theirs."""
    q, kv = n_heads * head_dim, n_kv_heads * head_dim
    return QknormParams(n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim,
                        rot_dim=head_dim if rot_dim is None else rot_dim, interleaved=int(interleaved),
                        dtype=_DTYPES.get(dtype, dtype), eps=eps, reserved=0, q_stride=q, k_stride=kv,
                        q_out_stride=q, k_out_stride=kv)


def nat_qknorm_workspace_bytes(params, cap):
    return load().nat_qknorm_workspace_bytes(ctypes.byref(params), cap)


def _qknorm_call(params, B, cu_seqlens, positions, n_rows, cap, w_q, w_k, inv_freq, tensors):
    """(params with the tensors' strides, leading arguments, weights and frequencies, pointers, device) of a call."""
    dev, D = _device(), params.head_dim
    dtype = torch.float32 if params.dtype == NAT_F32 else torch.bfloat16
    p = QknormParams.from_buffer_copy(params)
    strides, ptrs = {}, []
    for name, t, field, heads in tensors:
        if t is None:
            ptrs.append(None)
            continue
        ptr, stride = _heads(name, t, dtype, (cap, heads, D), dev)
        ptrs.append(ptr)
        if stride is not None:
            if field not in strides:
                strides[field] = stride
                setattr(p, field, stride)
            elif strides[field] != stride:
                raise NatError(f"{name}: token stride {stride}, its counterpart has {strides[field]}")
    i32, f32 = torch.int32, torch.float32
    where = (B, _rows("cu_seqlens", cu_seqlens, i32, (B + 1,), dev), _rows("positions", positions, i32, (cap,), dev),
             _rows("n_rows", n_rows, i32, (1,), dev), cap)
    laws = (_rows("w_q", w_q, f32, (D,), dev), _rows("w_k", w_k, f32, (D,), dev),
            _rows("inv_freq", inv_freq, torch.float64, (p.rot_dim // 2,), dev))
    return p, where, laws, ptrs, dev


def nat_qknorm_fwd(params, B, cu_seqlens, positions, n_rows, cap, q, k, w_q, w_k, inv_freq, q_out, k_out):
    """q_out and k_out from q and k, each head normed (w_q, w_k; both None: not) and turned by its token's position
    (positions None: from cu_seqlens).  Rows that no sequence of cu_seqlens owns are left alone (cu_seqlens None: none are
    told apart)."""
    h, kv = params.n_heads, params.n_kv_heads
    p, where, laws, (q, k, q_out, k_out), dev = _qknorm_call(
        params, B, cu_seqlens, positions, n_rows, cap, w_q, w_k, inv_freq,
        (("q", q, "q_stride", h), ("k", k, "k_stride", kv), ("q_out", q_out, "q_out_stride", h),
         ("k_out", k_out, "k_out_stride", kv)))
    _check(load().nat_qknorm_fwd(ctypes.byref(p), *where, q, k, *laws, q_out, k_out, _raw_stream(dev)))


def nat_qknorm_bwd(params, B, cu_seqlens, positions, n_rows, cap, q, k, w_q, w_k, inv_freq, dq_out, dk_out, dq, dk,
                   dw_q, dw_k, workspace):
    """dq, dk have the token strides of q, k.  Without norms (w_q, w_k None) q, k, dw_q, dw_k and the workspace may be
    None."""
    h, kv = params.n_heads, params.n_kv_heads
    p, where, laws, (q, k, dq_out, dk_out, dq, dk), dev = _qknorm_call(
        params, B, cu_seqlens, positions, n_rows, cap, w_q, w_k, inv_freq,
        (("q", q, "q_stride", h), ("k", k, "k_stride", kv), ("dq_out", dq_out, "q_out_stride", h),
         ("dk_out", dk_out, "k_out_stride", kv), ("dq", dq, "q_stride", h), ("dk", dk, "k_stride", kv)))
    ws, nbytes = (None, 0) if workspace is None else _workspace(workspace, dev)
    f32, D = torch.float32, (params.head_dim,)
    _check(load().nat_qknorm_bwd(ctypes.byref(p), *where, q, k, *laws, dq_out, dk_out, dq, dk,
                                 _rows("dw_q", dw_q, f32, D, dev), _rows("dw_k", dw_k, f32, D, dev), ws, nbytes,
                                 _raw_stream(dev)))


def experts_params(n_experts, n_in, n_out, dtype, accumulate=False):
    """``accumulate``: dw is added to.  The strides are those of contiguous rows; nat_experts_fwd / nat_experts_bwd set
    them from their tensors'."""
    return ExpertsParams(n_experts=n_experts, n_in=n_in, n_out=n_out, dtype=_DTYPES.get(dtype, dtype),
                         accumulate=int(accumulate), reserved=0, x_stride=n_in, y_stride=n_out)


def nat_experts_workspace_bytes(params, cap):
    return load().nat_experts_workspace_bytes(ctypes.byref(params), cap)


def _experts_call(params, offsets, cap, w, workspace, tensors):
    """(params with the tensors' strides, offsets, pointers, w, workspace, its bytes, device) of a call."""
    dev = _device()
    dtype = torch.float32 if params.dtype == NAT_F32 else torch.bfloat16
    p = ExpertsParams.from_buffer_copy(params)
    strides, ptrs = {}, []
    for name, t, field, width in tensors:
        if t is None:
            ptrs.append(None)
            continue
        s, st = t.shape, t.stride()
        if t.dtype is not dtype or t.get_device() != dev or len(s) != 2 or s[0] < cap or s[1] != width or st[1] != 1:
            _bad(name, t, dtype, (cap, width), dev)
        ptrs.append(t.data_ptr())
        if s[0] > 1:
            if field not in strides:
                strides[field] = st[0]
                setattr(p, field, st[0])
            elif strides[field] != st[0]:
                raise NatError(f"{name}: row stride {st[0]}, its counterpart has {strides[field]}")
    ws, nbytes = _workspace(workspace, dev)
    E = params.n_experts
    if w is not None and w.shape[0] != E:
        _bad("w", w, dtype, (E, params.n_out, params.n_in), dev)
    return (p, _rows("offsets", offsets, torch.int32, (E + 1,), dev), ptrs,
            _rows("w", w, dtype, (E, params.n_out, params.n_in), dev), ws, nbytes, dev)


def nat_experts_fwd(params, offsets, cap, x, w, y, workspace):
    """y [cap, n_out] from x [cap, n_in], the rows offsets[e] .. offsets[e + 1] with w[e] [n_out, n_in]."""
    p, offsets, (x, y), w, ws, nbytes, dev = _experts_call(
        params, offsets, cap, w, workspace, (("x", x, "x_stride", params.n_in), ("y", y, "y_stride", params.n_out)))
    _check(load().nat_experts_fwd(ctypes.byref(p), offsets, cap, x, w, y, ws, nbytes, _raw_stream(dev)))


def nat_experts_bwd(params, offsets, cap, x, w, dy, dx, dw, workspace):
    """dx (with x's row stride) and dw (float32), either of which may be None, from dy (with y's)."""
    p, offsets, (x, dy, dx), w, ws, nbytes, dev = _experts_call(
        params, offsets, cap, w, workspace, (("x", x, "x_stride", params.n_in), ("dy", dy, "y_stride", params.n_out),
                                             ("dx", dx, "x_stride", params.n_in)))
    dw = _rows("dw", dw, torch.float32, (params.n_experts, params.n_out, params.n_in), dev)
    _check(load().nat_experts_bwd(ctypes.byref(p), offsets, cap, x, w, dy, dx, dw, ws, nbytes, _raw_stream(dev)))


def nat_trace_begin():
    _check(load().nat_trace_begin())


def nat_trace_end():
    """Returns {kind: (milliseconds, launches)} for the tensor-core kernels traced."""
    ms = (ctypes.c_float * len(TRACE_KINDS))()
    cnt = (ctypes.c_int32 * len(TRACE_KINDS))()
    _check(load().nat_trace_end(ms, cnt))
    return {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(TRACE_KINDS)}


def alloc_workspace(nbytes, device):
    """256-byte aligned scratch (torch's caching allocator aligns to 512 bytes)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def nat_poll_status(workspace):
    """The NAT_DEV_* bits the last loss, attention, embedding or experts call left in its workspace (waits for the
    stream)."""
    word = ctypes.c_uint32(0)
    _check(load().nat_poll_status(_ptr(workspace), _stream(), ctypes.byref(word)))
    return int(word.value)


device_status = nat_poll_status
