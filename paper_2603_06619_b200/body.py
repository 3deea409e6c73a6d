"""One sublayer of the model body on packed prefixes, forward and backward, through the C-ABI library.

Under prefix cutting the model processes the prefixes only (Section 4, the paragraph on compute
savings): ``nat_gather_rows`` packs them, ``sel_offsets`` is their ``cu_seqlens`` and ``n_sel`` the
number of rows.  A token attends to the packed tokens of its sequence and to nothing else, so responses that follow
prompts are packed behind them, by ``nat_compact_prefix`` on the bounds of prompt and response together:

    nat.nat_compact_prefix(B, cu_whole, n_whole, prompt_len + cut_len, idx, resp, offs, n_sel, cap)

``PackedSublayer`` owns what one attention sublayer keeps and writes for batches of up
to ``cap`` such rows (torch is only the allocator and the stream) and exposes its calls in the
order a trainer makes them, forward and, reversed, backward:

    qkv = h @ W_qkv                     (the caller's projections)
    out = sub.attend(qkv, cu_seqlens)
    y = out @ W_o
    r, h_next = sub.join(x, y, ...)     post-norm, gate and residual scale, the next block's pre-norm
    ...
    dx, dy = sub.join_backward(dr, dh_next, ...)
    dqkv = sub.attend_backward(qkv, cu_seqlens, dout)

What a sublayer keeps from its forward to its backward pass is allocated with it: out and lse of the attention, the
reciprocal norms and, with ``ckpt8``, 8-bit checkpoints of y and r, which the backward of the join reads in
place of the rows (0.52 of the rows' bytes in bfloat16, 0.26 in float32).  Everything else that it writes only passes
through: r, h, dx, dy and dqkv go to tensors that the caller gives, which many sublayers can share, or else to
buffers of its own that are allocated when first needed (so make a first call before capturing a graph).
"""
import torch

from . import nat


class PackedSublayer:
    def __init__(self, cap, B, d, n_heads, n_kv_heads, head_dim, dtype, gate="none", eps=1e-6, alpha=1.0,
                 scale=None, ckpt8=True, device="cuda"):
        self.cap, self.B, self.d, self.ckpt8 = int(cap), int(B), d, ckpt8
        self.n_heads, self.n_kv_heads = n_heads, n_kv_heads
        dev, f32 = torch.device(device), torch.float32
        self.attn = nat.attn_params(n_heads, n_kv_heads, head_dim, dtype, scale=scale)
        self.norm = nat.resnorm_params(d, dtype, eps=eps, alpha=alpha, gate=gate)
        rows = max(self.cap, 1)
        self.out = torch.empty(rows, n_heads, head_dim, dtype=dtype, device=dev)
        self.lse = torch.empty(rows, n_heads, dtype=f32, device=dev)
        self._shapes = dict.fromkeys(("r", "h", "dx", "dy"), (rows, d))
        self._shapes["dqkv"] = (rows, n_heads + 2 * n_kv_heads, head_dim)
        self._own, self._empty = {}, lambda shape: torch.empty(shape, dtype=dtype, device=dev)
        self._joined = None  # r of the last join, where the backward pass reads its rows
        self.rstd_y, self.rstd_r = (torch.empty(rows, dtype=f32, device=dev) for _ in range(2))
        self.dw_post, self.dw_pre = (torch.empty(d, dtype=f32, device=dev) for _ in range(2))
        self.dgate = None if gate == "none" else torch.empty(d if gate == "channel" else rows, dtype=f32, device=dev)
        self.y8 = self.r8 = None
        if ckpt8:
            groups = -(-d // nat.GROUP8)
            self.y8, self.r8 = ((torch.empty(rows, d, dtype=torch.int8, device=dev),
                                 torch.empty(rows, groups, dtype=f32, device=dev)) for _ in range(2))
        self.attn_ws = nat.alloc_workspace(nat.nat_attn_workspace_bytes(self.attn, self.B, self.cap), dev)
        self.attn_ws[:4].zero_()  # the status word: a call without rows leaves it alone
        # the forward's and the backward's words, which share a workspace and would overwrite one another
        self.status_words = [torch.zeros(4, dtype=torch.uint8, device=dev) for _ in range(2)]
        self.norm_ws = nat.alloc_workspace(nat.nat_resnorm_workspace_bytes(self.norm, self.cap), dev)

    def _buffer(self, name):
        if name not in self._own:
            self._own[name] = self._empty(self._shapes[name])
        return self._own[name]

    r, h, dx, dy, dqkv = (property(lambda self, name=name: self._buffer(name)) for name in ("r", "h", "dx", "dy", "dqkv"))

    def _split(self, qkv):
        return qkv.split([self.n_heads, self.n_kv_heads, self.n_kv_heads], dim=1)

    def attend(self, qkv, cu_seqlens):
        """qkv [>= cap, n_heads + 2 n_kv_heads, head_dim] -> out [cap, n_heads, head_dim]."""
        q, k, v = self._split(qkv)
        nat.nat_attn_fwd(self.attn, self.B, cu_seqlens, self.cap, q, k, v, self.out, self.lse, self.attn_ws)
        self.status_words[0].copy_(self.attn_ws[:4])
        return self.out

    def join(self, x, y, w_post, gate, w_pre, n_rows, r=None, h=None):
        """(r, h): the residual stream and the next block's input, in the tensors given for them (r may be x, h may
        be y or x) or in the sublayer's own; h is None where there is no w_pre.  Without ``ckpt8`` the backward pass
        reads y and r: leave them alone."""
        r = self.r if r is None else r
        h = None if w_pre is None else self.h if h is None else h
        nat.nat_resnorm_fwd(self.norm, x, y, w_post, gate, w_pre, n_rows, self.cap, r, h, self.rstd_y,
                            self.rstd_r, y8=self.y8, r8=self.r8)
        self._joined = None if self.ckpt8 else r
        return r, h

    def join_backward(self, dr, dh, w_post, gate, w_pre, n_rows, y=None, dx=None, dy=None):
        """(dx, dy), in the tensors given for them (which may be dr and dh) or in the sublayer's own; dw_post, dgate
        and dw_pre are left in the attributes of these names.  `y` is needed where no checkpoint was left."""
        rows = (None, None) if self.ckpt8 else (y, self._joined)
        dx, dy = self.dx if dx is None else dx, self.dy if dy is None else dy
        nat.nat_resnorm_bwd(self.norm, *rows, w_post, gate, w_pre, self.rstd_y, self.rstd_r, n_rows, self.cap, dr,
                            dh, dx, dy, self.dw_post if w_post is not None else None, self.dgate,
                            self.dw_pre if w_pre is not None else None, self.norm_ws, y8=self.y8, r8=self.r8)
        return dx, dy

    def attend_backward(self, qkv, cu_seqlens, dout, dqkv=None):
        """dqkv, laid out like qkv, from the gradient of ``attend``'s out; in the tensor given for it or the
        sublayer's own."""
        dqkv = self.dqkv if dqkv is None else dqkv
        q, k, v = self._split(qkv)
        nat.nat_attn_bwd(self.attn, self.B, cu_seqlens, self.cap, q, k, v, self.out, self.lse, dout,
                         *self._split(dqkv), self.attn_ws)
        self.status_words[1].copy_(self.attn_ws[:4])
        return dqkv

    def status(self):
        """The NAT_DEV_* bits of the last ``attend`` and the last ``attend_backward`` together (waits for the
        stream); 0 before the first."""
        return nat.nat_poll_status(self.status_words[0]) | nat.nat_poll_status(self.status_words[1])
