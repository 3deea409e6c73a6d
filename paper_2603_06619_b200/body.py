"""One sublayer of the model body on packed prefixes, forward and backward, through the C-ABI library.

Under prefix cutting the model processes the prefixes only (Section 4, the paragraph on compute
savings): ``nat_gather_rows`` packs them, ``sel_offsets`` is their ``cu_seqlens`` and ``n_sel`` the
number of rows.  ``PackedSublayer`` owns what one attention sublayer keeps and writes for batches of up
to ``cap`` such rows (torch is only the allocator and the stream) and exposes its calls in the
order a trainer makes them, forward and, reversed, backward:

    qkv = h @ W_qkv                     (the caller's projections)
    out = sub.attend(qkv, cu_seqlens)
    y = out @ W_o
    r, h_next = sub.join(x, y, ...)     post-norm, gate and residual scale, the next block's pre-norm
    ...
    dx, dy = sub.join_backward(dr, dh_next, ...)
    dqkv = sub.attend_backward(qkv, cu_seqlens, dout)

With ``ckpt8`` the backward of the join reads 8-bit checkpoints of y and r that ``join`` leaves, so the
caller may drop both rows (a quarter to a half of their memory).
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
        self.dqkv = torch.empty(rows, n_heads + 2 * n_kv_heads, head_dim, dtype=dtype, device=dev)
        self.r, self.h, self.dx, self.dy = (torch.empty(rows, d, dtype=dtype, device=dev) for _ in range(4))
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

    def _split(self, qkv):
        return qkv.split([self.n_heads, self.n_kv_heads, self.n_kv_heads], dim=1)

    def attend(self, qkv, cu_seqlens):
        """qkv [>= cap, n_heads + 2 n_kv_heads, head_dim] -> out [cap, n_heads, head_dim]."""
        q, k, v = self._split(qkv)
        nat.nat_attn_fwd(self.attn, self.B, cu_seqlens, self.cap, q, k, v, self.out, self.lse, self.attn_ws)
        self.status_words[0].copy_(self.attn_ws[:4])
        return self.out

    def join(self, x, y, w_post, gate, w_pre, n_rows):
        """(r, h): the residual stream and the next block's input."""
        nat.nat_resnorm_fwd(self.norm, x, y, w_post, gate, w_pre, n_rows, self.cap, self.r, self.h, self.rstd_y,
                            self.rstd_r, y8=self.y8, r8=self.r8)
        return self.r, self.h

    def join_backward(self, dr, dh, w_post, gate, w_pre, n_rows, y=None):
        """(dx, dy); dw_post, dgate and dw_pre are left in the attributes of these names.  `y` is
        needed where no checkpoint was left."""
        rows = (None, None) if self.ckpt8 else (y, self.r)
        nat.nat_resnorm_bwd(self.norm, *rows, w_post, gate, w_pre, self.rstd_y, self.rstd_r, n_rows, self.cap, dr,
                            dh, self.dx, self.dy, self.dw_post if w_post is not None else None, self.dgate,
                            self.dw_pre if w_pre is not None else None, self.norm_ws, y8=self.y8, r8=self.r8)
        return self.dx, self.dy

    def attend_backward(self, qkv, cu_seqlens, dout):
        """dqkv, laid out like qkv, from the gradient of ``attend``'s out."""
        q, k, v = self._split(qkv)
        nat.nat_attn_bwd(self.attn, self.B, cu_seqlens, self.cap, q, k, v, self.out, self.lse, dout,
                         *self._split(self.dqkv), self.attn_ws)
        self.status_words[1].copy_(self.attn_ws[:4])
        return self.dqkv

    def status(self):
        """The NAT_DEV_* bits of the last ``attend`` and the last ``attend_backward`` together (waits for the
        stream); 0 before the first."""
        return nat.nat_poll_status(self.status_words[0]) | nat.nat_poll_status(self.status_words[1])
