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
    qk = sub.rotate(qkv, cu_seqlens, ...)   the heads' norms and the rotation by position, where the model has them
    out = sub.attend(qkv, cu_seqlens, qk)
    y = out @ W_o
    r, h_next = sub.join(x, y, ...)     post-norm, gate and residual scale, the next block's pre-norm
    ...
    dx, dy = sub.join_backward(dr, dh_next, ...)
    dqkv = sub.attend_backward(qkv, cu_seqlens, dout, qk=qk)
    sub.rotate_backward(qkv, cu_seqlens, ..., dqkv)

What a sublayer keeps from its forward to its backward pass is allocated with it: out and lse of the attention, the
reciprocal norms and, with ``ckpt8``, 8-bit checkpoints of y and r, which the backward of the join reads in
place of the rows (0.52 of the rows' bytes in bfloat16, 0.26 in float32).  Everything else that it writes only passes
through: r, h, dx, dy and dqkv go to tensors that the caller gives, which many sublayers can share, or else to
buffers of its own that are allocated when first needed (so make a first call before capturing a graph).  So does qk, of
which the backward pass needs what the forward pass left, kept or made anew by another ``rotate``.

``PackedEmbedding`` gives the first rows from the packed tokens' ids, and its table's gradient; ``PackedExperts`` multiplies
rows that are grouped by expert.  ``nat_gather_rows`` brings them there, a token's row to each of its experts; back brings
``nat_scatter_rows`` where a token has one expert.  It writes a row to one place and adds nothing up: with several experts a
token their rows are weighted and summed by the caller, and so are the gradients of the rows that were gathered.
"""
import torch

from . import nat


class PackedSublayer:
    def __init__(self, cap, B, d, n_heads, n_kv_heads, head_dim, dtype, gate="none", eps=1e-6, alpha=1.0,
                 scale=None, ckpt8=True, device="cuda", rot_dim=None, interleaved=False):
        self.cap, self.B, self.d, self.ckpt8 = int(cap), int(B), d, ckpt8
        self.n_heads, self.n_kv_heads = n_heads, n_kv_heads
        dev, f32 = torch.device(device), torch.float32
        self.attn = nat.attn_params(n_heads, n_kv_heads, head_dim, dtype, scale=scale)
        self.norm = nat.resnorm_params(d, dtype, eps=eps, alpha=alpha, gate=gate)
        self.heads = nat.qknorm_params(n_heads, n_kv_heads, head_dim, dtype, rot_dim=rot_dim, interleaved=interleaved, eps=eps)
        rows = max(self.cap, 1)
        self.out = torch.empty(rows, n_heads, head_dim, dtype=dtype, device=dev)
        self.lse = torch.empty(rows, n_heads, dtype=f32, device=dev)
        self._shapes = dict.fromkeys(("r", "h", "dx", "dy"), (rows, d))
        self._shapes["dqkv"] = (rows, n_heads + 2 * n_kv_heads, head_dim)
        self._shapes["qk"] = self._shapes["dqk"] = (rows, n_heads + n_kv_heads, head_dim)
        self.dw_q = self.dw_k = self.heads_ws = None  # made by the first rotate_backward with norms
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

    r, h, dx, dy, dqkv, qk, dqk = (property(lambda self, name=name: self._buffer(name))
                                   for name in ("r", "h", "dx", "dy", "dqkv", "qk", "dqk"))

    def _split(self, qkv):
        return qkv.split([self.n_heads, self.n_kv_heads, self.n_kv_heads], dim=1)

    def _split_qk(self, qk):
        return qk.split([self.n_heads, self.n_kv_heads], dim=1)

    def rotate(self, qkv, cu_seqlens, w_q, w_k, inv_freq, positions=None, qk=None):
        """qk [cap, n_heads + n_kv_heads, head_dim]: queries and keys of qkv, each head normed (w_q and w_k None: not)
        and turned by its token's position (in its sequence, or as given), in the tensor given for it or the
        sublayer's own.  inv_freq: ``nat.rope_freqs``, or any law."""
        qk = self.qk if qk is None else qk
        q, k, _ = self._split(qkv)
        nat.nat_qknorm_fwd(self.heads, self.B, cu_seqlens, positions, None, self.cap, q, k, w_q, w_k, inv_freq,
                           *self._split_qk(qk))
        return qk

    def attend(self, qkv, cu_seqlens, qk=None):
        """qkv [>= cap, n_heads + 2 n_kv_heads, head_dim] -> out [cap, n_heads, head_dim]; with ``qk`` the queries and
        keys are that tensor's."""
        q, k, v = self._split(qkv)
        if qk is not None:
            q, k = self._split_qk(qk)
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

    def attend_backward(self, qkv, cu_seqlens, dout, dqkv=None, qk=None, dqk=None):
        """dqkv, laid out like qkv, from the gradient of ``attend``'s out; in the tensor given for it or the
        sublayer's own.  With ``qk`` only the values' part of it is written, and the gradients of qk go to dqk (or the
        sublayer's own), from which ``rotate_backward`` makes the rest."""
        dqkv = self.dqkv if dqkv is None else dqkv
        q, k, v = self._split(qkv)
        dq, dk, dv = self._split(dqkv)
        if qk is not None:
            q, k = self._split_qk(qk)
            dq, dk = self._split_qk(self.dqk if dqk is None else dqk)
        nat.nat_attn_bwd(self.attn, self.B, cu_seqlens, self.cap, q, k, v, self.out, self.lse, dout, dq, dk, dv,
                         self.attn_ws)
        self.status_words[1].copy_(self.attn_ws[:4])
        return dqkv

    def rotate_backward(self, qkv, cu_seqlens, w_q, w_k, inv_freq, dqkv, positions=None, dqk=None):
        """Writes the queries' and keys' part of dqkv from dqk; dw_q and dw_k are left in the attributes of these
        names."""
        if w_q is not None and self.heads_ws is None:
            self.dw_q, self.dw_k = (torch.empty_like(w_q) for _ in range(2))
            self.heads_ws = nat.alloc_workspace(nat.nat_qknorm_workspace_bytes(self.heads, self.cap), w_q.device)
        q, k, _ = self._split(qkv)
        dq, dk, _ = self._split(dqkv)
        norms = (self.dw_q, self.dw_k, self.heads_ws) if w_q is not None else (None, None, None)
        nat.nat_qknorm_bwd(self.heads, self.B, cu_seqlens, positions, None, self.cap, q, k, w_q, w_k, inv_freq,
                           *self._split_qk(self.dqk if dqk is None else dqk), dq, dk, *norms)
        return dqkv

    def status(self):
        """The NAT_DEV_* bits of the last ``attend`` and the last ``attend_backward`` together (waits for the
        stream); 0 before the first."""
        return nat.nat_poll_status(self.status_words[0]) | nat.nat_poll_status(self.status_words[1])


class PackedEmbedding:
    """The first rows of the body: rows of a table [V, d] by the packed tokens' ids, times ``scale``; backward the table's
    gradient in float32, which may be that of the loss's output projection (``accumulate`` adds to it)."""

    def __init__(self, cap, V, d, dtype, scale=1.0, accumulate=False, device="cuda"):
        self.cap = int(cap)
        self.params = nat.embed_params(V, d, dtype, scale=scale, accumulate=accumulate)
        self.ws = nat.alloc_workspace(nat.nat_embed_workspace_bytes(self.params, self.cap), torch.device(device))
        self.ws[:4].zero_()  # the status word, before the first gradient

    def lookup(self, table, ids, x, sel_idx=None, n_rows=None):
        """x [cap, d]: row k from the table's row ids[sel_idx[k]] (sel_idx None: ids[k]).  n_rows: a device scalar (None:
        cap), behind which sel_idx and ids are not read and x is not written."""
        nat.nat_embed_fwd(self.params, table, ids, sel_idx, n_rows, self.cap, x)
        return x

    def gradient(self, ids, dx, dtable, sel_idx=None, n_rows=None):
        nat.nat_embed_bwd(self.params, ids, sel_idx, n_rows, self.cap, dx, dtable, self.ws)
        return dtable

    def status(self):
        """The NAT_DEV_* bits of the last ``gradient`` (waits for the stream)."""
        return nat.nat_poll_status(self.ws)


class PackedExperts:
    """One product of rows grouped by expert: offsets int32 [n_experts + 1], weights w [n_experts, n_out, n_in]."""

    def __init__(self, cap, n_experts, n_in, n_out, dtype, accumulate=False, device="cuda"):
        self.cap = int(cap)
        self.params = nat.experts_params(n_experts, n_in, n_out, dtype, accumulate=accumulate)
        self.ws = nat.alloc_workspace(nat.nat_experts_workspace_bytes(self.params, self.cap), torch.device(device))
        self.ws[:4].zero_()

    def forward(self, x, w, offsets, y):
        nat.nat_experts_fwd(self.params, offsets, self.cap, x, w, y, self.ws)
        return y

    def backward(self, x, w, offsets, dy, dx=None, dw=None):
        """dx and dw, those that are given."""
        nat.nat_experts_bwd(self.params, offsets, self.cap, x, w, dy, dx, dw, self.ws)
        return dx, dw

    def status(self):
        """The NAT_DEV_* bits of the last call (waits for the stream)."""
        return nat.nat_poll_status(self.ws)
