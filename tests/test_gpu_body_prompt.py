"""Responses behind their prompts: prefix cutting, packing of prompt and prefix, attention, and the way back to the loss's
rows, against float64 attention over the whole, uncut sequences."""
import numpy as np
import pytest
import torch

from oracle import nat_body as ob
from paper_2603_06619_b200 import nat
from paper_2603_06619_b200.body import PackedSublayer
from test_gpu_body import _close, _half, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_prompt_and_prefix_in_one_sequence(dtype):
    G, Hq, Hkv, D = 4, 4, 2, 64
    prompts = np.repeat([37, 129, 0], G)                       # a prompt for each group, once for each response
    T = np.array([50, 1, 200, 0, 64, 300, 7, 128, 90, 33, 2, 140])
    B, scale = len(T), D ** -0.5
    whole, resp = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (prompts + T, T))
    n_whole, n_tot = int(whole[-1]), int(resp[-1])
    dev = lambda x, t=torch.int32: torch.as_tensor(x, dtype=t, device="cuda")  # noqa: E731
    empty = lambda n, t=torch.int32: torch.empty(n, dtype=t, device="cuda")  # noqa: E731
    mask, pi, cut = empty(n_tot, torch.uint8), empty(n_tot, torch.float32), empty(B)
    nat.nat_select(nat.select_params("rpc", min_cut=3, seed=5), B, dev(resp), n_tot, mask, pi, cut)
    idx, of, offs, n_rows = empty(n_whole), empty(n_whole), empty(B + 1), empty(1)
    nat.nat_compact_prefix(B, dev(whole), n_whole, dev(prompts) + cut, idx, of, offs, n_rows, n_whole)

    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    qkv = torch.randn(n_whole, Hq + 2 * Hkv, D, generator=g, device="cuda").to(dtype)
    packed = torch.full_like(qkv, float("nan"))
    nat.nat_gather_rows(qkv, idx, n_rows, n_whole, packed)
    sub = PackedSublayer(n_whole, B, Hq * D, Hq, Hkv, D, dtype)
    out = sub.attend(packed, offs)
    assert sub.status() == 0

    # the response's rows, in the order of the loss's compact lists
    s_idx, s_resp, s_offs, n_sel = empty(n_tot), empty(n_tot), empty(B + 1), empty(1)
    nat.nat_compact_prefix(B, dev(resp), n_tot, cut, s_idx, s_resp, s_offs, n_sel, n_tot)
    n = int(n_sel.item())
    at = torch.zeros(n_tot, dtype=torch.int32, device="cuda")
    r = s_resp[:n].long()
    at[:n] = offs[r] + dev(prompts)[r] + s_idx[:n] - dev(resp)[r]
    hidden = torch.empty(n_tot, Hq, D, dtype=dtype, device="cuda")
    nat.nat_gather_rows(out, at, n_sel, n_tot, hidden)

    Q, K, V = (_np(x) for x in qkv.split([Hq, Hkv, Hkv], dim=1))
    O, _, mag = ob.attn_fwd(Q, K, V, whole, scale)
    token = whole[:-1][r.cpu().numpy()] + prompts[r.cpu().numpy()] + (s_idx[:n] - dev(resp)[r]).cpu().numpy()
    assert n > 200 and (token < whole[1:][r.cpu().numpy()]).all()
    # as in test_gpu_body: P rounded to bfloat16, the result once more, and the 32-bit parts
    u, bf16 = _half(dtype), dtype == torch.bfloat16
    z = scale * np.linalg.norm(Q, axis=2).max() * np.linalg.norm(K, axis=2).max()
    e = ((D + 4) * z + (prompts + T).max() + 16) * 2.0 ** -23 + 2.0 ** -21
    _close("out", hidden[:n], O[token], (u if bf16 else 2.0 ** -24) * np.abs(O[token]) + ((u if bf16 else 0.0) + 2 * e) * 1.01 * mag[token])
