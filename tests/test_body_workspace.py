"""Sizes of the attention workspace, and which sizes a call accepts (no GPU needed: nothing is enqueued)."""
import ctypes
import random

import pytest
import torch

from paper_2603_06619_b200 import nat

A = 4096                                   # a fake device address: nothing is dereferenced


def size(p, B, cap):
    return nat.nat_attn_workspace_bytes(p, B, cap)


def accepted(p, B, cap, nbytes, back):
    """Whether a call takes a workspace of that size: with one that is also misaligned it is refused either
    way, for its alignment only after its size."""
    fn, n = (nat.load().nat_attn_bwd, 9) if back else (nat.load().nat_attn_fwd, 5)
    status = fn(ctypes.byref(p), B, A, cap, *[A] * n, A + 16, nbytes, None)
    assert status in (-1, -3)
    return status == -1


def draw(r):
    Hkv, g = r.choice([1, 1, 2, 3, 4, 8]), r.choice([1, 2, 3, 4, 7, 8, 20, 64])
    p = nat.attn_params(Hkv * g, Hkv, 8 * r.randint(1, 16), r.choice([torch.float32, torch.bfloat16, torch.bfloat16]))
    return p, r.choice([1, 2, 5, 17, 64, 300, 5000]), r.choice([1, 700, 1024, 1025, 4096, 7000, 20000, 74000])


def bound(p, B, cap, pieces=True):
    """What include/nat.h says of the size."""
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    rows = cap * p.n_heads
    if p.dtype == nat.NAT_F32:
        return 256 + up(4 * rows) + (up(32 * (cap // 64 + B)) if B * p.n_heads > 2048 else 0)
    g = p.n_heads // p.n_kv_heads
    lists = sum(up(32 * (cap // t + B)) for t in (2 * (128 // g), 128 // g, 128))
    return 256 + 2 * up(4 * rows) + lists + (115 * 10 ** 6 if pieces else 0)


@pytest.mark.parametrize("seed", range(200))
def test_size_keeps_to_the_documented_bound(seed):
    p, B, cap = draw(random.Random(seed))
    assert 0 < size(p, B, cap) <= bound(p, B, cap)
    if p.dtype == nat.NAT_F32:
        assert size(p, B, cap) == bound(p, B, cap)


@pytest.mark.parametrize("seed", range(200))
def test_workspace_of_a_larger_batch_serves_a_smaller_one(seed):
    r = random.Random(seed)
    p, B, cap = draw(r)
    least_B, least_cap = r.randint(1, B), r.randint(1, cap)
    for back in (False, True):
        assert accepted(p, B, cap, size(p, B, cap), back)
        assert accepted(p, least_B, least_cap, size(p, B, cap), back)
        # no more than the parts that grow with B and cap is ever needed, and never less than a row's
        assert accepted(p, B, cap, bound(p, B, cap, pieces=False), back)
        assert not accepted(p, B, cap, 4 * cap * p.n_heads, back)
