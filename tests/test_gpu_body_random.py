"""Seeded random draws from the shape space of the body's operators, against the float64 forms."""
import random

import pytest
import torch

from test_gpu_body import Attn, Join

pytestmark = pytest.mark.gpu


def draw_attn(r):
    dtype = r.choice([torch.float32, torch.bfloat16, torch.bfloat16])
    Hkv = r.choice([1, 1, 2, 3])
    g = r.choice([1, 1, 2, 3, 4, 5, 6, 8, 11, 16])
    D = 8 * r.randint(1, 16)
    law = r.choice(["short", "mixed", "long", "one"])
    if law == "short":
        lengths = [r.randint(0, 40) for _ in range(r.randint(1, 60))]
    elif law == "mixed":
        lengths = [r.choice([0, 1, r.randint(2, 300), r.choice([63, 64, 65, 127, 128, 129, 255, 256, 257])])
                   for _ in range(r.randint(1, 6))]
    elif law == "long":
        lengths = [r.randint(900, 1700)] + [r.randint(0, 200) for _ in range(r.randint(0, 2))]
        g = min(g, 4)
        Hkv = 1
    else:
        lengths = [r.randint(1, 700)]
    lengths[0] = max(1, lengths[0])
    return lengths, Hkv * g, Hkv, D, dtype, r.choice([0, 1, 130]), r.random() < 0.5, r.choice([0.5, 2.0, 8.0])


@pytest.mark.parametrize("seed", range(40))
def test_random_attention(seed):
    lengths, Hq, Hkv, D, dtype, spare, fused, sharp = draw_attn(random.Random(seed))
    Attn(lengths, Hq, Hkv, D, dtype, seed=seed, spare=spare, fused=fused, sharp=sharp).check()


@pytest.mark.parametrize("seed", range(40))
def test_random_join(seed):
    r = random.Random(1000 + seed)
    d = 8 * r.choice([r.randint(1, 64), r.randint(65, 512), r.randint(513, 1024)])
    n = r.randint(1, max(1, min(900, 300000 // d)))
    Join(n, d, r.choice([torch.float32, torch.bfloat16]), gate=r.choice(["none", "channel", "row"]),
         parts=r.choice(["all", "all", "no_post", "no_pre", "no_dr"]), ckpt=r.random() < 0.5, seed=seed,
         spare=r.randint(0, 5), eps=r.choice([1e-6, 1e-2]), alpha=r.choice([1.0, 0.3, -0.7])).check()
