"""Packed attention over many short sequences, against the float64 form; and how its time grows with them."""
import random

import pytest
import torch

from paper_2603_06619_b200 import nat
from test_gpu_body import DT, Attn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,heads", [(1024, (2, 1, 64)), (1025, (2, 1, 64)), (3000, (2, 2, 32)), (300, (8, 2, 128))])
def test_many_short_sequences(B, heads, dtype):
    r = random.Random(B)
    Attn([r.choice([0, 1, 2, 3, 5, r.randint(0, 70)]) for _ in range(B)], *heads, DT[dtype], seed=B).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_faults_among_many_sequences(dtype):
    B = 1500
    a, b = (Attn([2] * B, 2, 1, 64, DT[dtype], seed=1, spare=0) for _ in range(2))
    a.fwd()
    a.bwd()
    b.cu[-1] = 4000                                # more rows than the buffers hold
    for run in (b.fwd, b.bwd):
        run()
        assert nat.nat_poll_status(b.ws) == nat.NAT_DEV_CAPACITY
    for name in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    b.cu[700] = 5                                  # bounds that do not ascend
    for t in (b.out, b.dq, b.dk, b.dv):
        t.fill_(7.0)
    for run in (b.fwd, b.bwd):
        run()
        assert nat.nat_poll_status(b.ws) == nat.NAT_DEV_CAPACITY
    for t in (b.out, b.dq, b.dk, b.dv):
        assert (t == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("back", [False, True])
def test_time_grows_with_the_sequences_not_with_their_square(back, dtype):
    """16,384 and 65,536 sequences of 4 tokens: a factor of 4 in the work; a search of all bounds in every
    block would make it 16."""
    took = []
    for B in (16384, 65536):
        a = Attn([4] * B, 2, 1, 64, DT[dtype], seed=2, spare=0)
        a.fwd()
        run = a.bwd if back else a.fwd
        run()
        times = []
        for _ in range(5):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            run()
            end.record()
            end.synchronize()
            times.append(begin.elapsed_time(end))
        took.append(min(times))
    assert took[1] < 8 * took[0], took
