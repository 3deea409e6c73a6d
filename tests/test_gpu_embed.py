"""GPU parity of the embedding and its table's gradient against the float64 forms in ``oracle/nat_packed.py``.

Tolerances, by arithmetic: a looked-up element is one product, rounded in 32 bits (2^-24) and to its type (half a step,
u = finfo.eps / 2); a gradient's element is a sum of m rows in 32 bits, (m + 2) 2^-24 of the sum of their
magnitudes, the scale's product among it, and one more of the old value where it is added to that.
"""
import numpy as np
import pytest
import torch

from oracle import nat_packed as op
from paper_2603_06619_b200 import nat

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _np(t):
    return t.detach().double().cpu().numpy()


class Embed:
    """A batch with NaN gradients behind the last row and poisoned outputs."""

    def __init__(self, n, V, d, dtype, seed=0, spare=5, scale=1.0, picked=False, accumulate=False, ids=None):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.n, self.V, self.d, self.cap, self.dtype, self.scale = n, V, d, n + spare, dtype, float(np.float32(scale))
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        n_tot = 2 * self.cap + 1 if picked else max(self.cap, 1)
        # a few ids are far more frequent than the others
        u = torch.rand(n_tot, generator=g, device="cuda")
        all_ids = (u ** 3 * V).long().clamp(max=V - 1) * 7919 % V
        self.sel = None
        if picked:
            order = torch.rand(n_tot, generator=g, device="cuda").argsort()[:self.cap].sort().values
            self.sel = order.to(torch.int32)
        if ids is not None:
            at = torch.arange(n, device="cuda") if self.sel is None else self.sel[:n].long()
            all_ids[at] = torch.as_tensor(ids, device="cuda")
        self.ids = all_ids.to(torch.int32)
        self.of_rows = (self.ids[:n] if self.sel is None else self.ids[self.sel[:n].long()]).cpu().numpy()
        self.table = rand(V, d).to(dtype)
        self.x = torch.full((max(self.cap, 1), d), 7.0, dtype=dtype, device="cuda")
        self.dx = rand(max(self.cap, 1), d).to(dtype)
        self.dx[n:] = float("nan")
        self.old = rand(V, d)
        self.dtable = self.old.clone() if accumulate else torch.full((V, d), 7.0, device="cuda")
        self.n_rows = torch.tensor([n], dtype=torch.int32, device="cuda")
        self.params = nat.embed_params(V, d, dtype, scale=scale, accumulate=accumulate)
        self.ws = nat.alloc_workspace(nat.nat_embed_workspace_bytes(self.params, self.cap), "cuda")
        self.ws.random_(0, 255)

    def fwd(self):
        nat.nat_embed_fwd(self.params, self.table, self.ids, self.sel, self.n_rows, self.cap, self.x)

    def bwd(self):
        nat.nat_embed_bwd(self.params, self.ids, self.sel, self.n_rows, self.cap, self.dx, self.dtable, self.ws)

    def check(self):
        self.fwd()
        ref = op.embed_fwd(_np(self.table), self.of_rows, self.scale)
        u = 2.0 ** -24 + (2.0 ** -8 if self.dtype == torch.bfloat16 else 0.0)
        got = _np(self.x[:self.n])
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        assert (np.nan_to_num(np.abs(got - ref)) <= 1.001 * u * np.nan_to_num(np.abs(ref)) + 1e-37).all()
        assert (self.x[self.n:] == 7).all()
        self.bwd()
        bad = ((self.of_rows < 0) | (self.of_rows >= self.V)).any()
        assert nat.nat_poll_status(self.ws) == (nat.NAT_DEV_BAD_TARGET if bad else 0)
        ref, mag, count = op.embed_bwd(_np(self.dx[:self.n]), self.of_rows, self.V, self.scale)
        tol = (count[:, None] + 2) * 2.0 ** -24 * mag
        if self.params.accumulate:
            assert torch.equal(self.dtable[torch.from_numpy(count == 0).cuda()], self.old[torch.from_numpy(count == 0).cuda()])
            ref = ref + _np(self.old)
            tol = tol + 2.0 ** -24 * (np.abs(_np(self.old)) + mag)
        over = np.abs(_np(self.dtable) - ref) - 1.001 * tol - 1e-37
        assert (over <= 0).all(), (float(over.max()), np.argwhere(over > 0)[:4].tolist())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,V,d", [(0, 5, 8), (1, 1, 8), (1, 700, 64), (290, 512, 64), (128, 3, 136), (129, 1, 40),
                                   (700, 2, 256), (4096, 300, 72), (4097, 300, 72), (9001, 70000, 24), (500, 50, 2056),
                                   (20000, 37, 16), (300, 9, 4096), (40, 1000, 8200), (2049, 5, 8), (1024, 700, 40), (1025, 9, 72), (70001, 400, 8),
                                   (70001, 1 << 20, 8), (300001, 150000, 8), (262144, 200, 8)])
def test_embed_parity(n, V, d, dtype):
    Embed(n, V, d, DT[dtype], seed=n + V, scale=0.75 if d > 64 else 1.0, picked=n % 2 == 1).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [100, 5000])
def test_embed_added_to_a_table_gradient(n, dtype):
    Embed(n, 400, 136, DT[dtype], seed=3, scale=-2.5, accumulate=True, picked=True).check()


@pytest.mark.parametrize("n", [60, 6000])
@pytest.mark.parametrize("picked", [False, True])
def test_embed_ids_outside_the_table(picked, n):
    ids = np.arange(n) % 50
    ids[5], ids[17], ids[40], ids[41] = -1, 50, 2 ** 31 - 1, -2 ** 31
    e = Embed(n, 50, 64, torch.bfloat16, seed=4, ids=ids, picked=picked)
    assert (e.of_rows[[5, 17, 40, 41]] == [-1, 50, 2 ** 31 - 1, -2 ** 31]).all()
    e.check()
    # none valid at all
    e = Embed(n, 50, 64, torch.float32, seed=5, ids=np.full(n, 77), picked=picked)
    e.check()
    assert (e.dtable == 0).all()


@pytest.mark.parametrize("lengths", [[129, 127, 128, 1], [1, 255, 256, 257], [128, 128, 129, 383, 5], [1000], [127, 2000, 3],
                                     [65, 63, 64, 1], [1, 63, 64, 65, 66], [64, 64, 65, 191, 5], [64], [65], [63, 1, 64, 2]])
def test_embed_rows_that_end_where_pieces_do(lengths):
    """Table rows of lengths around a piece's, in the order of their ids."""
    ids = np.repeat(np.arange(len(lengths)) * 3, lengths)
    np.random.default_rng(0).shuffle(ids)
    Embed(len(ids), 3 * len(lengths) + 4, 264, torch.float32, seed=6, ids=ids).check()


def test_embed_order_of_the_sums_is_the_tokens():
    """One large term first: the small ones behind it are lost one by one, in the tokens' order and no other."""
    n, d = 60, 8
    e = Embed(n, 4, d, torch.float32, seed=7, ids=np.full(n, 2))
    e.dx[:n] = 1.0
    e.dx[0] = 2.0 ** 24
    e.bwd()
    assert (e.dtable[2] == 2.0 ** 24).all()
    e.dx[0], e.dx[n - 1] = 1.0, 2.0 ** 24
    e.bwd()
    assert (e.dtable[2] == 2.0 ** 24 + 60).all()      # 59 ones, then a tie to even


def test_embed_repeats_bit_for_bit_and_replays_with_other_rows():
    e = Embed(7000, 900, 128, torch.bfloat16, seed=8, picked=True)
    e.fwd()
    e.bwd()
    first = [e.x.clone(), e.dtable.clone()]
    e.ws.random_(0, 255)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        e.fwd()
        e.bwd()
    e.x.fill_(7.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(e.x, first[0]) and torch.equal(e.dtable, first[1])
    e.n_rows.fill_(100)
    e.x.fill_(7.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(e.x[:100], first[0][:100]) and (e.x[100:] == 7).all()
    ref, mag, count = op.embed_bwd(_np(e.dx[:100]), e.of_rows[:100], e.V, 1.0)
    assert (np.abs(_np(e.dtable) - ref) <= 1.01 * (count[:, None] + 2) * 2.0 ** -24 * mag).all()
    # more rows than there is room for: as many as there are
    e.n_rows.fill_(1 << 30)
    e.dx[e.n:] = 0
    e.x.fill_(7.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(e.x[:7000], first[0][:7000]) and not (e.x[7000:] == 7).any()


def test_embed_two_calls_at_once():
    a, b = Embed(5000, 300, 256, torch.bfloat16, seed=9), Embed(3000, 5000, 64, torch.float32, seed=10)
    want = []
    for e in (a, b):
        e.fwd()
        e.bwd()
        want += [e.x.clone(), e.dtable.clone()]
        e.x.fill_(7.0)
        e.dtable.fill_(7.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, e in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            e.fwd()
            e.bwd()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, (a.x, a.dtable, b.x, b.dtable)))


def test_embed_past_32_bits():
    """A table whose elements lie more than 2^31 behind its first, and rows as far."""
    V, d, n = 140000, 16384, 140001
    assert V * d > 1 << 31
    table = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    table.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    ids = (torch.arange(n, device="cuda") * 7919 % V).to(torch.int32)
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    p = nat.embed_params(V, d, torch.bfloat16)
    nat.nat_embed_fwd(p, table, ids, None, None, n, x)
    assert torch.equal(x[-64:], table[ids[-64:].long()]) and torch.equal(x[:64], table[ids[:64].long()])
    del table
    dtable = torch.empty(V, d, device="cuda")
    ws = nat.alloc_workspace(nat.nat_embed_workspace_bytes(p, n), "cuda")
    nat.nat_embed_bwd(p, ids, None, None, n, x, dtable, ws)
    for v in (0, 1, 70000, V - 1):
        want = torch.zeros(d, device="cuda")
        for k in (ids == v).nonzero().flatten().tolist():
            want += x[k].float()
        assert torch.equal(dtable[v], want)


def test_embed_nan_and_infinities_stay_in_their_row():
    a, b = (Embed(3000, 200, 64, torch.bfloat16, seed=11) for _ in range(2))
    b.dx[17], b.table[5] = float("nan"), float("inf")
    for e in (a, b):
        e.fwd()
        e.bwd()
    keep = torch.arange(200, device="cuda") != int(a.of_rows[17])
    assert torch.equal(a.dtable[keep], b.dtable[keep]) and b.dtable[~keep].isnan().all()
    rows = torch.from_numpy(a.of_rows != 5).cuda()
    assert torch.equal(a.x[:3000][rows], b.x[:3000][rows])
