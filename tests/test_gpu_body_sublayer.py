"""What a PackedSublayer keeps and reports."""
import pytest
import torch

from paper_2603_06619_b200 import nat
from paper_2603_06619_b200.body import PackedSublayer

pytestmark = pytest.mark.gpu


def _sublayer(cap=64, B=2, dtype=torch.bfloat16, **kw):
    return PackedSublayer(cap, B, 64, 2, 1, 64, dtype, **kw)


def _cu(*bounds):
    return torch.tensor(bounds, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("captured", [False, True])
def test_status_keeps_what_either_direction_found(captured, dtype):
    sub = _sublayer(dtype=dtype)
    qkv = torch.randn(64, 4, 64, device="cuda").to(dtype)
    dout = torch.randn(64, 2, 64, device="cuda").to(dtype)
    forward, backward = _cu(0, 30, 64), _cu(0, 30, 64)   # bounds of their own, to go wrong one by one

    def step():
        sub.attend(qkv, forward)
        sub.attend_backward(qkv, backward, dout)

    step()
    if captured:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        step = g.replay
    step()
    assert sub.status() == 0
    for of in (forward, backward):
        of[2] = 4000                                     # more rows than there are
        step()
        assert sub.status() == nat.NAT_DEV_CAPACITY
        of[2] = 64
        step()
        assert sub.status() == 0                         # of the last calls, not of all


def _steps(subs, shared, cap=512, d=256, Hq=4, Hkv=2, D=64, dtype=torch.bfloat16):
    """Forward and backward of a stack of sublayers; `shared` gives them their outputs, else they use their own.
    Returns the last dx and all weights' gradients."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    cu, n_rows = _cu(0, 100, cap - 7), _cu(cap - 7)
    w = 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
    x, qkvs, ys = rand(cap, d), [], []
    give = (lambda **kw: kw) if shared else (lambda **kw: {})
    r, h, dx, dy = (torch.empty(cap, d, dtype=dtype, device="cuda") for _ in range(4))
    dqkv = torch.empty(cap, Hq + 2 * Hkv, D, dtype=dtype, device="cuda")
    for sub in subs:
        qkvs.append(rand(cap, Hq + 2 * Hkv, D))
        ys.append(sub.attend(qkvs[-1], cu).reshape(cap, d))
        x, _ = sub.join(x, ys[-1], w, None, w, n_rows, **give(r=r, h=h))
        x = x.clone()
    grad, out = rand(cap, d), []
    for sub, qkv, y in reversed(list(zip(subs, qkvs, ys))):
        grad, gy = sub.join_backward(grad, rand(cap, d), w, None, w, n_rows, y=y, **give(dx=dx, dy=dy))
        grad = grad.clone()
        got = sub.attend_backward(qkv, cu, gy.view(cap, Hq, D), **give(dqkv=dqkv))
        out += [grad[:cap - 7].clone(), got[:cap - 7].clone(), sub.dw_post.clone(), sub.dw_pre.clone()]
    return out


def _stack(ckpt8, n=4):
    return [PackedSublayer(512, 2, 256, 4, 2, 64, torch.bfloat16, ckpt8=ckpt8) for _ in range(n)]


def test_sublayers_share_the_tensors_that_they_are_given():
    apart, shared = (_steps(_stack(True), s) for s in (False, True))
    assert all(torch.equal(a, b) for a, b in zip(apart, shared))


def test_join_backward_reads_the_r_that_its_join_wrote():
    """Without checkpoints: r in a tensor of the caller's."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, y, dr, dh, w, n_rows = rand(64, 64), rand(64, 64), rand(64, 64), rand(64, 64), 1 + 0.1 * rand(64), _cu(50)
    got = []
    for r in (None, torch.empty(64, 64, device="cuda")):
        sub = _sublayer(dtype=torch.float32, ckpt8=False)
        sub.r.fill_(7.0)
        out, _ = sub.join(x, y, w, None, w, n_rows, r=r)
        assert out is (sub.r if r is None else r)
        got.append([t[:50].clone() for t in sub.join_backward(dr, dh, w, None, w, n_rows, y=y)] + [sub.dw_pre])
    assert all(torch.equal(a, b) for a, b in zip(*got))
    with pytest.raises(nat.NatError, match="null pointer"):
        _sublayer(dtype=torch.float32, ckpt8=False).join_backward(dr, dh, w, None, w, n_rows, y=y)


def test_a_sublayer_holds_what_its_backward_pass_reads_and_no_more():
    cap, d, Hq, Hkv, D = 512, 256, 4, 2, 64
    _steps(_stack(True, 1), True)
    torch.cuda.synchronize()
    begin = torch.cuda.memory_allocated()
    subs = _stack(True)
    _steps(subs, True)
    held = (torch.cuda.memory_allocated() - begin) / len(subs)
    kept = cap * Hq * (2 * D + 4) + 2 * 4 * cap + 2 * cap * (d + 4 * 2)   # out, lse, norms, checkpoints
    spaces = subs[0].attn_ws.numel() + subs[0].norm_ws.numel()
    # and two rows of gradients, the status words, and the allocator's rounding of a dozen tensors to 512 bytes
    assert held <= kept + spaces + 2 * 4 * d + 16 * 512, (held, kept, spaces)


@pytest.mark.parametrize("ckpt8", [False, True])
def test_join_without_a_pre_norm_has_no_next_input(ckpt8):
    """The last sublayer of a stack: no h, and none of an earlier call in its place."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, y, dr, w, n_rows = rand(64, 64), rand(64, 64), rand(64, 64), 1 + 0.1 * rand(64), _cu(50)
    sub = _sublayer(dtype=torch.float32, ckpt8=ckpt8)
    assert sub.join(x, y, w, None, w, n_rows)[1] is sub.h
    r, h = sub.join(x, y, w, None, None, n_rows)
    assert h is None
    rstd = (y[:50].double().square().mean(dim=1, keepdim=True) + 1e-6).rsqrt()
    # three products and a sum in 32 bits, and a norm of 64 terms
    assert (r[:50] - (x[:50] + y[:50] * rstd * w)).abs().max() <= 80 * 2.0 ** -24 * 8
    dx, _ = sub.join_backward(dr, None, w, None, None, n_rows, y=y)
    assert torch.equal(dx[:50], dr[:50])
