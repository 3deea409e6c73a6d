"""The two quotients of an 8-bit checkpoint, 1 / top and top / 127, for every mantissa of a group's largest magnitude.

Both are checked against float64, rounded once more.  That rounding is safe: m h of a 24-bit m and a 25-bit midpoint h
is a multiple of 2^-48, so 1 / m keeps at least 2^-49 from h, and top / 127 a 254th of a step: neither is lost in 53
bits.  The factor (1 / top) 127 itself is not stored; it is seen through the codes of elements next to the
borders between two codes, where one unit in its last place decides.
"""
import pytest
import torch

from paper_2603_06619_b200 import nat

pytestmark = pytest.mark.gpu

N = 1 << 23


def _bits(x):
    return x.view(torch.int32)


# 2^-120 is the smallest magnitude that is kept; below 2^-119 and a little the scale is subnormal; above 2^126 the
# reciprocal would be
@pytest.mark.parametrize("exponent", [-120, -119, -118, -1, 0, 1, 64, 125, 126, 127])
def test_quotients_of_every_mantissa(exponent):
    top = torch.arange(N, dtype=torch.int32, device="cuda").add_((exponent + 127) << 23).view(torch.float32)
    mantissa = top.double() * 2.0 ** -exponent
    inv = ((1.0 / mantissa).float() * 127.0).double() * 2.0 ** -exponent     # normal for every exponent here
    inv = inv.float()
    x = torch.empty(N, 8, device="cuda")
    x[:, 0] = -top
    lane = torch.arange(N, device="cuda")
    for j in range(1, 8):      # seven of the 127 borders each, another seven in the next row, and their neighbours
        border = ((lane * 7 + j * 18) % 126 + 0.5).double() / inv.double()
        near = border.float()
        step = (lane + j) % 3 - 1
        x[:, j] = (_bits(near) + step.int()).view(torch.float32)
    assert (x.abs().amax(dim=1) == top).all()
    codes, scales = torch.empty(N, 8, dtype=torch.int8, device="cuda"), torch.empty(N, 1, device="cuda")
    nat.nat_ckpt8_store(x, None, N, codes, scales)
    assert torch.equal(_bits(scales[:, 0]), _bits((top.double() / 127.0).float()))
    want = torch.round(x * inv[:, None])
    assert torch.equal(codes.float(), want)
    # the borders are met: some products lie on one, and both sides of it occur
    off = (x[:, 1:] * inv[:, None]).abs() % 1.0 - 0.5
    assert (off == 0).any() and (off > 0).any() and (off < 0).any()


def test_magnitudes_around_the_smallest_kept():
    x = torch.zeros(4, 8, device="cuda")
    x[:, 3] = torch.tensor([2.0 ** -120, 2.0 ** -120 * (1 - 2.0 ** -24), -(2.0 ** -149), 2.0 ** -119], device="cuda")
    codes, scales = torch.full((4, 8), 9, dtype=torch.int8, device="cuda"), torch.full((4, 1), 9.0, device="cuda")
    nat.nat_ckpt8_store(x, None, 4, codes, scales)
    assert codes[:, 3].tolist() == [127, 0, 0, 127] and (codes[:, [0, 1, 2, 4, 5, 6, 7]] == 0).all()
    assert (scales[1:3] == 0).all() and (scales[[0, 3]] > 0).all()
