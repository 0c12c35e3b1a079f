"""The 8-bit outputs of the norms, code by code: what include/lq.h says of their rounding.

scale: one product of two roundings, within 2^-23 of max / 448.  code: y times a reciprocal of the scale that is within a step (2^-23), one rounding more (2^-24):
the quotient that is rounded to e4m3 is within 2^-22 of y / scale.
"""
import pytest
import torch

import linear_ref as ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu

VALUES = torch.arange(127, dtype=torch.uint8).view(ref.E4M3).double()             # 0 .. 448
MIDDLES = (VALUES[1:] + VALUES[:-1]) / 2


def index(x):
    """Number of the code that is nearest to a magnitude, the even one of two."""
    low, high = torch.searchsorted(MIDDLES, x), torch.searchsorted(MIDDLES, x, right=True)
    return torch.where(low % 2 == 0, low, high)


def test_index():
    assert torch.equal(index(VALUES), torch.arange(127)) and torch.equal(index(MIDDLES), (torch.arange(126) + 1) // 2 * 2)
    assert index(torch.tensor([1e9], dtype=torch.float64)).item() == 126


def check(y, code, scale):
    y, code, scale = y.double(), code.cpu(), scale.cpu().double()
    s = ref.scales(y)
    assert ((scale - s).abs() <= 2.0 ** -23 * s).all()
    q = (y / ref.spread(scale, y.shape[1])).abs()
    bits = code.view(torch.uint8).long()
    assert (index(q * (1 - 2.0 ** -22)) <= bits % 128).all() and (bits % 128 <= index(q * (1 + 2.0 ** -22))).all()
    assert ((bits >= 128) == torch.signbit(y)).all()


def rows(tokens, dim, seed, size=1.0):
    """Blocks of 128 whose values are next to the middle between two codes, every other row of any values."""
    g = torch.Generator().manual_seed(seed)
    blocks = -(-dim // 128)
    c = size * torch.exp(2 * torch.randn(tokens, blocks, 1, generator=g)).float()
    pick = torch.randint(0, 126, (tokens, blocks, 128), generator=g)
    near = c * MIDDLES[pick].float() * (1 + torch.randint(-4, 5, pick.shape, generator=g) * 2.0 ** -23)
    near[..., 0] = 448 * c[..., 0]
    any_ = c * 20 * torch.randn(tokens, blocks, 128, generator=g)
    y = torch.where((torch.arange(tokens) % 2 == 0)[:, None, None], near, any_)
    return (y * torch.sign(torch.randn(y.shape, generator=g))).flatten(1)[:, :dim].contiguous()


@pytest.mark.parametrize("dim", [128, 2048, 2001, 16384])
@pytest.mark.parametrize("size", [1.0, 1e-20, 1e30])
def test_codes_of_rows(dim, size):
    y = rows(40, dim, dim, size)
    code, scale = torch.empty((40, dim), dtype=ref.E4M3, device="cuda"), torch.empty((-(-dim // 128), 40), device="cuda")
    lq.norm_add(lq.AddShape(40, dim, norm=lq.NORM_NONE, type=lq.F32), y.cuda(), out8=code, scale=scale)
    check(y, code, scale)


@pytest.mark.parametrize("shift", [0, 1])
def test_codes_of_heads(shift):
    """A sigmoid of 200 is 1."""
    y = rows(40, 512, 9)
    wide = torch.zeros((40, 512 + shift), device="cuda")[:, shift:]
    wide.copy_(y)
    z = torch.full((40, 4, 128), 200.0, device="cuda")
    code, scale, out = torch.empty((40, 512), dtype=ref.E4M3, device="cuda"), torch.empty((4, 40), device="cuda"), torch.empty((40, 512), device="cuda")
    lq.norm_gate(lq.GatedShape(40, 4, norm=lq.NORM_NONE, silu=0, type=lq.F32), wide.unflatten(-1, (4, 128)), z, out=out, out8=code, scale=scale)
    assert torch.equal(out.cpu(), y)
    check(y, code, scale)
