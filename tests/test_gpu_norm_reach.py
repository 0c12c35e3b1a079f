"""The norms of the 8-bit linear layer at the ends of their range: sizes, strides, values; against their definitions in 64 bits.

Tolerances as in test_gpu_rownorm.py: 2^-18 of the value and one rounding to the type.
"""
import pytest
import torch

import linear_ref as ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [1e-25, 1e15, 1e18, 1e19, 1e25])
@pytest.mark.parametrize("norm", [lq.NORM_L2, lq.NORM_RMS])
def test_sums_of_squares_beyond_binary32(size, norm):
    """A row whose sum of squares is not finite in binary32 becomes 0, as the header says; below that nothing happens to it."""
    x = size * torch.randn(6, 256, generator=torch.Generator().manual_seed(1))
    over = (x.double() ** 2).sum(-1) > 2.0 ** 128
    out = torch.empty((6, 256), device="cuda")
    lq.norm_add(lq.AddShape(6, 256, norm=norm, type=lq.F32, eps=1e-30), x.cuda(), out=out)
    heads = torch.empty((6, 256), device="cuda")
    lq.norm_gate(lq.GatedShape(6, 1, dim=256, norm=norm, silu=0, type=lq.F32, eps=1e-30), x.cuda()[:, None], torch.full((6, 1, 256), 200.0, device="cuda"), out=heads)
    want = ref.norm(x.double(), norm, None, 1e-30)
    want[over] = 0.0
    assert over.all() == (size >= 1e19)
    for got in (out, heads):
        assert ((got.cpu().double() - want).abs() <= (2.0 ** -18 + 2.0 ** -24) * want.abs()).all()


@pytest.mark.parametrize("dim", [1, 130, 4096])
def test_one_row_of_any_stride(dim):
    """A slice of one row: its stride is not looked at."""
    x = torch.randn((1, dim), generator=torch.Generator().manual_seed(dim)).bfloat16().cuda()
    wide = torch.zeros((1, 3 * dim), dtype=torch.bfloat16, device="cuda")
    view, out, own = wide[:, dim:2 * dim], torch.empty_like(x), torch.empty_like(x)
    view.copy_(x)
    lq.norm_add(lq.AddShape(1, dim), x, out=own)
    lq.norm_add(lq.AddShape(1, dim), view, out=out)
    assert torch.equal(out, own)
    lq.norm_add(lq.AddShape(1, dim), view, out=view)
    assert torch.equal(view, own) and (wide[:, :dim] == 0).all() and (wide[:, 2 * dim:] == 0).all()


def test_columns_of_one_element():
    """Rows of one channel, strided: the channels of a larger array one by one."""
    wide = torch.randn((50, 7), generator=torch.Generator().manual_seed(2)).cuda()
    before = wide.clone()
    out = torch.empty((50, 1), device="cuda")
    lq.norm_add(lq.AddShape(50, 1, type=lq.F32, eps=0.0), wide[:, 3:4], out=out)
    assert torch.allclose(out, torch.sign(before[:, 3:4]), rtol=1e-6)
    lq.norm_add(lq.AddShape(50, 1, type=lq.F32, eps=0.0), wide[:, 3:4], out=wide[:, 3:4])
    want = before.clone()
    want[:, 3:4] = out
    assert torch.equal(wide, want)
