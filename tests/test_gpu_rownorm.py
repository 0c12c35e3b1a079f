"""Norms around the projections (whole rows with the residual, heads with a gate), against their definitions in 64 bits.

Tolerance: one rounding to the result's type (half a step; e4m3 relative to the block's scale below 2^-6 of it), and binary32 inside: a sum of
squares has at most 32 + 5 + 16 additions on its way, 2^-24 each and half of that after the root, a root of 2^-22, products and the scale's
quotient - below 2^-18 of the value.  The gate: an exponential whose argument is off by 1.5 * 2^-24 * 1.45 |z|, 2^-21.3 for the two functions: below 2^-21 +
2^-23 |z|, and what is below 2^-119 may be 0.
"""
import pytest
import torch

import linear_ref as ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
FILL = 7.0


def wide(rows, cols, pad, dtype, values=None, shift=None):
    """A [rows, cols] slice of a buffer that is FILL elsewhere."""
    buf = torch.full((rows, cols + pad), FILL, device="cuda").to(dtype)
    at = pad // 2 if shift is None else shift
    view = buf[:, at:at + cols]
    if values is not None:
        view.copy_(values)
    return buf, view


def untouched(buf, view):
    at = view.storage_offset()
    rest = buf.clone().float()
    rest[:, at:at + view.shape[1]] = FILL
    return bool((rest == FILL).all())


def check(outs, want, dtype, extra=0.0):
    """outs: out, out8, scale or None; want [rows, channels]"""
    out, out8, scale = outs
    slack = (2.0 ** -18 + extra) * want.abs() + (2.0 ** -119 if torch.is_tensor(extra) else 0.0)
    if out is not None:
        assert ref.off(out.cpu(), want, dtype, slack) <= 1
    if out8 is not None:
        s = ref.scales(want)
        got = scale.cpu().double()
        most = float(extra.max()) if torch.is_tensor(extra) else extra
        assert ((got - s).abs() <= (2.0 ** -18 + most) * s).all()
        by = ref.spread(got, want.shape[1])
        d = (out8.cpu().double() * by - want).abs()
        assert (d <= 2.0 ** -4 * want.abs() + 2.0 ** -10 * by + 2 * slack).all(), float((d / by).max())


def add(tokens, dim, norm, dtype, residual=True, outs="both", pad=0, shift=None, weights=True, in_place=False, seed=0, size=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (size * torch.randn(tokens, dim, generator=g)).to(dtype)
    r = (3 * size * torch.randn(tokens, dim, generator=g)).to(dtype) if residual else None
    w = 1 + 0.3 * torch.randn(dim, generator=g) if weights and norm == lq.NORM_RMS else None
    bx, dx = wide(tokens, dim, pad, dtype, x, shift)
    br, dr = wide(tokens, dim, pad, dtype, r, shift) if residual else (None, None)
    bo, do = (bx, dx) if in_place else wide(tokens, dim, pad, dtype, shift=shift) if outs in ("both", "out") else (None, None)
    b8, d8 = wide(tokens, dim, pad, ref.E4M3, shift=shift) if outs in ("both", "out8") else (None, None)
    bs, ds = wide(-(-dim // 128), tokens, pad, torch.float32, shift=shift) if d8 is not None else (None, None)
    sh = lq.AddShape(tokens, dim, norm=norm, type=lq.TYPES[dtype], eps=1e-5)
    lq.norm_add(sh, dx, residual=dr, w=None if w is None else w.cuda(), out=do, out8=d8, scale=ds)
    h = x.double() + (r.double() if residual else 0.0)
    if residual:
        assert ref.off(dr.cpu(), h, dtype, 2.0 ** -24 * h.abs()) <= 1
    check((do, d8, ds), ref.norm(h, norm, w, 1e-5), dtype)
    for b, v in ((bx, dx), (br, dr), (bo, do), (b8, d8), (bs, ds)):
        assert b is None or untouched(b, v)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("norm", [lq.NORM_NONE, lq.NORM_L2, lq.NORM_RMS])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("outs", ["out", "out8", "both"])
def test_every_form_of_rows(dtype, norm, residual, outs):
    add(5, 640, norm, dtype, residual, outs, pad=16, shift=8)


@pytest.mark.parametrize("dim", [1, 2, 7, 8, 100, 127, 128, 129, 256, 264, 1000, 1291, 2048, 2056, 4096, 4104, 8192, 8200, 12345, 16384])
def test_channels_of_rows(dim):
    add(3, dim, lq.NORM_RMS, torch.bfloat16, seed=dim)
    add(3, dim, lq.NORM_RMS, torch.float32, residual=False, seed=dim)


@pytest.mark.parametrize("tokens", [1, 2, 7, 8, 9, 300])
@pytest.mark.parametrize("dim", [64, 136, 520, 1024])
def test_rows_that_share_a_cta(tokens, dim):
    add(tokens, dim, lq.NORM_RMS, torch.bfloat16, seed=tokens)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("pad,shift", [(1, 0), (3, 1), (8, 4), (16, 8), (1, 1)])
def test_rows_of_any_alignment(dtype, pad, shift):
    add(6, 384, lq.NORM_RMS, dtype, pad=pad, shift=shift)
    add(6, 384, lq.NORM_L2, dtype, pad=pad, shift=shift, in_place=True)


def test_rows_in_place():
    add(40, 4096, lq.NORM_RMS, torch.bfloat16, in_place=True)
    add(40, 200, lq.NORM_RMS, torch.bfloat16, residual=False, in_place=True)


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e12])
def test_sizes_of_values(size):
    add(9, 512, lq.NORM_NONE, torch.float32, size=size)
    add(9, 512, lq.NORM_RMS, torch.float32, size=size, weights=False)


def test_blocks_of_zeros_and_of_what_is_not_finite():
    x = torch.randn(4, 512, generator=torch.Generator().manual_seed(1))
    x[0] = 0.0
    x[1, 130], x[2, 300], x[3, 5] = float("nan"), float("inf"), 1e-38
    out8, scale = torch.empty((4, 512), dtype=ref.E4M3, device="cuda"), torch.empty((4, 4), device="cuda")
    lq.norm_add(lq.AddShape(4, 512, norm=lq.NORM_NONE, type=lq.F32), x.cuda(), out8=out8, scale=scale)
    y = (out8.float() * ref.spread(scale, 512)).cpu()
    assert (y[0] == 0).all() and (scale[:, 0] == 2.0 ** -100).all()
    assert torch.isnan(y[1, 130]) and torch.isnan(y[1]).sum() == 1
    assert torch.isnan(y[2, 256:384]).all() and torch.isnan(y[2]).sum() == 128
    assert torch.isfinite(y[3]).all()
    rows = torch.zeros(3, 256, device="cuda")
    rows[1, 7] = float("nan")
    rows[2] = 1.0
    out = torch.empty_like(rows)
    lq.norm_add(lq.AddShape(3, 256, type=lq.F32, eps=1e-6), rows, out=out)
    assert (out[0] == 0).all() and torch.isnan(out[1]).all() and torch.allclose(out[2], torch.ones(256, device="cuda"))


def gate(tokens, heads, dim, norm, dtype, o_type=torch.float32, silu=True, outs="both", pad=0, shift=None, weights=True, seed=0, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    o = torch.randn(tokens, heads, dim, generator=g).to(o_type)
    z = (spread * torch.randn(tokens, heads, dim, generator=g)).to(dtype)
    w = 1 + 0.3 * torch.randn(dim, generator=g) if weights and norm == lq.NORM_RMS else None
    width = heads * dim
    bo, do = wide(tokens, width, pad, o_type, o.flatten(1), shift)
    bz, dz = wide(tokens, width, pad, dtype, z.flatten(1), shift)
    by, dy = wide(tokens, width, pad, dtype, shift=shift) if outs in ("both", "out") else (None, None)
    b8, d8 = wide(tokens, width, pad, ref.E4M3, shift=shift) if outs in ("both", "out8") else (None, None)
    bs, ds = wide(-(-width // 128), tokens, pad, torch.float32, shift=shift) if d8 is not None else (None, None)
    sh = lq.GatedShape(tokens, heads, dim=dim, norm=norm, silu=int(silu), o_type=lq.TYPES[o_type], type=lq.TYPES[dtype], eps=1e-5)
    lq.norm_gate(sh, do.unflatten(-1, (heads, dim)), dz.unflatten(-1, (heads, dim)), w=None if w is None else w.cuda(), out=dy, out8=d8, scale=ds)
    zz = z.double()
    want = ref.norm(o.double(), norm, w, 1e-5) * torch.sigmoid(zz) * (zz if silu else 1.0)
    check((dy, d8, ds), want.flatten(1), dtype, (2.0 ** -21 + 2.0 ** -23 * zz.abs()).flatten(1))
    for b, v in ((by, dy), (b8, d8), (bs, ds)):
        assert b is None or untouched(b, v)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("o_type", TYPES, ids=str)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("norm,silu,outs", [(lq.NORM_RMS, True, "both"), (lq.NORM_RMS, False, "out8"), (lq.NORM_L2, True, "out"), (lq.NORM_NONE, False, "both")])
def test_every_form_of_heads(dtype, o_type, dim, norm, silu, outs):
    gate(5, 3, dim, norm, dtype, o_type, silu, outs)


@pytest.mark.parametrize("tokens", [1, 2, 9, 100])
@pytest.mark.parametrize("heads,dim", [(1, 64), (1, 128), (1, 256), (7, 64), (32, 128), (5, 256), (33, 64)])
def test_rows_and_heads(tokens, heads, dim):
    gate(tokens, heads, dim, lq.NORM_RMS, torch.bfloat16, seed=tokens)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("pad,shift", [(1, 0), (3, 1), (8, 4), (16, 8), (1, 1)])
def test_heads_of_any_alignment(dtype, pad, shift):
    gate(6, 3, 128, lq.NORM_RMS, dtype, pad=pad, shift=shift)
    gate(6, 3, 64, lq.NORM_RMS, dtype, o_type=torch.bfloat16, pad=pad, shift=shift)


@pytest.mark.parametrize("silu", [False, True])
def test_gates_over_their_range(silu):
    gate(64, 2, 128, lq.NORM_NONE, torch.float32, silu=silu, spread=30.0, weights=False)
    z = torch.tensor([200.0, -200.0, 90.0, -90.0, 0.0, -87.0, 1e30, -1e30], device="cuda").repeat(16).reshape(1, 1, 128)
    y = torch.empty((1, 128), device="cuda")
    lq.norm_gate(lq.GatedShape(1, 1, norm=lq.NORM_NONE, silu=int(silu), type=lq.F32), torch.ones_like(z), z, out=y)
    want = torch.sigmoid(z.double()) * (z.double() if silu else 1.0)
    assert ((y.double() - want[0]).abs() <= 2.0 ** -15 * want[0].abs() + 2.0 ** -119).all()
