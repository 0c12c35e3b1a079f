"""Norms of queries and keys with the position rotation, against their definition in 64 bits.

Tolerance: one rounding to the result's type (half a step), and binary32 inside: the sum of squares is off by at most 2^-24 times the
additions on its way (8 + 5), half of that after the root, the root itself, three products and the pair's two - below 2^-19 of the pair's
magnitude; the fraction of a turn below one half is rounded to 2^-25 of a turn, 2^-22.3 as an angle.  fp16 results below 2^-14 are
rounded to steps of 2^-24.
"""
import pytest
import torch

import ops_ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
FILL = 55.0


def run(tokens, hq, hk, dim, rot, pairs, norm, dtype, pad=0, in_place=False, far=1 << 20, weights=True, positions=None, scale=(0.125, 1.0), shift=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    sides, outs, ref = [], [], []
    pos = positions if positions is not None else torch.randint(0, far, (tokens,), generator=g, dtype=torch.int32)
    freq = (10000.0 ** -(torch.arange(rot // 2, dtype=torch.float64) * 2 / max(rot, 1))).float()
    wts = [1 + 0.3 * torch.randn(dim, generator=g) if weights and norm == 2 else None for _ in range(2)]
    for h in (hq, hk):
        wide = torch.randn((tokens, h * dim + pad), generator=g).to(dtype)
        x = wide[:, shift:shift + h * dim].unflatten(-1, (h, dim)) if h else None
        xd = wide.cuda()[:, shift:shift + h * dim].unflatten(-1, (h, dim)) if h else None
        sides.append(xd)
        outs.append(xd if in_place else torch.full((tokens, h, dim), FILL, dtype=dtype, device="cuda") if h else None)
        ref.append(x)
    sh = lq.NormShape(tokens, hq, hk, dim=dim, rot=rot, pairs=int(pairs), norm=norm, type=lq.TYPES[dtype], eps=1e-5, scale_q=scale[0], scale_k=scale[1])
    use = rot > 0 or positions is not None
    lq.norm_rotate(sh, sides[0], sides[1], outs[0], outs[1], w_q=None if wts[0] is None else wts[0].cuda(), w_k=None if wts[1] is None else wts[1].cuda(),
                   positions=pos.cuda() if use else None, inv_freq=freq.cuda() if rot else None)
    for x, out, w, s in zip(ref, outs, wts, scale):
        if x is None:
            continue
        want, size = ops_ref.norm_rotate(x, w, norm, 1e-5, s, pos, freq, pairs)
        got = out.cpu()
        live = pos >= 0 if use else torch.ones(tokens, dtype=torch.bool)
        assert torch.equal(got[~live], x[~live] if in_place else torch.full_like(got[~live], FILL))
        bound = ops_ref.half_step(dtype) * want.abs() + 2.0 ** -19 * size + (2.0 ** -25 if dtype is torch.float16 else 1e-37)
        off = ((got.double() - want).abs() / bound)[live]
        assert off.numel() == 0 or off.max() <= 1, float(off.max())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("norm", [lq.NORM_NONE, lq.NORM_L2, lq.NORM_RMS])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rot,pairs", [(0, False), (16, False), (16, True), (48, False), (64, True), ("all", False), ("all", True)])
def test_every_form(dtype, norm, dim, rot, pairs):
    run(5, 3, 2, dim, dim if rot == "all" else rot, pairs, norm, dtype)


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 63, 1000])
@pytest.mark.parametrize("hq,hk", [(1, 1), (16, 16), (32, 8), (5, 0), (0, 7), (33, 3)])
def test_rows_and_heads(tokens, hq, hk):
    run(tokens, hq, hk, 128, 64, False, lq.NORM_RMS, torch.bfloat16, pad=64, shift=32, seed=tokens)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("pad,shift", [(3, 1), (8, 8), (1, 0), (2, 2)])
def test_rows_of_any_alignment(dtype, pad, shift):
    run(9, 4, 3, 128, 96, False, lq.NORM_L2, dtype, pad=pad, shift=shift)
    run(9, 4, 3, 64, 32, True, lq.NORM_RMS, dtype, pad=pad, shift=shift, in_place=True)


@pytest.mark.parametrize("pairs", [False, True])
def test_in_place_with_padding_rows(pairs):
    pos = torch.tensor([0, 5, -1, 2 ** 31 - 1, -7, 1, 123456789], dtype=torch.int32)
    run(7, 4, 2, 128, 128, pairs, lq.NORM_L2, torch.float32, in_place=True, positions=pos)
    run(7, 4, 2, 128, 128, pairs, lq.NORM_L2, torch.bfloat16, positions=pos)
    run(7, 4, 2, 128, 0, pairs, lq.NORM_RMS, torch.bfloat16, positions=pos, weights=False)


def test_a_row_of_zeros_and_large_values():
    x = torch.zeros((3, 1, 128), device="cuda")
    x[1] = 1e18
    x[2, 0, 5] = float("nan")
    y = torch.empty_like(x)
    lq.norm_rotate(lq.NormShape(3, 1, 0, type=lq.F32), x, None, y, None)
    assert torch.equal(y[0], torch.zeros_like(y[0])) and torch.allclose(y[1], torch.full_like(y[1], 128 ** -0.5), rtol=1e-6)
    assert torch.isnan(y[2]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("pairs", [False, True])
def test_frequencies_that_are_not_finite(dtype, dim, pairs):
    """The channels that they turn are NaN, at position 0 too; all others stay as they are, bit for bit."""
    T, H, half = 21, 3, dim // 4
    x = torch.randn((T, H, dim), generator=torch.Generator().manual_seed(dim)).to(dtype).cuda()
    freq = (10000.0 ** -(torch.arange(half) / half)).float()
    pos = torch.arange(T, dtype=torch.int32).cuda()
    sh = lq.NormShape(T, H, 0, dim=dim, rot=2 * half, pairs=int(pairs), type=lq.TYPES[dtype])
    want, got = torch.empty_like(x), torch.empty_like(x)
    lq.norm_rotate(sh, x, None, want, None, positions=pos, inv_freq=freq.cuda())
    freq[1], freq[4], freq[half - 1] = float("nan"), float("inf"), float("-inf")
    lq.norm_rotate(sh, x, None, got, None, positions=pos, inv_freq=freq.cuda())
    i = torch.tensor([1, 4, half - 1])
    bad = torch.zeros(dim, dtype=torch.bool)
    bad[torch.cat([2 * i, 2 * i + 1] if pairs else [i, i + half])] = True
    assert torch.isnan(got.cpu()[..., bad]).all()
    assert torch.equal(got.cpu()[..., ~bad], want.cpu()[..., ~bad]) and torch.isfinite(want).all()
