"""The gate of norm_gate where z and out are binary32, against its definition in 64 bits.

Tolerance: an exponential within 2 steps of 2^-23, its sum with 1 half a step, a reciprocal within a step and the product with z half a step: 8 * 2^-24, 2^-21 whatever z
is; what is below 2^-119 may be 0.
The norm in front of it: a sum of squares with at most 16 + 4 additions, half of their 2^-24 each after the root, a root of 2^-22, three products: below 2^-19.
"""
import pytest
import torch

import linear_ref as ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu


def gates(z, silu):
    z = z.double()
    return torch.sigmoid(z) * (z if silu else 1.0)


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("o_type", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("shift", [0, 1])
def test_gate_alone(silu, o_type, shift):
    tokens, heads, dim = 64, 3, 128
    width = heads * dim
    z = torch.linspace(-88.0, 88.0, tokens * width).view(tokens, width)
    z[1::2] = 2 * torch.randn(tokens // 2, width, generator=torch.Generator().manual_seed(3))
    wide = torch.zeros((tokens, width + shift), device="cuda")[:, shift:]
    wide.copy_(z)
    out = torch.empty((tokens, width), device="cuda")
    o = torch.ones((tokens, heads, dim), dtype=o_type, device="cuda")
    lq.norm_gate(lq.GatedShape(tokens, heads, norm=lq.NORM_NONE, silu=int(silu), o_type=lq.TYPES[o_type], type=lq.F32), o, wide.unflatten(-1, (heads, dim)), out=out)
    want = gates(z, silu)
    d = (out.cpu().double() - want).abs() / (2.0 ** -21 * want.abs() + 2.0 ** -119)
    assert float(d.max()) <= 1, float(z.flatten()[d.argmax()])


@pytest.mark.parametrize("silu", [False, True])
def test_what_is_far_out(silu):
    z = torch.tensor([0.0, -0.0, 200.0, -200.0, 1e30, -1e30, float("inf"), float("nan"), -87.0, -88.5, -89.5, 1e-40] + [1.0] * 52, device="cuda").view(1, 1, 64)
    y = torch.empty((1, 64), device="cuda")
    lq.norm_gate(lq.GatedShape(1, 1, dim=64, norm=lq.NORM_NONE, silu=int(silu), type=lq.F32), torch.ones_like(z), z, out=y)
    want = gates(z.cpu(), silu).view(1, 64)
    got = y.cpu().double()
    assert torch.isnan(got[0, 7]) and got[0, 6] == (float("inf") if silu else 1.0)
    keep = [i for i in range(64) if i not in (6, 7)]
    assert ((got - want).abs() <= 2.0 ** -21 * want.abs() + 2.0 ** -119)[0, keep].all()


def test_with_the_norm_in_front():
    g = torch.Generator().manual_seed(5)
    o, z, w = torch.randn(50, 5, 256, generator=g), 30 * torch.randn(50, 5, 256, generator=g), 1 + 0.3 * torch.randn(256, generator=g)
    out = torch.empty((50, 1280), device="cuda")
    lq.norm_gate(lq.GatedShape(50, 5, dim=256, type=lq.F32, eps=1e-5), o.cuda(), z.cuda(), w=w.cuda(), out=out)
    front = ref.norm(o.double(), 2, w, 1e-5)
    want = (front * gates(z, True)).flatten(1)
    # (a gate below 2^-119 may be 0, and is multiplied with what stands in front of it: off by 2^-119 |front| at most)
    assert ((out.cpu().double() - want).abs() <= (2.0 ** -21 + 2.0 ** -19) * want.abs() + 2.0 ** -119 * (1 + front.abs()).flatten(1)).all()
