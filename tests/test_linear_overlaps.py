"""Outputs of the 8-bit linear layer over its small inputs - a norm's weights, the groups' first rows - are refused (no GPU is touched); next to them they are not."""
import pytest
import torch

from paper_2609_38166_b200 import lq
from test_linear_abi import L, OUT, OUT8, R, SCALE, UNSUPPORTED, add, gate, product   # noqa: F401


@pytest.mark.parametrize("tokens", [1, 40])
@pytest.mark.parametrize("call,kind,channels", [(add, lq.AddShape, 256), (gate, lq.GatedShape, 128)], ids=["add", "gate"])
def test_weights_of_a_norm(L, call, kind, channels, tokens):   # noqa: F811
    sh = kind(tokens, 256) if call is add else kind(tokens, 2)
    outs = [(OUT, tokens * 512), (OUT8, tokens * 256), (SCALE, 2 * tokens * 4)] + ([(R, tokens * 512)] if call is add else [])
    for start, size in outs:
        for at in (start, start + size - 4, start - channels * 4 + 4):
            assert call(L, sh, w=at) == UNSUPPORTED, (hex(start), at - start)


def test_first_rows_of_groups(L):   # noqa: F811
    sh = lq.ProductShape(40, 256, 300, groups=3)
    for at in (OUT, OUT - 12, OUT + 39 * 600, OUT + 40 * 600 - 4):
        assert product(L, sh, groups=True, start=at) == UNSUPPORTED, at - OUT


@pytest.mark.gpu
def test_neighbours_are_no_overlap():
    tokens, dim = 3, 256
    rows = torch.zeros((tokens + 4) * dim, device="cuda")
    out, w = rows[2 * dim:5 * dim].view(tokens, dim), rows[5 * dim:6 * dim]
    w.fill_(2.0)
    front = rows[dim:2 * dim].fill_(3.0)
    x = torch.randn((tokens, dim), device="cuda")
    for weights, by in ((w, 2.0), (front, 3.0)):
        lq.norm_add(lq.AddShape(tokens, dim, type=lq.F32), x, w=weights, out=out)
        want = by * x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        assert torch.allclose(out, want, rtol=1e-5) and (weights == by).all()
    ints = torch.zeros(3 + 2 * 16 + 3, dtype=torch.int32, device="cuda")
    y = ints[3:35].view(torch.float32).view(2, 16)
    a, s = torch.ones((2, 16), device="cuda").to(lq.E4M3), torch.ones((1, 2), device="cuda")
    b, t = torch.ones((2, 16, 16), device="cuda").to(lq.E4M3), torch.ones((2, 1, 1), device="cuda")
    for starts in (ints[:3], ints[35:]):
        starts.copy_(torch.tensor([0, 1, 2]))
        y.zero_()
        lq.product_groups(lq.ProductShape(2, 16, 16, groups=2, type=lq.F32), a, s, b, t, y, starts)
        assert (y == 16).all() and starts.tolist() == [0, 1, 2]
    assert lq.check_device() == 0


@pytest.mark.gpu
def test_weights_that_are_not_read_may_lie_anywhere():
    x, out = torch.randn((3, 256), device="cuda"), torch.empty((3, 256), device="cuda")
    for norm in (lq.NORM_NONE, lq.NORM_L2):
        lq.norm_add(lq.AddShape(3, 256, norm=norm, type=lq.F32, eps=0.0), x, w=out.view(-1)[:256], out=out)
        assert torch.allclose(out, x if norm == lq.NORM_NONE else x / torch.linalg.norm(x, dim=-1, keepdim=True), rtol=1e-5)
    assert lq.check_device() == 0
