"""Products of 8-bit rows with 8-bit weights, whole and by groups of rows, against their definition in 64 bits.

Tolerance: one rounding to the result's type; products of codes are exact, and each of a block's 128 additions and of the additions over blocks is off by a step at
most (the tensor cores may cut off where binary32 would round), 2^-23 of the sum over magnitudes, the scales' product and the one with it by half a step each.
"""
import pytest
import torch

import linear_ref as ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
FILL = 7.0


def operands(rows, cin, cout, groups=1, seed=0):
    g = torch.Generator().manual_seed(seed)
    x, s = ref.quantize(torch.randn(rows, cin, generator=g) * torch.exp(torch.randn(rows, 1, generator=g)))
    w = (100 * torch.randn(groups, cout, cin, generator=g)).clamp(-448, 448).to(ref.E4M3)
    ws = torch.exp(0.5 * torch.randn(groups, -(-cout // 128), -(-cin // 128), generator=g)) / (100 * cin ** 0.5)
    return x, s, w, ws


def close(got, want, size, dtype, cin):
    live = ~torch.isnan(want)
    slack = (128 + -(-cin // 128) + 2) * 2.0 ** -23 * size
    assert ref.off(got[live], want[live], dtype, slack[live]) <= 1
    assert (got[~live] == FILL).all()


def run(rows, cin, cout, dtype=torch.bfloat16, starts=None, groups=1, pad=(0, 0, 0), seed=0, guard=8):
    x, s, w, ws = operands(rows, cin, cout, groups, seed)
    dx = torch.zeros((rows, cin + pad[0]), device="cuda").to(ref.E4M3)[:, :cin]
    dx.copy_(x)
    dx = dx if pad[0] else dx.contiguous()
    ds = torch.full((s.shape[0], rows + pad[1]), float("nan"), device="cuda")[:, :rows]
    ds.copy_(s)
    buf = torch.full((rows + 2 * guard, cout + pad[2]), FILL, dtype=dtype, device="cuda")
    at = 8 if pad[2] >= 16 else 0 if pad[2] % 8 else pad[2] // 2
    out = buf[guard:guard + rows, at:at + cout]
    sh = lq.ProductShape(rows, cin, cout, groups=groups, type=lq.TYPES[dtype])
    if starts is None:
        lq.product(sh, dx, ds, w[0].cuda(), ws[0].cuda(), out)
    else:
        lq.product_groups(sh, dx, ds, w.cuda(), ws.cuda(), out, torch.tensor(starts, dtype=torch.int32, device="cuda"))
    got = out.cpu()
    assert lq.check_device() == 0
    want, size = ref.product(x, s, w, ws, starts)
    close(got, want, size, dtype, cin)
    rest = buf.cpu()
    rest[guard:guard + rows, at:at + cout] = FILL
    assert (rest == FILL).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cin,cout", [(1, 16, 1), (1, 128, 128), (3, 4096, 300), (17, 272, 129), (64, 1024, 256), (129, 640, 1000), (300, 2048, 520)])
def test_types_and_sizes(dtype, rows, cin, cout):
    run(rows, cin, cout, dtype)


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500, 513, 1025])
def test_rows(rows):
    run(rows, 512, 384, seed=rows)
    run(rows, 400, 200, torch.float32, seed=rows)


@pytest.mark.parametrize("cin", [16, 32, 112, 128, 144, 240, 256, 272, 1024, 1040, 4096, 8192])
def test_channels_in(cin):
    run(5, cin, 160, torch.float32, seed=cin)
    run(200, cin, 160, torch.float32, seed=cin)


@pytest.mark.parametrize("cout", [1, 2, 7, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1999])
def test_channels_out(cout):
    run(5, 256, cout, seed=cout)
    run(300, 256, cout, seed=cout)


@pytest.mark.parametrize("pad", [(16, 0, 0), (0, 3, 0), (0, 0, 1), (48, 5, 8), (16, 1, 32)])
@pytest.mark.parametrize("rows", [7, 260])
def test_strides(pad, rows):
    run(rows, 384, 256, pad=pad)
    run(rows, 384, 256, torch.float32, pad=pad)


@pytest.mark.parametrize("rows,cin,cout", [(4000, 1024, 4096), (1000, 4096, 4096), (256, 4096, 12352), (40, 4096, 12352), (1, 4096, 4096)])
def test_layers(rows, cin, cout):
    run(rows, cin, cout)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("starts", [[0, 10, 10, 50], [3, 3, 40, 41], [0, 0, 0, 0], [0, 50, 50, 50], [0, 0, 0, 50], [1, 2, 3, 4], [50, 50, 50, 50]], ids=str)
def test_groups(dtype, starts):
    run(50, 272, 200, dtype, starts, groups=3)


@pytest.mark.parametrize("groups,rows", [(1, 5), (33, 40), (100, 700), (128, 2048), (7, 3000), (1024, 1500)])
def test_ragged_groups(groups, rows):
    g = torch.Generator().manual_seed(groups)
    cuts = sorted(torch.randint(0, rows + 1, (groups + 1,), generator=g).tolist())
    run(rows, 256, 160, starts=cuts, groups=groups, seed=rows)


def test_starts_that_make_no_sense():
    """Row numbers that go down or out of range: no access outside of the arrays."""
    x, s, w, ws = operands(300, 256, 256, 4)
    sh = lq.ProductShape(300, 256, 256, groups=4)
    for starts in ([-5, 400, 100, 2 ** 31 - 1, -2 ** 31], [300, 200, 100, 50, 0], [2 ** 31 - 1] * 5, [-1] * 5):
        buf = torch.full((364, 256), FILL, dtype=torch.bfloat16, device="cuda")
        lq.product_groups(sh, x.cuda(), s.cuda(), w.cuda(), ws.cuda(), buf[32:332], torch.tensor(starts, dtype=torch.int32, device="cuda"))
        assert lq.check_device() == 0
        assert (buf[:32] == FILL).all() and (buf[332:] == FILL).all()


@pytest.mark.parametrize("rows", [20, 300])
def test_what_is_not_finite_stays_in_its_row(rows):
    x, s, w, ws = operands(rows, 512, 256)
    sh = lq.ProductShape(rows, 512, 256, type=lq.F32)
    clean, out = torch.empty((rows, 256), device="cuda"), torch.empty((rows, 256), device="cuda")
    lq.product(sh, x.cuda(), s.cuda(), w[0].cuda(), ws[0].cuda(), clean)
    y, t = x.float(), s.clone()
    y[3, 100] = float("nan")
    t[2, 7] = float("inf")
    t[1, 11] = 0.0
    lq.product(sh, y.to(ref.E4M3).cuda(), t.cuda(), w[0].cuda(), ws[0].cuda(), out)
    assert torch.isnan(out[3]).all() and not torch.isfinite(out[7]).any() and torch.isfinite(out[11]).all()
    same = [r for r in range(rows) if r not in (3, 7, 11)]
    assert torch.equal(out[same], clean[same])


def test_the_same_call_gives_the_same_bits():
    for rows in (1, 100, 256, 1000):
        x, s, w, ws = (t.cuda() for t in operands(rows, 2048, 640))
        sh = lq.ProductShape(rows, 2048, 640, type=lq.F32)
        a, b = torch.empty((rows, 640), device="cuda"), torch.empty((rows, 640), device="cuda")
        lq.product(sh, x, s, w[0], ws[0], a)
        for _ in range(5):
            lq.product(sh, x, s, w[0], ws[0], b)
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows", [5, 100, 300])
@pytest.mark.parametrize("cout", [100, 1001])
def test_rows_of_outputs_that_end_inside_a_piece(dtype, rows, cout):
    """Rows that start at multiples of 16 bytes and end elsewhere: what lies behind them stays."""
    run(rows, 256, cout, dtype, pad=(0, 0, -cout % 8 + 8))
    run(rows, 256, cout, dtype, starts=[0, rows // 3, rows - 1], groups=2, pad=(0, 0, -cout % 8 + 8))


@pytest.mark.parametrize("rows,cout", [(20000, 288), (20000, 32), (15000, 480)])
def test_many_short_products(rows, cout):
    """Tiles with an odd number of pieces of outputs, one after another in the same places of shared memory."""
    run(rows, 128, cout)
