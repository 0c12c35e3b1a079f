"""Short causal convolution (prompts and single tokens) against its definition in 64 bits.

Tolerance: one rounding to the result's type (half a step, relative), and binary32 inside: at most width + 1 roundings of the sum, 2^-24
of its terms' magnitudes each, and the exponential and quotient of SiLU, whose slope is below 1.1 - 2^-20 of that magnitude covers
them.  fp16 results below 2^-14 are rounded to steps of 2^-24.  State rows are copies: equal bit by bit.
"""
import pytest
import torch

import ops_ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
FILL = 77.0


def make(seed, tokens, channels, width, dtype, n_slots, pad=0, bias=True):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)                                    # noqa: E731
    wide = r(tokens, channels + pad).to(dtype)
    return wide, r(channels, width).mul(0.5).to(dtype), r(channels).mul(0.2).to(dtype) if bias else None, r(n_slots, width - 1, channels).to(dtype)


def check_rows(got, want, scale, dtype):
    there = ~torch.isnan(want)
    assert torch.equal(got[~there], torch.full_like(got[~there], FILL)), "rows of no sequence are not written"
    tiny = 2.0 ** -25 if dtype is torch.float16 else 1e-37
    bound = ops_ref.half_step(dtype) * want.abs() + 2.0 ** -20 * scale + tiny
    off = ((got.double() - want).abs() / bound)[there]
    assert off.numel() == 0 or off.max() <= 1, float(off.max())


def run_prompt(x, w, bias, state, lens, slots=None, resume=None, silu=1, lead=0, view=None):
    """One call on packed sequences that start at row `lead`; checks everything against the definition."""
    dtype, C, W = x.dtype, w.shape[0], w.shape[1]
    starts = [lead]
    for n in lens:
        starts.append(starts[-1] + n)
    dev = lambda t: None if t is None else torch.as_tensor(t, dtype=torch.int32).cuda()    # noqa: E731
    xd = x.cuda()
    xs = xd if view is None else xd[:, view:view + C]
    out = torch.full((x.shape[0], C), FILL, dtype=dtype, device="cuda")
    st = state.cuda() if state is not None else None
    sh = lq.ConvShape(x.shape[0], len(lens), C, width=W, n_slots=0 if st is None else st.shape[0], silu=silu, type=lq.TYPES[dtype])
    lq.conv_prompt(sh, xs, w.cuda(), None if bias is None else bias.cuda(), st, out, dev(starts), slots=dev(slots), resume=dev(resume))
    torch.cuda.synchronize()
    want, scale, after = ops_ref.conv(xs.cpu(), w, bias, state, starts, slots, resume, silu)
    check_rows(out.cpu(), want, scale, dtype)
    if state is not None:
        assert torch.equal(st.cpu(), after)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("width", [2, 3, 4])
@pytest.mark.parametrize("channels,pad", [(1, 0), (129, 3), (256, 0), (1032, 64)])
def test_prompt_lengths_around_the_taps_and_the_tiles(dtype, width, channels, pad):
    lens = [1, 2, 3, 0, 4, 5, 31, 32, 33, 1, 1, 100, 0, 64, 2]
    x, w, bias, state = make(1, sum(lens) + 7, channels, width, dtype, len(lens) + 2, pad)
    slots = torch.randperm(len(lens) + 2, generator=torch.Generator().manual_seed(2))[:len(lens)].tolist()
    run_prompt(x, w, bias, state, lens, slots, [i % 3 != 0 for i in range(len(lens))], lead=3, view=pad)


@pytest.mark.parametrize("first", range(24, 36))
def test_sequences_that_start_next_to_a_tile_border(first):
    """The slot of a sequence is read and written where its first row is, whatever tile its second and third rows are in."""
    lens = [first, 70, 1, 2]
    x, w, bias, state = make(3, sum(lens), 64, 4, torch.bfloat16, 4)
    for _ in range(3):
        run_prompt(x, w, bias, state, lens, None, [1, 1, 1, 1])


def test_single_tokens_packed_and_no_bias_no_silu_no_state():
    x, w, _, state = make(4, 300, 72, 4, torch.float32, 300, bias=False)
    run_prompt(x, w, None, state, [1] * 300, None, [1] * 300, silu=0)
    run_prompt(x, w, None, None, [100, 200], silu=1)
    run_prompt(x, w, None, None, [100, 200], slots=[0, -1], silu=0)


def test_padding_sequences_and_slots_out_of_range():
    lens = [5, 6, 7, 8]
    x, w, bias, state = make(5, sum(lens), 64, 4, torch.float16, 3)
    run_prompt(x, w, bias, state, lens, [2, -1, 0, 3], [1, 1, 0, 1])          # slot 3 does not exist: padding


def test_no_sequence_sees_another_ones_nan():
    lens = [40, 1, 50]
    x, w, bias, state = make(6, 91 + 9, 64, 4, torch.bfloat16, 3)
    x[:3], x[43], x[94:] = float("nan"), float("inf"), float("nan")
    state[1] = float("nan")
    sh = lq.ConvShape(100, 3, 64, n_slots=3)
    out = torch.zeros((100, 64), dtype=torch.bfloat16, device="cuda")
    st = state.cuda()
    lq.conv_prompt(sh, x.cuda(), w.cuda(), bias.cuda(), st, out, torch.tensor([3, 43, 44, 94], dtype=torch.int32).cuda(),
                   resume=torch.tensor([1, 1, 1], dtype=torch.int32).cuda())
    assert torch.isfinite(out[3:43]).all() and torch.isfinite(out[44:94]).all() and not torch.isfinite(out[43]).any()
    assert torch.isfinite(st[0]).all() and torch.isfinite(st[2]).all()


def test_a_prompt_in_pieces_is_the_prompt():
    x, w, bias, state = make(7, 200, 128, 4, torch.bfloat16, 1)
    w_, b_ = w.cuda(), bias.cuda()
    whole, parts = torch.zeros((200, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((200, 128), dtype=torch.bfloat16, device="cuda")
    st_a, st_b, xd = state.cuda(), state.cuda(), x.cuda()
    start = lambda n: torch.tensor([0, n], dtype=torch.int32, device="cuda")      # noqa: E731
    lq.conv_prompt(lq.ConvShape(200, 1, 128, n_slots=1), xd, w_, b_, st_a, whole, start(200))
    at = 0
    for i, n in enumerate([1, 1, 2, 30, 66, 1, 99]):
        r = torch.tensor([int(i > 0)], dtype=torch.int32, device="cuda")
        if n == 1 and i:
            lq.conv_step(lq.ConvShape(1, 1, 128, n_slots=1), xd[at:at + 1], w_, b_, st_b, parts[at:at + 1])
        else:
            lq.conv_prompt(lq.ConvShape(n, 1, 128, n_slots=1), xd[at:at + n], w_, b_, st_b, parts[at:at + n], start(n), resume=r)
        at += n
    assert torch.equal(whole, parts) and torch.equal(st_a, st_b)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("batch,channels,width", [(1, 8, 4), (3, 1025, 2), (70, 264, 3), (256, 1024, 4)])
@pytest.mark.parametrize("in_place", [False, True])
def test_step(dtype, batch, channels, width, in_place):
    wide, w, bias, state = make(8, batch, channels, width, dtype, batch + 1, pad=16)
    slots = torch.randperm(batch + 1, generator=torch.Generator().manual_seed(9))[:batch].tolist()
    if batch > 2:
        slots[1] = -1
    xd = wide.cuda()[:, 8:8 + channels]
    x = xd.cpu().clone()
    out = xd if in_place else torch.full((batch, channels), FILL, dtype=dtype, device="cuda")
    st = state.cuda()
    sh = lq.ConvShape(batch, batch, channels, width=width, n_slots=batch + 1, type=lq.TYPES[dtype])
    lq.conv_step(sh, xd, w.cuda(), bias.cuda(), st, out, slots=torch.tensor(slots, dtype=torch.int32).cuda())
    want, scale, after = ops_ref.conv(x, w, bias, state, list(range(batch + 1)), slots, [1] * batch, 1)
    got = out.cpu()
    if in_place and batch > 2:
        assert torch.equal(got[1], x[1])
        got[1] = FILL
    check_rows(got, want, scale, dtype)
    assert torch.equal(st.cpu(), after)


def test_large_strides_and_rows_beyond_32_bits():
    """Rows that lie more than 2^32 bytes into their buffer."""
    rows, stride, C = 70, 1 << 26, 64
    buf = torch.empty((rows * stride,), dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, C), (stride, 1))
    vals, w, bias, state = make(10, rows, C, 4, torch.bfloat16, 1)
    x.copy_(vals)
    out = torch.empty((rows, C), dtype=torch.bfloat16, device="cuda")
    st = state.cuda()
    lq.conv_prompt(lq.ConvShape(rows, 1, C, n_slots=1), x, w.cuda(), bias.cuda(), st, out, torch.tensor([0, rows], dtype=torch.int32).cuda())
    want, scale, after = ops_ref.conv(vals, w, bias, state, [0, rows], None, None, 1)
    check_rows(out.cpu(), want, scale, torch.bfloat16)
    assert torch.equal(st.cpu(), after)


@pytest.mark.parametrize("channels", [64, 63])
def test_silu_over_its_range(channels):
    """y / (1 + exp(-y)) in binary32: exp2 to 2^-22, its argument -y log2(e) rounded twice (|y| (2^-24 + 2^-25)), 1 + exp to 2^-24, the reciprocal to 2^-23, the
    product to 2^-24: below 2^-21 + 2^-23 |y| of the value together.  Where exp(-y) has no reciprocal of 2^-126 or more the result is 0."""
    y = torch.cat([torch.linspace(-130, 130, 4097), torch.linspace(-90, -84, 1024), 10.0 ** torch.linspace(-30, 30, 128), -(10.0 ** torch.linspace(-30, 30, 128))])
    y = y[:y.numel() // channels * channels].view(-1, channels).contiguous()
    w = torch.tensor([0.0, 1.0]).repeat(channels, 1)
    out = torch.empty(y.shape, device="cuda")
    lq.conv_prompt(lq.ConvShape(y.shape[0], 1, channels, width=2, type=lq.F32), y.cuda(), w.cuda(), None, None, out, torch.tensor([0, y.shape[0]], dtype=torch.int32).cuda())
    want = y.double() * torch.sigmoid(y.double())
    off = (out.cpu().double() - want).abs()
    assert (off <= (2.0 ** -21 + 2.0 ** -23 * y.double().abs()) * want.abs() + 2.0 ** -119).all()
    assert (out.cpu()[y < -87.4] == 0).all()
