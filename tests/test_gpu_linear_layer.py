"""A layer from the residual stream back to it, as it runs: norm, projections, convolution, norms of q and k, the window's decode step (or the prompt's scan), gated
norm, output projection, experts behind them - on the current stream, on another one, captured and replayed, two at once.

Tolerances: every stage is compared with its definition in 64 bits on the values that it was given (their own tests derive the bounds); the same calls
in another way give the same bits.
"""
import pytest
import torch

import linear_ref as ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu
D, HQ, HV, HIDDEN = 128, 2, 4, 640
C = (2 * HQ + HV) * D
OUTS = C + HV * D + 2 * HV                                                        # q, k, v | z | beta, alpha
GROUPS = 5


def weight(g, *shape):
    w = (100 * torch.randn(*shape, generator=g)).clamp(-448, 448).to(ref.E4M3)
    s = torch.exp(0.3 * torch.randn(*shape[:-2], -(-shape[-2] // 128), -(-shape[-1] // 128), generator=g)) / (100 * shape[-1] ** 0.5)
    return w.cuda(), s.cuda()


class Layer:
    """`rows` tokens: one each of as many sequences (the decode step), or a packed prompt of one sequence (the scan)."""

    def __init__(self, rows, prompt, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g)                                # noqa: E731
        self.rows, self.prompt = rows, prompt
        self.x, self.residual0 = r(rows, HIDDEN).bfloat16().cuda(), (2 * r(rows, HIDDEN)).bfloat16().cuda()
        self.w_in, self.w_head, self.w_out = (1 + 0.2 * r(HIDDEN)).cuda(), (1 + 0.2 * r(D)).cuda(), (1 + 0.2 * r(HIDDEN)).cuda()
        self.proj, self.back, self.experts = weight(g, OUTS, HIDDEN), weight(g, HIDDEN, HV * D), weight(g, GROUPS, 384, HIDDEN)
        self.taps = (0.4 * r(C, 4)).bfloat16().cuda()
        cuts = sorted(torch.randint(0, rows + 1, (GROUPS - 1,), generator=g).tolist())
        self.cuts = [0, *cuts, rows]
        self.group_start = torch.tensor(self.cuts, dtype=torch.int32).cuda()
        self.starts = torch.tensor([0, rows], dtype=torch.int32).cuda()
        e = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")   # noqa: E731
        f32 = torch.float32
        self.h8, self.hs = e(rows, HIDDEN, dtype=ref.E4M3), e(HIDDEN // 128, rows, dtype=f32)
        self.p, self.mixed = e(rows, OUTS), e(rows, C)
        self.o = e(rows, HV, D, dtype=torch.bfloat16 if prompt else f32)
        self.y8, self.ys = e(rows, HV * D, dtype=ref.E4M3), e(HV * D // 128, rows, dtype=f32)
        self.out, self.f, self.f8, self.fs = e(rows, HIDDEN), e(rows, HIDDEN), e(rows, HIDDEN, dtype=ref.E4M3), e(HIDDEN // 128, rows, dtype=f32)
        self.expert = e(rows, 384)
        self.S = torch.zeros((1 if prompt else rows, HV, D, D), device="cuda")
        self.conv = torch.zeros((1 if prompt else rows, 3, C), dtype=torch.bfloat16, device="cuda")
        self.residual = self.residual0.clone()
        self.qkv = [e(rows, h, D) for h in (HQ, HQ, HV)]
        self.gates = [e(rows, HV) for _ in range(2)]
        if not prompt:
            self.shape = lq.Shape(rows, HV, HQ, delta=1, W=8)
            self.state = lq.State(self.shape)
            S0 = (0.1 * r(rows, HV, D, D)).cuda()
            lq.quantize_state(self.shape, S0, self.state)
        else:
            self.scan = lq.ScanShape(rows, 1, HV, HQ, max_len=rows, n_slots=1)
            self.work = torch.empty((max(16, lq.scan_prompt_bytes(self.scan)),), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()

    def run(self, stream=None):
        rows, kw = self.rows, dict(stream=stream)
        lq.norm_add(lq.AddShape(rows, HIDDEN), self.x, residual=self.residual, w=self.w_in, out8=self.h8, scale=self.hs, **kw)
        lq.product(lq.ProductShape(rows, HIDDEN, OUTS), self.h8, self.hs, *self.proj, self.p, **kw)
        if self.prompt:
            lq.conv_prompt(lq.ConvShape(rows, 1, C, n_slots=1), self.p[:, :C], self.taps, None, self.conv, self.mixed, self.starts, **kw)
        else:
            lq.conv_step(lq.ConvShape(rows, rows, C, n_slots=rows), self.p[:, :C], self.taps, None, self.conv, self.mixed, **kw)
        q, k, v = (t.unflatten(-1, (-1, D)) for t in self.mixed.split([HQ * D, HQ * D, HV * D], -1))
        lq.norm_rotate(lq.NormShape(rows, HQ, HQ), q, k, self.qkv[0], self.qkv[1], **kw)
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
            self.qkv[2].copy_(v)
            for gate, raw in zip(self.gates, self.p[:, C + HV * D:].split([HV, HV], -1)):
                torch.sigmoid(raw, out=gate)
        if self.prompt:
            lq.scan_prompt(self.scan, *self.qkv, *self.gates, self.o, self.S, self.starts, work=self.work, **kw)
        else:
            bits = lambda t: t.view(torch.int16)                                  # noqa: E731
            lq.decode_step(self.shape, self.state, *(bits(t) for t in self.qkv), *(bits(t) for t in self.gates), self.o, **kw)
        z = self.p[:, C:C + HV * D].unflatten(-1, (HV, D))
        lq.norm_gate(lq.GatedShape(rows, HV, o_type=lq.TYPES[self.o.dtype]), self.o, z, w=self.w_head, out8=self.y8, scale=self.ys, **kw)
        lq.product(lq.ProductShape(rows, HV * D, HIDDEN), self.y8, self.ys, *self.back, self.out, **kw)
        lq.norm_add(lq.AddShape(rows, HIDDEN), self.out, residual=self.residual, w=self.w_out, out=self.f, out8=self.f8, scale=self.fs, **kw)
        lq.product_groups(lq.ProductShape(rows, HIDDEN, 384, groups=GROUPS), self.f8, self.fs, *self.experts, self.expert, self.group_start, **kw)

    def written(self):
        return [self.h8.view(torch.uint8), self.hs, self.p, self.mixed, self.o, self.y8.view(torch.uint8), self.ys, self.out, self.f, self.f8.view(torch.uint8), self.fs,
                self.expert, self.residual]


def values(code, scale):
    return code.cpu().double() * ref.spread(scale.cpu().double(), code.shape[1])


def near(code, scale, want):
    by = ref.spread(scale.cpu().double(), want.shape[1])
    return bool(((values(code, scale) - want).abs() <= (2.0 ** -4 + 2.0 ** -16) * want.abs() + 2.0 ** -10 * by).all())


@pytest.mark.parametrize("rows,prompt", [(1, False), (3, False), (40, False), (1, True), (150, True), (700, True)])
def test_every_stage_on_what_it_was_given(rows, prompt):
    a = Layer(rows, prompt, seed=rows)
    a.run()
    torch.cuda.synchronize()
    assert lq.check_device() == 0
    h = a.x.cpu().double() + a.residual0.cpu().double()
    assert near(a.h8, a.hs, ref.norm(h, 2, a.w_in.cpu(), 1e-6))
    slack = lambda size, cin: (128 + -(-cin // 128) + 2) * 2.0 ** -23 * size      # noqa: E731
    for out, x, s, (w, ws), cin, starts in ((a.p, a.h8, a.hs, a.proj, HIDDEN, None), (a.out, a.y8, a.ys, a.back, HV * D, None),
                                            (a.expert, a.f8, a.fs, a.experts, HIDDEN, a.cuts)):
        w, ws = (w, ws) if starts else (w[None], ws[None])
        want, size = ref.product(x.cpu(), s.cpu(), w.cpu(), ws.cpu(), starts)
        assert ref.off(out.cpu(), want, torch.bfloat16, slack(size, cin)) <= 1
    z = a.p[:, C:C + HV * D].cpu().double().unflatten(-1, (HV, D))
    assert near(a.y8, a.ys, (ref.norm(a.o.cpu().double(), 2, a.w_head.cpu(), 1e-6) * torch.sigmoid(z) * z).flatten(1))
    h1 = h.bfloat16().double() + a.out.cpu().double()
    assert ref.off(a.residual.cpu(), h1, torch.bfloat16, 2.0 ** -24 * h1.abs()) <= 1
    f = ref.norm(h1, 2, a.w_out.cpu(), 1e-6)
    assert ref.off(a.f.cpu(), f, torch.bfloat16, 2.0 ** -18 * f.abs()) <= 1 and near(a.f8, a.fs, f)


@pytest.mark.parametrize("rows,prompt", [(40, False), (300, True)])
def test_on_another_stream_and_captured(rows, prompt):
    a, b, c = (Layer(rows, prompt) for _ in range(3))
    a.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b.run(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    fresh = [t.clone() for t in (c.residual, c.conv, c.S)]
    state = [t.clone() for t in c.state.tensors()] if not prompt else []
    c.run()                                   # (first calls outside of the capture)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for _ in range(2):
        for t, was in zip((c.residual, c.conv, c.S, *(c.state.tensors() if not prompt else [])), (*fresh, *state)):
            t.copy_(was)
        for t in (c.p, c.out, c.expert):
            t.fill_(7.0)
        graph.replay()
    torch.cuda.synchronize()
    assert lq.check_device() == 0
    for x, y, z in zip(a.written(), b.written(), c.written()):
        assert torch.equal(x, y) and torch.equal(x, z)


def test_layers_at_once_on_several_streams():
    want = [Layer(rows, prompt, seed=i) for i, (rows, prompt) in enumerate([(30, False), (500, True), (7, False), (260, True)])]
    for a in want:
        a.run()
    torch.cuda.synchronize()
    got = [Layer(a.rows, a.prompt, seed=i) for i, a in enumerate(want)]
    streams = [torch.cuda.Stream() for _ in got]
    for a, s in zip(got, streams):
        a.run(stream=s)
    torch.cuda.synchronize()
    assert lq.check_device() == 0
    for a, b in zip(want, got):
        for x, y in zip(a.written(), b.written()):
            assert torch.equal(x, y)


def test_slices_side_by_side_in_one_buffer():
    """Column slices of one buffer and a product's output behind its input: neighbours, not overlaps; the bits are those of arrays of their own."""
    rows, cin, cout = 37, 256, 192
    g = torch.Generator(device="cuda").manual_seed(9)
    buf = torch.zeros((rows, 2 * cin + cin + 2 * cout), dtype=torch.uint8, device="cuda")
    x, h8, out = buf[:, :2 * cin].view(torch.bfloat16), buf[:, 2 * cin:3 * cin].view(lq.E4M3), buf[:, 3 * cin:].view(torch.bfloat16)
    x.copy_(torch.randn((rows, cin), generator=g, device="cuda"))
    scale, (w, ws) = torch.empty((2, rows), device="cuda"), weight(torch.Generator().manual_seed(3), cout, cin)
    own8, own_scale, own = torch.empty((rows, cin), dtype=lq.E4M3, device="cuda"), torch.empty_like(scale), torch.empty((rows, cout), dtype=torch.bfloat16, device="cuda")
    add, sh = lq.AddShape(rows, cin), lq.ProductShape(rows, cin, cout)
    lq.norm_add(add, x.contiguous(), out8=own8, scale=own_scale)
    lq.product(sh, own8, own_scale, w, ws, own)
    lq.norm_add(add, x, out8=h8, scale=scale)
    lq.product(sh, h8, scale, w, ws, out)
    assert torch.equal(own8.view(torch.uint8), h8.view(torch.uint8)) and torch.equal(own_scale, scale) and torch.equal(own, out)


@pytest.mark.parametrize("rows", [1, 30, 300, 5000])
def test_calls_right_behind_one_another(rows):
    """Every call takes what the one in front of it has just written, into the same arrays over and over: as with a wait between all of them."""
    g = torch.Generator().manual_seed(rows)
    x0 = torch.randn((rows, HIDDEN), generator=g).bfloat16().cuda()
    w, ws = weight(g, HIDDEN, HIDDEN)

    def chain(wait):
        x, r = x0.clone(), torch.zeros_like(x0)
        h8, hs = torch.empty((rows, HIDDEN), dtype=ref.E4M3, device="cuda"), torch.empty((HIDDEN // 128, rows), device="cuda")
        add, sh = lq.AddShape(rows, HIDDEN), lq.ProductShape(rows, HIDDEN, HIDDEN)
        for _ in range(30):
            for call in (lambda: lq.norm_add(add, x, residual=r, out8=h8, scale=hs), lambda: lq.product(sh, h8, hs, w, ws, x)):
                call()
                if wait:
                    torch.cuda.synchronize()
        return x, r

    slow = chain(True)
    for _ in range(3):
        for a, b in zip(slow, chain(False)):
            assert torch.equal(a, b)
    assert torch.isfinite(slow[0].float()).all() and lq.check_device() == 0


def test_rows_beyond_two_to_the_31_elements():
    """70000 rows, 32768 elements apart: the same bits as of rows side by side."""
    rows, far, cin, cout = 70000, 32768, 128, 48
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((rows, cin), generator=g, device="cuda").bfloat16()
    w, ws = weight(torch.Generator().manual_seed(2), cout, cin)
    add, gated, sh = lq.AddShape(rows, cin), lq.GatedShape(rows, 1, o_type=lq.BF16), lq.ProductShape(rows, cin, cout)

    def chain(of, of8):
        o, z, y, y8 = of(cin), of(cin), of(cout), of8(cin)
        scale = torch.empty((1, rows), device="cuda")
        lq.norm_add(add, x, out=o)
        z.copy_(x.flip(0))
        lq.norm_gate(gated, o[:, None], z[:, None], out8=y8, scale=scale)
        lq.product(sh, y8, scale, w, ws, y)
        lq.norm_add(add, o, out=o)
        return [t.contiguous().view(torch.uint8) for t in (o, y, y8)]

    here = chain(lambda n: torch.empty((rows, n), dtype=torch.bfloat16, device="cuda"), lambda n: torch.empty((rows, n), dtype=ref.E4M3, device="cuda"))
    buf, buf8 = torch.empty((rows, far), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, far), dtype=torch.uint8, device="cuda")
    at = iter((0, 512, 1024))

    def apart(n):
        k = next(at)
        return buf[:, k:k + n]

    there = chain(apart, lambda n: buf8[:, 256:256 + n].view(ref.E4M3))
    for a, b in zip(here, there):
        assert torch.equal(a, b)
    assert lq.check_device() == 0
