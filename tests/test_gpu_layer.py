"""The operators around the decode step, run together as a layer runs them: convolution, norms with rotation, the scan over prompts, the
window representation, and single tokens behind it - on the current stream, on another one, captured and replayed.

Tolerances: the chain is compared with the same chain in 64 bits on the values that each stage was given (every stage's own test bounds
its errors), and with itself - the same calls in another way give the same bits.
"""
import pytest
import torch

import ops_ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu
D, HQ, HV, W = 128, 2, 4, 4
C = (2 * HQ + HV) * D
LENS = [130, 1, 0, 257, 40]
N = len(LENS)


class Layer:
    """A layer without the delta rule (scalar gate), its weights and states, prompts and a token at a time."""

    def __init__(self, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g)                                # noqa: E731
        self.T = sum(LENS)
        self.proj = r(self.T, C + HV + 8).bfloat16().cuda()                       # conv channels, then dt
        self.token = r(N, C + HV + 8).bfloat16().cuda()
        self.w, self.bias = (0.4 * r(C, W)).bfloat16().cuda(), (0.1 * r(C)).bfloat16().cuda()
        self.A, self.dt_bias, self.skip = (x.cuda() for x in (-torch.rand(HV, generator=g) * 2 - 0.1, r(HV) - 2, r(HV)))
        self.freq = (10000.0 ** -(torch.arange(32) / 32.0)).float().cuda()
        starts = [0]
        for n in LENS:
            starts.append(starts[-1] + n)
        self.starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in LENS]).cuda()
        self.last = torch.tensor(LENS, dtype=torch.int32, device="cuda")
        self.conv_shape = lq.ConvShape(self.T, N, C, n_slots=N)
        self.norm_shape = lq.NormShape(self.T, HQ, HQ, rot=64)
        self.scan_shape = lq.ScanShape(self.T, N, HV, HQ, max_len=max(LENS), n_slots=N, select=1)
        self.work = torch.empty((lq.scan_prompt_bytes(self.scan_shape),), dtype=torch.uint8, device="cuda")
        self.conv_state = torch.zeros((N, W - 1, C), dtype=torch.bfloat16, device="cuda")
        self.S = torch.full((N, HV, D, D), float("nan"), device="cuda")
        self.mixed = torch.empty((self.T, C), dtype=torch.bfloat16, device="cuda")
        self.o = torch.empty((self.T, HV, D), dtype=torch.bfloat16, device="cuda")
        self.mixed1 = torch.empty((N, C), dtype=torch.bfloat16, device="cuda")
        self.o1 = torch.empty((N, HV, D), device="cuda")

    def split(self, x):
        q, k, v = x[:, :HQ * D], x[:, HQ * D:2 * HQ * D], x[:, 2 * HQ * D:]
        return q.unflatten(-1, (HQ, D)), k.unflatten(-1, (HQ, D)), v.unflatten(-1, (HV, D))

    def prompt(self, stream=None):
        lq.conv_prompt(self.conv_shape, self.proj[:, :C], self.w, self.bias, self.conv_state, self.mixed, self.starts, stream=stream)
        q, k, v = self.split(self.mixed)
        lq.norm_rotate(self.norm_shape, q, k, q, k, positions=self.positions, inv_freq=self.freq, stream=stream)
        lq.scan_prompt(self.scan_shape, q, k, v, self.proj[:, C:C + HV], None, self.o, self.S, self.starts, A=self.A, dt_bias=self.dt_bias, skip=self.skip,
                       work=self.work, stream=stream)

    def step(self, stream=None):
        lq.conv_step(lq.ConvShape(N, N, C, n_slots=N), self.token[:, :C], self.w, self.bias, self.conv_state, self.mixed1, stream=stream)
        q, k, v = self.split(self.mixed1)
        lq.norm_rotate(lq.NormShape(N, HQ, HQ, rot=64), q, k, q, k, positions=self.last, inv_freq=self.freq, stream=stream)
        lq.scan_step(lq.ScanShape(N, N, HV, HQ, n_slots=N, select=1), q, k, v, self.token[:, C:C + HV], None, self.o1, self.S, A=self.A,
                     dt_bias=self.dt_bias, skip=self.skip, stream=stream)


def test_prompt_then_tokens_against_the_definition_and_the_window_representation():
    a = Layer()
    a.prompt()
    torch.cuda.synchronize()
    assert lq.check_device() == 0
    starts = a.starts.tolist()
    q, k, v = a.split(a.mixed)
    wo, so, wS, sS = ops_ref.scan(q.cpu(), k.cpu(), v.cpu(), a.proj[:, C:C + HV].cpu(), None, torch.zeros(N, HV, D, D), starts, None, [0] * N, a.A.cpu(),
                                  a.dt_bias.cpu(), a.skip.cpu())
    assert ((a.o.cpu().double() - wo).abs() / (2.0 ** -8 * wo.abs() + (2.0 ** -8 + 2.0 ** -14) * so + 1e-30)).max() <= 1
    assert ((a.S.cpu().double() - wS).abs() / (2.0 ** -16 * sS + 1e-30)).max() <= 1
    # the dense states go over to the 8-bit representation, and the next token is taken on both
    sh = lq.Shape(N, HV, HQ, delta=0, W=8)
    st = lq.State(sh)
    lq.quantize_state(sh, a.S, st)
    before = a.S.cpu()
    a.step()
    q1, k1, v1 = (x.contiguous() for x in a.split(a.mixed1))
    dt = torch.nn.functional.softplus(a.token[:, C:C + HV].float() + a.dt_bias)
    beta, alpha = dt.bfloat16(), torch.exp(dt * a.A).bfloat16()
    o8 = torch.empty((N, HV, D), device="cuda")
    bits = lambda x: x.contiguous().view(torch.int16)                             # noqa: E731
    lq.decode_step(sh, st, bits(q1), bits(k1), bits(v1), bits(beta), bits(alpha), o8)
    dense = a.o1 - a.skip[:, None] * v1.float()
    # gates rounded to bf16 (2^-8 each) and 8-bit codes (half of 1/127 of a column's largest value, averaged over 128 channels)
    assert torch.linalg.norm(o8 - dense) <= 0.03 * torch.linalg.norm(dense)
    # and in 64 bits, from the states that the step was given
    o64, so64, S64, sS64 = ops_ref.scan(q1.cpu(), k1.cpu(), v1.cpu(), a.token[:, C:C + HV].cpu(), None, before, list(range(N + 1)), None, [1] * N, a.A.cpu(),
                                        a.dt_bias.cpu(), a.skip.cpu())
    assert ((a.o1.cpu().double() - o64).abs() / (2.0 ** -16 * so64 + 1e-30)).max() <= 1
    assert ((a.S.cpu().double() - S64).abs() / (2.0 ** -16 * sS64 + 1e-30)).max() <= 1


def test_the_prompt_and_the_step_captured_and_replayed_and_on_another_stream():
    a, b, c = Layer(), Layer(), Layer()
    a.prompt()
    a.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b.prompt(stream=side)
    b.step(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    c.prompt()                                # (first calls outside of the capture)
    c.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.prompt()
        c.step()
    for _ in range(3):
        for x in (c.o, c.o1, c.S, c.mixed, c.conv_state):
            x.fill_(7.0)
        graph.replay()
    torch.cuda.synchronize()
    # (sequence 2 has no rows: its slot of the convolution is left as it is, and its token goes on from what it holds - another thing in c)
    for name in ("o", "mixed", "o1", "S", "conv_state"):
        x, y, z = (getattr(l, name).clone() for l in (a, b, c))
        if name not in ("o", "mixed"):
            x[2] = y[2] = z[2] = 0.0
        assert torch.equal(x, y) and torch.equal(x, z), name


def test_two_prompts_at_once_on_two_streams_with_a_workspace_each():
    g = torch.Generator(device="cuda").manual_seed(3)
    sh = lq.ScanShape(4096, 2, 2, 1, max_len=3000, n_slots=2)
    assert lq.scan_prompt_bytes(sh) > 0       # cut into pieces
    q = torch.nn.functional.normalize(torch.randn((4096, 1, D), device="cuda", generator=g), dim=-1).bfloat16()
    k, v = q.flip(0).contiguous(), torch.randn((4096, 2, D), device="cuda", generator=g).bfloat16()
    beta, alpha = torch.rand((4096, 2), device="cuda", generator=g).bfloat16(), (1 - 0.05 * torch.rand((4096, 2), device="cuda", generator=g)).bfloat16()
    starts = torch.tensor([0, 3000, 4096], dtype=torch.int32, device="cuda")
    runs = []
    for _ in range(3):
        runs.append((torch.cuda.Stream(), torch.zeros((4096, 2, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 2, D, D), device="cuda"),
                     torch.empty((lq.scan_prompt_bytes(sh),), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o, S, work in runs:
            lq.scan_prompt(sh, q, k, v, beta, alpha, o, S, starts, work=work, stream=s)
    torch.cuda.synchronize()
    assert lq.check_device() == 0
    for _, o, S, _ in runs[1:]:
        assert torch.equal(o, runs[0][1]) and torch.equal(S, runs[0][2])


def test_the_binding_refuses_what_the_shape_does_not_say():
    a = Layer()
    x = a.proj[:, :C]
    with pytest.raises(lq.LqError):
        lq.conv_prompt(a.conv_shape, x.cpu(), a.w, a.bias, a.conv_state, a.mixed, a.starts)
    with pytest.raises(lq.LqError):
        lq.conv_prompt(a.conv_shape, x.float(), a.w, a.bias, a.conv_state, a.mixed, a.starts)
    with pytest.raises(lq.LqError):
        lq.conv_prompt(a.conv_shape, x, a.w.t().contiguous().t(), a.bias, a.conv_state, a.mixed, a.starts)
    with pytest.raises(lq.LqError):
        lq.conv_prompt(a.conv_shape, x, a.w, a.bias, a.conv_state, a.mixed, a.starts.long())
    with pytest.raises(lq.LqError):
        lq.conv_prompt(a.conv_shape, x, a.w, a.bias, a.conv_state[:2], a.mixed, a.starts)
    with pytest.raises(lq.LqError):
        lq.conv_prompt(a.conv_shape, a.mixed, a.w, a.bias, a.conv_state, a.mixed, a.starts)          # in place
    q, k, v = a.split(a.mixed)
    with pytest.raises(lq.LqError):
        lq.norm_rotate(a.norm_shape, q, k, k, q, positions=a.positions, inv_freq=a.freq)              # crossed
    with pytest.raises(lq.LqError):
        lq.scan_prompt(a.scan_shape, q, k, v, a.proj[:, C:C + HV], None, a.o, a.S, a.starts)          # A is missing
    with pytest.raises(lq.LqError):
        lq.scan_prompt(a.scan_shape, q, k, v.transpose(1, 2), a.proj[:, C:C + HV], None, a.o, a.S, a.starts, A=a.A)
    long = lq.ScanShape(4096, 1, 1, 1, max_len=4096, n_slots=1)
    big = torch.zeros((4096, 1, D), dtype=torch.bfloat16, device="cuda")
    gates = torch.zeros((4096, 1), dtype=torch.bfloat16, device="cuda")
    for work in (None, torch.empty((lq.scan_prompt_bytes(long) - 1,), dtype=torch.uint8, device="cuda")):
        with pytest.raises(lq.LqError):
            lq.scan_prompt(long, big, big, big, gates, gates, torch.empty_like(big), torch.zeros((1, 1, D, D), device="cuda"),
                           torch.tensor([0, 4096], dtype=torch.int32, device="cuda"), work=work)


def test_arrays_of_sequences_that_make_no_sense_touch_nothing_else():
    """Row numbers that go down or out of range and slots that do not exist: no access outside of the arrays."""
    a = Layer()
    guard = 5.0
    mixed = torch.full((a.T + 64, C), guard, dtype=torch.bfloat16, device="cuda")
    state = torch.full((N + 2, W - 1, C), guard, dtype=torch.bfloat16, device="cuda")
    S = torch.full((N + 2, HV, D, D), guard, device="cuda")
    o = torch.full((a.T + 64, HV, D), guard, dtype=torch.bfloat16, device="cuda")
    q, k, v = a.split(a.proj[:, :C].contiguous())
    bad = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in
           ([-5, 300, 200, 10 ** 9, -7, 2 ** 31 - 1], [400, 300, 200, 100, 50, 0], [0, 0, 0, 0, 0, -1], [428, 428, 428, 428, 428, 2 ** 31 - 1])]
    slots = torch.tensor([-2 ** 31, 7, 2 ** 31 - 1, -1, 1], dtype=torch.int32, device="cuda")
    for starts in bad:
        for sl in (None, slots):
            lq.conv_prompt(a.conv_shape, a.proj[:, :C], a.w, a.bias, state[1:1 + N], mixed[32:32 + a.T], starts, slots=sl,
                           resume=torch.ones(N, dtype=torch.int32, device="cuda"))
            lq.scan_prompt(a.scan_shape, q, k, v, a.proj[:, C:C + HV], None, o[32:32 + a.T], S[1:1 + N], starts, slots=sl, A=a.A, work=a.work,
                           resume=torch.ones(N, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert lq.check_device() == 0
    for x, lead, tail in ((mixed, 32, 32), (o, 32, 32), (state, 1, 1), (S, 1, 1)):
        assert bool((x[:lead] == guard).all()) and bool((x[-tail:] == guard).all())


def test_arrays_side_by_side_in_one_buffer():
    """Column slices of one buffer and the states right behind its last row: neighbours, not overlaps; the bits are those of arrays of their own."""
    T, H, G, D = 150, 2, 1, 128
    g = torch.Generator(device="cuda").manual_seed(5)
    W = (2 * G + 2 * H) * D                                                       # q | k | v | o
    n = T * W * 2
    buf = torch.empty(n + H * D * D * 4, device="cuda", dtype=torch.uint8)
    rows, S = buf[:n].view(torch.bfloat16).view(T, W), buf[n:].view(torch.float32).view(1, H, D, D)
    rows.copy_(torch.randn(T, W, device="cuda", generator=g) * 0.1)
    cut = lambda a, b, h: rows[:, a * D:b * D].unflatten(1, (h, D))               # noqa: E731
    q, k, v, o = cut(0, G, G), cut(G, 2 * G, G), cut(2 * G, 2 * G + H, H), cut(2 * G + H, 2 * G + 2 * H, H)
    beta, alpha = (torch.rand(T, H, device="cuda", generator=g).bfloat16() for _ in range(2))
    start = torch.tensor([0, T], device="cuda", dtype=torch.int32)
    sh = lq.ScanShape(T, 1, H, G, max_len=T, n_slots=1)
    own_o, own_S = torch.empty(T, H, D, device="cuda", dtype=torch.bfloat16), torch.empty(1, H, D, D, device="cuda")
    work = torch.empty(lq.scan_prompt_bytes(sh), device="cuda", dtype=torch.uint8)
    lq.scan_prompt(sh, q.contiguous(), k.contiguous(), v.contiguous(), beta, alpha, own_o, own_S, start, work=work)
    lq.scan_prompt(sh, q, k, v, beta, alpha, o, S, start, work=work)
    assert torch.equal(o, own_o) and torch.equal(S, own_S)

    C = 64
    n = T * 2 * C * 2
    buf = torch.empty(n + 3 * C * 2, device="cuda", dtype=torch.uint8)
    rows, state = buf[:n].view(torch.bfloat16).view(T, 2 * C), buf[n:].view(torch.bfloat16).view(1, 3, C)
    rows.copy_(torch.randn(T, 2 * C, device="cuda", generator=g))
    w = torch.randn(C, 4, device="cuda", generator=g).bfloat16()
    x, out = rows[:, :C], rows[:, C:]
    own, own_state = torch.empty(T, C, device="cuda", dtype=torch.bfloat16), torch.empty(1, 3, C, device="cuda", dtype=torch.bfloat16)
    sh = lq.ConvShape(T, 1, C, n_slots=1)
    lq.conv_prompt(sh, x.contiguous(), w, None, own_state, own, start)
    lq.conv_prompt(sh, x, w, None, state, out, start)
    assert torch.equal(out, own) and torch.equal(state, own_state)
