"""Selective scan over prompts and for single tokens, against the recurrence in 64 bits.

Tolerances, elementwise, against the sums of the terms' magnitudes (`scale`, the same recurrence over absolute values):
S is held in binary32.  Weights are exact to a few steps of 2^-23 (exponentials of sums of at most 128 logarithms, each off by 2^-23 of
itself where at most about 30 of the sum matters: 2^-18), products with them are kept to 24 bits, and sums over a block of 128 rows
pass at most 24 accumulations: together below 2^-16.
o of the prompt is rounded to bf16 (2^-8 of the value), and so are, in front of the last two products, the weighted scores and the
state: 2^-8 of the magnitudes that enter them, which `scale` bounds.  o of a single token is binary32: 2^-16 of `scale`.
"""
import pytest
import torch

import ops_ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu
D = 128
BF = 2.0 ** -8
FILL = 33.0


class Case:
    def __init__(self, lens, hv, hq, select=False, gates=torch.bfloat16, skip=False, lead=0, tail=0, pad=0, slots=None, n_slots=None, resume=None, seed=0,
                 slow=0.05, bias=True):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g)                                # noqa: E731
        T = lead + sum(lens) + tail
        self.lens, self.hv, self.hq, self.T, self.resume, self.slots = lens, hv, hq, T, resume, slots
        self.n_slots = n_slots or len(lens)
        self.starts = [lead]
        for n in lens:
            self.starts.append(self.starts[-1] + n)
        unit = lambda x: x / x.norm(dim=-1, keepdim=True)                         # noqa: E731
        self.q, self.k = unit(r(T, hq, D)).bfloat16(), unit(r(T, hq, D)).bfloat16()
        self.v = r(T, hv, D).bfloat16()
        self.A = self.dt_bias = self.alpha = None
        if select:
            self.beta = r(T, hv).to(gates)
            self.A, self.dt_bias = -torch.rand(hv, generator=g) * 2, r(hv) - 2 if bias else None
        else:
            self.beta = torch.sigmoid(r(T, hv)).to(gates)
            self.alpha = torch.exp(-slow * torch.nn.functional.softplus(r(T, hv))).to(gates)
        self.skip = r(hv) if skip else None
        self.S = 0.3 * r(self.n_slots, hv, D, D)
        self.pad, self.gates, self.select = pad, gates, select

    def dev(self, x, dtype=None):
        return None if x is None else torch.as_tensor(x, dtype=dtype).cuda()

    def wide(self, x):
        T, h = x.shape[:2]
        buf = torch.full((T, h * D + self.pad), float("nan"), dtype=x.dtype, device="cuda")
        buf[:, self.pad // 2:self.pad // 2 + h * D] = x.cuda().flatten(1)
        return buf[:, self.pad // 2:self.pad // 2 + h * D].unflatten(-1, (h, D))

    def shape(self, **kw):
        return lq.ScanShape(self.T, len(self.lens), self.hv, self.hq, max_len=max(self.lens, default=0), n_slots=self.n_slots, select=int(self.select),
                            gate_type=lq.TYPES[self.gates], **kw)

    def prompt(self, sh=None, work=None, stream=None, apart=False):
        sh = sh or self.shape()
        o = torch.full((self.T, self.hv * D + self.pad), FILL, dtype=torch.bfloat16, device="cuda")
        S = self.S.cuda()
        S0, S = (S, torch.full_like(S, float("nan"))) if apart else (None, S)
        n = lq.scan_prompt_bytes(sh)
        work = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if work is None else work
        i32 = torch.int32
        lq.scan_prompt(sh, self.wide(self.q), self.wide(self.k), self.wide(self.v), self.dev(self.beta), self.dev(self.alpha),
                       o[:, :self.hv * D].unflatten(-1, (self.hv, D)), S, self.dev(self.starts, i32), slots=self.dev(self.slots, i32),
                       resume=self.dev(self.resume, i32), A=self.dev(self.A), dt_bias=self.dev(self.dt_bias), skip=self.dev(self.skip), S0=S0, work=work, stream=stream)
        torch.cuda.synchronize()
        assert lq.check_device() == 0
        assert S0 is None or torch.equal(S0.cpu(), self.S)
        assert bool((o[:, self.hv * D:] == FILL).all())
        return o[:, :self.hv * D].unflatten(-1, (self.hv, D)).cpu(), S.cpu()

    def want(self):
        return ops_ref.scan(self.q, self.k, self.v, self.beta, self.alpha, self.S, self.starts, self.slots, self.resume if self.resume else [0] * len(self.lens),
                            self.A, self.dt_bias, self.skip)

    def check(self):
        o, S = self.prompt()
        wo, so, wS, sS = self.want()
        there = ~torch.isnan(wo)
        assert torch.equal(o[~there], torch.full_like(o[~there], FILL))
        off = ((o.double() - wo).abs() / (BF * wo.abs() + (BF + 2.0 ** -14) * so + 1e-30))[there]
        assert off.numel() == 0 or off.max() <= 1, float(off.max())
        off = (S.double() - wS).abs() / (2.0 ** -16 * sS + 1e-30)
        assert off.max() <= 1, float(off.max())


@pytest.mark.parametrize("n", [1, 2, 7, 8, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300])
def test_lengths(n):
    Case([n], 2, 1, resume=[1], seed=n).check()


@pytest.mark.parametrize("hv,hq", [(1, 1), (3, 3), (6, 2), (8, 1), (4, 4)])
@pytest.mark.parametrize("select", [False, True])
@pytest.mark.parametrize("gates", [torch.bfloat16, torch.float32], ids=str)
def test_heads_and_gates(hv, hq, select, gates):
    Case([150, 40], hv, hq, select=select, gates=gates, skip=True, resume=[0, 1], pad=64, seed=hv).check()


def test_select_without_bias():
    Case([150], 2, 1, select=True, bias=False).check()


def test_ragged_packed_with_empty_and_padding_sequences():
    lens = [0, 1, 130, 0, 5, 128, 1, 200, 64, 0]
    slots = [9, 0, 4, 2, -1, 1, 12, 3, 5, 6]                                      # 12 is not a slot: padding, as is -1
    Case(lens, 4, 2, slots=slots, n_slots=11, resume=[1, 1, 0, 0, 1, 0, 1, 1, 0, 0], lead=5, tail=9, skip=True).check()


def test_single_tokens_packed():
    Case([1] * 40, 2, 2, resume=[i % 2 for i in range(40)]).check()


@pytest.mark.parametrize("resume", ["none", "all", "some"])
@pytest.mark.parametrize("lens", [[128] * 60, [3, 128, 64, 200, 0, 1] * 10, [256, 130] * 30])
def test_many_heads_to_a_multiprocessor(lens, resume):
    """Several heads one after the other in a CTA, with and without a state in front of them."""
    Case(lens, 8, 2, resume=[{"none": 0, "all": 1, "some": i % 3 % 2}[resume] for i in range(len(lens))], skip=True).check()


def test_decays_of_zero_and_one():
    """alpha 0 empties the state in the middle of a prompt, also many times in a block; alpha 1 keeps all."""
    c = Case([300, 260], 2, 1, gates=torch.float32, resume=[1, 1])
    c.alpha[::7] = 0.0
    c.alpha[400:] = 1.0
    c.alpha[:, 1] = torch.where(torch.rand(560) < 0.5, 0.0, 0.9)
    c.check()
    c.alpha[:] = 0.0
    c.check()
    c.alpha[:] = 1.0
    c.check()


def test_strong_and_weak_decays():
    c = Case([400], 3, 1, gates=torch.float32, resume=[1])
    g = torch.Generator().manual_seed(5)
    c.alpha[:, 0] = torch.exp(-60 * torch.rand(400, generator=g))                 # logarithms that sum to thousands
    c.alpha[:, 1] = 1 - 2.0 ** -20
    c.alpha[:, 2] = torch.where(torch.arange(400) % 64 == 9, 1e-38, 0.999)
    c.check()


def test_signs_and_sizes_of_beta():
    c = Case([200], 2, 2, gates=torch.float32)
    c.beta = torch.randn(200, 2) * 1e3
    c.beta[::5] = 0.0
    c.check()


def test_one_long_prompt_behind_many_short_ones():
    """More heads than multiprocessors: the long prompt's are handed out first, whatever its place."""
    lens = [20] * 18 + [1700] + [33, 0]
    Case(lens, 8, 4, resume=[i % 2 for i in range(len(lens))], slots=list(range(len(lens)))[::-1], skip=True).check()


def test_large_values_behind_strong_decays():
    """Outputs of 10^9 and more where the decays since the start of a block are far below 2^-60."""
    c = Case([300], 2, 1, gates=torch.float32, resume=[1], slow=3.0)
    c.v = (c.v.float() * 2.0 ** 30).bfloat16()
    c.S = c.S * 2.0 ** 20
    c.check()


def test_long_prompt_few_heads():
    """Cut into pieces along the prompt."""
    Case([2500], 1, 1, resume=[1], slow=0.01, skip=True).check()
    Case([1500, 3, 700], 2, 1, resume=[1, 0, 1], slow=0.003, select=True).check()


def test_values_of_other_sequences_never_arrive():
    """NaN and infinities in rows of no sequence and in a neighbour, on both sides, leave a sequence bit for bit as it is."""
    a = Case([100, 70, 150], 2, 1, lead=6, tail=11, resume=[1, 1, 1], skip=True)
    o, S = a.prompt()
    for x in (a.q, a.k, a.v, a.beta, a.alpha):
        x[:6], x[106:176], x[326:] = float("nan"), float("inf"), float("nan")
    o2, S2 = a.prompt()
    for rows in (slice(6, 106), slice(176, 326)):
        assert torch.equal(o[rows], o2[rows])
    assert torch.equal(S[0], S2[0]) and torch.equal(S[2], S2[2])


def test_infinite_values_in_a_fresh_slot_are_not_read():
    a = Case([100], 1, 1, resume=[0])
    a.S[:] = float("nan")
    o, S = a.prompt()
    assert torch.isfinite(o).all() and torch.isfinite(S).all()


def test_the_same_call_gives_the_same_bits():
    a = Case([900, 10], 2, 1, resume=[1, 0])
    o, S = a.prompt()
    for _ in range(3):
        o2, S2 = a.prompt()
        assert torch.equal(o, o2) and torch.equal(S, S2)


def test_longer_than_max_len_is_cut():
    a = Case([100, 50], 2, 1)
    sh = a.shape()
    sh.max_len = 60
    o, S = a.prompt(sh)
    b = Case([100, 50], 2, 1)
    want, _ = b.prompt()
    assert torch.equal(o[:60], want[:60]) and torch.equal(o[100:], want[100:])
    assert bool((o[60:100] == FILL).all())


@pytest.mark.parametrize("lens", [[100, 0, 300, 0], [1500, 0, 2]])
def test_resumed_from_a_state_that_stays(lens):
    a = Case(lens, 2, 1, resume=[1, 1, 0, 0][:len(lens)])
    o, S = a.prompt()
    o2, S2 = a.prompt(apart=True)
    assert torch.equal(o, o2) and torch.equal(S, S2)


def test_no_rows_at_all():
    a = Case([0, 0], 2, 1, resume=[1, 0])
    _, S = a.prompt()
    assert torch.equal(S[0], a.S[0]) and not S[1].any()


@pytest.mark.parametrize("batch,hv,hq", [(1, 1, 1), (3, 6, 2), (40, 4, 4)])
@pytest.mark.parametrize("select", [False, True])
@pytest.mark.parametrize("gates", [torch.bfloat16, torch.float32], ids=str)
def test_step(batch, hv, hq, select, gates):
    slots = torch.randperm(batch + 2, generator=torch.Generator().manual_seed(1))[:batch].tolist()
    if batch > 2:
        slots[1] = -1
    c = Case([1] * batch, hv, hq, select=select, gates=gates, skip=select, slots=slots, n_slots=batch + 2, resume=[1] * batch, pad=64)
    o = torch.full((batch, hv, D), FILL, device="cuda")
    S = c.S.cuda()
    lq.scan_step(c.shape(), c.wide(c.q), c.wide(c.k), c.wide(c.v), c.dev(c.beta), c.dev(c.alpha), o, S, slots=c.dev(c.slots, torch.int32), A=c.dev(c.A),
                 dt_bias=c.dev(c.dt_bias), skip=c.dev(c.skip))
    wo, so, wS, sS = c.want()
    there = ~torch.isnan(wo)
    assert torch.equal(o.cpu()[~there], torch.full_like(o.cpu()[~there], FILL))
    assert (((o.cpu().double() - wo).abs() / (2.0 ** -16 * so + 1e-30))[there]).max() <= 1
    assert ((S.cpu().double() - wS).abs() / (2.0 ** -16 * sS + 1e-30)).max() <= 1


def test_prompt_then_steps_are_the_longer_prompt():
    a = Case([140], 4, 2, select=True, skip=True)
    wo, so, wS, sS = a.want()
    sh = lq.ScanShape(130, 1, 4, 2, max_len=130, n_slots=1, select=1)
    o = torch.empty((130, 4, D), dtype=torch.bfloat16, device="cuda")
    S = a.S.cuda()
    q, k, v, dt = (x.cuda() for x in (a.q, a.k, a.v, a.beta))
    kw = dict(A=a.dev(a.A), dt_bias=a.dev(a.dt_bias), skip=a.dev(a.skip))
    work = torch.empty((lq.scan_prompt_bytes(sh),), dtype=torch.uint8, device="cuda")
    lq.scan_prompt(sh, q[:130], k[:130], v[:130], dt[:130], None, o, S, torch.tensor([0, 130], dtype=torch.int32, device="cuda"), work=work, **kw)
    one = lq.ScanShape(1, 1, 4, 2, n_slots=1, select=1)
    for t in range(130, 140):
        ot = torch.empty((1, 4, D), device="cuda")
        lq.scan_step(one, q[t:t + 1], k[t:t + 1], v[t:t + 1], dt[t:t + 1], None, ot, S, **kw)
        assert ((ot.cpu()[0].double() - wo[t]).abs() / (2.0 ** -16 * so[t])).max() <= 1
    assert ((S.cpu().double() - wS).abs() / (2.0 ** -16 * sS + 1e-30)).max() <= 1


@pytest.mark.parametrize("lens,hv,hq,select,slow", [([300, 128, 77], 4, 2, False, 0.05), ([300, 128, 77], 4, 2, False, 1.0), ([520], 6, 6, True, 0.05),
                                                    ([2500], 1, 1, False, 0.01)])
def test_all_outputs_together(lens, hv, hq, select, slow):
    """The 2-norm of what all outputs are off by, below that of three roundings to bf16 at independent places.

    A rounding to bf16 (steps of 2^-7 of the power of two below) is off by 2^-7 / sqrt(12) = 2.26e-3 of the value in the mean square at most.
    The output has one; in front of it are one of the state's elements, which q weighs, and one of the weighted scores, which weigh v.  These are
    sums of many terms with errors that do not know of one another, so that each part is off by 2.26e-3 of its own size, and the parts, which
    do not know of one another either, have the output's size together: sqrt(2) * 2.26e-3 = 3.2e-3, and half a percent for the number of
    outputs (50 thousand at least) and for binary32.
    """
    c = Case(lens, hv, hq, select=select, slow=slow, resume=[1] * len(lens), gates=torch.float32)
    o, S = c.prompt()
    wo, _, wS, _ = c.want()
    off = float(torch.linalg.norm(o.double() - wo) / torch.linalg.norm(wo))
    print(f"o {off:.3e}, S {float(torch.linalg.norm(S.double() - wS) / torch.linalg.norm(wS)):.3e}")
    assert off <= 1.005 * 2 ** 0.5 * 2.0 ** -7 / 12 ** 0.5
