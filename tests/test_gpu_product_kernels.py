"""Every instance of the product kernels on calls that reach it: which kernel a call launches is read from a captured graph of it, so that a test of a kernel cannot
come to be one of another.

Tolerance as in test_gpu_product.py: one rounding to the result's type; each of a block's 128 additions and of the additions over blocks is off by 2^-23 of the sum over
magnitudes at most, the scales' product and the one with it by half a step each.
"""
import ctypes as C
import re

import pytest
import torch

import linear_ref as ref
from paper_2609_38166_b200 import lq

pytestmark = pytest.mark.gpu
TYPES = {torch.bfloat16: "13__nv_bfloat16", torch.float16: "6__half", torch.float32: "f"}
FILL = 7.0
MANY, FEW = "many", "few"


class KernelNode(C.Structure):
    _fields_ = [("func", C.c_void_p), ("grid", C.c_uint * 3), ("block", C.c_uint * 3), ("shared", C.c_uint), ("params", C.c_void_p), ("extra", C.c_void_p),
                ("kern", C.c_void_p), ("ctx", C.c_void_p)]


def launched(call):
    """(kernel, type, wide, rows of a tile or None) of a call, from the driver's graph of it."""
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    driver, raw = C.CDLL("libcuda.so.1"), C.c_void_p(graph.raw_cuda_graph())
    count = C.c_size_t(0)
    assert driver.cuGraphGetNodes(raw, None, C.byref(count)) == 0 and count.value == 1
    node, of, name = C.c_void_p(), KernelNode(), C.c_char_p()
    assert driver.cuGraphGetNodes(raw, C.byref(node), C.byref(count)) == 0
    assert driver.cuGraphKernelNodeGetParams_v2(node, C.byref(of)) == 0
    named = driver.cuFuncGetName(C.byref(name), C.c_void_p(of.func)) if of.func else driver.cuKernelGetName(C.byref(name), C.c_void_p(of.kern))
    assert named == 0
    found = re.search(r"product_(many|few)_kernelI(13__nv_bfloat16|6__half|f)Lb([01])E(?:Li(\d+)E)?", name.value.decode())
    assert found, name.value
    kernel, kind, wide, rows = found.groups()
    return kernel, {v: k for k, v in TYPES.items()}[kind], wide == "1", int(rows) if rows else None


def operands(rows, cin, cout, groups, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")                      # noqa: E731
    blocks = -(-cin // 128)
    x = (100 * r(rows, cin)).clamp(-448, 448).to(ref.E4M3)
    s = torch.exp(r(blocks, rows)) / 100
    w = (100 * r(groups, cout, cin)).clamp(-448, 448).to(ref.E4M3)
    ws = torch.exp(0.5 * r(groups, -(-cout // 128), blocks)) / (100 * cin ** 0.5)
    return x, s, w, ws


def definition(x, s, w, ws, starts):
    """In 64 bits: (out, the same sum over magnitudes); NaN in rows of no group."""
    a = x.double() * s.double().t().repeat_interleave(128, 1)[:, :x.shape[1]]
    out = torch.full((x.shape[0], w.shape[1]), float("nan"), dtype=torch.float64, device="cuda")
    size = torch.ones_like(out)
    for g in range(len(starts) - 1):
        r, b = slice(starts[g], starts[g + 1]), ref.weights(w[g], ws[g]).t()
        out[r], size[r] = a[r] @ b, a[r].abs() @ b.abs()
    return out, size


class Call:
    def __init__(self, rows, cin, cout, dtype, wide, starts=None, seed=0):
        groups = len(starts) - 1 if starts else 1
        self.sh = lq.ProductShape(rows, cin, cout, groups=groups, type=lq.TYPES[dtype])
        self.x, self.s, self.w, self.ws = operands(rows, cin, cout, groups, seed)
        piece = 16 // dtype.itemsize
        self.pad = -cout % piece if wide else 1 + cout % 2                         # (an odd number of elements from row to row)
        self.buf = torch.full((rows + 2, cout + self.pad), FILL, dtype=dtype, device="cuda")
        if wide and self.buf.shape[1] % piece:
            raise AssertionError
        self.out, self.starts = self.buf[1:rows + 1, :cout], starts
        self.start = torch.tensor(starts, dtype=torch.int32, device="cuda") if starts else None

    def __call__(self):
        if self.starts:
            lq.product_groups(self.sh, self.x, self.s, self.w, self.ws, self.out, self.start)
        else:
            lq.product(self.sh, self.x, self.s, self.w[0], self.ws[0], self.out)

    def check(self):
        self.buf.fill_(FILL)
        self()
        want, size = definition(self.x, self.s, self.w, self.ws, self.starts or [0, self.x.shape[0]])
        live = ~torch.isnan(want)
        slack = (128 + self.s.shape[0] + 2) * 2.0 ** -23 * size[live]
        assert ref.off(self.out[live], want[live], self.out.dtype, slack) <= 1
        assert (self.out[~live] == FILL).all()
        rest = self.buf.clone()
        rest[1:-1, :self.out.shape[1]] = FILL
        assert (rest == FILL).all() and lq.check_device() == 0
        first = self.buf.clone()
        for _ in range(3):                                                        # the same bits again
            self.out.zero_()
            self()
            assert torch.equal(self.out[live], first[1:-1, :self.out.shape[1]][live])


def ragged(rows, groups, seed, first=0, last=None):
    g = torch.Generator().manual_seed(seed)
    last = rows if last is None else last
    cuts = (first + torch.rand(groups - 1, generator=g) * (last - first)).int().sort().values.tolist()
    cuts[groups // 2] = cuts[groups // 2 - 1]                                     # an empty one
    return [first, *sorted(cuts), last]


every = pytest.mark.parametrize("dtype,wide", [(t, w) for t in TYPES for w in (True, False)], ids=str)


@every
@pytest.mark.parametrize("cin", [384, 400, 640])
def test_many_rows(dtype, wide, cin):
    """304 tiles of 256 x 256 on 74 pairs of CTAs, 3, 4 (the last a part) and 5 K blocks, rows and outputs that end inside a tile."""
    call = Call(4000, cin, 4735, dtype, wide, seed=cin)
    assert launched(call) == (MANY, dtype, wide, None)
    call.check()


@every
@pytest.mark.parametrize("cin", [128, 720])
def test_many_rows_of_groups(dtype, wide, cin):
    """Ragged groups, about 400 tiles; rows of nobody in front and behind."""
    call = Call(12000, cin, 1300, dtype, wide, ragged(12000, 24, cin, 100, 11900), seed=cin)
    assert launched(call) == (MANY, dtype, wide, None)
    call.check()


@every
def test_hundreds_of_rows_of_groups(dtype, wide):
    """Tiles of 128 rows by groups, a CTA from one group to the next: more than 300 tiles on 148 CTAs, 4 and 6 K blocks."""
    for cin in (400, 720):
        call = Call(4500, cin, 599, dtype, wide, ragged(4500, 64, cin, 3, 4490), seed=cin)
        assert launched(call) == (FEW, dtype, wide, 128)
        call.check()


@every
def test_hundreds_of_rows(dtype, wide):
    """Tiles of 128 rows in three rounds, five K blocks."""
    call = Call(40000, 640, 100, dtype, wide)
    assert launched(call) == (FEW, dtype, wide, 128)
    call.check()


@every
def test_few_rows(dtype, wide):
    """Tiles of 32 rows, by groups in several rounds, and shared by the CTAs of a cluster."""
    call = Call(2500, 400, 1003, dtype, wide, ragged(2500, 100, 7))
    assert launched(call) == (FEW, dtype, wide, 32)
    call.check()
    for rows in (1, 13, 32):
        call = Call(rows, 1296, 1003, dtype, wide, seed=rows)
        assert launched(call) == (FEW, dtype, wide and rows > 1, 32)              # (a row alone is as far from the next as it is wide: 1003)
        call.check()


@every
def test_hundreds_of_rows_shared(dtype, wide):
    """Tiles of 128 rows whose K blocks are shared by the CTAs of a cluster, with the sums in either place."""
    for rows in (33, 129, 200):
        call = Call(rows, 1296, 1003, dtype, wide, seed=rows)
        assert launched(call) == (FEW, dtype, wide, 128)
        call.check()


@pytest.mark.parametrize("kernel,rows,cin,cout,starts", [(MANY, 4000, 400, 2049, None), (MANY, 12000, 272, 1300, [0, 5000, 5000, 12000]), (FEW, 4500, 400, 599, "64 groups"),
                                                          (FEW, 40000, 640, 100, None)], ids=str)
def test_what_is_not_finite_stays_in_its_row(kernel, rows, cin, cout, starts):
    starts = ragged(rows, 64, 1) if starts == "64 groups" else starts
    call = Call(rows, cin, cout, torch.float32, False, starts)
    assert launched(call)[0] == kernel
    call()
    clean = call.out.clone()
    bad = [3, 7, 130, 299, 1023]
    codes = call.x.view(torch.uint8)
    codes[bad[0], 100] = codes[bad[2]] = codes[bad[3], 5] = 0x7F
    call.s[1, bad[1]] = float("inf")
    call.s[0, bad[4]] = float("nan")
    call()
    assert torch.isnan(call.out[[bad[0], bad[2], bad[3], bad[4]]]).all() and not torch.isfinite(call.out[bad[1]]).any()
    same = torch.ones(rows, dtype=torch.bool, device="cuda")
    same[bad] = False
    assert torch.equal(call.out[same], clean[same])


@pytest.mark.parametrize("codes,steps", [("of one size", 1), ("of every size", 37), ("one and the rest", 37)])
@pytest.mark.parametrize("kernel,rows,cout", [(MANY, 16384, 2048), (FEW, 40, 2048)])
def test_sums_of_a_block(kernel, rows, cout, codes, steps):
    """One K block and factors of 1: outputs are the accumulators.  An instruction adds 32 products to the sum so far; terms are cut off 2^-25 below the largest of
    them, 33 * 2^-25 of it in all, and the sum at 2^-23 of itself: 9.25 * 2^-23 of the sum over magnitudes, four times 37.  Where they are of one size, next to nothing
    is cut off: a step in all."""
    call = Call(rows, 128, cout, torch.float32, True)
    g = torch.Generator(device="cuda").manual_seed(1)
    if codes != "of one size":
        for t in (call.x, call.w):
            any_ = torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8)
            any_[any_ % 128 == 127] = 0                                           # (NaN)
            t.view(torch.uint8).copy_(any_)
    if codes == "one and the rest":                                               # 127 of the smallest
        call.x.view(torch.uint8).copy_(1 + 128 * (torch.arange(128, device="cuda") % 3 == 0).to(torch.uint8))
        call.x.view(torch.uint8)[:, 77] = 0x7E
    call.s.fill_(1.0), call.ws.fill_(1.0)
    assert launched(call)[0] == kernel
    call()
    want, size = definition(call.x, call.s, call.w, call.ws, [0, rows])
    assert ((call.out.double() - want).abs() <= steps * 2.0 ** -23 * size).all()


@pytest.mark.parametrize("share", range(2, 9))
def test_clusters_of_every_size(share):
    """A tile's K blocks shared by 2 to 8 CTAs, evenly and not."""
    for cin in (256 * share, 256 * share + 16):
        for rows in (5, 40, 128):
            Call(rows, cin, 250, torch.bfloat16, True, seed=cin).check()


def test_weights_beyond_two_to_the_32_bytes():
    """600 groups of 8 MB: rows in the first, in one on either side of 2^32 bytes, and in the last."""
    groups, cin, cout, rows = 600, 2048, 4096, 60
    assert groups * cin * cout > 2 ** 32
    x, s, w, ws = operands(rows, cin, cout, 4, 4)
    big = torch.full((groups, cout, cin), 0x7F, dtype=torch.uint8, device="cuda").view(ref.E4M3)   # (NaN)
    scales = torch.full((groups, cout // 128, cin // 128), float("nan"), device="cuda")
    at = [0, 511, 512, 599]
    for k, n in enumerate(at):
        big[n], scales[n] = w[k], ws[k]
    cuts = [0, 13, 20, 45, rows]
    starts = [cuts[sum(n < m for n in at)] for m in range(groups + 1)]
    out = torch.empty((rows, cout), dtype=torch.float32, device="cuda")
    lq.product_groups(lq.ProductShape(rows, cin, cout, groups=groups, type=lq.F32), x, s, big, scales, out, torch.tensor(starts, dtype=torch.int32, device="cuda"))
    want, size = definition(x, s, w, ws, cuts)
    assert ref.off(out, want, torch.float32, (128 + cin // 128 + 2) * 2.0 ** -23 * size) <= 1 and lq.check_device() == 0
