"""Refusals of the operators on packed rows, each with nothing else in the call that could be refused (no GPU is touched).

Addresses that are never looked at: arrays that are not meant to meet lie 2^40 bytes and more apart."""
import ctypes as C
import dataclasses

import pytest
import torch

from paper_2609_38166_b200 import build, lq

OK, NULL, SHAPE, ALIGN, UNSUPPORTED = 0, 1, 2, 3, 4
X, OUT, TAPS, STATE, STARTS = 1 << 40, 1 << 52, 1 << 57, 1 << 58, 1 << 61


@pytest.fixture(scope="module")
def L():
    build.build()
    return lq.lib()


def conv(L, sh, step, x=X, xs=None, out=OUT, outs=None, state=STATE):
    s, xs, outs = C.byref(sh.c()), sh.channels if xs is None else xs, sh.channels if outs is None else outs
    if step:
        return L.lq_conv_step(s, x, xs, TAPS, None, state, out, outs, None, None)
    return L.lq_conv_prompt(s, x, xs, TAPS, None, state, out, outs, STARTS, None, None, None)


# rows of 64 bf16 channels, 128 bytes; 40 of them
OVERLAPS = [
    dict(out=X + 2), dict(out=X + 128), dict(out=X - 128), dict(out=X + 39 * 128 + 126), dict(out=X - 39 * 128 - 126),
    dict(xs=128, outs=128, out=X + 2 * 63), dict(xs=128, outs=128, out=X - 2 * 63), dict(xs=128, outs=128, out=X + 256 * 39 + 2 * 63),
    dict(xs=128, outs=128, out=X + 256 * 7 - 2 * 63), dict(xs=128, outs=192, out=X + 128), dict(xs=128, outs=64, out=X), dict(xs=64, outs=128, out=X),
    dict(state=X), dict(state=X + 39 * 128 + 126), dict(state=X - 4 * 3 * 128 + 2),                 # (slots of 3 rows)
    dict(state=OUT), dict(state=OUT + 39 * 128 + 126), dict(state=OUT - 4 * 3 * 128 + 2),
]


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("kw", OVERLAPS, ids=str)
def test_conv_arrays_that_overlap(L, step, kw):
    sh = lq.ConvShape(40, 40 if step else 4, 64, n_slots=4)
    assert conv(L, sh, step, **kw) == UNSUPPORTED


def test_conv_prompt_in_place(L):
    assert conv(L, lq.ConvShape(40, 4, 64, n_slots=4), False, out=X) == UNSUPPORTED


@pytest.mark.parametrize("step", [False, True])
def test_conv_more_than_a_grid(L, step):
    """2^20 rows of 2^30 channels: 2^34 CTAs and more, in arrays of 2^51 bytes that do not meet."""
    sh = lq.ConvShape(1 << 20, 1 << 20 if step else 4, 1 << 30, n_slots=4)
    assert conv(L, sh, step) == UNSUPPORTED


# ---- the binding: what the shape says of a tensor, argument by argument.  Host tensors pass for tensors of the device, and the library is not there ----

class Called(Exception):
    pass


class Library:
    def __getattr__(self, name):
        def call(*args):
            raise Called(name)
        return call


@pytest.fixture
def host(monkeypatch):
    monkeypatch.setattr(lq, "_lib", Library())
    monkeypatch.setattr(lq, "_device", lambda: -1)                                # (what get_device() says of a host tensor)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 7


def wrong(t, rows):
    """Tensors that are not like t: another type, another shape, missing elements between neighbours, one row too few, another device."""
    yield t.double() if t.is_floating_point() else t.long()
    yield t[None]
    yield t[:-1] if t.shape[0] > 1 else torch.cat([t, t])
    yield t.as_subclass(Elsewhere)
    if t.shape[-1] > 1:
        yield torch.stack([t, t], -1)[..., 0]
    if rows and t.dim() == 3 and t.shape[1] > 1:
        yield t.transpose(1, 2).contiguous().transpose(1, 2)
    if not rows and t.dim() > 1:
        yield torch.cat([t, t], -1)[..., :t.shape[-1]]


def check(call, args, rows):
    with pytest.raises(Called):
        call(args)
    for name, t in args.items():
        if t is None:
            continue
        for bad in wrong(t, name in rows or name == "alpha"):                   # (rows may be strided)
            with pytest.raises(lq.LqError, match=rf"^{name}: "):
                call({**args, name: bad})
    for name in rows:
        with pytest.raises(lq.LqError, match=rf"^{name}: missing"):
            call({**args, name: None})


def rand(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def ints(n):
    return torch.zeros(n, dtype=torch.int32)


def test_binding_conv(host):
    sh = lq.ConvShape(6, 3, 16, width=4, n_slots=4)
    args = dict(x=rand(6, 16), w=rand(16, 4), bias=rand(16), state=rand(4, 3, 16), out=rand(6, 16), seq_start=ints(4), slots=ints(3), resume=ints(3))
    check(lambda a: lq.conv_prompt(sh, stream=0, **a), args, ("x", "out"))
    sh = dataclasses.replace(sh, tokens=3)
    del args["seq_start"], args["resume"]
    args.update(x=rand(3, 16), out=rand(3, 16))
    check(lambda a: lq.conv_step(sh, stream=0, **a), args, ("x", "out"))


def test_binding_norm(host):
    sh = lq.NormShape(5, 3, 2, dim=64, rot=32)
    args = dict(q=rand(5, 3, 64), k=rand(5, 2, 64), out_q=rand(5, 3, 64), out_k=rand(5, 2, 64), w_q=rand(64, dtype=torch.float32),
                w_k=rand(64, dtype=torch.float32), positions=ints(5), inv_freq=rand(16, dtype=torch.float32))
    check(lambda a: lq.norm_rotate(sh, stream=0, **a), args, ("q", "k", "out_q", "out_k"))


@pytest.mark.parametrize("select", [0, 1])
def test_binding_scan(host, select):
    T, H, G = 4, 4, 2
    sh = lq.ScanShape(T, 4, H, G, max_len=4, n_slots=5, select=select)
    f32 = torch.float32
    args = dict(q=rand(T, G, 128), k=rand(T, G, 128), v=rand(T, H, 128), beta=rand(T, H), alpha=None if select else rand(T, H), o=rand(T, H, 128),
                S=rand(5, H, 128, 128, dtype=f32), seq_start=ints(5), slots=ints(4), resume=ints(4), A=rand(H, dtype=f32) if select else None,
                dt_bias=rand(H, dtype=f32), skip=rand(H, dtype=f32), S0=rand(5, H, 128, 128, dtype=f32))
    check(lambda a: lq.scan_prompt(sh, stream=0, **a), args, ("q", "k", "v", "beta", "o"))
    del args["seq_start"], args["resume"]
    args["o"] = rand(T, H, 128, dtype=f32)
    check(lambda a: lq.scan_step(sh, stream=0, **a), args, ("q", "k", "v", "beta", "o"))


# ---- counts near 2^31: row numbers up to a tile, sequence numbers up to a CTA and items up to a wave beyond the last are formed in 32 bits ----

MOST = 2 ** 31 - 1024


def scan(L, sh, step):
    w = (sh.heads_qk * 128, sh.heads_v * 128)
    io = lq._ScanIo(q=X, k=X, v=X, q_stride=w[0], k_stride=w[0], v_stride=w[1], beta=X, alpha=X, beta_stride=sh.heads_v, alpha_stride=sh.heads_v, S=STATE,
                    seq_start=STARTS)
    if step:
        return L.lq_scan_step(C.byref(sh.c()), C.byref(io), OUT, w[1], None)
    return L.lq_scan_prompt(C.byref(sh.c()), C.byref(io), OUT, w[1], TAPS, None)


@pytest.mark.parametrize("n", [MOST + 1, 2 ** 31 - 129, 2 ** 31 - 1])
def test_conv_counts_near_two_to_the_31(L, n):
    assert conv(L, lq.ConvShape(n, 4, 64, n_slots=4), False) == UNSUPPORTED
    assert conv(L, lq.ConvShape(40, n, 64, n_slots=4), False) == UNSUPPORTED
    assert conv(L, lq.ConvShape(n, n, 64, n_slots=4), True) == UNSUPPORTED


@pytest.mark.parametrize("seqs,heads", [(2 ** 31 - 1, 1), (2 ** 24 - 1, 128), (2 ** 23 + 1, 128)])
def test_scan_counts_near_two_to_the_31(L, seqs, heads):
    """Few rows in very many sequences: 2^30 heads at most."""
    sh = lq.ScanShape(8, seqs, heads, 1, max_len=8, n_slots=8)
    assert scan(L, sh, False) == UNSUPPORTED and L.lq_scan_prompt_bytes(C.byref(sh.c())) == 0
    assert scan(L, dataclasses.replace(sh, tokens=seqs), True) == UNSUPPORTED
    assert scan(L, lq.ScanShape(MOST + 1, 8, 1, 1, max_len=8, n_slots=8), False) == UNSUPPORTED
