"""CPU checks of the operators on packed rows: bad arguments are refused before anything is launched (no GPU is touched)."""
import ctypes as C
import dataclasses

import pytest
import torch

from paper_2609_38166_b200 import build, lq

OK, NULL, SHAPE, ALIGN, UNSUPPORTED = 0, 1, 2, 3, 4
P = 0x100000                                   # an address that is never looked at


@pytest.fixture(scope="module")
def L():
    build.build()
    return lq.lib()


def conv(L, sh, x=P, xs=None, w=P, bias=None, state=P, out=P << 8, outs=None, start=P, slots=None, resume=None, step=False):
    s, xs, outs = C.byref(sh.c()) if sh else None, sh.channels if sh and xs is None else xs, sh.channels if sh and outs is None else outs
    if step:
        return L.lq_conv_step(s, x, xs or 0, w, bias, state, out, outs or 0, slots, None)
    return L.lq_conv_prompt(s, x, xs or 0, w, bias, state, out, outs or 0, start, slots, resume, None)


def test_conv_refusals(L):
    sh = lq.ConvShape(40, 4, 64, n_slots=4)
    rep = lambda **kw: dataclasses.replace(sh, **kw)                              # noqa: E731
    assert conv(L, None) == NULL
    for bad in (rep(tokens=-1), rep(seqs=-1), rep(channels=0), rep(width=0), rep(n_slots=-1), rep(silu=2), rep(type=3), rep(type=-1)):
        assert conv(L, bad) == SHAPE, bad
    for bad in (rep(width=1), rep(width=5), rep(channels=1 << 30)):
        assert conv(L, bad, outs=1 << 31) == UNSUPPORTED, bad
    assert conv(L, sh, xs=63) == SHAPE and conv(L, sh, outs=63) == SHAPE
    for kw in (dict(x=None), dict(w=None), dict(out=None), dict(start=None), dict(state=None, resume=P)):
        assert conv(L, sh, **kw) == NULL, kw
    for kw in (dict(x=P + 1), dict(w=P + 1), dict(out=P + 1), dict(bias=P + 1), dict(state=P + 1), dict(start=P + 2), dict(slots=P + 2), dict(resume=P + 2)):
        assert conv(L, sh, **kw) == ALIGN, kw
    # overlap: the same rows, a shifted view of them; slices of one buffer side by side are none
    assert conv(L, sh, out=P) == UNSUPPORTED and conv(L, sh, out=P + 2 * 64) == UNSUPPORTED
    assert conv(L, sh, xs=128, out=P + 2 * 63, outs=128) == UNSUPPORTED and conv(L, sh, xs=128, out=P - 2 * 63, outs=128) == UNSUPPORTED
    assert conv(L, sh, xs=128, out=P + 2 * 64, outs=192) == UNSUPPORTED
    # nothing to do is no error
    assert conv(L, rep(tokens=0)) == OK and conv(L, rep(seqs=0)) == OK
    one = rep(tokens=4)
    assert conv(L, rep(tokens=5), step=True) == SHAPE
    assert conv(L, one, state=None, step=True) == NULL
    assert conv(L, one, out=P, xs=128, outs=64, step=True) == UNSUPPORTED       # the same address with another stride
    assert conv(L, one, out=P + 2, step=True) == UNSUPPORTED


def norm(L, sh, q=P, qs=None, k=2 * P, ks=None, oq=3 * P, oqs=None, ok=4 * P, oks=None, wq=None, wk=None, pos=P, freq=P):
    s = C.byref(sh.c()) if sh else None
    d = lambda x, h: x if x is not None else (h * sh.dim if sh else 0)            # noqa: E731
    hq, hk = (sh.heads_q, sh.heads_k) if sh else (0, 0)
    return L.lq_norm_rotate(s, q, d(qs, hq), k, d(ks, hk), oq, d(oqs, hq), ok, d(oks, hk), wq, wk, pos, freq, None)


def test_norm_refusals(L):
    sh = lq.NormShape(10, 4, 2, rot=64)
    rep = lambda **kw: dataclasses.replace(sh, **kw)                              # noqa: E731
    assert norm(L, None) == NULL
    for bad in (rep(tokens=-1), rep(heads_q=-1), rep(heads_k=-1), rep(dim=0), rep(rot=-16), rep(rot=144), rep(norm=3), rep(norm=-1), rep(pairs=2), rep(type=7)):
        assert norm(L, bad) == SHAPE, bad
    for bad in (rep(dim=96, rot=0), rep(dim=512), rep(rot=8), rep(rot=72), rep(heads_q=1 << 16, heads_k=1)):
        assert norm(L, bad) == UNSUPPORTED, bad
    for kw in (dict(q=None), dict(k=None), dict(oq=None), dict(ok=None), dict(pos=None), dict(freq=None)):
        assert norm(L, sh, **kw) == NULL, kw
    for kw in (dict(q=P + 1), dict(ok=P + 1), dict(wq=P + 2), dict(wk=P + 1), dict(pos=P + 2), dict(freq=P + 1)):
        assert norm(L, sh, **kw) == ALIGN, kw
    for kw in (dict(qs=511), dict(ks=255), dict(oqs=511), dict(oks=255)):
        assert norm(L, sh, **kw) == SHAPE, kw
    # an output over the other input, over the other output, over its own input shifted
    for kw in (dict(oq=2 * P), dict(ok=P), dict(ok=3 * P), dict(oq=P + 2), dict(oq=P, oqs=1024)):
        assert norm(L, sh, **kw) == UNSUPPORTED, kw
    assert norm(L, rep(tokens=0)) == OK and norm(L, rep(heads_q=0, heads_k=0)) == OK


def scan(L, sh, o=P << 4, os=None, work=None, step=False, no_io=False, **kw):
    H, G = (sh.heads_v, sh.heads_qk) if sh else (1, 1)
    io = dict(q=P, k=P, v=P, q_stride=G * 128, k_stride=G * 128, v_stride=H * 128, beta=P, alpha=P, beta_stride=H, alpha_stride=H, A=None, dt_bias=None,
              skip=None, S0=None, S=P, seq_start=P, slots=None, resume=None)
    io.update(kw)
    f = L.lq_scan_step if step else L.lq_scan_prompt
    args = [C.byref(sh.c()) if sh else None, None if no_io else C.byref(lq._ScanIo(**io)), o, H * 128 if os is None else os]
    return f(*args, None) if step else f(*args, work, None)


@pytest.mark.parametrize("step", [False, True])
def test_scan_refusals(L, step):
    sh = lq.ScanShape(4, 4, 4, 2, max_len=4, n_slots=4)
    rep = lambda **kw: dataclasses.replace(sh, **kw)                              # noqa: E731
    go = lambda s, **kw: scan(L, s, step=step, **kw)                              # noqa: E731
    assert go(None) == NULL and go(sh, no_io=True) == NULL
    for bad in (rep(tokens=-1), rep(seqs=-1), rep(heads_v=0), rep(heads_qk=0), rep(heads_qk=3), rep(d_k=0), rep(d_v=-1), rep(n_slots=-1), rep(select=2)):
        assert go(bad) == SHAPE, bad
    assert go(rep(tokens=5) if step else rep(max_len=-1)) == SHAPE
    for bad in (rep(d_k=64), rep(d_v=256), rep(gate_type=lq.F16)):
        assert go(bad) == UNSUPPORTED, bad
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(beta=None), dict(alpha=None), dict(S=None), dict(o=None)):
        assert go(sh, **kw) == NULL, kw
    assert go(rep(select=1)) == NULL                                              # A is missing
    for kw in (dict(q=P + 2), dict(k=P + 8), dict(v=P + 4), dict(S=P + 4), dict(S0=P + 8), dict(beta=P + 1), dict(alpha=P + 1), dict(A=P + 2), dict(dt_bias=P + 1), dict(skip=P + 2),
               dict(slots=P + 2), dict(o=P + 1), dict(q_stride=260), dict(k_stride=257), dict(v_stride=513)):
        assert go(sh, **kw) == ALIGN, kw
    assert go(rep(gate_type=lq.F32), beta=P + 2) == ALIGN
    for kw in (dict(q_stride=248), dict(k_stride=0), dict(v_stride=504), dict(os=511), dict(beta_stride=3), dict(alpha_stride=3)):
        assert go(sh, **kw) == SHAPE, kw
    assert go(rep(seqs=0, tokens=0)) == OK
    if not step:
        assert go(sh, seq_start=None) == NULL and go(sh, resume=P + 1) == ALIGN


def test_binding_refuses_tensors_that_are_not_what_the_shape_says():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    sh = lq.ConvShape(4, 4, 64, n_slots=4)
    with pytest.raises((lq.LqError, AssertionError, RuntimeError)):
        lq.conv_step(sh, x, x, None, x, x)                                        # not on the device


@pytest.mark.parametrize("step", [False, True])
def test_scan_refuses_arrays_that_overlap(L, step):
    """Offsets in bytes: a state of 4 slots of 4 heads has 1 MB (2^20), four rows of o 4 KB (bf16) or 8 KB (fp32)."""
    sh = lq.ScanShape(4, 4, 4, 2, max_len=4, n_slots=4)
    at = dict(q=P, k=P + 0x10000, v=P + 0x20000, S=P + 0x100000)
    go = lambda **kw: scan(L, sh, step=step, **{**at, **kw})                      # noqa: E731
    row = 4 * 128 * (4 if step else 2)
    for kw in (dict(o=P), dict(o=P + 0x10000 + 16), dict(o=P + 0x20000), dict(o=P + 0x20000 - 4 * row + 16)):        # over q, k, v
        assert go(**kw) == UNSUPPORTED, kw
    for kw in (dict(o=P + 0x100000), dict(o=P + 0x200000 - 16), dict(o=P + 0x100000 - 4 * row + 16)):                # over S
        assert go(**kw) == UNSUPPORTED, kw
    for kw in (dict(q=P + 0x100000), dict(k=P + 0x200000 - 16), dict(v=P + 0x180000)):                               # S over an input
        assert go(**kw) == UNSUPPORTED, kw
    for kw in (dict(S0=P + 0x100000 + 16), dict(S0=P + 16), dict(S0=P + 0x200000 - 16), dict(S0=P << 3, o=P << 3)):   # S0 over S, o over S0
        assert go(**kw) == UNSUPPORTED, kw


def test_conv_refuses_a_state_that_overlaps(L):
    sh = lq.ConvShape(4, 4, 64, n_slots=4)                                        # a state of 1536 bytes, rows of 512
    for step in (False, True):
        for state in (P, P + 510, P - 1534, 2 * P, 2 * P + 510, 2 * P - 1534):
            assert conv(L, sh, x=P, out=2 * P, w=4 * P, state=state, step=step) == UNSUPPORTED, state

