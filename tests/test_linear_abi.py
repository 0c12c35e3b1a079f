"""CPU checks of the 8-bit linear layer's boundary: bad arguments are refused before anything is launched (no GPU is touched).

Addresses that are never looked at: arrays that are not meant to meet lie 2^40 bytes and more apart."""
import ctypes as C
import dataclasses

import pytest
import torch

from paper_2609_38166_b200 import build, lq

OK, NULL, SHAPE, ALIGN, UNSUPPORTED = 0, 1, 2, 3, 4
X, R, OUT, OUT8, SCALE, W = (i << 44 for i in range(1, 7))


@pytest.fixture(scope="module")
def L():
    build.build()
    return lq.lib()


def add(L, sh, x=X, xs=None, r=R, rs=None, w=W, out=OUT, outs=None, out8=OUT8, out8s=None, scale=SCALE, scales=None, no_io=False):
    d = lambda v: v if v is not None else sh.dim if sh else 0                     # noqa: E731
    io = lq._NormIo(x=x, x_stride=d(xs), residual=r, residual_stride=d(rs), w=w, out=out, out_stride=d(outs), out8=out8, out8_stride=d(out8s), scale=scale,
                    scale_stride=scales if scales is not None else sh.tokens if sh else 0)
    return L.lq_norm_add(C.byref(sh.c()) if sh else None, None if no_io else C.byref(io), None)


def gate(L, sh, o=X, os=None, z=R, zs=None, w=W, out=OUT, outs=None, out8=OUT8, out8s=None, scale=SCALE, scales=None, no_io=False):
    d = lambda v: v if v is not None else sh.heads * sh.dim if sh else 0          # noqa: E731
    io = lq._NormIo(x=o, x_stride=d(os), z=z, z_stride=d(zs), w=w, out=out, out_stride=d(outs), out8=out8, out8_stride=d(out8s), scale=scale,
                    scale_stride=scales if scales is not None else sh.tokens if sh else 0)
    return L.lq_norm_gate(C.byref(sh.c()) if sh else None, None if no_io else C.byref(io), None)


def product(L, sh, x=X, xs=None, s=SCALE, ss=None, w=W, ws=R, out=OUT, outs=None, start=None, groups=False, no_io=False):
    io = lq._ProductIo(x=x, x_stride=xs if xs is not None else sh.channels_in if sh else 0, x_scale=s, x_scale_stride=ss if ss is not None else sh.rows if sh else 0, w=w,
                       w_scale=ws, out=out, out_stride=outs if outs is not None else sh.channels_out if sh else 0, group_start=start)
    return (L.lq_product_groups if groups else L.lq_product)(C.byref(sh.c()) if sh else None, None if no_io else C.byref(io), None)


@pytest.mark.parametrize("call,sh", [(add, lq.AddShape(40, 256)), (gate, lq.GatedShape(40, 2, dim=128))], ids=["add", "gate"])
def test_norm_refusals(L, call, sh):
    rep = lambda **kw: dataclasses.replace(sh, **kw)                              # noqa: E731
    first, second = ("x", "r") if call is add else ("o", "z")
    assert call(L, None) == NULL and call(L, sh, no_io=True) == NULL
    for bad in (rep(tokens=-1), rep(dim=0), rep(dim=-1), rep(norm=-1), rep(norm=3), rep(type=-1), rep(type=3)):
        assert call(L, bad) == SHAPE, bad
    if call is add:
        assert call(L, rep(dim=16385)) == UNSUPPORTED and call(L, rep(tokens=2 ** 31 - 1)) == UNSUPPORTED
    else:
        for bad in (rep(heads=0), rep(silu=2), rep(silu=-1), rep(o_type=3), rep(o_type=-1)):
            assert call(L, bad) == SHAPE, bad
        for bad in (rep(dim=96), rep(dim=32), rep(dim=512), rep(heads=65537), rep(tokens=2 ** 31 - 1), rep(tokens=2 ** 25, heads=65536)):
            assert call(L, bad) == UNSUPPORTED, bad
        assert call(L, sh, z=None) == NULL
    assert call(L, sh, **{first: None}) == NULL
    assert call(L, sh, out=None, out8=None) == NULL and call(L, sh, scale=None) == NULL
    for kw in ({first: X + 1}, {second: R + 1}, dict(out=OUT + 1), dict(w=W + 2), dict(scale=SCALE + 2)):
        assert call(L, sh, **kw) == ALIGN, kw
    for kw in ({first + "s": 255}, {second + "s": 255}, dict(outs=255), dict(out8s=255), dict(scales=39)):
        assert call(L, sh, **kw) == SHAPE, kw
    row = 256 * (4 if call is gate else 2)                                        # of the first input
    for kw in (dict(out8=X), dict(out=X + 2), dict(out8=X + 39 * row + row - 1), dict(scale=X), dict(out=R), dict(out8=R), dict(scale=R + 512),     # an output over an input
               dict(out8=OUT), dict(out=OUT8), dict(scale=OUT), dict(scale=OUT8), dict(out8=OUT + 40 * 512 - 1), dict(scale=OUT8 - 2 * 40 * 4 + 4)):  # or another output
        assert call(L, sh, **kw) == UNSUPPORTED, kw
    if call is add:
        assert call(L, sh, r=X) == UNSUPPORTED and call(L, sh, out=X, outs=300) == UNSUPPORTED
    else:
        assert call(L, sh, out=X) == UNSUPPORTED and call(L, sh, out=R) == UNSUPPORTED
    assert call(L, rep(tokens=0)) == OK


def test_product_refusals(L):
    sh = lq.ProductShape(40, 256, 300)
    rep = lambda **kw: dataclasses.replace(sh, **kw)                              # noqa: E731
    for groups in (False, True):
        go = lambda of, **kw: product(L, of, groups=groups, **{"start": X << 4, **kw})   # noqa: E731
        assert go(None) == NULL and go(sh, no_io=True) == NULL
        for bad in (rep(rows=-1), rep(channels_in=0), rep(channels_out=0), rep(groups=0), rep(groups=-1), rep(type=3), rep(type=-1)):
            assert go(bad) == SHAPE, bad
        for bad in (rep(channels_in=250), rep(channels_in=8), rep(channels_in=2 ** 20 + 16), rep(channels_out=2 ** 20 + 1), rep(rows=2 ** 31 - 1),
                    rep(rows=2 ** 30, channels_out=2 ** 14), rep(channels_in=2 ** 20, channels_out=2 ** 20)):
            assert go(bad) == UNSUPPORTED, bad
        for kw in (dict(x=None), dict(s=None), dict(w=None), dict(ws=None), dict(out=None)):
            assert go(sh, **kw) == NULL, kw
        for kw in (dict(x=X + 8), dict(w=W + 8), dict(s=SCALE + 2), dict(ws=R + 2), dict(out=OUT + 1), dict(xs=264)):
            assert go(sh, **kw) == ALIGN, kw
        for kw in (dict(xs=240), dict(ss=39), dict(outs=299)):
            assert go(sh, **kw) == SHAPE, kw
        assert go(sh, xs=2 ** 36) == UNSUPPORTED and go(rep(rows=2 ** 20), xs=2 ** 20) == UNSUPPORTED
        for kw in (dict(out=X), dict(out=X + 40 * 256 - 2), dict(out=SCALE + 4), dict(out=W + 300 * 256 - 2), dict(out=R + 20), dict(out=X - 40 * 600 + 2)):
            assert go(sh, **kw) == UNSUPPORTED, kw
        assert go(rep(rows=0)) == OK
    assert product(L, rep(groups=2)) == SHAPE
    assert product(L, rep(groups=1025), groups=True, start=X << 4) == UNSUPPORTED
    assert product(L, sh, groups=True) == NULL and product(L, sh, groups=True, start=(X << 4) + 2) == ALIGN


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


def wrong(t):
    """Tensors that are not like t: another type, another shape, one row too few, another device, elements that are not neighbours."""
    yield t.double() if t.is_floating_point() else t.long()
    yield t[None]
    yield t[:-1] if t.shape[0] > 1 else torch.cat([t.float(), t.float()]).to(t.dtype)
    yield t.as_subclass(Elsewhere)
    yield torch.stack([t.float(), t.float()], -1).to(t.dtype)[..., 0]


def check(call, args, required):
    with pytest.raises(Called):
        call(args)
    for name, t in args.items():
        for bad in wrong(t):
            with pytest.raises(lq.LqError, match=rf"^{name}: "):
                call({**args, name: bad})
    for name in required:
        with pytest.raises(lq.LqError, match=rf"^{name}: missing"):
            call({**args, name: None})


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape).to(dtype)


def test_packed_arguments_are_the_structs(host):
    f32 = torch.float32
    assert lq._NORM_IO.size == C.sizeof(lq._NormIo) and lq._PRODUCT_IO.size == C.sizeof(lq._ProductIo)
    names = [n for n, _ in lq._NormIo._fields_]
    io = lq._NormIo.from_buffer_copy(lq._NORM_IO.pack(*range(1, 14)))
    assert [getattr(io, n) for n in names] == list(range(1, 14))
    names = [n for n, _ in lq._ProductIo._fields_]
    io = lq._ProductIo.from_buffer_copy(lq._PRODUCT_IO.pack(*range(1, 10)))
    assert [getattr(io, n) for n in names] == list(range(1, 10))
    x, r = zeros(5, 300), zeros(5, 320)[:, 10:310]
    out8, scale, w = zeros(5, 300, dtype=lq.E4M3), zeros(3, 8, dtype=f32)[:, :5], zeros(300, dtype=f32)
    got = lq._NormIo.from_buffer_copy(lq._norm_io(-1, lq._rows(x, "x", x.dtype, (5, 300), -1), lq._rows(r, "r", r.dtype, (5, 300), -1), (0, 0), w, (300,), None, out8, scale,
                                                  x.dtype, (5, 300), (3, 5)))
    assert (got.x, got.x_stride, got.residual, got.residual_stride, got.z, got.w) == (x.data_ptr(), 300, r.data_ptr(), 320, None, w.data_ptr())
    assert (got.out, got.out8, got.out8_stride, got.scale, got.scale_stride) == (None, out8.data_ptr(), 300, scale.data_ptr(), 8)


def test_binding_norms(host):
    f32 = torch.float32
    check(lambda a: lq.norm_add(lq.AddShape(5, 300), stream=0, **a),
          dict(x=zeros(5, 300), residual=zeros(5, 300), w=zeros(300, dtype=f32), out=zeros(5, 300), out8=zeros(5, 300, dtype=lq.E4M3), scale=zeros(3, 5, dtype=f32)), ("x",))
    check(lambda a: lq.norm_gate(lq.GatedShape(5, 3, dim=64), stream=0, **a),
          dict(o=zeros(5, 3, 64, dtype=f32), z=zeros(5, 3, 64), w=zeros(64, dtype=f32), out=zeros(5, 192), out8=zeros(5, 192, dtype=lq.E4M3), scale=zeros(2, 5, dtype=f32)),
          ("o", "z"))


def test_binding_products(host):
    f32 = torch.float32
    args = dict(x=zeros(5, 272, dtype=lq.E4M3), x_scale=zeros(3, 5, dtype=f32), w=zeros(130, 272, dtype=lq.E4M3), w_scale=zeros(2, 3, dtype=f32), out=zeros(5, 130))
    check(lambda a: lq.product(lq.ProductShape(5, 272, 130), stream=0, **a), args, ("x", "x_scale", "out"))
    args.update(w=zeros(4, 130, 272, dtype=lq.E4M3), w_scale=zeros(4, 2, 3, dtype=f32), group_start=torch.zeros(5, dtype=torch.int32))
    check(lambda a: lq.product_groups(lq.ProductShape(5, 272, 130, groups=4), stream=0, **a), args, ("x", "x_scale", "out"))
