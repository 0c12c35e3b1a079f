"""The 8-bit linear layer from its definitions, in 64 bits on the CPU."""
import torch

BLOCK, TOP, LEAST = 128, 448.0, 2.0 ** -100
E4M3 = torch.float8_e4m3fn
# one rounding to the type, relative; below the smallest normal number, absolute
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24, E4M3: 2.0 ** -4}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150, E4M3: 2.0 ** -10}


def norm(x, kind, w, eps):
    if kind == 1:
        return x / torch.sqrt((x * x).sum(-1, keepdim=True) + eps)
    if kind == 2:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        return x * w.double() if w is not None else x
    return x


def scales(y):
    """[blocks, rows]"""
    n = -(-y.shape[1] // BLOCK)
    wide = torch.nn.functional.pad(y, (0, n * BLOCK - y.shape[1]))
    return (wide.reshape(y.shape[0], n, BLOCK).abs().amax(-1).clamp_min(TOP * LEAST) / TOP).t()


def spread(scale, channels):
    """[blocks, rows] as a factor of every element, [rows, channels]"""
    return scale.t().repeat_interleave(BLOCK, 1)[:, :channels]


def quantize(y):
    """(codes, scales) of rows in binary32"""
    s = scales(y.double()).float().contiguous()
    return (y / spread(s, y.shape[1])).clamp(-TOP, TOP).to(E4M3), s


def weights(w, scale):
    return w.double() * scale.double().repeat_interleave(BLOCK, -2)[..., :w.shape[-2], :].repeat_interleave(BLOCK, -1)[..., :w.shape[-1]]


def product(x, x_scale, w, w_scale, starts=None):
    """(out, the same sum over magnitudes); NaN in rows of no group.  w [groups, out, in]"""
    a = x.double() * spread(x_scale.double(), x.shape[1])
    b = weights(w, w_scale)
    out = torch.full((x.shape[0], w.shape[1]), float("nan"), dtype=torch.float64)
    size = torch.ones_like(out)
    starts = starts if starts is not None else [0, x.shape[0]]
    for g in range(len(starts) - 1):
        r = slice(starts[g], starts[g + 1])
        out[r], size[r] = a[r] @ b[g].t(), a[r].abs() @ b[g].abs().t()
    return out, size


def off(got, want, dtype, slack):
    """The largest error in units of its bound: a rounding to the type and `slack` in front of it."""
    d = (got.double() - want).abs() / (HALF[dtype] * want.abs() + slack * (1 + HALF[dtype]) + TINY[dtype])
    return float(d.max()) if d.numel() else 0.0
