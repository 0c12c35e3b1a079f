"""The operators on packed rows from their definitions, in 64 bits on the CPU, and how far binary32 and a result's type may be off.

Every function returns (value, scale): ``scale`` is the same sum over the magnitudes of its terms, which is what rounding errors
of the sum are relative to.
"""
import torch


def half_step(dtype) -> float:
    """A rounding to ``dtype`` is off by at most this, relative to the value."""
    return torch.finfo(dtype).eps / 2


def conv(x, w, bias, state, starts, slots, resume, silu):
    """(out, scale, state) with NaN in rows of no sequence; state rows move bit by bit."""
    T, C = x.shape
    W = w.shape[1]
    out, scale = torch.full((T, C), float("nan"), dtype=torch.float64), torch.ones((T, C), dtype=torch.float64)
    state = state.clone() if state is not None else None
    for n in range(len(starts) - 1):
        a, b = starts[n], starts[n + 1]
        slot = slots[n] if slots is not None else n
        if a == b or slot < 0 or (state is not None and slot >= state.shape[0]):
            continue
        old = state[slot] if resume is not None and resume[n] else torch.zeros((W - 1, C), dtype=x.dtype)
        rows = torch.cat([old, x[a:b]])
        y, s = torch.zeros((b - a, C), dtype=torch.float64), torch.zeros((b - a, C), dtype=torch.float64)
        for i in range(W):
            term = rows[i:i + b - a].double() * w[:, i].double()
            y, s = y + term, s + term.abs()
        if bias is not None:
            y, s = y + bias.double(), s + bias.double().abs()
        out[a:b], scale[a:b] = y * torch.sigmoid(y) if silu else y, s
        if state is not None:
            state[slot] = rows[rows.shape[0] - (W - 1):]
    return out, scale, state


def norm_rotate(x, w, norm, eps, scale, positions, inv_freq, pairs):
    """(y, size of the pair that an element is in)"""
    y = x.double()
    if norm == 1:
        y = y / torch.sqrt((y ** 2).sum(-1, keepdim=True) + eps)
    elif norm == 2:
        y = y / torch.sqrt((y ** 2).mean(-1, keepdim=True) + eps)
        y = y * w.double() if w is not None else y
    y = y * scale
    size = y.abs()
    if inv_freq is not None and inv_freq.numel():
        half = inv_freq.numel()
        i = torch.arange(half)
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
        z = torch.complex(y[..., a], y[..., b])
        angle = positions.double()[:, None] * inv_freq.double()
        z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
        y[..., a], y[..., b] = z.real, z.imag
        size[..., a] = size[..., b] = z.abs()
    return y, size


def gates(beta, alpha, A, dt_bias):
    """(beta, alpha) of the recurrence from what a call is given"""
    if A is None:
        return beta.double(), alpha.double()
    dt = torch.nn.functional.softplus(beta.double() + (dt_bias.double() if dt_bias is not None else 0.0), threshold=1e6)
    return dt, torch.exp(dt * A.double())


def scan(q, k, v, beta, alpha, S, starts, slots, resume, A=None, dt_bias=None, skip=None):
    """(o, scale of o, S, scale of S): the recurrence token by token; NaN in rows of no sequence."""
    T, H = v.shape[:2]
    ratio = H // q.shape[1]
    b, a = gates(beta, alpha, A, dt_bias)
    q, k, v = (x.double() for x in (q.repeat_interleave(ratio, 1), k.repeat_interleave(ratio, 1), v))
    o, so = torch.full(v.shape, float("nan"), dtype=torch.float64), torch.ones(v.shape, dtype=torch.float64)
    S, sS = S.double().clone(), S.double().abs()
    for n in range(len(starts) - 1):
        slot = slots[n] if slots is not None else n
        if slot < 0 or slot >= S.shape[0]:
            continue
        X = S[slot] if resume is None or resume[n] else torch.zeros_like(S[slot])
        Y = X.abs()
        for t in range(starts[n], starts[n + 1]):
            add = b[t][:, None, None] * k[t][..., None] * v[t][:, None, :]
            X, Y = a[t][:, None, None] * X + add, a[t][:, None, None] * Y + add.abs()
            o[t] = (q[t][:, None, :] @ X)[:, 0]
            so[t] = (q[t].abs()[:, None, :] @ Y)[:, 0]
            if skip is not None:
                o[t] += skip.double()[:, None] * v[t]
                so[t] += (skip.double()[:, None] * v[t]).abs()
        S[slot], sS[slot] = X, Y
    return o, so, S, sS
