"""The 8-bit linear layer around the decode step, as timed cases: what is between the residual stream and a layer with a recurrent state.

In front of the projections the residual is added and normalised (``norm_add``), behind the recurrence every head's output is
normalised and gated (``norm_gate``); both leave rows of e4m3 codes with a scale for each 128 channels.  The projections are products
of such rows with e4m3 weights that have a scale for each block of 128 x 128 (``product``), for experts with a weight for each group
of rows (``product_groups``).  32 value heads over 16 query/key heads of 128 channels are this repository's benchmark: the output has 4096
channels, and the projections of q, k, v, the output gate and two gates a head 2 * 2048 + 4096 + 4096 + 64 = 12352.

``own`` false: elementary torch operations in 32 bits, on any tree.  What is held in 8 bits is returned as torch's e4m3 type, the values
that the codes stand for in units of the block's scale, next to the scales.
"""
import math
import random

import torch

own = False

BLOCK = 128            # channels (and, of weights, outputs) to a scale
LARGEST = 448.0        # of e4m3
LEAST = 2.0 ** -100    # of a scale
E4M3 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

ADD = {"op": "norm_add", "tokens": 256, "dim": 4096, "norm": "rms", "residual": True, "eight": True, "pad": 0, "type": "bf16"}
GATE = {"op": "norm_gate", "tokens": 256, "heads": 32, "dim": 128, "norm": "rms", "gate": "silu", "eight": True, "pad": 0, "o": "f32", "type": "bf16"}
PRODUCT = {"op": "product", "rows": 256, "cin": 4096, "cout": 12352, "groups": 1, "type": "bf16"}


def listed():
    return [
        # one token of one request in front of the projections: the smallest call, where latency counts
        {**ADD, "name": "norm_add_1", "tokens": 1},
        # one token of the benchmark batch
        {**ADD, "name": "norm_add_256"},
        # packed prompts, the addend a slice of a wider buffer
        {**ADD, "name": "norm_add_16k", "tokens": 16384, "pad": 1024},
        # 32 bits and no 8-bit output, a number of channels that no vector width divides
        {**ADD, "name": "norm_add_odd", "tokens": 779, "dim": 1291, "eight": False, "type": "f32"},
        # outputs of the decode step (binary32) of the benchmark batch, the gate a slice of the projection
        {**GATE, "name": "norm_gate_256", "pad": 8256},
        # outputs of a prompt's scan
        {**GATE, "name": "norm_gate_16k", "tokens": 16384, "o": "bf16", "pad": 8256},
        # the output projection of one token: the weights are read and little else
        {**PRODUCT, "name": "product_1", "rows": 1, "cout": 4096},
        # the input projections of the benchmark batch
        {**PRODUCT, "name": "product_256"},
        # few channels, sizes that no tile divides
        {**PRODUCT, "name": "product_odd", "rows": 779, "cin": 1296, "cout": 1999, "type": "f16"},
        # the input projections of packed prompts
        {**PRODUCT, "name": "product_8k", "rows": 8192},
        # experts, one token of the benchmark batch, eight experts a token of 128
        {**PRODUCT, "name": "groups_2k", "op": "product_groups", "rows": 2048, "cin": 2048, "cout": 1536, "groups": 128},
        # experts, a prompt's rows over 64 of them, loads far apart
        {**PRODUCT, "name": "groups_16k", "op": "product_groups", "rows": 16384, "cin": 2048, "cout": 1536, "groups": 64},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["norm_add", "norm_add", "norm_gate", "norm_gate", "product", "product", "product", "product_groups", "product_groups"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "norm_add":
        dim = _log(rng, 256, 8192)
        dim = rng.choice([dim, dim // 8 * 8, dim // 128 * 128])
        return {**ADD, "tokens": _log(rng, 1, min(16384, 16384 * 2048 // dim)), "dim": dim, "norm": rng.choice(["rms", "rms", "l2", "none"]),
                "residual": rng.random() < 0.6, "eight": rng.random() < 0.6, "pad": rng.choice([0, 64, 1000]), "type": kind}
    if op == "norm_gate":
        dim = rng.choice([64, 128, 128, 256])
        heads = rng.randint(1, 4096 // dim)
        return {**GATE, "tokens": _log(rng, 1, 8192), "heads": heads, "dim": dim, "norm": rng.choice(["rms", "rms", "l2", "none"]),
                "gate": rng.choice(["silu", "sigmoid"]), "eight": rng.random() < 0.7, "pad": rng.choice([0, 64, 512]), "o": rng.choice(["f32", "bf16"]), "type": kind}
    if op == "product":
        cin, cout = _log(rng, 256, 8192) // 16 * 16, _log(rng, 64, 12352)
        return {**PRODUCT, "rows": _log(rng, 1, min(8192, 8192 * 4096 * 12352 // (cin * cout))), "cin": rng.choice([cin, max(128, cin // 128 * 128)]),
                "cout": rng.choice([cout, max(64, cout // 64 * 64)]), "type": kind}
    groups = rng.randint(2, 128)
    return {**PRODUCT, "op": op, "rows": _log(rng, 1, 16384), "cin": _log(rng, 256, 2048) // 16 * 16, "cout": rng.choice([_log(rng, 64, 2048), 512, 1536]),
            "groups": groups, "type": kind}


def _lengths(case):
    """Rows of every group: far from even, empty ones among them."""
    rows, groups = case["rows"], case["groups"]
    if case["op"] == "product":
        return [rows]
    rng = random.Random(1000003 * groups + rows)
    share = [math.exp(rng.gauss(0.0, 0.8)) for _ in range(groups)]
    share[rng.randrange(groups)] = 0.0
    lens = [int(rows * s / sum(share)) for s in share]
    for _ in range(rows - sum(lens)):
        lens[rng.choice([g for g in range(groups) if share[g] > 0.0])] += 1
    return lens


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    def strided(rows, cols, pad, dtype, scale=1.0):
        """[rows, cols] as a slice of a wider buffer, as projections come."""
        wide = torch.zeros((rows, cols + pad), dtype=dtype, device=dev)
        at = pad // 2 // 8 * 8
        wide[:, at:at + cols] = scale * normal(rows, cols)
        return wide[:, at:at + cols]

    s = {"case": case}
    dt = TYPES[case["type"]]
    if case["op"].startswith("norm"):
        tokens = case["tokens"]
        if case["op"] == "norm_add":
            width = case["dim"]
            s["x"] = strided(tokens, width, case["pad"], dt)
            s["residual"] = (3 * normal(tokens, width)).to(dt) if case["residual"] else None
        else:                                # (outputs of a recurrence are small, and some heads much smaller than others)
            width = case["heads"] * case["dim"]
            size = torch.exp(normal(1, case["heads"], 1) - 2)
            s["o"] = (size * normal(tokens, case["heads"], case["dim"])).to(TYPES[case["o"]])
            s["z"] = strided(tokens, width, case["pad"], dt, 2.0).unflatten(-1, (case["heads"], case["dim"]))
        s["w"] = 1 + 0.2 * normal(case["dim"]) if case["norm"] == "rms" else None
        if case["eight"]:
            s["out8"] = torch.empty((tokens, width), dtype=E4M3, device=dev)
            s["scale"] = torch.empty((-(-width // BLOCK), tokens), device=dev)
        else:
            s["out"] = torch.empty((tokens, width), dtype=dt, device=dev)
        return s
    rows, cin, cout, groups = case["rows"], case["cin"], case["cout"], case["groups"]
    blocks = -(-cin // BLOCK)
    # rows of a norm, some channels larger than others; weights as trained ones are kept
    x = normal(rows, cin) * torch.exp(0.5 * normal(cin))
    top = torch.nn.functional.pad(x, (0, blocks * BLOCK - cin)).unflatten(-1, (blocks, BLOCK)).abs().amax(-1)
    scale = top.clamp_min(LARGEST * LEAST) / LARGEST
    s["x"], s["x_scale"] = (x / scale.repeat_interleave(BLOCK, 1)[:, :cin]).clamp(-LARGEST, LARGEST).to(E4M3), scale.t().contiguous()
    s["w"] = torch.empty((groups, cout, cin), dtype=E4M3, device=dev)
    for k in range(groups):
        s["w"][k] = (110.0 * normal(cout, cin)).clamp(-LARGEST, LARGEST).to(E4M3)
    s["w_scale"] = torch.exp(0.3 * normal(groups, -(-cout // BLOCK), blocks)) / (110.0 * math.sqrt(cin))
    s["out"] = torch.empty((rows, cout), dtype=dt, device=dev)
    lens = _lengths(case)
    s["max_len"] = max(lens)
    if case["op"] == "product":
        s["w"], s["w_scale"] = s["w"][0], s["w_scale"][0]
    else:
        s["group_start"] = torch.tensor([0] + lens, device=dev).cumsum(0).to(torch.int32)
    return s


# ---- plain forms ----

def _rounded(s, y):
    """The outputs of a norm: of the case's type, or codes and scales."""
    tokens, width = y.shape
    if not s["case"]["eight"]:
        return {"out": y.to(TYPES[s["case"]["type"]])}
    blocks = -(-width // BLOCK)
    top = torch.nn.functional.pad(y, (0, blocks * BLOCK - width)).unflatten(-1, (blocks, BLOCK)).abs().amax(-1)
    scale = top.clamp_min(LARGEST * LEAST) / LARGEST
    code = (y / scale.repeat_interleave(BLOCK, 1)[:, :width]).clamp(-LARGEST, LARGEST).to(E4M3)
    return {"out8": code, "scale": scale.t().contiguous()}


def _normed(y, norm, w):
    if norm == "none":
        return y
    square = (y * y).sum(-1, keepdim=True)
    return y * torch.rsqrt(square + 1e-6) if norm == "l2" else y * torch.rsqrt(square / y.shape[-1] + 1e-6) * w


def _plain_norm_add(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
        s["residual"].copy_(h)
    got = _rounded(s, _normed(h, s["case"]["norm"], s["w"]))
    return {**got, "residual": s["residual"]}


def _plain_norm_gate(s):
    z = s["z"].float()
    gate = 1 / (1 + torch.exp(-z))
    y = _normed(s["o"].float(), s["case"]["norm"], s["w"]) * (z * gate if s["case"]["gate"] == "silu" else gate)
    return _rounded(s, y.flatten(1))


def _wide(w, scale):
    """Weights in 32 bits."""
    cout, cin = w.shape[-2:]
    return w.float() * scale.repeat_interleave(BLOCK, -2)[..., :cout, :].repeat_interleave(BLOCK, -1)[..., :cin]


def _plain_product(s):
    x = s["x"].float() * s["x_scale"].t().repeat_interleave(BLOCK, 1)[:, :s["case"]["cin"]]
    w = _wide(s["w"], s["w_scale"])
    dt = TYPES[s["case"]["type"]]
    if s["case"]["op"] == "product":
        return {"out": (x @ w.t()).to(dt)}
    # every group's rows behind zeros up to the longest group's length, all groups in one product
    start = s["group_start"].long()
    row = start[:-1, None] + torch.arange(s["max_len"], device=x.device)
    there = row < start[1:, None]
    y = (x[row.clamp_max(x.shape[0] - 1)] * there[..., None]) @ w.transpose(1, 2)
    out = torch.empty((x.shape[0], w.shape[1]), dtype=dt, device=x.device)
    out[row[there]] = y[there].to(dt)
    return {"out": out}


PLAIN = {"norm_add": _plain_norm_add, "norm_gate": _plain_norm_gate, "product": _plain_product, "product_groups": _plain_product}


# ---- the library's calls ----

def _own_shape(lq, case):
    kind = lq.TYPES[TYPES[case["type"]]]
    if case["op"].startswith("product"):
        return lq.ProductShape(case["rows"], case["cin"], case["cout"], groups=case["groups"], type=kind)
    norm = {"none": lq.NORM_NONE, "l2": lq.NORM_L2, "rms": lq.NORM_RMS}[case["norm"]]
    if case["op"] == "norm_add":
        return lq.AddShape(case["tokens"], case["dim"], norm=norm, type=kind, eps=1e-6)
    return lq.GatedShape(case["tokens"], case["heads"], dim=case["dim"], norm=norm, silu=int(case["gate"] == "silu"), o_type=lq.TYPES[TYPES[case["o"]]],
                         type=kind, eps=1e-6)


def _own(s):
    from paper_2609_38166_b200 import lq
    case = s["case"]
    sh = s.get("shape")
    if sh is None:                           # (a program keeps it between calls)
        sh = s["shape"] = _own_shape(lq, case)
    if case["op"] == "product":
        lq.product(sh, s["x"], s["x_scale"], s["w"], s["w_scale"], s["out"])
        return {"out": s["out"]}
    if case["op"] == "product_groups":
        lq.product_groups(sh, s["x"], s["x_scale"], s["w"], s["w_scale"], s["out"], s["group_start"])
        return {"out": s["out"]}
    outs = {n: s[n] for n in ("out", "out8", "scale") if n in s}
    if case["op"] == "norm_add":
        lq.norm_add(sh, s["x"], residual=s["residual"], w=s["w"], **outs)
        return {**outs, "residual": s["residual"]}
    lq.norm_gate(sh, s["o"], s["z"], w=s["w"], **outs)
    return outs


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    if case["op"].startswith("norm"):
        width = case["dim"] * case.get("heads", 1)
        into = size[case["type"]] * (1 + 2 * case["residual"]) if case["op"] == "norm_add" else size[case["type"]] + size[case["o"]]
        out = 1 + 4 / BLOCK if case["eight"] else size[case["type"]]
        return {"bytes": case["tokens"] * width * (into + out), "flops": 8 * case["tokens"] * width}
    rows, cin, cout = case["rows"], case["cin"], case["cout"]
    live = sum(n > 0 for n in _lengths(case))
    return {"bytes": rows * cin * (1 + 4 / BLOCK) + live * cin * cout * (1 + 4 / BLOCK ** 2) + rows * cout * size[case["type"]], "flops": 2 * rows * cin * cout}


# ---- the definitions, in 64 bits ----

def _exact_out(case, y):
    if not case["eight"]:
        return {"out": y}
    tokens, width = y.shape
    code, scale = torch.empty_like(y), []
    for at in range(0, width, BLOCK):        # (in front of the rounding to 8 bits)
        part = y[:, at:at + BLOCK]
        scale.append(part.abs().max(1).values.clamp(min=LARGEST * LEAST) / LARGEST)
        code[:, at:at + BLOCK] = part / scale[-1][:, None]
    return {"out8": code, "scale": torch.stack(scale)}


def _exact_norm(x, norm, w):
    if norm == "l2":
        return x / torch.sqrt(torch.linalg.vecdot(x, x)[..., None] + 1e-6)
    if norm == "rms":
        return x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6) * w.double()
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm_add":
        h = s["x"].double() + (s["residual"].double() if case["residual"] else 0.0)
        return {**_exact_out(case, _exact_norm(h, case["norm"], s["w"])), "residual": h if case["residual"] else None}
    if case["op"] == "norm_gate":
        z = s["z"].double()
        y = _exact_norm(s["o"].double(), case["norm"], s["w"]) * torch.sigmoid(z) * (z if case["gate"] == "silu" else 1.0)
        return _exact_out(case, y.reshape(case["tokens"], -1))
    # group by group, and block by block of channels with the scales behind the sums
    out = torch.zeros((case["rows"], case["cout"]), dtype=torch.float64, device=s["x"].device)
    weights, scales = s["w"].reshape(-1, case["cout"], case["cin"]), s["w_scale"].reshape(case["groups"], -1, s["w_scale"].shape[-1])
    at = 0
    for g, n in enumerate(_lengths(case)):
        x, sx = s["x"][at:at + n].double(), s["x_scale"][:, at:at + n].double()
        for b in range(sx.shape[0] if n else 0):
            k = slice(b * BLOCK, (b + 1) * BLOCK)
            of_out = scales[g, :, b].double().repeat_interleave(BLOCK)[:case["cout"]]
            out[at:at + n] += sx[b][:, None] * of_out * (x[:, k] @ weights[g, :, k].double().t())
        at += n
    return {"out": out}
