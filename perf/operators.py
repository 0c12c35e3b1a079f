"""The operators around the decode step, as timed cases: what a prompt and a token go through before and beside it.

A layer with a recurrent state takes its projections through a short causal convolution (``conv_prompt`` for packed prompts,
``conv_step`` for one token of every request), normalises and rotates queries and keys per head (``norm_rotate``), and runs the
selective scan: over packed prompts (``scan_prompt``, whose dense states ``quantize_state`` takes over) or for one token on the
dense state (``scan_step``).  Head counts, channels and batches are those of this repository's benchmark (32 value heads over
16 query/key heads of 128 channels, 256 sequences: 2 * 16 * 128 + 32 * 128 = 8192 convolved channels) or generic ones of the
same kind.

``own`` false: elementary torch operations in 32 bits (64 for angles and sums of log decays), on any tree.
"""
import math
import random

import torch

own = False

D = 128                # channels of a head
BLOCK = 64             # tokens to a block of the plain scan
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

CONV = {"op": "conv_prompt", "seqs": 1, "tokens": 1, "channels": 8192, "pad": 0, "width": 4, "silu": True, "bias": True, "type": "bf16", "resume": 0.5}
NORM = {"op": "norm_rotate", "tokens": 256, "heads_q": 16, "heads_k": 16, "dim": 128, "rot": 0, "pairs": False, "norm": "l2", "pad": 0, "type": "bf16",
        "far": 65536}
SCAN = {"op": "scan_prompt", "seqs": 1, "tokens": 1, "heads_v": 32, "heads_qk": 16, "select": False, "gates": "bf16", "skip": False, "pad": 0, "resume": 0.0}


def listed():
    return [
        # one token of one request: the smallest call, where latency counts
        {**CONV, "name": "conv_step_1", "op": "conv_step", "seqs": 1, "tokens": 1},
        # one token of the benchmark batch, states in slots in no particular order
        {**CONV, "name": "conv_step_256", "op": "conv_step", "seqs": 256, "tokens": 256},
        # a few short prompts of odd sizes, one filter tap less, in 32 bits, channels that no vector width divides
        {**CONV, "name": "conv_prompt_odd", "seqs": 5, "tokens": 701, "channels": 1291, "width": 3, "type": "f32"},
        # long packed prompts, the channels a slice of a wider projection
        {**CONV, "name": "conv_prompt_32k", "seqs": 6, "tokens": 32768, "pad": 4096},
        # queries and keys of one token of the benchmark batch: unit length, no rotation (gated delta rule)
        {**NORM, "name": "norm_step_256"},
        # packed prompts at far positions: RMS norm with weights, half of the channels rotated, slices of a projection
        {**NORM, "name": "norm_rotate_16k", "tokens": 16384, "heads_q": 32, "heads_k": 8, "rot": 64, "norm": "rms", "pad": 1024, "far": 1 << 20},
        # every channel rotated in neighbouring pairs, no norm, odd counts, 32 bits
        {**NORM, "name": "rotate_odd", "tokens": 779, "heads_q": 7, "heads_k": 3, "rot": 128, "pairs": True, "norm": "none", "type": "f32"},
        # one token of a small batch on dense states, gates selected from dt
        {**SCAN, "name": "scan_step_4", "op": "scan_step", "seqs": 4, "tokens": 4, "select": True, "skip": True},
        # one token of the benchmark batch on dense states
        {**SCAN, "name": "scan_step_256", "op": "scan_step", "seqs": 256, "tokens": 256},
        # many short prompts, single tokens and empty ones among them
        {**SCAN, "name": "scan_prompt_64x120", "seqs": 64, "tokens": 64 * 120, "pad": 512},
        # one long prompt, gates selected from dt, few query/key groups: work has to be split along the prompt
        {**SCAN, "name": "scan_prompt_1x16k", "seqs": 1, "tokens": 16384, "heads_qk": 4, "select": True, "gates": "f32", "skip": True},
        # packed ragged prompts, half of them continuing earlier pieces
        {**SCAN, "name": "scan_prompt_12x2k", "seqs": 12, "tokens": 24000, "gates": "f32", "resume": 0.5},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["conv_prompt", "conv_step", "norm_rotate", "norm_rotate", "scan_prompt", "scan_prompt", "scan_step"])
    if op.startswith("conv"):
        c = _log(rng, 256, 8192)
        c = rng.choice([c, c // 8 * 8, c // 8 * 8])
        seqs = _log(rng, 1, 512 if op == "conv_step" else 64)
        tokens = seqs if op == "conv_step" else _log(rng, 1, 32768 * 8192 // max(c, 8192))
        return {**CONV, "op": op, "seqs": seqs, "tokens": tokens, "channels": c, "pad": rng.choice([0, 64, 1000]), "width": rng.choice([2, 3, 4, 4]),
                "silu": rng.random() < 0.8, "bias": rng.random() < 0.5, "type": rng.choice(["bf16", "bf16", "f16", "f32"]), "resume": rng.choice([0.0, 0.5, 1.0])}
    if op == "norm_rotate":
        hk = rng.randint(1, 16)
        dim = rng.choice([64, 128, 128, 256])
        rot = rng.choice([0, 32, dim // 2, dim])
        return {**NORM, "tokens": _log(rng, 1, 8192), "heads_q": rng.randint(1, 32), "heads_k": hk, "dim": dim, "rot": rot, "pairs": rng.random() < 0.4,
                "norm": rng.choice(["l2", "rms", "rms", "none"]), "pad": rng.choice([0, 64, 128]), "type": rng.choice(["bf16", "bf16", "f16", "f32"]),
                "far": _log(rng, 64, 1 << 20)}
    qk = rng.choice([1, 2, 3, 4, 5, 8, 16])
    heads = qk * rng.randint(1, 32 // qk)
    case = {**SCAN, "op": op, "heads_v": heads, "heads_qk": qk, "select": rng.random() < 0.5, "gates": rng.choice(["bf16", "f32"]), "skip": rng.random() < 0.5,
            "pad": rng.choice([0, 64, 512])}
    if op == "scan_step":
        seqs = _log(rng, 1, 256)
        return {**case, "seqs": seqs, "tokens": seqs}
    return {**case, "seqs": _log(rng, 1, 32), "tokens": _log(rng, 1, 16384), "resume": rng.choice([0.0, 0.5, 1.0])}


def _lengths(case):
    """The lengths of the packed sequences: uneven, empty ones and single tokens among them where there are many."""
    seqs, tokens = case["seqs"], case["tokens"]
    rng = random.Random(1000003 * seqs + tokens)
    share = [rng.uniform(0.2, 1.8) for _ in range(seqs)]
    lens = [int(tokens * s / sum(share)) for s in share]
    if seqs >= 8:
        lens[3], lens[5] = 0, min(1, lens[5])
    lens[rng.randrange(seqs)] += tokens - sum(lens)
    return lens


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    def strided(rows, cols, pad, dtype, make=None):
        """[rows, cols] as a slice of a wider buffer, as projections come."""
        x = (make or normal)(rows, cols)
        wide = torch.zeros((rows, cols + pad), dtype=dtype, device=dev)
        wide[:, pad // 2 // 8 * 8: pad // 2 // 8 * 8 + cols] = x
        return wide[:, pad // 2 // 8 * 8: pad // 2 // 8 * 8 + cols]

    op, s = case["op"], {"case": case}
    if op == "norm_rotate":
        dt, dim, tokens = TYPES[case["type"]], case["dim"], case["tokens"]
        for n in ("q", "k"):
            h = case["heads_" + n]
            s[n] = strided(tokens, h * dim, case["pad"], dt).unflatten(-1, (h, dim))
            s["w_" + n] = 1 + 0.2 * normal(dim) if case["norm"] == "rms" else None
            s["out_" + n] = torch.empty((tokens, h, dim), dtype=dt, device=dev)
        s["positions"] = s["inv_freq"] = None
        if case["rot"]:
            s["positions"] = torch.randint(0, case["far"], (tokens,), generator=g, device=dev, dtype=torch.int32)
            s["inv_freq"] = (10000.0 ** -(torch.arange(case["rot"] // 2, device=dev, dtype=torch.float64) * 2 / case["rot"])).float()
        return s
    seqs, tokens = case["seqs"], case["tokens"]
    slots = seqs + (3 if op.startswith("conv") else 0)
    s["n_slots"] = slots
    s["slots"] = torch.randperm(slots, generator=g, device=dev)[:seqs].to(torch.int32)
    if op.endswith("prompt"):
        lens = _lengths(case)
        s["max_len"], s["lens"] = max(lens), lens
        s["seq_start"] = torch.tensor([0] + lens, device=dev).cumsum(0).to(torch.int32)
        s["resume"] = (torch.rand((seqs,), generator=g, device=dev) < case["resume"]).to(torch.int32)
    if op.startswith("conv"):
        dt, c, w = TYPES[case["type"]], case["channels"], case["width"]
        s["x"] = strided(tokens, c, case["pad"], dt)
        s["w"] = (0.4 * normal(c, w)).to(dt)
        s["bias"] = (0.1 * normal(c)).to(dt) if case["bias"] else None
        s["state"] = normal(slots, w - 1, c).to(dt)
        s["out"] = torch.empty((tokens, c), dtype=dt, device=dev)
        return s
    hv, hq = case["heads_v"], case["heads_qk"]

    def unit(rows, cols):
        x = normal(rows, cols // D, D)
        return (x * torch.rsqrt((x * x).sum(-1, keepdim=True))).reshape(rows, cols)

    s["q"] = strided(tokens, hq * D, case["pad"], torch.bfloat16, unit).unflatten(-1, (hq, D))
    s["k"] = strided(tokens, hq * D, case["pad"], torch.bfloat16, unit).unflatten(-1, (hq, D))
    s["v"] = strided(tokens, hv * D, case["pad"], torch.bfloat16).unflatten(-1, (hv, D))
    gates = TYPES[case["gates"]]
    s["A"] = s["dt_bias"] = s["skip"] = s["alpha"] = None
    if case["select"]:                       # steps between 0.001 and 0.1, decay rates between 1 and 16
        step = torch.exp(torch.rand((hv,), generator=g, device=dev) * math.log(100.0) + math.log(0.001))
        s["dt_bias"] = step + torch.log(-torch.expm1(-step))
        s["A"] = -(1 + 15 * torch.rand((hv,), generator=g, device=dev))
        s["beta"] = normal(tokens, hv).to(gates)
    else:                                    # the gate distributions of the benchmark; every fourth head forgets slowly
        slow = torch.where(torch.arange(hv, device=dev) % 4 == 3, 0.02, 1.0)
        s["beta"] = torch.sigmoid(normal(tokens, hv)).to(gates)
        s["alpha"] = torch.exp(-slow * torch.nn.functional.softplus(normal(tokens, hv))).to(gates)
    if case["skip"]:
        s["skip"] = 1 + 0.3 * normal(hv)
    s["S"] = 0.3 * normal(slots, hv, D, D)
    s["o"] = torch.empty((tokens, hv, D), dtype=torch.bfloat16 if op == "scan_prompt" else torch.float32, device=dev)
    return s


# ---- plain forms ----

def _rows(s):
    """Sequence, its first row and its end, of every packed row."""
    start = s["seq_start"].long()
    seq = torch.repeat_interleave(torch.arange(s["case"]["seqs"], device=start.device), start[1:] - start[:-1], output_size=s["case"]["tokens"])
    return seq, start[seq], start[seq + 1]


def _conv_sum(taps, s):
    w = s["w"].float()
    y = sum(taps(i) * w[:, i] for i in range(w.shape[1]))
    y = y + s["bias"].float() if s["bias"] is not None else y
    y = y * (1 / (1 + torch.exp(-y))) if s["case"]["silu"] else y
    return y.to(s["x"].dtype)


def _plain_conv_prompt(s):
    x, state, h = s["x"], s["state"], s["case"]["width"] - 1
    seq, first, _ = _rows(s)
    slot, resume, start = s["slots"].long(), s["resume"] != 0, s["seq_start"].long()
    t = torch.arange(x.shape[0], device=x.device)
    old = torch.where(resume[:, None, None], state[slot], 0).float()             # [seqs, h, C]

    def tap(i):
        back = h - i
        inside = t - back >= first
        row = x[(t - back).clamp_min(0)].float()
        return torch.where(inside[:, None], row, old[seq, (i + t - first).clamp_max(h - 1)]) if back else row

    out = _conv_sum(tap, s)
    n = (start[1:] - start[:-1])[:, None]
    at = n + torch.arange(h, device=x.device)[None]                               # row of (old, x), h rows of old first
    src = torch.where((at < h)[..., None], old.gather(1, at.clamp_max(h - 1)[..., None].expand_as(old)), x[(start[:-1, None] + at - h).clamp(0, x.shape[0] - 1)].float())
    state[slot] = torch.where((n > 0)[..., None], src.to(state.dtype), state[slot])
    return {"out": out, "state": state}


def _plain_conv_step(s):
    slot = s["slots"].long()
    rows = torch.cat([s["state"][slot], s["x"][:, None]], 1)
    out = _conv_sum(lambda i: rows[:, i].float(), s)
    s["state"][slot] = rows[:, 1:]
    return {"out": out, "state": s["state"]}


def _plain_norm(s):
    case = s["case"]
    rot, scale = case["rot"], 1 / math.sqrt(case["dim"]) if case["norm"] == "rms" else 1.0
    if rot:
        angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def one(x, w, scale):
        y = x.float()
        if case["norm"] == "l2":
            y = y * torch.rsqrt((y * y).sum(-1, keepdim=True) + 1e-6)
        elif case["norm"] == "rms":
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w
        y = y * scale
        if rot:
            a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if case["pairs"] else (y[..., :rot // 2], y[..., rot // 2:rot])
            turned = (a * cos - b * sin, b * cos + a * sin)
            y = torch.cat([torch.stack(turned, -1).flatten(-2) if case["pairs"] else torch.cat(turned, -1), y[..., rot:]], -1)
        return y.to(x.dtype)

    return {"q": one(s["q"], s["w_q"], scale), "k": one(s["k"], s["w_k"], 1.0)}


def _gates(s, dtype=torch.float64):
    """(beta, log decay) of every token and head."""
    b = s["beta"].to(dtype)
    if not s["case"]["select"]:
        return b, torch.log(s["alpha"].to(dtype)).clamp_min(-800.0)
    x = b + s["dt_bias"]
    dt = x.clamp_min(0) + torch.log1p(torch.exp(-x.abs()))
    return dt, dt * s["A"]


def _plain_scan_prompt(s):
    case, dev = s["case"], s["q"].device
    hv, ratio, lens = case["heads_v"], case["heads_v"] // case["heads_qk"], s["lens"]
    nb = sum(-(-n // BLOCK) for n in lens)                                        # blocks of all sequences
    start = s["seq_start"].long()
    blocks = (start[1:] - start[:-1] + BLOCK - 1) // BLOCK
    seq = torch.repeat_interleave(torch.arange(case["seqs"], device=dev), blocks, output_size=nb)
    first = blocks.cumsum(0) - blocks                                             # a sequence's first block
    row = start[seq][:, None] + (torch.arange(nb, device=dev) - first[seq])[:, None] * BLOCK + torch.arange(BLOCK, device=dev)
    valid = row < start[seq + 1][:, None]
    row = row.clamp_max(case["tokens"] - 1)
    q, k, v = (x[row].float().transpose(1, 2) * valid[:, None, :, None] for x in (s["q"], s["k"], s["v"]))   # [nb, heads, BLOCK, D]
    beta, g = (x[row].transpose(1, 2) * valid[:, None] for x in _gates(s))        # [nb, hv, BLOCK], 64 bits
    cum = g.cumsum(-1)
    low = torch.ones((BLOCK, BLOCK), dtype=torch.bool, device=dev).tril()
    decay = torch.exp((cum[..., :, None] - cum[..., None, :]).masked_fill(~low, -1e4)).float()
    wide = lambda x: x.repeat_interleave(ratio, 1)                                # noqa: E731
    o = (wide(q @ k.transpose(-1, -2)) * decay * beta[..., None, :].float()) @ v
    total = cum[..., -1]
    local = wide(k).transpose(-1, -2) @ (v * (beta * torch.exp(total[..., None] - cum)).float()[..., None])   # [nb, hv, D, D]
    # states: what every block adds, decayed to where it is read
    upto = total.cumsum(0)                                                        # [nb, hv], over all sequences
    same = seq[:, None] == seq[None]
    order = torch.arange(nb, device=dev)
    before = same & (order[None] < order[:, None])
    old = torch.where((s["resume"] != 0)[:, None, None, None], s["S"][s["slots"].long()], 0)
    base = (upto - total)[first.clamp_max(nb - 1)]                                # [seqs, hv]
    into = torch.exp(((upto - total)[:, None] - upto[None]).masked_fill(~before[..., None], -1e4)).float()    # [block, source, hv]
    flat = local.flatten(-2).transpose(0, 1)                                      # [hv, nb, D*D]
    S_in = (into.permute(2, 0, 1) @ flat).transpose(0, 1).unflatten(-1, (D, D)) + torch.exp((upto - total) - base[seq]).float()[..., None, None] * old[seq]
    o = o + torch.exp(cum).float()[..., None] * (wide(q) @ S_in)
    if s["skip"] is not None:
        o = o + s["skip"][:, None, None] * v
    out = torch.zeros_like(s["o"])
    out[row[valid]] = o.transpose(1, 2)[valid].to(out.dtype)
    last = torch.where((blocks > 0)[:, None], upto[(first + blocks - 1).clamp(0, nb - 1)], 0)
    base = torch.where((blocks > 0)[:, None], base, 0)
    mine = torch.arange(case["seqs"], device=dev)[:, None] == seq[None]
    ends = torch.exp((last[:, None] - upto[None]).masked_fill(~mine[..., None], -1e4)).float()
    S = (ends.permute(2, 0, 1) @ flat).transpose(0, 1).unflatten(-1, (D, D)) + torch.exp(last - base).float()[..., None, None] * old
    state = s["S"].clone()
    state[s["slots"].long()] = S
    return {"o": out, "S": state}


def _plain_scan_step(s):
    ratio, slot = s["case"]["heads_v"] // s["case"]["heads_qk"], s["slots"].long()
    q, k = (s[n].float().repeat_interleave(ratio, 1) for n in ("q", "k"))
    v = s["v"].float()
    beta, g = _gates(s)
    S = torch.exp(g).float()[..., None, None] * s["S"][slot] + (beta.float()[..., None] * k)[..., None] * v[..., None, :]
    s["S"][slot] = S
    o = (S * q[..., None]).sum(-2)
    return {"o": o + s["skip"][:, None] * v if s["skip"] is not None else o, "S": s["S"]}


PLAIN = {"conv_prompt": _plain_conv_prompt, "conv_step": _plain_conv_step, "norm_rotate": _plain_norm, "scan_prompt": _plain_scan_prompt,
         "scan_step": _plain_scan_step}


# ---- the library's calls ----

def _own_shape(lq, s):
    case = s["case"]
    if case["op"].startswith("conv"):
        return lq.ConvShape(case["tokens"], case["seqs"], case["channels"], width=case["width"], n_slots=s["n_slots"], silu=int(case["silu"]),
                            type=lq.TYPES[s["x"].dtype])
    if case["op"] == "norm_rotate":
        rms = case["norm"] == "rms"
        return lq.NormShape(case["tokens"], case["heads_q"], case["heads_k"], dim=case["dim"], rot=case["rot"], pairs=int(case["pairs"]),
                            norm={"none": lq.NORM_NONE, "l2": lq.NORM_L2, "rms": lq.NORM_RMS}[case["norm"]], type=lq.TYPES[s["q"].dtype], eps=1e-6,
                            scale_q=1 / math.sqrt(case["dim"]) if rms else 1.0, scale_k=1.0)
    return lq.ScanShape(case["tokens"], case["seqs"], case["heads_v"], case["heads_qk"], max_len=s.get("max_len", 1), n_slots=s["n_slots"],
                        select=int(case["select"]), gate_type=lq.TYPES[s["beta"].dtype])


def _own(s):
    from paper_2609_38166_b200 import lq
    op = s["case"]["op"]
    sh = s.get("shape")
    if sh is None:                           # (what a program keeps between calls: the shape, the scan's workspace)
        sh = s["shape"] = _own_shape(lq, s)
        if op == "scan_prompt":
            s["work"] = torch.empty((lq.scan_prompt_bytes(sh),), dtype=torch.uint8, device="cuda")
            s["S_out"] = torch.empty_like(s["S"])
    if op == "conv_prompt":
        lq.conv_prompt(sh, s["x"], s["w"], s["bias"], s["state"], s["out"], s["seq_start"], slots=s["slots"], resume=s["resume"])
        return {"out": s["out"], "state": s["state"]}
    if op == "conv_step":
        lq.conv_step(sh, s["x"], s["w"], s["bias"], s["state"], s["out"], slots=s["slots"])
        return {"out": s["out"], "state": s["state"]}
    if op == "norm_rotate":
        lq.norm_rotate(sh, s["q"], s["k"], s["out_q"], s["out_k"], w_q=s["w_q"], w_k=s["w_k"], positions=s["positions"], inv_freq=s["inv_freq"])
        return {"q": s["out_q"], "k": s["out_k"]}
    gates = {"A": s["A"], "dt_bias": s["dt_bias"], "skip": s["skip"]}
    if op == "scan_prompt":
        lq.scan_prompt(sh, s["q"], s["k"], s["v"], s["beta"], s["alpha"], s["o"], s["S_out"], s["seq_start"], slots=s["slots"], resume=s["resume"], S0=s["S"],
                       work=s["work"], **gates)
        return {"o": s["o"], "S": s["S_out"]}
    lq.scan_step(sh, s["q"], s["k"], s["v"], s["beta"], s["alpha"], s["o"], s["S"], slots=s["slots"], **gates)
    return {"o": s["o"], "S": s["S"]}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    tokens = case["tokens"]
    if case["op"] == "norm_rotate":
        n = tokens * (case["heads_q"] + case["heads_k"]) * case["dim"]
        return {"bytes": 2 * n * size[case["type"]] + 4 * tokens * (case["rot"] > 0), "flops": 6 * n}
    if case["op"].startswith("conv"):
        c, b = case["channels"], size[case["type"]]
        old = 1.0 if case["op"] == "conv_step" else case["resume"]
        return {"bytes": b * c * (2 * tokens + (1 + old) * case["seqs"] * (case["width"] - 1) + case["width"] + case["bias"]),
                "flops": tokens * c * (2 * case["width"] + 5 * case["silu"])}
    hv, hq, step = case["heads_v"], case["heads_qk"], case["op"] == "scan_step"
    rows = tokens * D * (4 * hq + 2 * hv + (4 if step else 2) * hv) + tokens * hv * size[case["gates"]] * (1 if case["select"] else 2)
    states = 4 * case["seqs"] * hv * D * D * (1 + (1.0 if step else case["resume"]))
    return {"bytes": rows + states, "flops": 4 * tokens * hv * D * D}


# ---- the definitions, in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm_rotate":
        return _exact_norm(s)
    if case["op"].startswith("conv"):
        return _exact_conv(s)
    return _exact_scan(s)


def _exact_norm(s):
    case = s["case"]
    got = {}
    for n in ("q", "k"):
        y = s[n].double()
        if case["norm"] == "l2":
            y = y / torch.sqrt((y ** 2).sum(-1, keepdim=True) + 1e-6)
        if case["norm"] == "rms":
            y = y / torch.sqrt((y ** 2).mean(-1, keepdim=True) + 1e-6) * s["w_" + n].double()
        if case["norm"] == "rms" and n == "q":
            y = y / math.sqrt(case["dim"])
        if case["rot"]:                      # as a product with the unit complex number of the angle
            half = case["rot"] // 2
            i = torch.arange(half, device=y.device)
            a, b = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + half)
            angle = torch.outer(s["positions"].double(), s["inv_freq"].double())
            z = torch.complex(y[..., a], y[..., b]) * torch.polar(torch.ones_like(angle), angle)[:, None]
            y[..., a], y[..., b] = z.real, z.imag
        got[n] = y
    return got


def _exact_conv(s):
    """Sequence by sequence: the rows so far and the new ones in one array, and the sum over the taps."""
    case, x, w = s["case"], s["x"].double(), s["w"].double()
    h = case["width"] - 1
    state = s["state"].double()
    out = torch.zeros_like(x)
    starts = s["seq_start"].tolist() if case["op"] == "conv_prompt" else list(range(case["seqs"] + 1))
    slots = s["slots"].tolist()
    resume = s["resume"].tolist() if case["op"] == "conv_prompt" else [1] * case["seqs"]
    for n, slot in enumerate(slots):
        a, b = starts[n], starts[n + 1]
        if a == b:
            continue
        rows = torch.cat([state[slot] * (1.0 if resume[n] else 0.0), x[a:b]])
        y = torch.zeros_like(x[a:b])
        for i in range(case["width"]):
            y += rows[i:i + b - a] * w[:, i]
        if s["bias"] is not None:
            y += s["bias"].double()
        out[a:b] = y * torch.sigmoid(y) if case["silu"] else y
        state[slot] = rows[-h:]
    return {"out": out, "state": state}


def _exact_scan(s):
    """The recurrence, token by token, all sequences side by side."""
    case = s["case"]
    ratio, step = case["heads_v"] // case["heads_qk"], case["op"] == "scan_step"
    lens = [1] * case["seqs"] if step else s["lens"]
    # a token takes about ten launches and six trips over the states
    if max(lens) * (150e-6 + 6 * 8 * case["seqs"] * case["heads_v"] * D * D / 4e12) > 18:
        return None
    slot = s["slots"].long()
    q, k, v = s["q"], s["k"], s["v"].double()
    beta, g = _gates(s)
    alpha = torch.exp(g) if case["select"] else s["alpha"].double()
    state = s["S"].double()
    starts = list(range(case["seqs"])) if step else s["seq_start"].tolist()[:-1]
    order = sorted(range(case["seqs"]), key=lambda n: -lens[n])                   # the longest first: those that go on are the first rows
    at = torch.tensor([starts[n] for n in order], device=q.device)
    S = state[slot][order]
    if not step:
        S = S * (s["resume"][order] != 0).double()[:, None, None, None]
    o = torch.zeros((case["tokens"], case["heads_v"], D), dtype=torch.float64, device=q.device)
    for t in range(max(lens)):
        n = sum(x > t for x in lens) if case["seqs"] > 1 else 1
        r = at[:n] + t
        kt, qt, vt = k[r].double().repeat_interleave(ratio, 1), q[r].double().repeat_interleave(ratio, 1), v[r]
        S[:n].mul_(alpha[r][..., None, None])
        S[:n].addcmul_((beta[r][..., None] * kt)[..., None], vt[..., None, :])
        o[r] = (qt[..., None, :] @ S[:n])[..., 0, :]
    if s["skip"] is not None:
        o += s["skip"].double()[:, None] * v
    state[slot[order]] = S
    return {"o": o, "S": state}
