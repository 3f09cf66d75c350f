"""What the operators that fit laws are timed on: code lengths of symbols under logits, their gradient,
layer norm, and the AdamW step that moves the weights.

A program that learns the laws its coder works under runs these per training step; one that only asks
what a stream would cost runs the first of them.  `listed` holds one case for each use, `draw` takes
further ones from the same ranges.  `run` is the plain form in 32 bits, or with `own` the framework.

Lengths are in nats.  Everywhere below, a negative target is one that does not count, and a row whose
logits are all -inf has no law: its log probabilities are -inf, its entropy and gradient 0.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TARGETS = {"u8": torch.uint8, "i32": torch.int32, "i64": torch.int64}

# AdamW as every case runs it
LR, BETA1, BETA2, EPS, DECAY, STEP = 3e-4, 0.9, 0.999, 1e-8, 0.1, 1000
BLOCK = 256          # values that share a scale where states are held in 8 bits


def _logits(name, op, rows, vocab, pad, dtype, target, top, masked):
    """masked: share of the logits that are -inf; with it one row in 97 is empty and one target in 13 does not count."""
    return {"name": name, "op": op, "rows": rows, "vocab": vocab, "pad": pad, "dtype": dtype, "target": target,
            "top": top, "masked": masked}


def _norm(name, op, rows, width, pad, dtype, weight):
    return {"name": name, "op": op, "rows": rows, "width": width, "pad": pad, "dtype": dtype, "weight": weight}


def _adamw(name, tensors, values, param, grad, bits, apart):
    """tensors of sizes spread around values / tensors; apart: values between the end of one and a multiple of 256 at
    which the next begins are left out of it (as in a bucket), or with `apart` 0 the tensors follow one another at once."""
    return {"name": name, "op": "adamw", "tensors": tensors, "values": values, "param": param, "grad": grad,
            "bits": bits, "apart": apart}


def listed():
    return [
        # one row at a time while a stream is decoded: what the next symbol costs, and what else it might have been
        _logits("one_row", "logprobs", 1, 131072, 0, "bf16", "i64", 20, 0.0),
        # the length of an index stream under its predicted laws: 256 images of 16 x 16 indices out of 256
        _logits("index_lengths", "logprobs", 65536, 256, 0, "f32", "u8", 0, 0.0),
        # scoring long streams over a large alphabet whose size divides by nothing, rows padded, some symbols ruled out
        _logits("scoring", "logprobs", 4093, 100003, 29, "bf16", "i64", 5, 0.02),
        # the gradient by itself, from the log sums that the forward pass left, with an entropy term
        _logits("gradient", "grad", 8190, 50001, 7, "f16", "i32", 0, 0.02),
        # the loss of a training step and its gradient in one call: a small and a large alphabet
        _logits("index_training", "train", 65536, 256, 0, "bf16", "u8", 0, 0.0),
        _logits("training", "train", 16384, 65536, 0, "bf16", "i64", 0, 0.0),
        # the norm before the head: a few rows, and a whole batch
        _norm("norm_few_rows", "norm_forward", 16, 4096, 0, "bf16", "bf16"),
        _norm("norm_batch", "norm_forward", 16384, 8192, 0, "bf16", "f32"),
        _norm("norm_backward", "norm_backward", 32768, 4096, 0, "bf16", "bf16"),
        # a small network's tensors in one step: launches and latency only
        _adamw("adamw_small", 24, 200000, "f32", "f32", 32, 0),
        # a large network's: weights and states in 32 bits, and weights in 16 with states in 8
        _adamw("adamw_large", 291, 150000000, "f32", "f32", 32, 256),
        _adamw("adamw_bytes", 291, 300000000, "bf16", "bf16", 8, 256),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["logprobs", "logprobs", "grad", "train", "norm_forward", "norm_backward", "adamw", "adamw"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind in ("logprobs", "grad", "train"):
        vocab = _spread(rng, 2, 200000)
        rows = max(1, min(_spread(rng, 1, 65536), 500_000_000 // vocab))
        target = rng.choice(["u8", "i32", "i64"]) if vocab >= 256 else rng.choice(["i32", "i64"])
        c = _logits("", kind, rows, vocab, rng.choice([0, 0, rng.randrange(1, 64)]), dtype, target,
                    rng.choice([0, 1, 5, 20, 32]) if kind == "logprobs" else 0, rng.choice([0.0, 0.02, 0.3]))
    elif kind.startswith("norm"):
        width = _spread(rng, 8, 20000)
        rows = max(1, min(_spread(rng, 1, 100000), 250_000_000 // width))
        c = _norm("", kind, rows, width, rng.choice([0, 0, rng.randrange(1, 64)]), dtype, rng.choice([dtype, "f32"]))
    else:
        tensors = _spread(rng, 1, 600)
        values = max(tensors, _spread(rng, 1000, 100_000_000))
        bits = rng.choice([8, 32])
        param = rng.choice(["f32", "bf16", "f16"])
        c = _adamw("", tensors, values, param, rng.choice([param, "f32", "bf16"]), bits, 256 if bits == 8 else rng.choice([0, 256]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ inputs
def _sizes(case):
    """(begins, counts, values in all): the tensors' places in one flat buffer, from the case alone."""
    rng = random.Random(case["tensors"] * 1000003 + case["values"])
    share = [math.exp(rng.gauss(0.0, 1.5)) for _ in range(case["tensors"])]
    scale = max(1, case["values"] - case["tensors"]) / sum(share)
    counts = [1 + int(s * scale) for s in share]
    apart = case["apart"] or 1
    begins, at = [], 0
    for n in counts:
        begins.append(at)
        at = -(-(at + n) // apart) * apart
    return begins, counts, at


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device=DEVICE, dtype=dtype) * scale)


def _prepare_logits(case, g):
    rows, vocab, dtype = case["rows"], case["vocab"], TYPES[case["dtype"]]
    whole = torch.randn(rows, vocab + case["pad"], generator=g, device=DEVICE, dtype=dtype)
    whole.mul_(2.5)
    logits = whole[:, :vocab]
    target = torch.randint(0, min(vocab, 256) if case["target"] == "u8" else vocab, (rows,), generator=g, device=DEVICE)
    # a law that has been learned puts most of its mass on a few symbols, the given one often among them
    logits[torch.arange(rows, device=DEVICE), target] += (6.0 * torch.rand(rows, generator=g, device=DEVICE)).to(dtype)
    if case["masked"]:
        step = max(1, 2_000_000_000 // 8 // max(1, rows * vocab))   # the same columns are ruled out in groups of rows
        cols = torch.rand(min(rows, 64 * step), vocab, generator=g, device=DEVICE) < case["masked"]
        for a in range(0, rows, cols.shape[0]):
            b = min(rows, a + cols.shape[0])
            logits[a:b].masked_fill_(cols[: b - a], -math.inf)
        logits[96::97] = -math.inf
        if case["target"] != "u8":
            target[12::13] = -1
    whole[:, vocab:] = math.nan            # what lies between rows is nobody's
    each = (16384.0 if dtype == torch.float16 else 1.0) / rows      # a mean; gradients in f16 are scaled to stay in its range
    s = {"logits": logits, "target": target.to(TARGETS[case["target"]]), "up_logp": -each * torch.rand(rows, generator=g, device=DEVICE),
         "up_entropy": 0.1 * each * torch.rand(rows, generator=g, device=DEVICE)}
    f32 = dict(dtype=torch.float32, device=DEVICE)
    if case["op"] == "grad":
        top = logits.float().amax(1)
        z = logits.float() - torch.where(top == -math.inf, 0.0, top)[:, None]
        e = z.exp()
        total = e.sum(1)
        s["lse"] = top + total.log()
        s["lse"][top == -math.inf] = -math.inf
        s["entropy"] = torch.where(total > 0, total.log() - (e * z).nan_to_num(0.0, 0.0, 0.0).sum(1) / total, 0.0)
    else:
        s["lse"], s["entropy"], s["logp"] = (torch.empty(rows, **f32) for _ in range(3))
    if case["op"] == "logprobs":
        s["top_sym"] = torch.empty(rows, case["top"], dtype=torch.int32, device=DEVICE)
        s["top_logp"] = torch.empty(rows, case["top"], **f32)
    else:
        s["grad"] = torch.empty(rows, vocab, dtype=dtype, device=DEVICE)
    return s


def _prepare_norm(case, g):
    rows, width, dtype, wtype = case["rows"], case["width"], TYPES[case["dtype"]], TYPES[case["weight"]]
    made = lambda *shape, t=dtype: torch.empty(*shape, dtype=t, device=DEVICE)  # noqa: E731
    x = torch.randn(rows, width + case["pad"], generator=g, device=DEVICE, dtype=dtype)[:, :width]
    x.mul_(1.5)
    x.add_(_randn(g, rows, 1).to(dtype))
    s = {"x": x, "weight": (1 + _randn(g, width, scale=0.2)).to(wtype), "bias": _randn(g, width, scale=0.2).to(wtype),
         "eps": 1e-5}
    if case["op"] == "norm_forward":
        s.update(y=made(rows, width), mean=made(rows, t=torch.float32), rstd=made(rows, t=torch.float32))
    else:
        f = x.float()
        mean = f.mean(1)
        var = (f - mean[:, None]).square().mean(1)
        s.update(dy=torch.randn(rows, width + case["pad"], generator=g, device=DEVICE, dtype=dtype)[:, :width],
                 mean=mean, rstd=1 / torch.sqrt(var + 1e-5), dx=made(rows, width), dweight=made(width, t=wtype), dbias=made(width, t=wtype))
    return s


def _prepare_adamw(case, g):
    begins, counts, total = _sizes(case)
    s = {"begins": begins, "counts": counts, "step": STEP, "decayed": begins[len(begins) // 2]}
    flat = {"param": _randn(g, total, scale=0.02).to(TYPES[case["param"]]),
            "grad": _randn(g, total, scale=1e-3).to(TYPES[case["grad"]])}
    m, v = _randn(g, total, scale=1e-4), _randn(g, total, scale=1e-3).square()
    if case["apart"]:                      # nothing lies between the tensors of a bucket
        inside = torch.zeros(total + 1, dtype=torch.int32, device=DEVICE)
        inside[torch.tensor(begins, device=DEVICE)] += 1
        inside[torch.tensor([b + n for b, n in zip(begins, counts)], device=DEVICE)] -= 1
        inside = inside.cumsum(0)[:total] > 0
        for t in (flat["param"], flat["grad"], m, v):
            t.masked_fill_(~inside, 0)
    if case["bits"] == 32:
        flat["m"], flat["v"] = m, v
    else:
        none = torch.zeros(total, dtype=torch.int64, device=DEVICE)
        flat["m"], flat["m_scale"] = _pack(m, none, 15, True)
        flat["v"], flat["v_scale"] = _pack(v, none, 31, False)
        flat["m_values"], flat["v_values"] = torch.empty_like(m), torch.empty_like(v)
    s["flat"] = flat
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    if case["op"] in ("logprobs", "grad", "train"):
        s = _prepare_logits(case, g)
    elif case["op"].startswith("norm"):
        s = _prepare_norm(case, g)
    else:
        s = _prepare_adamw(case, g)
    s["case"] = case
    if own:     # the scratch memory and the list of tensors that a program keeps from step to step; the inputs are the same
        from paper_2206_05279_amd import binding as pb
        made = lambda n: torch.empty(n, dtype=torch.uint8, device=DEVICE)  # noqa: E731
        if case["op"] in ("logprobs", "train"):
            s["workspace"] = made(pb.pilc_logprobs_workspace_size(case["rows"], case["vocab"], case["top"]))
        elif case["op"] == "norm_backward":
            s["workspace"] = made(pb.pilc_norm_workspace_size(case["rows"], case["width"]))
        elif case["op"] == "adamw":
            part = lambda t: [t[b:b + n] for b, n in zip(s["begins"], s["counts"])]  # noqa: E731
            scale = lambda t: [t[b // BLOCK: b // BLOCK + -(-n // BLOCK)] for b, n in zip(s["begins"], s["counts"])]  # noqa: E731
            f = s["flat"]
            s["list"] = pb.make_adamw_tensors(
                part(f["param"]), part(f["grad"]), part(f["m"]), part(f["v"]),
                m_scales=scale(f["m_scale"]) if case["bits"] == 8 else None,
                v_scales=scale(f["v_scale"]) if case["bits"] == 8 else None,
                decay=[DECAY if b < s["decayed"] else 0.0 for b in s["begins"]])
    return s


# ------------------------------------------------------------------------------------------ the plain forms
def _law(x):
    """(lse, entropy, p, ln p) of rows in 32 bits; where there is no law: -inf, 0, zeros."""
    top = x.amax(1, keepdim=True)
    empty = top == -math.inf
    z = x - torch.where(empty, 0.0, top)
    e = z.exp()
    total = torch.where(empty, 1.0, e.sum(1, keepdim=True))
    log_total = total.log()
    inside = (e * torch.where(e > 0, z, 0.0)).sum(1, keepdim=True)
    entropy = log_total - inside / total
    lse = torch.where(empty, -math.inf, top + log_total)
    return lse[:, 0], torch.where(empty, 0.0, entropy)[:, 0], e / total, z - log_total


def _target_logp(x, target, lse):
    counts = target >= 0
    at = x.gather(1, target.clamp(min=0)[:, None])[:, 0]
    return torch.where(counts, torch.where(lse == -math.inf, -math.inf, at - lse), 0.0)


def _alternatives(x, lse, k):
    """The k largest of each row, the lower symbol first where they are equal; -1 and -inf where a row has fewer."""
    rows, vocab = x.shape
    bits = (x + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(torch.int64)          # integers in the order of the values
    key = (order << 32) + torch.arange(vocab - 1, -1, -1, device=x.device)
    best = torch.topk(key, min(k, vocab), dim=1).values
    sym = vocab - 1 - (best & 0xFFFFFFFF)
    value = x.gather(1, sym)
    there = value > -math.inf
    sym = torch.where(there, sym, -1).to(torch.int32)
    logp = torch.where(there, value - lse[:, None], -math.inf)
    if k > vocab:
        sym = torch.cat([sym, torch.full((rows, k - vocab), -1, dtype=torch.int32, device=x.device)], 1)
        logp = torch.cat([logp, torch.full((rows, k - vocab), -math.inf, device=x.device)], 1)
    return sym, logp


def _gradient(x, target, entropy, p, logp, a, b):
    a = torch.where(target >= 0, a, 0.0)
    d = -p * a[:, None] - b[:, None] * p * (torch.where(p > 0, logp, 0.0) + entropy[:, None])
    full = (x > -math.inf).any(1)
    return d.scatter_add_(1, target.clamp(min=0)[:, None], torch.where(full, a, 0.0)[:, None])


def _plain_logits(s):
    case, x, target = s["case"], s["logits"].float(), s["target"].to(torch.int64)
    if case["op"] == "grad":
        lse = s["lse"][:, None]
        logp = x - torch.where(lse == -math.inf, 0.0, lse)
        d = _gradient(x, target, s["entropy"], logp.exp(), logp, s["up_logp"], s["up_entropy"])
        return [d.to(s["logits"].dtype)]
    lse, entropy, p, logp = _law(x)
    out = [_target_logp(x, target, lse), entropy, lse]
    if case["op"] == "train":
        out.append(_gradient(x, target, entropy, p, logp, s["up_logp"], s["up_entropy"]).to(s["logits"].dtype))
    elif case["top"]:
        out += _alternatives(x, lse, case["top"])
    return out


def _plain_norm(s):
    x, w = s["x"].float(), s["weight"].float()
    if s["case"]["op"] == "norm_forward":
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = 1 / torch.sqrt(d.square().mean(1) + s["eps"])
        return [(d * rstd[:, None] * w + s["bias"].float()).to(s["x"].dtype), mean, rstd]
    dy = s["dy"].float()
    xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
    q = dy * w
    dx = s["rstd"][:, None] * (q - q.mean(1, keepdim=True) - xh * (q * xh).mean(1, keepdim=True))
    return [dx.to(s["x"].dtype), (dy * xh).sum(0).to(s["weight"].dtype), dy.sum(0).to(s["weight"].dtype)]


def _times_power(x, e):
    """x * 2^e for whole e that one 32-bit factor would not hold."""
    half = e >> 1
    power = lambda k: ((k + 127) << 23).view(torch.float32)  # noqa: E731
    return x * power(half) * power(e - half)


def _pack(x, noise, octaves, signed):
    """(codes, scales): a block's values over the power of two above its largest, plus 2^-octaves, cut to three bits
    behind the leading one after `noise` (16 bits) has been added below them; a value above 0 without a sign is never code 0."""
    n = x.numel()
    x = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    noise = torch.nn.functional.pad(noise, (0, -n % BLOCK)).view(-1, BLOCK)
    e = (x.abs().amax(1, keepdim=True).view(torch.int32) >> 23).clamp(min=1)
    y = _times_power(x.abs(), 126 - e) + 2.0 ** -octaves
    code = ((y.view(torch.int32).to(torch.int64) + (noise << 4) + 8) >> 20) - ((127 - octaves) << 3)
    code = code + 128 * (x < 0) if signed else torch.maximum(code, (x > 0).to(torch.int64))
    return code.to(torch.uint8).view(-1)[:n], e.to(torch.uint8).view(-1)


def _unpack(code, scale, octaves, signed):
    n = code.numel()
    code = torch.nn.functional.pad(code, (0, -n % BLOCK)).view(-1, BLOCK).to(torch.int32)
    size = code & 127 if signed else code
    x = ((size + ((127 - octaves) << 3)) << 20).view(torch.float32) - 2.0 ** -octaves
    x = _times_power(x, scale.to(torch.int32)[:, None] - 126)
    return (torch.where(code > 127, -x, x) if signed else x).view(-1)[:n]


def _noise(begins, counts, total, dither):
    """32 bits a value, made from its number (whole blocks of 256 a tensor, in the list's order) and the step's dither."""
    low = torch.arange(total, device=DEVICE, dtype=torch.int64)      # tensors here begin at whole blocks, one after the other
    mask = 0xFFFFFFFF
    h = ((low & mask) * 0x9E3779B9 + (low >> 32) * 0x6A09E667 + (dither * 0xBB67AE85 & mask)) & mask
    h = h ^ (h >> 16)
    h = h * 0x3C6EF373 & mask
    h = h ^ (h >> 15)
    h = h * 0xA54FF53B & mask
    return h ^ (h >> 16)


def _plain_adamw(s):
    f, case = s["flat"], s["case"]
    p, g = f["param"].float(), f["grad"].float()
    if case["bits"] == 32:
        m, v = f["m"], f["v"]
    else:
        m, v = _unpack(f["m"], f["m_scale"], 15, True), _unpack(f["v"], f["v_scale"], 31, False)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    c1, c2 = 1 - BETA1 ** s["step"], 1 - BETA2 ** s["step"]
    move = (m / c1) / (torch.sqrt(v / c2) + EPS)
    d = s["decayed"]
    p[:d] -= LR * DECAY * p[:d]
    f["param"].copy_(p - LR * move)
    if case["bits"] == 32:
        f["m"].copy_(m)
        f["v"].copy_(v)
        out = [f["param"], f["m"], f["v"]]
    else:
        h = _noise(s["begins"], s["counts"], p.numel(), s["step"])
        for key, x, noise, octaves, signed in (("m", m, h & 0xFFFF, 15, True), ("v", v, h >> 16, 31, False)):
            code, scale = _pack(x, noise, octaves, signed)
            f[key].copy_(code)
            f[key + "_scale"].copy_(scale)
            f[key + "_values"].copy_(_unpack(code, scale, octaves, signed))
        out = [f["param"], f["m_values"], f["v_values"]]
    s["step"] += 1
    return out


# ------------------------------------------------------------------------------------------ the framework's
def _own(s):
    from paper_2206_05279_amd import binding as pb
    case, op = s["case"], s["case"]["op"]
    if op == "logprobs":
        pb.pilc_logprobs(s["logits"], s["target"], s["logp"], entropy=s["entropy"], lse=s["lse"],
                         top_sym=s["top_sym"] if case["top"] else None, top_logp=s["top_logp"] if case["top"] else None,
                         workspace=s["workspace"])
        return [s["logp"], s["entropy"], s["lse"]] + ([s["top_sym"], s["top_logp"]] if case["top"] else [])
    if op == "grad":
        pb.pilc_logprobs_grad(s["logits"], s["target"], s["lse"], s["up_logp"], s["grad"], entropy=s["entropy"],
                              up_entropy=s["up_entropy"])
        return [s["grad"]]
    if op == "train":
        pb.pilc_logprobs_train(s["logits"], s["target"], s["up_logp"], s["logp"], s["grad"], entropy=s["entropy"], lse=s["lse"],
                               up_entropy=s["up_entropy"], workspace=s["workspace"])
        return [s["logp"], s["entropy"], s["lse"], s["grad"]]
    if op == "norm_forward":
        pb.pilc_norm_forward(s["x"], s["weight"], s["bias"], s["y"], mean=s["mean"], rstd=s["rstd"], eps=s["eps"])
        return [s["y"], s["mean"], s["rstd"]]
    if op == "norm_backward":
        pb.pilc_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"], dweight=s["dweight"], dbias=s["dbias"],
                              workspace=s["workspace"])
        return [s["dx"], s["dweight"], s["dbias"]]
    f = s["flat"]
    pb.pilc_adamw_step(s["list"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, step=s["step"], dither=s["step"])
    s["step"] += 1
    if case["bits"] == 32:
        return [f["param"], f["m"], f["v"]]
    # what the bytes stand for, as a program that writes a checkpoint in 32 bits takes it
    pb.pilc_adamw_values(f["m"], f["m_scale"], f["m_values"], signed=True)
    pb.pilc_adamw_values(f["v"], f["v_scale"], f["v_values"], signed=False)
    return [f["param"], f["m_values"], f["v_values"]]


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_adamw(state) if op == "adamw" else _plain_norm(state) if op.startswith("norm") else _plain_logits(state)


def work(case):
    size = lambda t: {"f32": 4, "bf16": 2, "f16": 2}[t]  # noqa: E731
    if case["op"] in ("logprobs", "grad", "train"):
        values, each = case["rows"] * case["vocab"], size(case["dtype"])
        row = {"u8": 1, "i32": 4, "i64": 8}[case["target"]] + {"logprobs": 12 + 8 * case["top"], "grad": 16, "train": 20}[case["op"]]
        return {"bytes": values * each * (1 if case["op"] == "logprobs" else 2) + case["rows"] * row,
                "flops": values * {"logprobs": 6, "grad": 8, "train": 13}[case["op"]]}
    if case["op"].startswith("norm"):
        values, forward = case["rows"] * case["width"], case["op"] == "norm_forward"
        return {"bytes": values * size(case["dtype"]) * (2 if forward else 3) + 8 * case["rows"] + (2 if forward else 3) * case["width"] * size(case["weight"]),
                "flops": values * (8 if forward else 16)}
    n = sum(_sizes(case)[1])
    if case["bits"] == 32:
        return {"bytes": n * (2 * size(case["param"]) + size(case["grad"]) + 16), "flops": n * 14}
    return {"bytes": n * (2 * size(case["param"]) + size(case["grad"]) + 4 + 2 + 8) + 6 * (n // BLOCK), "flops": n * 60}


# ------------------------------------------------------------------------------------------ 64 bits
def _exact_logits(s):
    case, rows = s["case"], s["case"]["rows"]
    parts, step = [], max(1, 400_000_000 // case["vocab"])
    for r in range(0, rows, step):
        x, t = s["logits"][r:r + step].double(), s["target"][r:r + step].long()
        lse = torch.logsumexp(x, 1)
        none = torch.isneginf(lse)
        logp = x - lse.masked_fill(none, 0.0)[:, None]
        p = logp.exp()
        h = -(p * logp.masked_fill(p == 0, 0.0)).sum(1)
        here = torch.gather(logp, 1, t.clamp_min(0).unsqueeze(1)).squeeze(1)
        here = here.masked_fill(none, -math.inf).masked_fill(t < 0, 0.0)
        out = []
        if case["op"] != "grad":
            out += [here, h, lse]
        if case["op"] != "logprobs":
            a = s["up_logp"][r:r + step].double() * (t >= 0) * ~none
            b = s["up_entropy"][r:r + step].double()
            one = torch.zeros_like(p).scatter_(1, t.clamp_min(0).unsqueeze(1), 1.0)
            out.append(a[:, None] * (one - p) - b[:, None] * p * (logp.masked_fill(p == 0, 0.0) + h[:, None]))
        elif case["top"]:
            k = min(case["top"], case["vocab"])
            best = torch.topk(x, k, dim=1).values
            values = (best - lse.masked_fill(none, 0.0)[:, None])
            out.append(torch.nn.functional.pad(values, (0, case["top"] - k), value=-math.inf))
        parts.append(out)
    out = [torch.cat([p[i] for p in parts]) for i in range(len(parts[0]))]
    if case["op"] == "logprobs" and case["top"]:
        out.insert(3, None)                                             # the symbols: whole numbers
    return out


def _exact_norm(s):
    x, w = s["x"].double(), s["weight"].double()
    if s["case"]["op"] == "norm_forward":
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + s["eps"]).rsqrt()
        return [torch.addcmul(s["bias"].double(), (x - mean[:, None]).mul_(rstd[:, None]), w), mean, rstd]
    n, rstd = x.shape[1], s["rstd"].double()[:, None]
    xh = x.sub_(s["mean"].double()[:, None]).mul_(rstd)
    dy = s["dy"].double()
    dw, db = (dy * xh).sum(0), dy.sum(0)
    q = dy.mul_(w)
    along = (q * xh).sum(1, keepdim=True)
    return [(q - (q.sum(1, keepdim=True) + xh * along) / n) * rstd, dw, db]


def _exact_bytes(x, noise, c, signed):
    """The values that 8 bits hold of `x`, in 64 bits: steps of an eighth of the power of two below |x| / scale + c."""
    n = x.numel()
    blocks = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    noise = torch.nn.functional.pad(noise, (0, -n % BLOCK)).view(-1, BLOCK)
    scale = torch.exp2(torch.frexp(blocks.abs().amax(1, keepdim=True)).exponent.double().clamp(min=-125))
    y = blocks.abs() / scale + c
    grid = torch.exp2(torch.frexp(y).exponent.double() - 4)
    held = torch.floor(y / grid + (noise.double() * 16 + 8) / 2 ** 20) * grid
    if not signed:
        held = torch.where((blocks > 0) & (held <= c), torch.full_like(held, c * 1.125), held)
    return ((held - c) * scale * torch.sign(blocks)).view(-1)[:n]


def _exact_adamw(s):
    f, case, t = s["flat"], s["case"], s["step"]
    p, g = f["param"].double(), f["grad"].double()
    if case["bits"] == 32:
        m, v = f["m"].double(), f["v"].double()
    else:
        m, v = _unpack(f["m"], f["m_scale"], 15, True).double(), _unpack(f["v"], f["v_scale"], 31, False).double()
    m, v = m.lerp_(g, 1 - BETA1), v.lerp_(g * g, 1 - BETA2)
    move = m / (1 - BETA1 ** t) / ((v / (1 - BETA2 ** t)).sqrt_() + EPS)
    keep = torch.ones_like(p)
    keep[: s["decayed"]] = 1 - LR * DECAY
    p = p * keep - LR * move
    if case["bits"] == 8:
        h = _noise(s["begins"], s["counts"], p.numel(), t)
        m, v = _exact_bytes(m, h & 0xFFFF, 2.0 ** -15, True), _exact_bytes(v, h >> 16, 2.0 ** -31, False)
    return [p, m, v]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    return _exact_adamw(s) if op == "adamw" else _exact_norm(s) if op.startswith("norm") else _exact_logits(s)
