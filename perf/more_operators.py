"""What the operators on the way from a network's last states to its laws, and to a smaller network's, are timed on:
root-mean-square norm with the residual's addition, matrices held in 8 bits under scales for blocks of 128, their
product, and distillation from a teacher's likeliest symbols.

A program that learns laws, or learns a small network from a large one, runs all of these per step; one that answers
with laws symbol by symbol runs the norm and the product on a row or a few.  `listed` holds one case for each use,
`draw` takes further ones from the same ranges.  `run` is the plain form in 32 bits, or with `own` the framework.

A block of 128 values in 8 bits shares a scale that is a power of two: the smallest under which its largest value is
no more than the type's largest.  What is held in 8 bits is returned as the values it stands for (bfloat16 holds them
all).  Lengths are in nats.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
BLOCK = 128
EPS = 1e-5


def _rms(name, op, rows, width, pad, dtype, weight, residual, out="same"):
    """residual: the forward pass adds a second tensor first, the backward pass takes a gradient of that sum too.  out: the
    type that the forward pass answers in, e4m3 and e5m2 under scales."""
    return {"name": name, "op": op, "rows": rows, "width": width, "pad": pad, "dtype": dtype, "weight": weight, "residual": residual, "out": out}


def _quantize(name, rows, width, pad, dtype, out, shared, both):
    """shared: rows that share a scale, 1 or 128.  both: the transposed matrix too, of the same type and sharing."""
    return {"name": name, "op": "quantize", "rows": rows, "width": width, "pad": pad, "dtype": dtype, "out": out, "shared": shared, "both": both}


def _product(name, rows, cols, depth, pad, a, b, shared, out):
    """rows x depth of type `a`, a scale a row and block, times the transpose of cols x depth of type `b`, a scale for
    `shared` rows and block."""
    return {"name": name, "op": "product", "rows": rows, "cols": cols, "depth": depth, "pad": pad, "a": a, "b": b, "shared": shared, "out": out}


def _distill(name, rows, vocab, pad, dtype, top, rest, temperature, grad, masked):
    """top: symbols that the teacher names.  rest: their probabilities are the teacher's own, and what is left of 1 stands
    against what the student leaves; otherwise they are weighed against one another alone.  masked: share of the logits that
    are -inf; with it some rows have no law and some no teacher, and some teachers name fewer symbols."""
    return {"name": name, "op": "distill", "rows": rows, "vocab": vocab, "pad": pad, "dtype": dtype, "top": top, "rest": rest,
            "temperature": temperature, "grad": grad, "masked": masked}


def listed():
    return [
        # the norm before a layer in 8 bits: of one symbol's states, and of a whole batch
        _rms("rms_token", "rms_forward", 1, 4096, 0, "bf16", "bf16", True, "e4m3"),
        _rms("rms_batch", "rms_forward", 16384, 8192, 0, "bf16", "f32", True, "e4m3"),
        # its backward pass, the residual stream's gradient among what comes in
        _rms("rms_backward", "rms_backward", 32768, 4096, 0, "bf16", "bf16", True),
        # weights from 32 bits into 8 after an optimiser's step, for the product forward and, transposed, for the one backward
        _quantize("quantize_weights", 8192, 8192, 0, "f32", "e4m3", 128, True),
        # gradients of logits of an alphabet whose size divides by nothing
        _quantize("quantize_gradient", 1021, 50001, 7, "bf16", "e5m2", 1, False),
        # logits of one symbol, and a layer for a few of them: weights are read once
        _product("product_token", 1, 131072, 4096, 0, "e4m3", "e4m3", 128, "f32"),
        _product("product_few", 33, 8192, 8192, 0, "e4m3", "e4m3", 128, "bf16"),
        # a layer for a batch
        _product("product_batch", 8192, 8192, 8192, 0, "e4m3", "e4m3", 128, "bf16"),
        # weights' gradient, the sum going over a batch's rows
        _product("product_weights", 2047, 1531, 32777, 3, "e5m2", "e4m3", 1, "f32"),
        # a student of the index stream's laws, 256 symbols; and what a stream would lose under one with a large alphabet
        _distill("distill_index", 65536, 256, 0, "bf16", 16, False, 2.0, True, 0.0),
        _distill("distill_scoring", 500, 100003, 29, "f16", 32, True, 1.0, False, 0.02),
        # a student's step with a large alphabet
        _distill("distill_training", 8192, 131072, 0, "bf16", 64, True, 1.0, True, 0.0),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["rms_forward", "rms_forward", "rms_backward", "quantize", "product", "product", "product", "distill", "distill"])
    dtype, pad = rng.choice(["f32", "bf16", "bf16", "f16"]), rng.choice([0, 0, rng.randrange(1, 64)])
    if kind.startswith("rms"):
        width = _spread(rng, 8, 20000)
        rows = max(1, min(_spread(rng, 1, 100000), 130_000_000 // width))
        c = _rms("", kind, rows, width, pad, dtype, rng.choice([dtype, "f32"]), rng.random() < 0.7,
                 rng.choice(["e4m3", "e4m3", "e5m2", "same"]) if kind == "rms_forward" else "same")
    elif kind == "quantize":
        width = _spread(rng, 1, 100000)
        rows = max(1, min(_spread(rng, 1, 100000), 60_000_000 // width))
        c = _quantize("", rows, width, pad, dtype, rng.choice(["e4m3", "e5m2"]), rng.choice([1, 128]), rng.random() < 0.5)
    elif kind == "product":
        depth = _spread(rng, 16, 50000)
        if rng.random() < 0.5:                                  # real layers mostly divide by 16, gradients' sums over rows do not
            depth = -(-depth // 16) * 16
        rows = max(1, min(_spread(rng, 1, 16384), 500_000_000 // depth))
        cols = max(1, min(_spread(rng, 16, 131072), 500_000_000 // depth, 250_000_000_000 // (depth * rows), 500_000_000 // rows))
        c = _product("", rows, cols, depth, pad, rng.choice(["e4m3", "e4m3", "e5m2"]), rng.choice(["e4m3", "e4m3", "e5m2"]),
                     rng.choice([1, 128]), rng.choice(["f32", "bf16", "bf16", "f16"]))
    else:
        vocab = _spread(rng, 2, 200000)
        rows = max(1, min(_spread(rng, 1, 65536), 400_000_000 // vocab))
        c = _distill("", rows, vocab, pad, dtype, min(vocab, rng.choice([1, 4, 16, 50, 128])), rng.random() < 0.5, rng.choice([1.0, 1.0, 2.0, 4.0]),
                     rng.random() < 0.7, rng.choice([0.0, 0.02, 0.3]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ values in 8 bits
def _times_blocks(x, factor, shared):
    """x times the factor [rows / shared, width / 128] of the block it lies in."""
    rows, width = x.shape
    return x * factor.repeat_interleave(shared, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :width]


def _into_blocks(x, dtype, shared):
    """(codes, scales): scales are bytes e that stand for 2^(e - 127), the smallest under which a block's largest value is
    1.75 times a power of two (448 and 57344) at most; codes are rounded to the nearest, ties to even."""
    rows, width = x.shape
    whole = torch.nn.functional.pad(x, (0, -width % BLOCK, 0, -rows % shared))
    largest = whole.abs().view(whole.shape[0] // shared, shared, whole.shape[1] // BLOCK, BLOCK).amax((1, 3))
    e = (((largest.view(torch.int32) + 0x1FFFFF) >> 23) - (8 if dtype == torch.float8_e4m3fn else 15)).clamp(min=0)
    codes = _times_blocks(x, ((254 - e) << 23).view(torch.float32), shared).to(dtype)
    return codes, e.to(torch.uint8)


def _from_blocks(codes, scales, shared):
    return _times_blocks(codes.float(), (scales.to(torch.int32) << 23).view(torch.float32), shared)


def _held(x, dtype, shared=1):
    """What 8 bits hold of x, in bfloat16."""
    return _from_blocks(*_into_blocks(x, dtype, shared), shared).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------ inputs
def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEVICE, dtype=dtype) * scale


def _padded(x, pad):
    """x with `pad` values that are nobody's between its rows."""
    if not pad:
        return x.contiguous()
    whole = torch.empty(x.shape[0], x.shape[1] + pad, dtype=x.dtype, device=x.device)
    whole.view(torch.uint8).fill_(0x7F)
    whole[:, : x.shape[1]] = x
    return whole[:, : x.shape[1]]


def _made(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device=DEVICE)


def _states(g, rows, width, dtype):
    """A residual stream: a few columns far larger than the others."""
    columns = torch.exp(0.5 * _randn(g, width))
    columns[torch.randint(0, width, (max(1, width // 500),), generator=g, device=DEVICE)] *= 20
    return torch.randn(rows, width, generator=g, device=DEVICE, dtype=dtype).mul_(columns.to(dtype))


def _prepare_rms(case, g):
    rows, width, dtype, wtype = case["rows"], case["width"], TYPES[case["dtype"]], TYPES[case["weight"]]
    s = {"x": _padded(_states(g, rows, width, dtype), case["pad"]), "weight": (1 + _randn(g, width, scale=0.2)).to(wtype), "add": None}
    if case["op"] == "rms_forward":
        if case["residual"]:
            s["add"] = _padded(torch.randn(rows, width, generator=g, device=DEVICE, dtype=dtype), case["pad"])
            s["sum"] = _made(rows, width, dtype=dtype)
        s["rstd"] = _made(rows)
        if case["out"] == "same":
            s["y"] = _made(rows, width, dtype=dtype)
        else:
            s["codes"], s["scales"] = _made(rows, width, dtype=TYPES[case["out"]]), _made(rows, -(-width // BLOCK), dtype=torch.uint8)
            s["values"] = _made(rows, width, dtype=torch.bfloat16)
    else:
        s["dy"] = _padded(torch.randn(rows, width, generator=g, device=DEVICE, dtype=dtype), case["pad"])
        s["dsum"] = _padded(torch.randn(rows, width, generator=g, device=DEVICE, dtype=dtype), case["pad"]) if case["residual"] else None
        s["rstd"] = 1 / torch.sqrt(s["x"].float().square().mean(1) + EPS)
        s["dx"], s["dweight"] = _made(rows, width, dtype=dtype), _made(width, dtype=wtype)
    return s


def _prepare_quantize(case, g):
    rows, width, shared, out = case["rows"], case["width"], case["shared"], TYPES[case["out"]]
    x = _states(g, rows, width, TYPES[case["dtype"]])
    x.mul_(0.02 * 2.0 ** torch.randint(-4, 5, (rows, 1), generator=g, device=DEVICE).to(x.dtype))
    s = {"x": _padded(x, case["pad"])}
    for key, (r, w) in {"": (rows, width), "_t": (width, rows)}.items():
        if not key or case["both"]:
            s["codes" + key], s["scales" + key] = _made(r, w, dtype=out), _made(-(-r // shared), -(-w // BLOCK), dtype=torch.uint8)
            s["values" + key] = _made(r, w, dtype=torch.bfloat16)
    return s


def _prepare_product(case, g):
    s = {"c": _made(case["rows"], case["cols"], dtype=TYPES[case["out"]])}
    for key, count, shared in (("a", case["rows"], 1), ("b", case["cols"], case["shared"])):
        x = _states(g, count, case["depth"], torch.float32) if key == "a" else _randn(g, count, case["depth"], scale=case["depth"] ** -0.5)
        codes, s[key + "_scales"] = _into_blocks(x, TYPES[case[key]], shared)
        s[key + "_codes"] = _padded(codes.view(torch.uint8), case["pad"]).view(codes.dtype)
    return s


def _prepare_distill(case, g):
    rows, vocab, dtype, top = case["rows"], case["vocab"], TYPES[case["dtype"]], case["top"]
    logits = _padded(torch.randn(rows, vocab, generator=g, device=DEVICE, dtype=dtype).mul_(2.5), case["pad"])
    for _ in range(3):                                          # a few symbols that are likely
        at = torch.randint(0, vocab, (rows,), generator=g, device=DEVICE)
        logits[torch.arange(rows, device=DEVICE), at] += (8.0 * torch.rand(rows, generator=g, device=DEVICE)).to(dtype)
    if case["masked"]:
        cols = torch.rand(min(rows, 64), vocab, generator=g, device=DEVICE) < case["masked"]
        for a in range(0, rows, cols.shape[0]):
            logits[a:a + cols.shape[0]].masked_fill_(cols[: min(rows - a, cols.shape[0])], -math.inf)
        logits[96::97] = -math.inf
    sym, value = _made(rows, top, dtype=torch.int32), _made(rows, top)
    step = max(1, 100_000_000 // vocab)
    for a in range(0, rows, step):                              # a teacher that agrees with the student more or less
        t = logits[a:a + step].float()
        t += torch.randn(t.shape, generator=g, device=DEVICE)
        best = torch.topk(t, top, dim=1)
        sym[a:a + step], value[a:a + step] = best.indices.to(torch.int32), best.values
        if case["rest"]:
            value[a:a + step] -= torch.logsumexp(t, 1).nan_to_num(0.0, 0.0, 0.0)[:, None]
    none = value == -math.inf
    if case["masked"]:
        none |= torch.arange(top, device=DEVICE)[None] >= torch.randint(1, 2 * top + 1, (rows, 1), generator=g, device=DEVICE)
        none[12::13] = True
    sym.masked_fill_(none, -1)
    value.masked_fill_(none, -math.inf)
    s = {"logits": logits, "sym": sym, "value": value, "loss": _made(rows)}
    if case["grad"]:
        each = (16384.0 if dtype == torch.float16 else 1.0) / rows      # a mean; gradients in f16 are scaled to stay in its range
        s["up"], s["grad"] = each * torch.rand(rows, generator=g, device=DEVICE), _made(rows, vocab, dtype=dtype)
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    op = case["op"]
    s = _prepare_rms(case, g) if op.startswith("rms") else _prepare_quantize(case, g) if op == "quantize" else \
        _prepare_product(case, g) if op == "product" else _prepare_distill(case, g)
    s["case"] = case
    if own:     # the handles of matrices and the scratch memory that a program keeps; the inputs are the same
        from paper_2206_05279_amd import binding as pb
        scratch = lambda n: _made(n, dtype=torch.uint8)  # noqa: E731
        if op == "product":
            s["a"], s["b"] = pb.make_block8(s["a_codes"], s["a_scales"]), pb.make_block8(s["b_codes"], s["b_scales"], block_rows=case["shared"])
            s["workspace"] = scratch(pb.pilc_block8_product_workspace_size(case["rows"], case["cols"], case["depth"]))
        elif op == "distill":
            s["workspace"] = scratch(pb.pilc_distill_workspace_size(case["rows"], case["vocab"], case["top"]))
        elif op == "rms_backward":
            s["workspace"] = scratch(pb.pilc_rms_workspace_size(case["rows"], case["width"]))
        else:
            for key in ("", "_t"):
                if "codes" + key in s:
                    s["held" + key] = pb.make_block8(s["codes" + key], s["scales" + key], block_rows=case.get("shared", 1))
    return s


# ------------------------------------------------------------------------------------------ the plain forms
def _plain_rms(s):
    case, w, x = s["case"], s["weight"].float(), s["x"]
    if case["op"] == "rms_forward":
        h = x if s["add"] is None else (x.float() + s["add"].float()).to(x.dtype)
        f = h.float()
        rstd = 1 / torch.sqrt(f.square().mean(1) + EPS)
        y = f * rstd[:, None] * w
        y = y.to(x.dtype) if case["out"] == "same" else _held(y, TYPES[case["out"]])
        return [y, rstd] if s["add"] is None else [y, rstd, h]
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = x.float() * rstd
    q = dy * w
    dx = rstd * (q - xh * (q * xh).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return [dx.to(x.dtype), (dy * xh).sum(0).to(s["weight"].dtype)]


def _plain_quantize(s):
    case, x = s["case"], s["x"].float()
    out = [_held(x, TYPES[case["out"]], case["shared"])]
    return out + [_held(x.t(), TYPES[case["out"]], case["shared"])] if case["both"] else out


def _plain_product(s):
    a, b = _from_blocks(s["a_codes"], s["a_scales"], 1), _from_blocks(s["b_codes"], s["b_scales"], s["case"]["shared"])
    return [(a @ b.t()).to(s["c"].dtype)]


def _powers(x):
    """(largest or 0, powers, their sum) of rows: e^(x - largest); ln of the sum of e^x is largest + ln sum."""
    top = x.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = (x - top).exp()
    return top, e, e.sum(1, keepdim=True)


def _plain_distill(s):
    """What a row has [rows, vocab] of is in 32 bits; what it has one of, or one for each symbol named, in 64: a loss is a
    small difference of large logarithms where student and teacher agree."""
    case, turn = s["case"], 1.0 / s["case"]["temperature"]
    x, value = s["logits"].float() * turn, s["value"].double()
    vocab, named = x.shape[1], s["sym"] >= 0
    at = torch.where(named, s["sym"], vocab).to(torch.int64)
    mine = torch.where(named, x.gather(1, at.clamp(max=vocab - 1)), -math.inf).double()
    bulk = x
    if case["rest"]:
        others = torch.zeros(x.shape[0], vocab + 1, device=DEVICE, dtype=torch.bool).scatter_(1, at, True)
        bulk = x.masked_fill(others[:, :-1], -math.inf)
    top, e, total = _powers(bulk)
    bulk_lse = top.double() + total.double().log()
    lse = bulk_lse
    if case["rest"]:
        big, _, both = _powers(torch.cat([bulk_lse, mine], 1))
        lse = big + both.log()
        log_q = torch.where(named, value, -math.inf)
        q = log_q.exp()
        left = torch.where(bulk_lse == -math.inf, 0.0, (1 - q.sum(1, keepdim=True)).clamp(min=0))
    else:
        scaled = torch.where(named, value * turn, -math.inf)
        big, _, both = _powers(scaled)
        log_q = scaled - (big + both.log())
        q = torch.where(named, log_q.exp(), 0.0)
    loss = torch.where(q > 0, q * (log_q - (mine - lse)), 0.0).sum(1, keepdim=True)
    if case["rest"]:
        loss = loss + torch.where(left > 0, left * (left.log() - (bulk_lse - lse)), 0.0)
    if not case["grad"]:
        return [loss[:, 0].float()]
    # symbols not named move by their probability and what there is for them all, named ones by the two probabilities' difference
    lawless, each = lse == -math.inf, s["up"].double()[:, None] * turn
    share = (bulk_lse - lse).exp() - left if case["rest"] else q.sum(1, keepdim=True)
    share = torch.where(lawless | (bulk_lse == -math.inf), 0.0, each * share / total.double())
    p = (mine - lse).exp()
    here = torch.where(lawless, 0.0, each * ((p if case["rest"] else p * q.sum(1, keepdim=True)) - q))
    grad = torch.cat([e * share.float(), _made(e.shape[0], 1)], 1).scatter_(1, at, here.float())[:, :-1]
    return [loss[:, 0].float(), grad.to(s["logits"].dtype)]


# ------------------------------------------------------------------------------------------ the framework's
def _own(s):
    from paper_2206_05279_amd import binding as pb
    case, op = s["case"], s["case"]["op"]
    if op == "rms_forward":
        plain = case["out"] == "same"
        pb.pilc_rms_forward(s["x"], s["weight"], y=s["y"] if plain else None, y8=None if plain else s["held"], add=s["add"], sum=s.get("sum"),
                            rstd=s["rstd"], eps=EPS)
        if not plain:
            pb.pilc_block8_values(s["held"], s["values"])
        return [s["y"] if plain else s["values"], s["rstd"]] + ([] if s["add"] is None else [s["sum"]])
    if op == "rms_backward":
        pb.pilc_rms_backward(s["dy"], s["x"], s["weight"], s["rstd"], dx=s["dx"], dweight=s["dweight"], dsum=s["dsum"], workspace=s["workspace"])
        return [s["dx"], s["dweight"]]
    if op == "quantize":
        pb.pilc_block8_quantize(s["x"], s["held"], s.get("held_t"))
        keys = ["", "_t"] if case["both"] else [""]
        for key in keys:
            pb.pilc_block8_values(s["held" + key], s["values" + key])
        return [s["values" + key] for key in keys]
    if op == "product":
        pb.pilc_block8_product(s["a"], s["b"], s["c"], workspace=s["workspace"])
        return [s["c"]]
    pb.pilc_distill(s["logits"], s["sym"], s["value"], s["loss"], up=s.get("up"), grad=s.get("grad"), temperature=case["temperature"],
                    rest=case["rest"], workspace=s["workspace"])
    return [s["loss"], s["grad"]] if case["grad"] else [s["loss"]]


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_rms(state) if op.startswith("rms") else _plain_quantize(state) if op == "quantize" else \
        _plain_product(state) if op == "product" else _plain_distill(state)


def work(case):
    size = lambda t: {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1 + 1 / BLOCK, "e5m2": 1 + 1 / BLOCK}[t]  # noqa: E731
    if case["op"].startswith("rms"):
        values, each = case["rows"] * case["width"], size(case["dtype"])
        if case["op"] == "rms_forward":
            each *= 3 if case["residual"] else 1
            each += size(case["dtype"]) if case["out"] == "same" else 2 * size(case["out"]) + 2        # the codes, and the values that are read off them
        else:
            each *= 4 if case["residual"] else 3
        return {"bytes": values * each + 4 * case["rows"] + (1 if case["op"] == "rms_forward" else 2) * case["width"] * size(case["weight"]),
                "flops": values * (9 if case["op"] == "rms_forward" else 12)}
    if case["op"] == "quantize":
        values, outputs = case["rows"] * case["width"], 2 if case["both"] else 1
        return {"bytes": values * (size(case["dtype"]) + outputs * (2 * size(case["out"]) + 2)), "flops": values * 4 * outputs}
    if case["op"] == "product":
        m, n, k = case["rows"], case["cols"], case["depth"]
        return {"bytes": m * k * size(case["a"]) + n * k * size(case["b"]) + m * n * size(case["out"]), "flops": 2 * m * n * k}
    values = case["rows"] * case["vocab"]
    return {"bytes": values * size(case["dtype"]) * (2 if case["grad"] else 1) + case["rows"] * (8 * case["top"] + 8),
            "flops": values * (7 if case["grad"] else 4)}


# ------------------------------------------------------------------------------------------ 64 bits
def _exact_held(y, out, shared=1):
    """y [rows, width] as steps of its blocks' grid: with 2^s the scale, a value of size 2^p 2^s has steps of 2^(p - digits) 2^s,
    none finer than the type's smallest."""
    digits, low, most = (3, -6, 448.0) if out == "e4m3" else (2, -14, 57344.0)
    rows, width = y.shape
    fill = torch.nn.functional.pad(y, (0, -width % BLOCK, 0, -rows % shared))
    tiles = fill.view(-1, shared, fill.shape[1] // BLOCK, BLOCK)
    largest = tiles.abs().amax((1, 3), keepdim=True)
    s = torch.ceil(torch.log2(torch.where(largest > 0, largest, most) / most))
    s = torch.where(torch.exp2(s) * most < largest, s + 1, s)
    s = torch.where(torch.exp2(s - 1) * most >= largest, s - 1, s).clamp(min=-127)
    z = tiles * torch.exp2(-s)
    step = torch.exp2((torch.frexp(z).exponent - 1).clamp(min=low).double() - digits)
    return (torch.round(z / step) * step * torch.exp2(s)).view(fill.shape)[:rows, :width]


def _exact_rms(s):
    case, x, w = s["case"], s["x"].double(), s["weight"].double()
    if case["op"] == "rms_forward":
        if s["add"] is not None:
            x = x.add_(s["add"].double()).to(s["x"].dtype).double()
        rstd = (torch.linalg.vector_norm(x, dim=1).square() / x.shape[1] + EPS).rsqrt()
        y = torch.einsum("rw,r,w->rw", x, rstd, w)
        out = [y if case["out"] == "same" else _exact_held(y, case["out"]), rstd]
        return out if s["add"] is None else out + [x]
    r, n = s["rstd"].double(), x.shape[1]
    dy = s["dy"].double()
    q = dy * w
    along = (q * x).sum(1) * r.pow(3) / n
    dx = q * r[:, None] - x * along[:, None]
    return [dx if s["dsum"] is None else dx + s["dsum"].double(), (dy * x * r[:, None]).sum(0)]


def _exact_product(s):
    sides = []
    for key, shared in (("a", 1), ("b", s["case"]["shared"])):
        power = torch.exp2(s[key + "_scales"].double() - 127)
        codes = s[key + "_codes"].float()
        n, k = codes.shape
        block = torch.arange(k, device=DEVICE) // BLOCK
        sides.append(codes.double().mul_(power[torch.arange(n, device=DEVICE) // shared][:, block]))
    return [torch.mm(sides[0], sides[1].t())]


def _exact_distill(s):
    case, t = s["case"], s["case"]["temperature"]
    losses, grads, step = [], [], max(1, 200_000_000 // case["vocab"])
    for r in range(0, case["rows"], step):
        x, sym = s["logits"][r:r + step].double() / t, s["sym"][r:r + step].long()
        there = sym >= 0
        n, v = x.shape
        value = s["value"][r:r + step].double().masked_fill(~there, -math.inf)
        log_p = torch.log_softmax(x, 1).masked_fill(torch.isneginf(x), -math.inf)
        mass = torch.zeros(n, v + 1, dtype=torch.float64, device=DEVICE)
        where = sym.masked_fill(~there, v)
        if case["rest"]:
            log_q = value
        else:
            log_q = torch.log_softmax(value / t, 1)
        log_q = log_q.masked_fill(torch.isneginf(value), -math.inf)
        q = log_q.exp()
        mass.scatter_add_(1, where, q)
        mass = mass[:, :v]
        named = torch.zeros(n, v + 1, dtype=torch.bool, device=DEVICE).scatter_(1, where, True)[:, :v]
        picked = log_p.gather(1, where.clamp(max=v - 1))
        loss = torch.where(q > 0, q * (log_q - picked), 0.0).sum(1)
        d = log_p.exp()
        lawless = torch.isneginf(x).all(1)
        if case["rest"]:
            outside = torch.logsumexp(log_p.masked_fill(named, -math.inf), 1)
            left = (1 - q.sum(1)).clamp(min=0).masked_fill(torch.isneginf(outside), 0.0)
            loss = loss + torch.where(left > 0, left * (left.log() - outside), 0.0)
            d = torch.where(named, d - mass, d * (1 - left * torch.exp(-outside.clamp(min=-700)))[:, None])
        else:
            d = d * q.sum(1, keepdim=True) - mass
        losses.append(loss.masked_fill(lawless, 0.0))      # where a row has no law these cases' teachers name nothing
        if case["grad"]:
            grads.append((d * (s["up"][r:r + step].double() / t)[:, None]).masked_fill(lawless[:, None], 0.0).float())
    return [torch.cat(losses)] + ([torch.cat(grads)] if case["grad"] else [])


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("rms"):
        return _exact_rms(s)
    if op == "quantize":
        x = s["x"].double()
        return [_exact_held(x, case["out"], case["shared"])] + ([_exact_held(x.t().contiguous(), case["out"], case["shared"])] if case["both"] else [])
    return _exact_product(s) if op == "product" else _exact_distill(s)
