"""Plain references in numpy for what fits the laws: log probabilities and their gradient, layer norm, AdamW.

Everything is computed in 64 bits from the definitions, one row or value at a time where that is
plainest; only the 8-bit states, whose codes are exact, are computed in 32 bits operation by operation.
Each function that a rounding analysis is made for also returns the sums that its bound is built of.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24          # half a unit in the last place of 32-bit numbers, relative


def chain(n: int) -> float:
    """Additions a value goes through in a sum over n values split over 64 threads at least, with the joins."""
    return min(n, n / 64 + 64) + 16


def apart_sums(n: int, first: float) -> float:
    """What a row's sum of powers may be off, in units of U of itself.  A power's exponent is rounded when the largest value is
    taken from it, when it goes from e to 2 and by log2 e having 24 bits, less than three units of its size together (`first` is
    the sizes' mean under the law); the power itself is two off; a common factor of all of a part's powers is taken out (three),
    and parts are joined by powers of their own (a few units each)."""
    return chain(n) + 24 + 3 * first


def logprobs(x, target, top):
    """x [rows, n] float64, target [rows] int64 or None.  Returns a dict: lse, entropy, logp, top_sym, top_logp,
    and the bounds of the errors that 32-bit arithmetic may make in lse, entropy and logp.  logp_apart is logp by the largest
    value and the logarithm of the sum one after the other, which lse, however many bits it has, swallows where the logits lie far
    from zero; its bound logp_apart_err has no share of |lse|."""
    rows, n = x.shape
    out = {k: np.zeros(rows) for k in ("lse", "entropy", "logp", "lse_err", "entropy_err", "logp_err", "logp_apart",
                                         "logp_apart_err")}
    out["top_sym"] = np.full((rows, top), -1, dtype=np.int32)
    out["top_logp"] = np.full((rows, top), -np.inf)
    for r in range(rows):
        v = x[r]
        bad = np.isnan(v).any() or (v == np.inf).any()
        t = None if target is None else int(target[r])
        if bad:
            out["lse"][r] = out["entropy"][r] = np.nan
            out["logp"][r] = out["logp_apart"][r] = 0.0 if t is not None and t < 0 else np.nan
            out["top_logp"][r] = np.nan
            continue
        there = v > -np.inf
        if not there.any():
            out["lse"][r] = -np.inf
            out["logp"][r] = out["logp_apart"][r] = 0.0 if t is not None and t < 0 else np.nan if t is not None and t >= n else -np.inf
            continue
        big = v.max()
        z = v[there] - big
        e = np.exp(z)
        total = e.sum()
        p = e / total
        log_total = np.log(total)
        out["lse"][r] = big + log_total
        out["entropy"][r] = log_total - (p * z).sum()
        # e: the product z log2 e is rounded (|z| U relative in e) and so is the power (2 U); the sum by its chain
        first, second = (p * -z).sum(), (p * z * z).sum()
        sums = chain(n) + 6 + first
        out["lse_err"][r] = U * (sums + 4 * log_total + 2 * abs(out["lse"][r]) + 1)
        out["entropy_err"][r] = U * (sums + 4 * log_total + (chain(n) + 10 + sums) * first + second + 2 * out["entropy"][r] + 1)
        if t is not None:
            out["logp"][r] = 0.0 if t < 0 else np.nan if t >= n else v[t] - out["lse"][r]
            if 0 <= t < n and v[t] > -np.inf:
                out["logp_err"][r] = U * (sums + 4 * log_total + 3 * abs(v[t] - big) + 3 * abs(out["logp"][r]) + 2 * abs(out["lse"][r]) + 1)
            out["logp_apart"][r] = 0.0 if t < 0 else np.nan if t >= n else (v[t] - big) - log_total
            if 0 <= t < n and v[t] > -np.inf:
                out["logp_apart_err"][r] = U * (apart_sums(n, first) + 4 * log_total + 3 * abs(v[t] - big) + 3 * abs(out["logp_apart"][r]) + 1)
        if top == 0:
            continue
        order = sorted(np.flatnonzero(there), key=lambda j: (-v[j], j))[:top]
        out["top_sym"][r, :len(order)] = order
        out["top_logp"][r, :len(order)] = v[order] - out["lse"][r]
    return out


def logprobs_grad(x, target, up_logp, up_entropy, apart=False):
    """(gradient, bound of its error before the last rounding) by the logits; up_entropy may be None.  apart: the law as it is by
    the largest value and the sum, not by an lse that was rounded; its bound has no share of |lse|."""
    rows, n = x.shape
    g, err = np.zeros_like(x), np.zeros_like(x)
    law = logprobs(x, target, 0)
    for r in range(rows):
        t = int(target[r])
        a = 0.0 if t < 0 else float(up_logp[r])
        b = 0.0 if up_entropy is None else float(up_entropy[r])
        lse, h = law["lse"][r], law["entropy"][r]
        if a == 0.0 and b == 0.0:
            continue
        if np.isnan(lse) or t >= n:
            g[r] = np.nan
            continue
        if lse == -np.inf:
            continue
        there = x[r] > -np.inf
        big = x[r][there].max()
        z = np.where(there, x[r] - big, -np.inf)
        total = np.exp(z).sum()
        lp = z - np.log(total) if apart else np.where(there, x[r] - lse, -np.inf)
        p = np.exp(lp)
        fall = np.where(p > 0, lp, 0.0)
        g[r] = -a * p - b * p * (fall + h)
        if t >= 0:
            g[r, t] += a
        if apart:       # of a power, of the sum and of what is made of both
            near = np.where(p > 0, -z, 0.0)
            off = U * (apart_sums(n, (p * near).sum()) + 3 * near + 2 * np.abs(fall) + 4 * np.log(total) + 12)
        else:
            off = law["lse_err"][r] + U * (2 * np.abs(fall) + abs(lse) + 4)         # relative error of p
        h_err = law["entropy_err"][r] * (3 if apart else 1)     # three roundings of an exponent for one
        err[r] = p * (abs(a) * (off + 4 * U) + abs(b) * ((np.abs(fall) + h) * (off + 6 * U) + off + h_err)) + U * np.abs(g[r])
        if t >= 0:
            err[r, t] += 2 * U * abs(a)
    return g, err


def norm_forward(x, weight, bias, eps):
    """(y, mean, rstd, bounds of their errors in the same order)."""
    rows, n = x.shape
    mean = x.mean(1)
    d = x - mean[:, None]
    var = (d * d).mean(1)
    rstd = 1 / np.sqrt(var + eps)
    w = np.ones(n) if weight is None else weight
    y = d * rstd[:, None] * w + (0 if bias is None else bias)
    mean_err = U * (chain(n) + 3) * np.abs(x).mean(1)
    # the mean's error enters the squares as its square, and what subtracting rounds as 2 U
    var_err = U * (chain(n) + 8) * var + mean_err ** 2 + 2 * U * np.abs(d).mean(1) * mean_err
    with np.errstate(divide="ignore", invalid="ignore"):
        rstd_rel = np.where(var + eps > 0, 0.5 * var_err / (var + eps), 0) * 1.5 + 6 * U
    y_err = np.abs(w) * rstd[:, None] * (mean_err[:, None] + np.abs(d) * (rstd_rel[:, None] + 4 * U)) + U * (np.abs(y) + (0 if bias is None else np.abs(bias)))
    return y, mean, rstd, y_err, mean_err, rstd * rstd_rel


def norm_backward(dy, x, weight, mean, rstd):
    """(dx, dweight, dbias, bounds of their errors in the same order)."""
    rows, n = x.shape
    w = np.ones(n) if weight is None else weight
    xh = (x - mean[:, None]) * rstd[:, None]
    q = dy * w
    c1, c2 = q.mean(1, keepdims=True), (q * xh).mean(1, keepdims=True)
    dx = rstd[:, None] * (q - c1 - xh * c2)
    c1_err, c2_err = U * (chain(n) + 4) * np.abs(q).mean(1, keepdims=True), U * (chain(n) + 8) * np.abs(q * xh).mean(1, keepdims=True)
    dx_err = np.abs(rstd[:, None]) * (8 * U * (np.abs(q) + np.abs(c1) + np.abs(xh * c2)) + c1_err + np.abs(xh) * c2_err)
    dw, db = (dy * xh).sum(0), dy.sum(0)
    return dx, dw, db, dx_err, U * (rows + 12) * np.abs(dy * xh).sum(0), U * (rows + 8) * np.abs(dy).sum(0)


def adamw(p, g, m, v, lr, beta1, beta2, eps, step, decay, grad_scale=1.0):
    """(param, m, v, bounds of their errors) in 64 bits."""
    g = g * grad_scale
    m0, m1, v0, v1 = m * beta1, g * (1 - beta1), v * beta2, g * g * (1 - beta2)
    m, v = m0 + m1, v0 + v1
    move = lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    new = p * (1 - lr * decay) - move
    m_err, v_err = 4 * U * (np.abs(m0) + np.abs(m1)), 6 * U * v + 2.0 ** -149
    with np.errstate(divide="ignore", invalid="ignore"):
        move_err = np.abs(move) * 20 * U + np.where(m != 0, np.abs(move / m) * m_err, 0) + np.where(v > 0, np.abs(move) * v_err / v, 0)
    return new, m, v, 3 * U * np.abs(p) + move_err + 2 * U * np.abs(new), m_err, v_err


# ---- states in 8 bits: 32-bit arithmetic, operation by operation --------------------------------
def moments32(m, v, g, beta1, beta2, grad_scale=1.0):
    f = np.float32
    m, v, g = m.astype(f), v.astype(f), g.astype(f) * f(grad_scale)
    return m * f(beta1) + g * f(1 - beta1), v * f(beta2) + g * g * f(1 - beta2)


def noise(numbers, dither):
    """32 bits for each value number (uint64)."""
    mask = np.uint64(0xFFFFFFFF)
    h = ((numbers & mask) * np.uint64(0x9E3779B9) & mask) + ((numbers >> np.uint64(32)) * np.uint64(0x6A09E667) & mask)
    h = (h + np.uint64(dither * 0xBB67AE85 & 0xFFFFFFFF)) & mask
    h ^= h >> np.uint64(16)
    h = h * np.uint64(0x3C6EF373) & mask
    h ^= h >> np.uint64(15)
    h = h * np.uint64(0xA54FF53B) & mask
    return (h ^ (h >> np.uint64(16))).astype(np.uint32)


def pack(x, bits16, signed):
    """(codes, scales) of float32 values, 256 a block."""
    k = 15 if signed else 31
    codes, scales = np.zeros(x.size, np.uint8), np.zeros(-(-x.size // 256), np.uint8)
    for b in range(scales.size):
        at = slice(256 * b, min(256 * b + 256, x.size))
        v = x[at].astype(np.float32)
        e = max(1, int((np.abs(v).view(np.uint32) >> 23).max()))
        scales[b] = e
        if e == 255:
            continue
        y = np.ldexp(np.abs(v), 126 - e) + np.float32(2.0 ** -k)
        code = ((y.view(np.uint32).astype(np.int64) + (bits16[at].astype(np.int64) << 4) + 8) >> 20) - ((127 - k) << 3)
        codes[at] = code | np.where(v < 0, 128, 0) if signed else np.where(v > 0, np.maximum(code, 1), code)
    return codes, scales


def unpack(codes, scales, signed):
    k = 15 if signed else 31
    size = (codes & 127 if signed else codes).astype(np.uint32)
    y = ((size + np.uint32((127 - k) << 3)) << np.uint32(20)).view(np.float32) - np.float32(2.0 ** -k)
    e = np.repeat(scales.astype(np.int32), 256)[: codes.size]
    x = np.ldexp(y, e - 126)
    x = np.where(codes > 127, -x, x) if signed else x
    return np.where(e == 255, np.float32(np.nan), x).astype(np.float32)
