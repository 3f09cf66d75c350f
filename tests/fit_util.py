"""Helpers for the tests of the operators that fit laws."""
import numpy as np
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half a unit in the last place, relative (2^-p for p digits, the leading one among them), and half the smallest step, of each type
UNIT = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25)}
LOWEST = {torch.float32: -3.4028234663852886e38, torch.bfloat16: -3.3895313892515355e38, torch.float16: -65504.0}
# below it 32-bit results may be taken for 0
TINY = 2.0 ** -125


def up(t):
    return t.detach().to("cpu").double().numpy()


def placed(values, dtype, pad=0, shift=0):
    """[rows, n] on the device with `pad` elements of NaN between rows, beginning `shift` elements into an allocation; the
    allocation too."""
    rows, n = values.shape
    whole = torch.full((shift + rows * (n + pad),), float("nan"), dtype=dtype, device="cuda:0")
    t = whole[shift:].view(rows, n + pad)[:, :n]
    t.copy_(torch.from_numpy(np.ascontiguousarray(values)).to(dtype))
    return t, whole


def close(got, want, err, dtype, what):
    """got (of `dtype`) is within err of want, and one rounding to dtype; what is not finite, or beyond dtype's range, is the same."""
    got = up(got)
    most = torch.finfo(dtype).max
    want = np.where(want > most, np.inf, np.where(want < -most, -np.inf, want))
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    rel, least = UNIT[dtype]
    bound = np.broadcast_to(err, want.shape) + rel * np.abs(want) * 1.01 + least + TINY
    off = np.abs(np.where(fine, got - np.where(fine, want, 0), 0)) - np.where(fine, bound, 0)
    assert (off <= 0).all(), "%s: %d values off, worst %g over its bound at %s" % (
        what, (off > 0).sum(), off.max(), np.unravel_index(off.argmax(), off.shape))
