"""The 64-bit references of the operators that fit laws, against their definitions: gradients against
differences, the short floating codes against their grid, the hash against uniform numbers."""
import numpy as np
import pytest

from oracle import fit_oracle as orc


def _difference(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


@pytest.mark.parametrize("rows,n", [(3, 5), (2, 1), (1, 17)])
def test_gradient_of_log_probabilities_is_the_difference(rows, n):
    rng = np.random.default_rng(rows * 100 + n)
    x = rng.normal(size=(rows, n)) * 2
    t = rng.integers(0, n, rows)
    t[0] = -1 if rows > 1 else t[0]
    a, b = rng.normal(size=rows), rng.normal(size=rows)

    def loss(v):
        law = orc.logprobs(v, t, 0)
        return (a * law["logp"]).sum() + (b * law["entropy"]).sum()

    g, _ = orc.logprobs_grad(x, t, a, b)
    assert np.abs(g - _difference(loss, x)).max() < 1e-7   # truncation h^2, cancellation 1e-16 / h


def test_rows_without_a_law_and_rows_that_are_not_numbers():
    x = np.array([[-np.inf, -np.inf], [0.0, np.nan], [np.inf, 0.0], [-np.inf, 3.0]])
    law = orc.logprobs(x, np.array([0, 1, -1, 1]), 2)
    assert law["lse"][0] == -np.inf and law["logp"][0] == -np.inf and law["entropy"][0] == 0
    assert np.isnan(law["lse"][1:3]).all() and np.isnan(law["logp"][1]) and law["logp"][2] == 0
    assert law["lse"][3] == 3 and law["logp"][3] == 0 and law["entropy"][3] == 0
    assert law["top_sym"].tolist() == [[-1, -1], [-1, -1], [-1, -1], [1, -1]]
    g, _ = orc.logprobs_grad(x, np.array([0, 1, -1, 1]), np.ones(4), None)
    assert (g[0] == 0).all() and np.isnan(g[1]).all() and (g[2] == 0).all() and (g[3] == 0).all()


def test_gradients_of_the_norm_are_the_differences():
    rng = np.random.default_rng(5)
    x, w, b, dy = rng.normal(size=(3, 6)), rng.normal(size=6), rng.normal(size=6), rng.normal(size=(3, 6))
    _, mean, rstd, *_ = orc.norm_forward(x, w, b, 1e-3)
    dx, dw, db, *_ = orc.norm_backward(dy, x, w, mean, rstd)
    loss = lambda xx, ww, bb: (orc.norm_forward(xx, ww, bb, 1e-3)[0] * dy).sum()  # noqa: E731
    for got, want in ((dx, _difference(lambda v: loss(v, w, b), x)), (dw, _difference(lambda v: loss(x, v, b), w)),
                      (db, _difference(lambda v: loss(x, w, v), b))):
        assert np.abs(got - want).max() < 1e-7


@pytest.mark.parametrize("signed", [True, False])
def test_codes_stand_for_a_grid_with_zero_in_it(signed):
    """Every code stands for another value, in order, evenly spaced near zero and an eighth apart above."""
    k, count = (15, 122) if signed else (31, 250)
    v = orc.unpack(np.arange(count, dtype=np.uint8), np.full(1, 126, np.uint8), signed).astype(np.float64)
    assert v[0] == 0 and (np.diff(v) > 0).all() and v[1] == 2.0 ** -(k + 3) and v[-1] >= 1
    assert (np.diff(v) <= (v[1:] + 2.0 ** -k) / 8 * 1.0001).all()


@pytest.mark.parametrize("signed", [True, False])
def test_codes_are_near_and_right_on_average(signed):
    rng = np.random.default_rng(11)
    x = (rng.normal(size=2560) * np.exp(rng.normal(size=2560) * 3)).astype(np.float32)
    x = x if signed else x * x
    x[7] = 0
    total, turns = np.zeros(x.size), 400
    for d in range(turns):
        h = orc.noise(np.arange(x.size, dtype=np.uint64), d)
        codes, scales = orc.pack(x, h & 0xFFFF if signed else h >> 16, signed)
        got = orc.unpack(codes, scales, signed).astype(np.float64)
        scale = np.ldexp(1.0, np.repeat(scales.astype(int), 256) - 126)
        step = np.maximum(np.abs(x), np.abs(got)) / 8 + scale * 2.0 ** (-18 if signed else -34)
        assert (np.abs(got - x) <= step * 1.001).all()
        total += got
    # a mean of 400 draws of a variable within one step: five deviations of at most step / 2 / sqrt(400).  A value
    # without a sign in the lowest step is held at that step
    low = (np.abs(x) < scale * 2.0 ** -34) & (not signed)
    assert (np.abs(total / turns - x) <= 5 * step / 2 / 20)[~low].all()
    assert not signed or total[7] == 0


def test_a_value_without_a_sign_above_zero_is_never_code_zero():
    x = np.zeros(256, np.float32)
    x[0], x[1], x[2] = 1.0, 1e-30, 0.0
    codes, _ = orc.pack(x, np.zeros(256, np.uint32), False)
    assert codes[1] == 1 and codes[2] == 0


def test_blocks_that_are_not_finite_say_so():
    x = np.ones(300, np.float32)
    x[299] = np.inf
    codes, scales = orc.pack(x, np.zeros(300, np.uint32), True)
    assert scales.tolist() == [127, 255]
    v = orc.unpack(codes, scales, True)
    assert (v[:256] == 1 - 2.0 ** -14).all() and np.isnan(v[256:]).all()     # 1 lies between two codes, rounded down without noise


def test_noise_is_even():
    h = orc.noise(np.arange(1 << 16, dtype=np.uint64) + np.uint64(1 << 33), 77)
    for part in (h & 0xFFFF, h >> 16):
        counts = np.bincount(part >> 8, minlength=256)
        assert ((counts - 256.0) ** 2 / 256).sum() < 255 + 6 * np.sqrt(2 * 255)     # chi squared, six deviations
    bits = ((h[:, None] >> np.arange(32)) & 1).astype(np.float64) - 0.5
    cross = np.abs((bits.T @ bits) / (0.25 * len(h)) - np.eye(32)).max()
    assert cross < 6 / np.sqrt(len(h))
    follow = np.abs((bits[:-1] * bits[1:]).mean(0) * 4).max()
    assert follow < 6 / np.sqrt(len(h))
