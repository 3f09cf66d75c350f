"""The references of what lies between states and laws, against their definitions: codes against the types' grids, gradients
against differences."""
import numpy as np
import pytest
import torch

from oracle import block8_oracle as orc

TORCH = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def _difference(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_codes_are_the_types(kind):
    every = torch.arange(256, dtype=torch.uint8)
    v = every.view(TORCH[kind]).float().double().numpy()
    assert np.array_equal(orc.decode(every.numpy(), kind), v, equal_nan=True)
    rng = np.random.default_rng(0)
    t = orc.TABLE[kind][np.isfinite(orc.TABLE[kind])]
    x = np.concatenate([t, (t[1:] + t[:-1]) / 2, rng.uniform(0, orc.MOST[kind], 4000), rng.uniform(0, 2.0 ** -4, 4000)])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).to(torch.float32).to(TORCH[kind]).view(torch.uint8).numpy()
    assert np.array_equal(orc.encode(x.astype(np.float32).astype(float), kind), want)


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_scales_are_the_smallest_that_hold(kind):
    most = orc.MOST[kind]
    for v in (most, np.nextafter(most, np.inf), most / 2, 1.0, 3e38, 1e-45, 1e-30):
        e = orc.scale_of(v, kind)
        assert v <= most * 2.0 ** (e - 127) and (e == 0 or v > most * 2.0 ** (e - 128))
    assert orc.scale_of(0.0, kind) == 0 and orc.scale_of(np.nan, kind) == 255 and orc.scale_of(np.inf, kind) == 255


@pytest.mark.parametrize("block_rows", [1, 128])
def test_a_block_is_off_by_half_a_step_at_most(block_rows):
    rng = np.random.default_rng(2)
    x = rng.normal(size=(130, 300)) * np.exp(rng.normal(size=(130, 1)) * 3)
    for kind, digits in (("e4m3", 3), ("e5m2", 2)):
        codes, scales = orc.quantize(x, kind, block_rows)
        v = orc.values(codes, scales, kind, block_rows)
        p = orc.powers(scales, x.shape, block_rows)
        least = 2.0 ** (-6 if kind == "e4m3" else -14) * p
        assert (np.abs(v - x) <= 2.0 ** -(digits + 1) * np.maximum(np.abs(x), least)).all()


def test_gradients_of_the_norm_are_the_differences():
    rng = np.random.default_rng(5)
    h, w, dy, ds = rng.normal(size=(3, 6)), rng.normal(size=6), rng.normal(size=(3, 6)), rng.normal(size=(3, 6))
    _, rstd, *_ = orc.rms_forward(h, w, 1e-3)
    dx, dw, *_ = orc.rms_backward(dy, h, w, rstd, ds)
    assert np.abs(dx - _difference(lambda v: (orc.rms_forward(v, w, 1e-3)[0] * dy + v * ds).sum(), h)).max() < 1e-7
    assert np.abs(dw - _difference(lambda v: (orc.rms_forward(h, v, 1e-3)[0] * dy).sum(), w)).max() < 1e-7


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("temperature", [1.0, 2.5])
def test_gradient_of_distillation_is_the_difference(rest, temperature):
    rng = np.random.default_rng(7)
    x = rng.normal(size=(4, 9)) * 2
    sym = np.array([[0, 3, 8], [5, -1, 5], [-1, -1, -1], [2, 1, 7]])
    value = np.log(rng.uniform(0.05, 0.3, size=(4, 3)))
    value[3, 1] = -np.inf
    up = rng.normal(size=4)
    _, g, *_ = orc.distill(x, sym, value, up, temperature, rest)
    assert np.abs(g - _difference(lambda v: (up * orc.distill(v, sym, value, None, temperature, rest)[0]).sum(), x)).max() < 1e-7


def test_a_student_that_agrees_loses_nothing():
    x = np.log(np.array([[0.4, 0.3, 0.2, 0.1]]))
    every = np.array([[2, 0, 1, 3]])
    for rest in (False, True):
        loss, g, *_ = orc.distill(x, every, x[0][every], np.ones(1), 1.0, rest)
        assert abs(loss[0]) < 1e-15 and np.abs(g).max() < 1e-15
    loss, g, *_ = orc.distill(x, every[:, :2], x[0][every[:, :2]], np.ones(1), 1.0, True)
    assert abs(loss[0]) < 1e-15 and np.abs(g).max() < 1e-15


def test_rows_without_a_law_or_a_teacher():
    inf = np.inf
    x = np.array([[-inf, -inf], [0.0, np.nan], [0.0, 1.0], [-inf, 3.0], [0.0, 1.0]])
    sym = np.array([[0], [1], [-1], [0], [2]])
    for rest in (False, True):
        loss, g, *_ = orc.distill(x, sym, np.full((5, 1), -0.5), np.ones(5), 1.0, rest)
        assert loss[0] == inf and (g[0] == 0).all() and np.isnan(loss[1]) and np.isnan(g[1]).all()
        assert loss[2] == 0 and (g[2] == 0).all() and loss[3] == inf and np.isfinite(g[3]).all() and np.isnan(loss[4])
