"""The 64-bit reference's law by largest value and sum apart: where the logits lie does not matter to it."""
import numpy as np
import pytest

from oracle import fit_oracle as orc


@pytest.mark.parametrize("offset", [0.0, -2.0 ** 30, 2.0 ** 45, -1e300])
def test_an_offset_changes_no_probability(offset):
    rng = np.random.default_rng(3)
    step = 2.0 ** -6 if abs(offset) < 2.0 ** 46 else 0.0      # what such an offset still holds exactly; the largest holds none
    x = rng.integers(-400, 400, (5, 60)) * step
    t, a, b = rng.integers(0, 60, 5), rng.normal(size=5), rng.normal(size=5)
    near, far = orc.logprobs(x, t, 0), orc.logprobs(x + offset, t, 0)
    assert np.array_equal(near["logp_apart"], far["logp_apart"]) and np.array_equal(near["logp_apart_err"], far["logp_apart_err"])
    assert np.abs(near["logp_apart"] - near["logp"]).max() < 1e-13
    g, err = orc.logprobs_grad(x, t, a, b, apart=True)
    g_far, err_far = orc.logprobs_grad(x + offset, t, a, b, apart=True)
    assert np.array_equal(g, g_far) and np.array_equal(err, err_far)
    assert np.abs(g - orc.logprobs_grad(x, t, a, b)[0]).max() < 1e-13
    assert np.abs(g.sum(1)).max() < 1e-13                     # probabilities add up to 1


def test_a_row_of_one_large_number_is_even():
    x = np.full((1, 8), -3.3895313892515355e38)
    assert orc.logprobs(x, np.array([2]), 0)["logp_apart"][0] == -np.log(8)
    g, _ = orc.logprobs_grad(x, np.array([2]), np.ones(1), None, apart=True)
    assert np.abs(g[0] - (np.arange(8) == 2) + 0.125).max() < 1e-15
