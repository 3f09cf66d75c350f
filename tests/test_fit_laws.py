"""The example that learns the laws of an index stream: its host side, and on a GPU the whole of it."""
import numpy as np
import pytest
import torch

from paper_2206_05279_amd import fit_laws


@pytest.mark.parametrize("prec_bits,num_sym", [(12, 256), (9, 256), (10, 5)])
def test_masses_are_what_the_coder_takes(prec_bits, num_sym):
    rng = np.random.default_rng(num_sym)
    p = rng.dirichlet(np.full(num_sym, 0.1), size=7)
    p[0] = 0
    p[0, 3] = 1
    m = fit_laws.masses_of(p, prec_bits)
    assert m.dtype == np.uint32 and (m >= 1).all() and (m.sum(1) == 1 << prec_bits).all()
    # a mass is one count and its share of the rest, off by the rounding of two edges
    assert np.abs(m - 1 - p * ((1 << prec_bits) - num_sym)).max() <= 1 + 1e-9


def test_law_numbers_go_by_cell_and_class():
    d = fit_laws.law_numbers(torch.tensor([0, 2]))
    assert d.shape == (2, 256) and d.dtype == torch.uint8
    image = d[0].reshape(16, 16).long()
    assert image[0, 0] == image[1, 1] == 0 and image[0, 2] == 1 and image[2, 0] == 8 and image[15, 15] == 63
    assert torch.equal(d[1].long(), d[0].long() + 128)


@pytest.mark.gpu
def test_laws_are_learned_and_code_the_stream():
    out = fit_laws.fit(images=2000, steps=200, batch=8192, say=lambda s: print(s, flush=True))
    assert out["lossless"]
    # the laws that the stream is drawn from differ: one law for all costs over half a bit more
    assert out["coded"] < out["static"] - 0.5
    # a coder's overhead: 8 bytes and an offset a piece of 256 indices, half a word of padding, masses of 12 bits, and what its
    # short state costs (at most 2 - log2 e bits a symbol)
    assert out["learned"] < out["coded"] < out["learned"] + 12 * 8 / 256 + 16 / 256 + 0.6
    assert (np.diff(out["best_logp"].numpy(), axis=1) <= 0).all() and (out["best"] >= 0).all()
