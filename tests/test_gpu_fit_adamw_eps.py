"""AdamW with very small eps."""
import numpy as np
import pytest
import torch

from paper_2206_05279_amd import binding as pb

DEV = "cuda:0"


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-38, 1e-40, 1e-60])
def test_weights_without_gradients_stay_where_eps_is_tiny(bits, eps):
    """m and v of 0 over an eps above 0 are no move, however little that eps is."""
    n = 700
    p = torch.randn(n, device=DEV)
    g, before = torch.zeros(n, device=DEV), p.clone()
    g[600:] = 0.01
    state = torch.float32 if bits == 32 else torch.uint8
    m, v = torch.zeros(n, dtype=state, device=DEV), torch.zeros(n, dtype=state, device=DEV)
    scales = [[torch.zeros(3, dtype=torch.uint8, device=DEV)] for _ in range(2)] if bits == 8 else [None, None]
    tensors = pb.make_adamw_tensors([p], [g], [m], [v], *scales)
    for step in (1, 2):
        pb.pilc_adamw_step(tensors, 1e-3, 0.9, 0.999, eps, step, dither=step)
    assert torch.equal(p[:600], before[:600])
    # the first step moves by lr times m / c1 over the root of v / c2, which are the gradient and its size; the second as much
    # but for what 8 bits make of m and v between (an eighth of each, one up and one down: a quarter)
    moved = (before - p)[600:].double().cpu().numpy()
    assert np.abs(moved / 2e-3 - 1).max() < (1e-3 if bits == 32 else 0.25)
