"""Log probabilities of rows of many runs: more of them, or more keys, than the threads that put a row together begin with."""
import numpy as np
import pytest
import torch

from fit_util import TYPES, close, up
from oracle import fit_oracle as orc
from paper_2206_05279_amd import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,top", [(1, 3000001, 0), (1, 3000001, 32), (1, 3000001, 1), (130, 250007, 32), (300, 130000, 31)])
@pytest.mark.parametrize("equals", [False, True])
def test_runs_put_together(dtype, rows, n, top, equals):
    g = torch.Generator(device=DEV).manual_seed(n + top)
    x = torch.empty(rows, n, dtype=TYPES[dtype], device=DEV)
    for r in range(rows):
        row = torch.randn(n, generator=g, device=DEV) * 3
        x[r] = row.round() if equals else row
    t = torch.randint(0, n, (rows,), generator=g, device=DEV)
    logp, entropy, lse = (torch.full((rows,), 77.0, device=DEV) for _ in range(3))
    sym, best = torch.full((rows, top), 77, dtype=torch.int32, device=DEV), torch.empty(rows, top, device=DEV)
    ws = torch.empty(pb.pilc_logprobs_workspace_size(rows, n, top), dtype=torch.uint8, device=DEV)
    pb.pilc_logprobs(x, t, logp, entropy=entropy, lse=lse, top_sym=sym if top else None, top_logp=best if top else None, workspace=ws)
    some = sorted({0, rows // 2, rows - 1})
    x64, t64 = up(x[some]), t[some].cpu().numpy()
    law = orc.logprobs(x64, t64, 0)
    close(lse[some], law["lse"], law["lse_err"], torch.float32, "lse")
    close(entropy[some], law["entropy"], 3 * law["entropy_err"], torch.float32, "entropy")
    close(logp[some], law["logp_apart"], law["logp_apart_err"], torch.float32, "logp")
    if top:
        order = np.argsort(-x64, axis=1, kind="stable")[:, :top]       # the lower symbol first among equals
        assert np.array_equal(sym[some].cpu().numpy(), order)
        for k in range(top):
            at = orc.logprobs(x64, order[:, k], 0) if k in (0, top - 1) else None
            if at is not None:
                close(best[some, k], at["logp_apart"], at["logp_apart_err"], torch.float32, "alternative %d" % k)
