"""Layer norm over widths between those of test_gpu_fit_norm.py, over many narrow rows, and over as many rows as are counted."""
import numpy as np
import pytest
import torch

from fit_util import TYPES, close, up
from oracle import fit_oracle as orc
from paper_2206_05279_amd import binding as pb
from test_gpu_fit_norm import backward, forward, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_as_many_rows_as_32_bits_count():
    """2^32 - 1 rows, all alike: the count of rows does not wrap."""
    torch.cuda.empty_cache()
    rows, n, step = 2 ** 32 - 1, 8, 1 << 28
    rng = np.random.default_rng(8)
    one, by = rng.normal(size=(1, n)) * 1.5 + 1, rng.normal(size=(1, n))
    x = torch.from_numpy(one).to(torch.bfloat16).to(DEV).expand(rows, n).contiguous()
    dy = torch.from_numpy(by).to(torch.bfloat16).to(DEV).expand(rows, n).contiguous()
    x64, dy64 = up(x[:1]), up(dy[:1])
    wy, wmean, wrstd, e, _, _ = orc.norm_forward(x64, None, None, float(np.float32(1e-5)))
    mean, rstd = (torch.full((rows,), float(np.float32(v[0])), device=DEV) for v in (wmean, wrstd))
    want = orc.norm_backward(dy64, x64, None, up(mean[:1]), up(rstd[:1]))
    ws = torch.empty(pb.pilc_norm_workspace_size(rows, n), dtype=torch.uint8, device=DEV)
    pb.pilc_norm_backward(dy, x, None, mean, rstd, dy, workspace=ws)
    pb.pilc_norm_forward(x, None, None, x)
    close(dy[-1:], want[0], want[3], torch.bfloat16, "dx")
    close(x[-1:], wy, e, torch.bfloat16, "y")
    for t in (dy, x):
        assert all(bool((t[a:a + step] == t[-1]).all()) for a in range(0, rows, step))
    del x, dy, mean, rstd, ws
    torch.cuda.empty_cache()


# rows that sixteen wavefronts hold as 32 values a lane, their weights read anew for each; 600: more than there are workgroups
LONG = [(3, 16385, 0, 0), (2, 20000, 3, 5), (1, 24576, 0, 1), (2, 32767, 1, 0), (2, 32768, 0, 0), (600, 17001, 0, 0)]
KINDS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")]


@pytest.mark.parametrize("dtype,wtype", KINDS)
@pytest.mark.parametrize("rows,n,pad,shift", LONG)
@pytest.mark.parametrize("in_place", [False, True])
def test_rows_of_sixteen_wavefronts(dtype, wtype, rows, n, pad, shift, in_place):
    rng = np.random.default_rng(rows + n)
    x, w = values(rng, rows, n), 1 + rng.normal(size=n) * 0.3
    forward(x, w, rng.normal(size=n), TYPES[dtype], TYPES[wtype], pad=pad, shift=shift, in_place=in_place)
    backward(rng.normal(size=(rows, n)), x, w, TYPES[dtype], TYPES[wtype], pad, shift, in_place=in_place)


@pytest.mark.parametrize("wanted", [(True, False, False), (False, True, True), (False, False, True)])
@pytest.mark.parametrize("n", [5, 20001])
def test_what_is_wanted_of_narrow_and_of_long_rows(n, wanted):
    rng = np.random.default_rng(n)
    backward(rng.normal(size=(300, n)), values(rng, 300, n), None, torch.bfloat16, torch.bfloat16, wanted=wanted)


@pytest.mark.parametrize("dtype,wtype", KINDS)
@pytest.mark.parametrize("rows,n", [(100000, 5), (70000, 7), (66000, 1)])
def test_many_rows_of_less_than_a_pack(dtype, wtype, rows, n):
    """More rows than a workgroup a compute unit has threads: each goes on to another, and there is more than one part."""
    rng = np.random.default_rng(n)
    x, w = values(rng, rows, n), 1 + rng.normal(size=n) * 0.3
    forward(x, w, rng.normal(size=n), TYPES[dtype], TYPES[wtype], in_place=n == 7)
    backward(rng.normal(size=(rows, n)), x, w, TYPES[dtype], TYPES[wtype], in_place=n == 7)


def test_weights_gradients_of_the_widest_rows():
    """More columns than one launch has threads for: 64 of them take 1024 threads."""
    torch.cuda.empty_cache()
    n = (1 << 28) + 72
    g = torch.Generator(device=DEV).manual_seed(3)
    x, dy = (torch.randint(-8, 9, (1, n), generator=g, device=DEV, dtype=torch.int8).to(torch.bfloat16) for _ in range(2))
    mean, rstd = torch.full((1,), 0.5, device=DEV), torch.full((1,), 2.0, device=DEV)
    dw, db = torch.full((n,), 77.0, dtype=torch.bfloat16, device=DEV), torch.full((n,), 77.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(pb.pilc_norm_workspace_size(1, n), dtype=torch.uint8, device=DEV)
    pb.pilc_norm_backward(dy, x, None, mean, rstd, None, dw, db, workspace=ws)
    assert torch.equal(db, dy[0])
    assert torch.equal(dw, (dy[0].float() * (2 * x[0].float() - 1)).to(torch.bfloat16))     # whole numbers up to 136
    del x, dy, dw, db, ws
    torch.cuda.empty_cache()
