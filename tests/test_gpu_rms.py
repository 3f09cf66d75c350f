"""pilc_rms_forward and pilc_rms_backward against the 64-bit reference."""
import numpy as np
import pytest
import torch

from block8_util import around, room, workspace
from fit_util import TYPES, close, placed, up
from oracle import block8_oracle as orc
from oracle.fit_oracle import U
from paper_2206_05279_amd import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

#       rows width pad shift
SIZES = [(1, 1, 0, 0), (3, 2, 0, 0), (4, 7, 1, 1), (9, 8, 0, 0), (2, 63, 0, 0), (40, 64, 0, 0), (4, 65, 3, 1), (300, 96, 0, 0), (5, 127, 0, 0),
         (5, 256, 0, 0), (7, 300, 0, 1), (7, 1024, 0, 0), (3, 1000, 24, 8), (5, 1537, 0, 0), (2, 2048, 0, 0), (9, 4096, 0, 0), (2, 4100, 4, 2),
         (3, 8192, 0, 0), (2, 12289, 0, 0), (1, 16384, 0, 0), (3, 20000, 0, 0), (2, 32767, 0, 0), (2, 40001, 1, 0), (2, 65536, 0, 0)]
KINDS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")]


def values(rng, rows, n):
    return rng.normal(size=(rows, n)) * np.exp(rng.normal(size=(1, n)) * 0.7)


def forward(x, add, w, dtype, wtype, kind="e4m3", pad=0, shift=0, sum_in=None, y_in=False, wanted="ycsr", eps=1e-5):
    rows, n = x.shape
    xt, x_whole = placed(x, dtype, pad, shift)
    at = None if add is None else placed(add, dtype, pad + 1, shift)[0]
    wt = None if w is None else torch.from_numpy(w).to(wtype).to(DEV)
    gaps = torch.isnan(x_whole)
    x64, a64 = up(xt), 0.0 if at is None else up(at)
    out = lambda: placed(np.full(x.shape, 55.0), dtype, pad)[0]  # noqa: E731
    s = {None: out, "x": lambda: xt, "add": lambda: at}[sum_in]() if "s" in wanted else None
    y = (xt if y_in else out()) if "y" in wanted else None
    held, codes, scales, whole = room(rows, n, kind, 1, pad, shift, pad) if "c" in wanted else (None,) * 4
    rstd = torch.full((rows,), 77.0, device=DEV) if "r" in wanted else None
    pb.pilc_rms_forward(xt, wt, y=y, y8=held, add=at, sum=s, rstd=rstd, eps=eps)
    total = x64 + a64
    if s is not None:
        close(s, total, U * np.abs(total), dtype, "sum")
        h = up(s)
    else:
        h = torch.from_numpy(total).to(torch.float32).to(dtype).double().numpy()
    want, want_rstd, y_rel, rstd_rel = orc.rms_forward(h, None if w is None else up(wt), float(np.float32(eps)))
    if rstd is not None:
        close(rstd, want_rstd, want_rstd * rstd_rel, torch.float32, "rstd")
    if y is not None:
        close(y, want, np.abs(want) * y_rel[:, None], dtype, "y")
    if held is not None:
        assert orc.held_by(codes.cpu().numpy(), scales.cpu().numpy(), want, y_rel, kind), "codes"
        assert around(whole[0], codes) and around(whole[1], scales)
    assert torch.isnan(x_whole[gaps]).all()


@pytest.mark.parametrize("dtype,wtype", KINDS)
@pytest.mark.parametrize("rows,n,pad,shift", SIZES)
def test_forward(dtype, wtype, rows, n, pad, shift):
    rng = np.random.default_rng(rows + n)
    x, add, w = values(rng, rows, n), rng.normal(size=(rows, n)), 1 + rng.normal(size=n) * 0.3
    forward(x, add, w, TYPES[dtype], TYPES[wtype], "e4m3" if n % 2 else "e5m2", pad, shift)
    forward(x, add, w, TYPES[dtype], TYPES[wtype], "e4m3", pad, shift, sum_in="x" if n % 2 else "add", wanted="csr")
    forward(x, None, w, TYPES[dtype], TYPES[wtype], "e4m3", pad, shift, y_in=True, wanted="yr")


@pytest.mark.parametrize("wanted", ["y", "c", "s", "r", "sy", "yc", "cr"])
@pytest.mark.parametrize("n", [200, 40000])
def test_what_is_not_wanted_is_left_out(wanted, n):
    rng = np.random.default_rng(4)
    forward(values(rng, 3, n), rng.normal(size=(3, n)), None, torch.bfloat16, torch.bfloat16, wanted=wanted)
    forward(values(rng, 3, n), None, rng.normal(size=n), torch.float32, torch.float32, wanted=wanted)


@pytest.mark.parametrize("n", [5, 100, 4096, 40000])
def test_rows_of_zeros_and_of_the_largest(n):
    """Zeros have nothing to divide by but eps; sums of squares up to 32 bits' range hold."""
    x = np.zeros((4, n))
    x[1], x[2, 0], x[3] = 1e-20, 1e15, 3e17 / np.sqrt(n)
    forward(x, None, None, torch.float32, torch.float32)


def test_what_is_not_a_number_stays_in_its_row():
    x = np.random.default_rng(5).normal(size=(4, 300))
    x[1, 7], x[2, 299] = np.nan, np.inf
    xt, _ = placed(x, torch.float32)
    y = torch.empty_like(xt)
    held, codes, scales, _ = room(4, 300, "e4m3")
    pb.pilc_rms_forward(xt, None, y, held)
    assert torch.isnan(y).any(1).cpu().numpy().tolist() == [False, True, True, False] and torch.isnan(y[1]).all()
    s = scales.cpu().numpy()
    assert (s[1] == 255).all() and s[2, 2] == 255 and (s[0] < 255).all() and (s[3] < 255).all()


def backward(dy, h, w, ds, dtype, wtype, pad=0, shift=0, dx_in=None, wanted="xw"):
    rows, n = h.shape
    ht, _ = placed(h, dtype, pad, shift)
    dyt, dy_whole = placed(dy, dtype, pad, shift)
    dst = None if ds is None else placed(ds, dtype, pad, 0)[0]
    wt = None if w is None else torch.from_numpy(w).to(wtype).to(DEV)
    rstd = (1 / torch.sqrt(ht.double().square().mean(1) + 1e-5)).float()
    gaps = torch.isnan(dy_whole)
    want = orc.rms_backward(up(dyt), up(ht), None if w is None else up(wt), up(rstd), None if ds is None else up(dst))
    dx = {None: lambda: placed(np.full(h.shape, 55.0), dtype, pad)[0], "dy": lambda: dyt, "ds": lambda: dst}[dx_in]() if "x" in wanted else None
    dw = torch.full((n,), 55.0, dtype=wtype, device=DEV) if "w" in wanted else None
    pb.pilc_rms_backward(dyt, ht, wt, rstd, dx=dx, dweight=dw, dsum=dst, workspace=workspace(pb.pilc_rms_workspace_size(rows, n)))
    if dx is not None:
        close(dx, want[0], want[2], dtype, "dx")
    if dw is not None:
        close(dw, want[1], want[3], wtype, "dweight")
    assert torch.isnan(dy_whole[gaps]).all()


@pytest.mark.parametrize("dtype,wtype", KINDS)
@pytest.mark.parametrize("rows,n,pad,shift", SIZES + [(600, 300, 0, 0), (3000, 20, 1, 0), (1200, 4096, 0, 0)])
def test_backward(dtype, wtype, rows, n, pad, shift):
    rng = np.random.default_rng(rows + n)
    dy, h, w, ds = rng.normal(size=(rows, n)), values(rng, rows, n), 1 + rng.normal(size=n) * 0.3, rng.normal(size=(rows, n))
    backward(dy, h, w, ds, TYPES[dtype], TYPES[wtype], pad, shift)
    backward(dy, h, None, None, TYPES[dtype], TYPES[wtype], pad, shift, dx_in="dy")


@pytest.mark.parametrize("n", [200, 20000, 40000])
def test_backward_where_one_is_wanted_and_in_place(n):
    rng = np.random.default_rng(6)
    dy, h, w, ds = rng.normal(size=(50, n)), values(rng, 50, n), 1 + rng.normal(size=n) * 0.3, rng.normal(size=(50, n))
    backward(dy, h, w, ds, torch.bfloat16, torch.float32, wanted="x")
    backward(dy, h, w, ds, torch.bfloat16, torch.float32, wanted="w")
    backward(dy, h, w, ds, torch.bfloat16, torch.bfloat16, dx_in="ds")
    backward(dy, h, w, ds, torch.float32, torch.float32, dx_in="dy")


def test_gradients_are_the_differences():
    """In 32 bits, with steps of 2^-6: truncation h^2 / 6 of the third derivative, rounding 2^-24 over h."""
    rng = np.random.default_rng(8)
    h = rng.normal(size=(2, 24))
    w, dy, ds = 1 + 0.3 * rng.normal(size=24), rng.normal(size=(2, 24)), rng.normal(size=(2, 24))
    on = lambda v: torch.from_numpy(v).float().to(DEV)  # noqa: E731
    ht, wt = on(h), on(w)

    def loss(v, u):
        y = torch.empty_like(v)
        pb.pilc_rms_forward(v, u, y)
        return float((up(y) * dy).sum() + (up(v) * ds).sum())

    y, rstd, dx, dw = torch.empty_like(ht), torch.empty(2, device=DEV), torch.empty_like(ht), torch.empty(24, device=DEV)
    pb.pilc_rms_forward(ht, wt, y, rstd=rstd)
    pb.pilc_rms_backward(on(dy), ht, wt, rstd, dx, dw, dsum=on(ds), workspace=workspace(pb.pilc_rms_workspace_size(2, 24)))
    step = 2.0 ** -6
    for base, g, f in ((ht, dx, lambda v: loss(v, wt)), (wt, dw, lambda v: loss(ht, v))):
        for i in np.ndindex(tuple(base.shape)):
            a, b = base.clone(), base.clone()
            a[i] += step
            b[i] -= step
            assert abs((f(a) - f(b)) / (2 * step) - float(g[i])) < 4e-3


def test_no_rows():
    e, w = torch.empty(0, 33, dtype=torch.bfloat16, device=DEV), torch.rand(33, dtype=torch.bfloat16, device=DEV)
    none, dw = torch.empty(0, device=DEV), torch.full((33,), 7.0, dtype=torch.bfloat16, device=DEV)
    pb.pilc_rms_forward(e, w, e)
    pb.pilc_rms_backward(e, e, w, none, e, dw, workspace=workspace(256))
    assert (dw == 0).all()


def test_rows_beyond_32_bits():
    n, rows = 70000, 33000
    some = [0, 30679, 32999]
    rng = np.random.default_rng(4)
    x, dy = torch.zeros(rows, n, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, n, dtype=torch.bfloat16, device=DEV)
    x[some] = torch.from_numpy(values(rng, 3, n)).to(torch.bfloat16).to(DEV)
    dy[some] = torch.from_numpy(rng.normal(size=(3, n))).to(torch.bfloat16).to(DEV)
    y, rstd = torch.empty_like(x), torch.empty(rows, device=DEV)
    pb.pilc_rms_forward(x, None, y, rstd=rstd)
    want, _, y_rel, _ = orc.rms_forward(up(x[some]), None, float(np.float32(1e-5)))
    close(y[some], want, np.abs(want) * y_rel[:, None], torch.bfloat16, "y")
    dw = torch.empty(n, dtype=torch.bfloat16, device=DEV)
    back = orc.rms_backward(up(dy[some]), up(x[some]), None, up(rstd[some]), None)
    pb.pilc_rms_backward(dy, x, None, rstd, dy, dw, workspace=workspace(pb.pilc_rms_workspace_size(rows, n)))
    close(dy[some], back[0], back[2], torch.bfloat16, "dx")
    close(dw, back[1], back[3], torch.bfloat16, "dweight")


@pytest.mark.parametrize("n", [1100, 4096, 20000])
def test_same_bits_every_time_on_another_stream_and_in_a_graph(n):
    rng = np.random.default_rng(1)
    rows = 700
    xt, dyt, add = (placed(values(rng, rows, n), torch.bfloat16)[0] for _ in range(3))
    w = torch.rand(n, device=DEV)
    s, dx, dw, rstd = torch.empty_like(xt), torch.empty_like(xt), torch.empty(n, device=DEV), torch.empty(rows, device=DEV)
    held, codes, scales, _ = room(rows, n, "e4m3")
    ws = workspace(pb.pilc_rms_workspace_size(rows, n))

    def both(stream=None):
        pb.pilc_rms_forward(xt, w, None, held, add=add, sum=s, rstd=rstd, stream=stream)
        pb.pilc_rms_backward(dyt, s, w, rstd, dx, dw, dsum=add, workspace=ws, stream=stream)

    outs = (s, dx, dw, rstd, codes, scales)
    both()
    torch.cuda.synchronize()
    first = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    both(side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for _ in range(4):
        xt.normal_()
        both()
        torch.cuda.synchronize()
        first = [t.clone() for t in outs]
        ws.fill_(0x5A)
        for t in outs:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, outs))
