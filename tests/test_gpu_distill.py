"""pilc_distill against the 64-bit reference."""
import numpy as np
import pytest
import torch

from block8_util import workspace
from fit_util import LOWEST, TYPES, close, placed, up
from oracle import block8_oracle as orc
from paper_2206_05279_amd import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

#        rows  n      top
SIZES = [(1, 1, 1), (5, 2, 2), (300, 3, 5), (4, 7, 128), (9, 8, 3), (70, 64, 16), (33, 65, 7), (35, 40, 128), (50, 200, 128), (40, 256, 16), (20, 500, 128), (9, 1000, 64), (7, 2048, 1),
         (5, 5003, 50), (3, 8192, 128), (4, 16385, 32), (2, 32769, 20), (3, 50001, 64), (1, 100003, 128), (2, 131072, 64)]


def inputs(rows, n, top, rest, seed=0):
    """A student, and a teacher who agrees with it more or less; entries in no order, some of them missing, some named twice."""
    rng = np.random.default_rng(rows * 7 + n * 3 + top + seed)
    x = rng.normal(size=(rows, n)) * 2.5
    t = x + rng.normal(size=(rows, n))
    sym = np.full((rows, top), -1, np.int32)
    value = np.full((rows, top), -np.inf)
    lse = np.log(np.exp(t - t.max(1, keepdims=True)).sum(1)) + t.max(1)
    for r in range(rows):
        k = min(n, top)
        best = rng.permutation(np.argsort(-t[r])[:k])
        sym[r, :k], value[r, :k] = best, t[r, best] - (lse[r] if rest else 0)
    if rows > 2:
        drop = rng.random(sym.shape) < 0.2
        drop[0] = False
        sym[drop] = -1
        sym[2] = -5
    if rows > 3 and top > 2:
        sym[3, 1] = sym[3, 0] = max(sym[3, 0], 0)
        value[3, :2] -= 0.5 * rest
    return x, sym, value.astype(np.float32)


def run(x, sym, value, dtype, temperature, rest, grad, pad=0, shift=0, in_place=False, up_zero=None):
    rows, n = x.shape
    xt, whole = placed(x, dtype, pad, shift)
    st, vt = torch.from_numpy(sym.astype(np.int32)).to(DEV), torch.from_numpy(value.astype(np.float32)).to(DEV)
    x64 = up(xt)
    gaps = torch.isnan(whole)
    rng = np.random.default_rng(1)
    weight = rng.normal(size=rows).astype(np.float32) if grad else None
    if grad and up_zero is not None:
        weight[up_zero] = 0
    ut = torch.from_numpy(weight).to(DEV) if grad else None
    g = None if not grad else xt if in_place else placed(np.full(x.shape, 55.0), dtype, pad + 1)[0]
    loss = torch.full((rows,), 55.0, device=DEV)
    pb.pilc_distill(xt, st, vt, loss, up=ut, grad=g, temperature=temperature, rest=rest,
                    workspace=workspace(pb.pilc_distill_workspace_size(rows, n, sym.shape[1])))
    want, want_g, err, g_err = orc.distill(x64, sym, value.astype(np.float64), weight, float(np.float32(temperature)), rest)
    close(loss, want, err, torch.float32, "loss")
    if grad:
        close(g, want_g, g_err, dtype, "gradient")
    if not np.isnan(x).any():
        assert torch.isnan(whole[gaps]).all()
    return loss, g


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n,top", SIZES)
@pytest.mark.parametrize("rest", [False, True])
def test_losses_and_gradients(dtype, rows, n, top, rest):
    x, sym, value = inputs(rows, n, top, rest)
    pad, shift = n % 3, n % 2
    run(x, sym, value, TYPES[dtype], 1.0, rest, True, pad, shift)
    run(x, sym, value, TYPES[dtype], 2.5, rest, True, pad, shift, in_place=True)
    run(x, sym, value, TYPES[dtype], 0.7, rest, False, pad, shift)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,n", [(300, 17000), (200, 40000), (140, 70000), (130, 131073)])
def test_many_long_rows(rows, n, rest):
    x, sym, value = inputs(8, n, 40, rest)
    many = lambda v: np.resize(v, (rows, v.shape[1]))  # noqa: E731
    xt = torch.from_numpy(x).to(torch.bfloat16).to(DEV).repeat(-(-rows // 8), 1)[:rows].contiguous()
    weight = torch.linspace(0.5, 2, rows, device=DEV)
    loss, g = torch.empty(rows, device=DEV), torch.empty_like(xt)
    pb.pilc_distill(xt, torch.from_numpy(many(sym)).to(DEV), torch.from_numpy(many(value)).to(DEV), loss, up=weight, grad=g, rest=rest,
                    workspace=workspace(pb.pilc_distill_workspace_size(rows, n, 40)))
    some = list(range(4)) + list(range(rows - 8, rows))
    want, want_g, err, g_err = orc.distill(up(xt[some]), many(sym)[some], many(value)[some].astype(float), up(weight[some]), 1.0, rest)
    close(loss[some], want, err, torch.float32, "loss")
    close(g[some], want_g, g_err, torch.bfloat16, "gradient")


SHAPES = [3, 100, 5000, 40000, 140000]


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n", SHAPES)
def test_masks(n, rest):
    """Logits ruled out, rows without a law, named symbols that are ruled out or everything there is, the lowest numbers."""
    x, sym, value = inputs(8, n, 6, rest)
    rng = np.random.default_rng(n)
    x[rng.random(x.shape) < 0.3] = -np.inf
    x[1] = -np.inf                            # no law
    x[4, :] = -np.inf
    x[4, sym[4][sym[4] >= 0]] = 1.0           # nothing but what is named
    x[5, np.maximum(sym[5], 0)] = -np.inf     # nothing of what is named
    x[6, ::2] = LOWEST[torch.float32]
    value[7] = -np.inf                        # named, without mass
    run(x, sym, value, torch.float32, 1.0, rest, True)
    run(np.where(x < -60000, -np.inf, x), sym, value, torch.float16, 2.0, rest, True, in_place=True)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n", SHAPES)
def test_rows_that_are_spoilt(n, rest):
    x, sym, value = inputs(9, n, 6, rest)
    sym[:, 0] = 0
    value[:, 0] = -1.0
    x[0, 0], x[1, n - 1] = np.nan, np.inf
    sym[2, 0], sym[4, 5] = n, 1 << 30
    value[5, 0] = np.nan
    x[6], x[7, :], value[7, 0] = np.nan, -np.inf, np.inf
    sym[8] = -1
    x[8, 0] = np.nan                          # not looked at
    run(x, sym, value, torch.float32, 1.0, rest, True)
    run(x, sym, value, torch.float32, 1.0, rest, False)
    run(x, sym, value, torch.bfloat16, 1.0, rest, True, up_zero=[0, 2, 5, 6])


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n,top", [(5, 128), (300, 128), (9000, 128), (40000, 128), (140000, 128), (40000, 65)])
def test_symbols_side_by_side_and_named_again_and_again(n, top, rest):
    """Entries that share 16 bytes of a row, all of the same symbol, and at the row's very end."""
    x, sym, value = inputs(6, n, top, rest)
    rng = np.random.default_rng(top)
    sym[0] = rng.permutation(np.arange(top) % n)
    sym[1] = n - 1
    sym[3] = n - 1 - rng.permutation(np.arange(top) % min(n, 40))
    sym[4] = rng.integers(0, min(n, 3), top)
    sym[5, ::2], sym[5, 1::2] = 0, n - 1
    value[:] = -np.log(2.0 * top) - rng.random(value.shape) if rest else value
    value[np.isinf(value)] = -20.0
    run(x, sym, value, torch.float32, 1.0, rest, True)
    run(x, sym, value, torch.bfloat16, 2.0, rest, True, in_place=True)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n", [5, 300, 40000, 140000])
def test_far_logits_and_one_sided_laws(n, rest):
    """Offsets that 32 bits hardly hold, a student that is certain of what is named, or of what is not: a rest of next to nothing."""
    x, sym, value = inputs(6, n, 3, rest)
    x[0] += 1e6
    x[1] -= 1e8
    named = np.maximum(sym, 0)
    x[3, named[3]] += 40.0
    x[4] += 60.0
    x[4, named[4]] -= 60.0
    x[5, named[5]] += 120.0                   # the rest's powers are no number of 32 bits beside theirs
    run(x, sym, value, torch.float32, 1.0, rest, True)
    run(x, sym, value, torch.float32, 4.0, rest, True)


@pytest.mark.parametrize("n", [256, 30000])
def test_gradient_is_the_difference(n):
    """Of the loss in 32 bits, along random directions: truncation h^2 of the third derivative, rounding 2^-24 of the loss over h."""
    for rest in (False, True):
        x, sym, value = inputs(1, n, 8, rest)
        rng = np.random.default_rng(2)
        xt = torch.from_numpy(x).float().to(DEV)
        st, vt, ws = torch.from_numpy(sym).to(DEV), torch.from_numpy(value).to(DEV), workspace(pb.pilc_distill_workspace_size(1, n, 8))
        loss, g, one = torch.empty(1, device=DEV), torch.empty_like(xt), torch.ones(1, device=DEV)
        pb.pilc_distill(xt, st, vt, loss, up=one, grad=g, rest=rest, workspace=ws)
        for _ in range(4):
            d = torch.from_numpy(rng.normal(size=x.shape)).float().to(DEV)
            at = []
            for h in (0.02, -0.02):
                pb.pilc_distill(xt + h * d, st, vt, loss, rest=rest, workspace=ws)
                at.append(float(loss))
            assert abs((at[0] - at[1]) / 0.04 - float((g.double() * d.double()).sum())) < 2e-3


def test_what_log_probabilities_answer_with_is_what_distillation_takes():
    """A teacher's top_sym and top_logp as they come; a student that is the teacher loses nothing."""
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.normal(size=(50, 700)) * 3).float().to(DEV)
    x[7, 3:] = -np.inf                        # fewer symbols than entries
    sym, logp = torch.empty(50, 32, dtype=torch.int32, device=DEV), torch.empty(50, 32, device=DEV)
    pb.pilc_logprobs(x, None, top_sym=sym, top_logp=logp, workspace=workspace(pb.pilc_logprobs_workspace_size(50, 700, 32)))
    loss, g, one = torch.empty(50, device=DEV), torch.empty_like(x), torch.ones(50, device=DEV)
    pb.pilc_distill(x, sym, logp, loss, up=one, grad=g, rest=True, workspace=workspace(pb.pilc_distill_workspace_size(50, 700, 32)))
    want, want_g, err, g_err = orc.distill(up(x), sym.cpu().numpy(), up(logp), up(one), 1.0, True)
    close(loss, want, err, torch.float32, "loss")
    close(g, want_g, g_err, torch.float32, "gradient")
    assert float(loss.abs().max()) < 1e-5 and float(g.abs().max()) < 1e-5


def test_no_rows():
    e = torch.empty(0, 33, device=DEV)
    pb.pilc_distill(e, torch.empty(0, 4, dtype=torch.int32, device=DEV), torch.empty(0, 4, device=DEV), torch.empty(0, device=DEV), workspace=workspace(256))


def test_rows_beyond_32_bits():
    rows, n, some = 33000, 131072, [0, 32768, 32999]
    x, sym, value = inputs(3, n, 5, True)
    sym[:] = np.abs(sym)
    xt = torch.zeros(rows, n, dtype=torch.bfloat16, device=DEV)
    xt[some] = torch.from_numpy(x).to(torch.bfloat16).to(DEV)
    st, vt = torch.full((rows, 5), -1, dtype=torch.int32, device=DEV), torch.zeros(rows, 5, device=DEV)
    st[some], vt[some] = torch.from_numpy(sym).to(DEV), torch.from_numpy(value).to(DEV)
    want, want_g, err, g_err = orc.distill(up(xt[some]), sym, value.astype(float), np.ones(3), 1.0, True)
    loss = torch.empty(rows, device=DEV)
    pb.pilc_distill(xt, st, vt, loss, up=torch.ones(rows, device=DEV), grad=xt, rest=True, workspace=workspace(pb.pilc_distill_workspace_size(rows, n, 5)))
    close(loss[some], want, err, torch.float32, "loss")
    close(xt[some], want_g, g_err, torch.bfloat16, "gradient")
    assert (xt[1:32768] == 0).all()


@pytest.mark.parametrize("rest", [False, True])
def test_more_rows_than_a_launch_takes(rest):
    """Rows of eight symbols go 32 to a workgroup and 2^20 workgroups to a launch: the rows of the second answer as the first's do."""
    rows, some = (1 << 25) + 77, 1000
    x, sym, value = inputs(some, 8, 2, rest)
    base = torch.from_numpy(x).to(torch.bfloat16).to(DEV)
    many = lambda t: t.repeat(-(-rows // some), 1)[:rows]  # noqa: E731
    xt, st, vt = many(base), many(torch.from_numpy(sym).to(DEV)), many(torch.from_numpy(value).to(DEV))
    loss, one = torch.empty(rows, device=DEV), torch.ones(rows, device=DEV)
    pb.pilc_distill(xt, st, vt, loss, up=one, grad=xt, rest=rest, workspace=workspace(pb.pilc_distill_workspace_size(rows, 8, 2)))
    want, want_g, err, g_err = orc.distill(up(base), sym, value.astype(float), np.ones(some), 1.0, rest)
    close(loss[:some], want, err, torch.float32, "loss")
    close(xt[:some], want_g, g_err, torch.bfloat16, "gradient")
    whole = rows // some * some
    assert (loss[:whole].view(-1, some) == loss[:some]).all() and torch.equal(loss[whole:], loss[:rows - whole])
    assert (xt[:whole].view(-1, some, 8) == xt[:some]).all() and torch.equal(xt[whole:], xt[:rows - whole])


@pytest.mark.parametrize("rows,n,rest", [(3000, 256, False), (40, 5000, True), (300, 40000, True), (5, 150000, True)])
def test_same_bits_every_time_on_another_stream_and_in_a_graph(rows, n, rest):
    x, sym, value = inputs(min(rows, 40), n, 16, rest)
    many = lambda v: torch.from_numpy(np.resize(v, (rows, v.shape[1]))).to(DEV)  # noqa: E731
    xt, st, vt = many(x.astype(np.float32)).to(torch.bfloat16), many(sym), many(value)
    loss, g, one = torch.empty(rows, device=DEV), torch.empty_like(xt), torch.rand(rows, device=DEV)
    ws = workspace(pb.pilc_distill_workspace_size(rows, n, 16))

    def go(stream=None):
        pb.pilc_distill(xt, st, vt, loss, up=one, grad=g, rest=rest, workspace=ws, stream=stream)

    go()
    torch.cuda.synchronize()
    first = [loss.clone(), g.clone()]
    side = torch.cuda.Stream()
    go(side)
    side.synchronize()
    assert torch.equal(first[0], loss) and torch.equal(first[1], g)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        go()
    for _ in range(4):
        xt.normal_()
        go()
        torch.cuda.synchronize()
        first = [loss.clone(), g.clone()]
        ws.fill_(0x5A)
        loss.fill_(7)
        g.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first[0], loss) and torch.equal(first[1], g)
