"""pilc_logprobs, pilc_logprobs_grad and pilc_logprobs_train against the 64-bit reference."""
import numpy as np
import pytest
import torch

from fit_util import LOWEST, TYPES, close, placed, up
from oracle import fit_oracle as orc
from paper_2206_05279_amd import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Case:
    def __init__(self, values, targets, dtype, target_type=torch.int64, top=0, pad=0, shift=0):
        self.dtype, self.top = dtype, top
        self.x, self.whole = placed(values, dtype, pad, shift)
        self.x64 = up(self.x)
        self.rows, self.n = values.shape
        self.t64 = np.asarray(targets, dtype=np.int64)
        self.t = torch.from_numpy(self.t64).to(target_type).to(DEV)
        self.ws = torch.full((pb.pilc_logprobs_workspace_size(self.rows, self.n, top),), 0xA5, dtype=torch.uint8, device=DEV)
        new = lambda *s, d=torch.float32: torch.full(s, 77, dtype=d, device=DEV)  # noqa: E731
        self.logp, self.entropy, self.lse = new(self.rows), new(self.rows), new(self.rows)
        self.top_sym, self.top_logp = new(self.rows, top, d=torch.int32), new(self.rows, top)
        self.law = orc.logprobs(self.x64, self.t64, top)

    def check_law(self):
        law = self.law
        close(self.lse, law["lse"], law["lse_err"], torch.float32, "lse")
        close(self.entropy, law["entropy"], law["entropy_err"], torch.float32, "entropy")
        close(self.logp, law["logp"], law["logp_err"], torch.float32, "logp")

    def forward(self):
        pb.pilc_logprobs(self.x, self.t, self.logp, entropy=self.entropy, lse=self.lse, top_sym=self.top_sym if self.top else None,
                         top_logp=self.top_logp if self.top else None, workspace=self.ws)
        self.check_law()
        if self.top:
            assert np.array_equal(self.top_sym.cpu().numpy(), self.law["top_sym"])
            lse = self.law["lse"][:, None]
            err = self.law["lse_err"][:, None] + orc.U * 4 * (np.abs(np.where(np.isfinite(lse), lse, 0)) + 1) + orc.U * 3 * np.where(
                np.isfinite(self.law["top_logp"]), np.abs(self.law["top_logp"]), 0)
            close(self.top_logp, self.law["top_logp"], err, torch.float32, "top_logp")

    def gradients(self, with_entropy=True, in_place=False, seed=3):
        rng = np.random.default_rng(seed)
        a = rng.normal(size=self.rows).astype(np.float32)
        b = rng.normal(size=self.rows).astype(np.float32) if with_entropy else None
        on = lambda v: None if v is None else torch.from_numpy(v).to(DEV)  # noqa: E731
        want, err = orc.logprobs_grad(self.x64, self.t64, a.astype(np.float64), None if b is None else b.astype(np.float64))
        gaps = torch.isnan(self.whole)
        grad, grad_whole = placed(np.full((self.rows, self.n), 55.0), self.dtype, pad=3, shift=1)
        pb.pilc_logprobs_train(self.x, self.t, on(a), self.logp, grad, entropy=self.entropy, lse=self.lse, up_entropy=on(b), workspace=self.ws)
        self.check_law()
        close(grad, want, err, self.dtype, "gradient, one call")
        pb.pilc_logprobs(self.x, self.t, self.logp, entropy=self.entropy, lse=self.lse, workspace=self.ws)
        target = self.x if in_place else placed(np.full((self.rows, self.n), 55.0), self.dtype)[0]
        pb.pilc_logprobs_grad(self.x, self.t, self.lse, on(a), target, entropy=self.entropy if with_entropy else None, up_entropy=on(b))
        close(target, want, err, self.dtype, "gradient by itself")
        if in_place:
            assert torch.isnan(self.whole[gaps]).all()          # nothing between the rows was written
            self.x.copy_(torch.from_numpy(self.x64).to(self.dtype))
            pb.pilc_logprobs_train(self.x, self.t, on(a), self.logp, self.x, entropy=self.entropy, lse=self.lse, up_entropy=on(b), workspace=self.ws)
            close(self.x, want, err, self.dtype, "gradient in place, one call")
            assert torch.isnan(self.whole[gaps]).all()


def law_values(rng, rows, n):
    return rng.normal(size=(rows, n)) * 3 + rng.normal(size=(rows, 1)) * 5


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,n,pad,shift", [
    (1, 1, 0, 0), (3, 2, 0, 0), (5, 63, 0, 0), (4, 64, 0, 0), (130, 256, 0, 0), (7, 255, 1, 0), (9, 257, 7, 3), (6, 1000, 24, 8),
    (3, 1024, 0, 1), (2, 4099, 5, 0), (5, 8192, 0, 0), (1, 32768, 0, 0), (2, 50001, 7, 0), (1, 131072, 0, 0), (1, 200003, 0, 5)])
def test_sizes_and_places(dtype, rows, n, pad, shift):
    rng = np.random.default_rng(rows * 7 + n)
    c = Case(law_values(rng, rows, n), rng.integers(0, n, rows), TYPES[dtype], top=5 if n < 60000 else 20, pad=pad, shift=shift)
    c.forward()
    c.gradients(in_place=n % 2 == 0)


@pytest.mark.parametrize("rows,n", [(9000, 3), (2050, 300), (40, 5000)])
def test_many_rows(rows, n):
    rng = np.random.default_rng(n)
    c = Case(law_values(rng, rows, n), rng.integers(0, n, rows), torch.float32, top=2)
    c.forward()
    c.gradients()


@pytest.mark.parametrize("target_type", [torch.uint8, torch.int32, torch.int64])
def test_types_of_targets_and_targets_that_do_not_count(target_type):
    rng = np.random.default_rng(1)
    t = rng.integers(0, 256, 33)
    if target_type != torch.uint8:
        t[[0, 5, 32]] = [-1, -100, -2 ** 31]
    c = Case(law_values(rng, 33, 256), t, torch.bfloat16, target_type)
    c.forward()
    c.gradients()
    c.gradients(with_entropy=False)


@pytest.mark.parametrize("n", [200, 20000, 150000])
def test_target_beyond_the_alphabet_is_nan(n):
    rng = np.random.default_rng(2)
    c = Case(law_values(rng, 3, n), [n, 1, 2 ** 40], torch.float32)
    c.forward()
    c.gradients()


@pytest.mark.parametrize("top", [0, 1, 5, 31, 32])
@pytest.mark.parametrize("n", [1, 20, 300, 3000, 70000])
def test_alternatives(n, top):
    rng = np.random.default_rng(n + top)
    Case(law_values(rng, 4, n), rng.integers(0, n, 4), torch.bfloat16, top=top).forward()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["same", "two", "rising", "falling", "signed_zero", "steps", "one_place"])
@pytest.mark.parametrize("n", [77, 256, 2500, 140000])
def test_alternatives_among_equals(dtype, kind, n):
    """The lower symbol comes first among equals, wherever the equals lie."""
    j = np.arange(n, dtype=np.float64)
    row = {"same": j * 0 + 1.5, "two": 1.0 + (j % 7 == 3), "rising": j / n, "falling": 1 - j / n, "signed_zero": np.where(j % 2, 0.0, -0.0),
           "steps": np.floor(j / 50) % 9, "one_place": np.where((j // 8) % 64 == 5, j / n + 4, -j / n)}[kind]
    values = np.stack([row, row[::-1], np.roll(row, n // 3)])
    Case(values, [0, n - 1, n // 2], TYPES[dtype], top=20).forward()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n", [5, 256, 999, 40000, 131073])
def test_masks(dtype, n):
    """Symbols ruled out by -inf or the type's lowest value, rows where nothing is left, rows that are not numbers."""
    rng = np.random.default_rng(n)
    v = law_values(rng, 12, n)
    v[0] = -np.inf
    v[1] = LOWEST[TYPES[dtype]]
    v[2, 1:] = -np.inf
    v[3, : n - 1] = LOWEST[TYPES[dtype]]
    v[4][rng.random(n) < 0.5] = -np.inf
    v[5, n // 2] = np.nan
    v[6, n - 1] = np.inf
    v[7] = -np.inf
    v[7, n // 2] = LOWEST[TYPES[dtype]]
    v[8] = -LOWEST[TYPES[dtype]]
    v[8, : n // 2] = LOWEST[TYPES[dtype]]
    v[9] = -np.inf
    v[9, n // 3] = np.nan
    v[10] = np.nan
    t = rng.integers(0, n, 12)
    t[4] = np.flatnonzero(v[4] == -np.inf)[0] if (v[4] == -np.inf).any() else 0     # a target that cannot occur
    t[10] = -1
    c = Case(v, t, TYPES[dtype], top=3, pad=2)
    c.forward()
    c.gradients()


def test_row_of_padding_gets_no_gradient_whatever_it_holds():
    v = np.full((2, 300), np.nan)
    c = Case(v, [-1, -1], torch.bfloat16)
    c.gradients(with_entropy=False)


def test_what_is_not_wanted_is_not_written_and_need_not_be_there():
    rng = np.random.default_rng(8)
    c = Case(law_values(rng, 5, 400), rng.integers(0, 400, 5), torch.float16, top=2)
    pb.pilc_logprobs(c.x, None, None, entropy=c.entropy, workspace=c.ws)
    close(c.entropy, c.law["entropy"], c.law["entropy_err"], torch.float32, "entropy alone")
    assert (c.lse == 77).all() and (c.logp == 77).all() and (c.top_sym == 77).all()
    pb.pilc_logprobs(c.x, c.t, None, top_sym=c.top_sym, top_logp=c.top_logp, workspace=c.ws)
    assert np.array_equal(c.top_sym.cpu().numpy(), c.law["top_sym"]) and (c.logp == 77).all()
    pb.pilc_logprobs(c.x, c.t, c.logp, workspace=c.ws)
    close(c.logp, c.law["logp"], c.law["logp_err"], torch.float32, "logp alone")


@pytest.mark.parametrize("rows,n", [(1, 3000), (100, 3000), (100, 1500), (127, 2500), (5, 70000), (40, 9000), (130, 200000), (3, 1100000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_training_without_lse_and_entropy_stays_in_its_workspace(rows, n, dtype):
    rng = np.random.default_rng(n)
    t = rng.integers(0, n, rows)
    x, _ = placed(rng.normal(size=(rows, n)), TYPES[dtype])
    size = pb.pilc_logprobs_workspace_size(rows, n)
    whole = torch.full((size + 8192,), 0x5A, dtype=torch.uint8, device=DEV)
    a, b = torch.ones(rows, device=DEV), torch.full((rows,), 0.5, device=DEV)
    logp, grad = torch.empty(rows, device=DEV), torch.empty_like(x)
    pb.pilc_logprobs_train(x, torch.from_numpy(t).to(DEV), a, logp, grad, up_entropy=b, workspace=whole[:size])
    assert (whole[size:] == 0x5A).all()
    some = [0, rows // 2, rows - 1]
    law = orc.logprobs(up(x[some]), t[some], 0)
    want, err = orc.logprobs_grad(up(x[some]), t[some], np.ones(3), np.full(3, 0.5))
    close(logp[some], law["logp"], law["logp_err"], torch.float32, "logp")
    close(grad[some], want, err, TYPES[dtype], "gradient")


def test_no_rows():
    e = torch.empty(0, 40, device=DEV)
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    none, t = torch.empty(0, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    assert pb.pilc_logprobs(e, t, none, workspace=ws) == pb.PILC_OK
    assert pb.pilc_logprobs_grad(e, t, none, none, e) == pb.PILC_OK
    assert pb.pilc_logprobs_train(e, t, none, none, e, workspace=ws) == pb.PILC_OK


def test_rows_beyond_32_bits():
    """Rows that begin more than 2^32 bytes and 2^31 elements into the tensor."""
    n, rows = 70000, 33000
    x = torch.zeros(rows, n, dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(4)
    some = [0, 30678, 32999]           # 30678 * 70000 is the first beyond 2^31
    x[some] = torch.from_numpy(law_values(rng, 3, n)).to(torch.bfloat16).to(DEV)
    t = torch.full((rows,), 3, dtype=torch.int32, device=DEV)
    logp, lse, up_logp = (torch.ones(rows, device=DEV) for _ in range(3))
    ws = torch.empty(pb.pilc_logprobs_workspace_size(rows, n), dtype=torch.uint8, device=DEV)
    x64 = up(x[some])
    law = orc.logprobs(x64, np.full(3, 3), 0)
    want, err = orc.logprobs_grad(x64, np.full(3, 3), np.ones(3), None)
    pb.pilc_logprobs_train(x, t, up_logp, logp, x, lse=lse, workspace=ws)
    close(logp[some], law["logp"], law["logp_err"], torch.float32, "logp")
    close(x[some], want, err, torch.bfloat16, "gradient")


def test_gradient_against_differences_of_the_kernel():
    """The kernel's own log probabilities, a step apart, against its gradient."""
    rng = np.random.default_rng(12)
    v, t = rng.normal(size=(1, 9)), np.array([4])
    c = Case(v, t, torch.float32)
    c.gradients(with_entropy=False, seed=1)
    a = np.random.default_rng(1).normal(size=1).astype(np.float32)
    h = 2.0 ** -7
    grad, _ = orc.logprobs_grad(c.x64, t, a.astype(np.float64), None)
    stepped = np.repeat(c.x64, 18, 0)
    for j in range(9):
        stepped[2 * j, j] += h
        stepped[2 * j + 1, j] -= h
    d = Case(stepped, np.repeat(t, 18), torch.float32)
    d.forward()
    got = up(d.logp)
    diff = a[0] * (got[0::2] - got[1::2]) / (2 * h)
    # truncation: h^2 / 6 times a third derivative of at most 1; the lengths' own errors over 2 h
    bound = abs(a[0]) * (h * h / 6 + (d.law["logp_err"].max() + 1e-7) / h)
    assert np.abs(diff - grad[0]).max() <= bound


def test_other_streams_and_replays_of_a_graph():
    rng = np.random.default_rng(6)
    c = Case(law_values(rng, 20, 30000), rng.integers(0, 30000, 20), torch.bfloat16, top=4)
    a = torch.rand(20, device=DEV)
    grad = torch.empty_like(c.x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def both():
        pb.pilc_logprobs(c.x, c.t, c.logp, entropy=c.entropy, lse=c.lse, top_sym=c.top_sym, top_logp=c.top_logp, workspace=c.ws)
        pb.pilc_logprobs_grad(c.x, c.t, c.lse, a, grad)

    with torch.cuda.stream(side):
        both()
    side.synchronize()
    c.check_law()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for turn in range(4):
        values = law_values(rng, 20, 30000)
        c.x.copy_(torch.from_numpy(values).to(c.dtype))
        for o in (c.logp, c.entropy, c.lse, c.top_logp, grad):
            o.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        seen = [o.clone() for o in (c.logp, c.entropy, c.lse, c.top_sym, c.top_logp, grad)]
        both()
        torch.cuda.synchronize()
        for s, o in zip(seen, (c.logp, c.entropy, c.lse, c.top_sym, c.top_logp, grad)):
            assert torch.equal(s, o), turn
        c.x64 = up(c.x)
        c.law = orc.logprobs(c.x64, c.t64, 4)
        c.check_law()


def test_same_bits_every_time():
    rng = np.random.default_rng(9)
    c = Case(law_values(rng, 3, 90000), rng.integers(0, 90000, 3), torch.bfloat16, top=10)
    c.forward()
    first = [t.clone() for t in (c.logp, c.entropy, c.lse, c.top_sym, c.top_logp)]
    for _ in range(5):
        c.forward()
        assert all(torch.equal(p, q) for p, q in zip(first, (c.logp, c.entropy, c.lse, c.top_sym, c.top_logp)))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n", [2, 3, 7])
def test_nearly_certain_symbol_of_a_short_row_keeps_its_digits(n, dtype):
    if n * torch.empty(0, dtype=TYPES[dtype]).element_size() >= 16:
        pytest.skip("as long as a pack")
    rng = np.random.default_rng(n)
    rows = 400
    values = rng.uniform(4.0, 6.0, (rows, n))
    targets = rng.integers(0, n, rows)
    values[np.arange(rows), targets] += rng.uniform(4.0, 12.0, rows)
    c = Case(values, targets, TYPES[dtype])
    c.forward()
    z = c.x64 - c.x64[np.arange(rows), targets][:, None]
    z[np.arange(rows), targets] = -np.inf
    want = -np.log1p(np.exp(z).sum(1))
    # a power of two's exponent is below 24, rounded twice (24 units of 2^-24 each), and the power, the sum of six, the quotient
    # and the logarithm take less than 16: 64 units are room enough, where 1 - p by itself would leave none
    off = np.abs(c.logp.cpu().double().numpy() / want - 1)
    assert off.max() <= 2.0 ** -18, off.max()
