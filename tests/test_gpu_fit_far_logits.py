"""Log probabilities of logits that lie far from zero: rows ruled out by large finite numbers, and offsets that leave little of
lse.  What does not pass through one 32-bit lse is held to bounds without a share of |lse|."""
import numpy as np
import pytest
import torch

from fit_util import LOWEST, TYPES, close, placed, up
from oracle import fit_oracle as orc
from paper_2206_05279_amd import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Rows:
    """Rows of logits, what the calls say of them and what they should."""

    def __init__(self, values, targets, dtype, seed=0):
        rng = np.random.default_rng(seed)
        self.dtype, (self.rows, self.n) = dtype, values.shape
        self.x, _ = placed(values, dtype, pad=1)
        self.x64, self.t64 = up(self.x), np.asarray(targets, dtype=np.int64)
        self.t = torch.from_numpy(self.t64).to(DEV)
        self.ws = torch.empty(pb.pilc_logprobs_workspace_size(self.rows, self.n, 3), dtype=torch.uint8, device=DEV)
        self.ws_train = torch.empty(pb.pilc_logprobs_workspace_size(self.rows, self.n), dtype=torch.uint8, device=DEV)
        self.a, self.b = (rng.normal(size=self.rows).astype(np.float32) for _ in range(2))
        self.law = orc.logprobs(self.x64, self.t64, 0)

    def outputs(self):
        return [torch.full((self.rows,), 77.0, device=DEV) for _ in range(3)]

    def check_law(self, logp, entropy, lse, what):
        law = self.law
        close(lse, law["lse"], law["lse_err"], torch.float32, what + ": lse")
        close(entropy, law["entropy"], 3 * law["entropy_err"], torch.float32, what + ": entropy")
        close(logp, law["logp_apart"], law["logp_apart_err"], torch.float32, what + ": logp")

    def forward(self, alternatives=False):
        logp, entropy, lse = self.outputs()
        sym, best = torch.empty(self.rows, 3, dtype=torch.int32, device=DEV), torch.empty(self.rows, 3, device=DEV)
        pb.pilc_logprobs(self.x, self.t, logp, entropy=entropy, lse=lse, top_sym=sym if alternatives else None,
                         top_logp=best if alternatives else None, workspace=self.ws)
        self.check_law(logp, entropy, lse, "law")
        if alternatives:
            law = orc.logprobs(self.x64, self.t64, 3)
            assert np.array_equal(sym.cpu().numpy(), law["top_sym"])
            for k in range(3):
                at = orc.logprobs(self.x64, law["top_sym"][:, k], 0)
                there = law["top_sym"][:, k] >= 0
                want = np.where(there, at["logp_apart"], np.where(np.isnan(law["lse"]), np.nan, -np.inf))
                close(best[:, k], want, at["logp_apart_err"], torch.float32, "alternative %d" % k)
        return lse, entropy

    def train(self, with_entropy=True, in_place=False):
        logp, entropy, lse = self.outputs()
        on = lambda v: torch.from_numpy(v).to(DEV)  # noqa: E731
        b = self.b if with_entropy else None
        want, err = orc.logprobs_grad(self.x64, self.t64, self.a.astype(np.float64), None if b is None else b.astype(np.float64), apart=True)
        grad = self.x if in_place else torch.full((self.rows, self.n), 55.0, dtype=self.dtype, device=DEV)
        pb.pilc_logprobs_train(self.x, self.t, on(self.a), logp, grad, entropy=entropy, lse=lse, up_entropy=on(b) if with_entropy else None,
                               workspace=self.ws_train)
        self.check_law(logp, entropy, lse, "training")
        close(grad, want, err, self.dtype, "training: gradient")
        if in_place:
            self.x.copy_(torch.from_numpy(self.x64).to(self.dtype))

    def gradient(self):
        """By an lse in 32 bits, which is what p is made of: its own rounding is the law's."""
        lse, entropy = self.forward()
        grad = torch.full((self.rows, self.n), 55.0, dtype=self.dtype, device=DEV)
        on = lambda v: torch.from_numpy(v).to(DEV)  # noqa: E731
        pb.pilc_logprobs_grad(self.x, self.t, lse, on(self.a), grad, entropy=entropy, up_entropy=on(self.b))
        lse64, h = up(lse)[:, None], up(entropy)[:, None]
        with np.errstate(over="ignore", invalid="ignore"):
            fall = np.where(self.x64 > -np.inf, self.x64 - lse64, -np.inf)
        p = np.exp(fall)
        fall = np.where(p > 0, fall, 0.0)
        a, b = (v.astype(np.float64)[:, None] for v in (self.a, self.b))
        want = -a * p - b * p * (fall + h)
        want[np.arange(self.rows), self.t64] += a[:, 0]
        # a power's exponent is rounded three times, the power and its factors make up twelve units; then two products of p
        off = orc.U * (3 * np.abs(fall) + 16)
        err = p * (np.abs(a) * off + np.abs(b) * (np.abs(fall) + h + 1) * 2 * off) + 2 * orc.U * (np.abs(want) + np.abs(a))
        close(grad, want, err, self.dtype, "gradient by lse")


def blocks(rng, n, *values):
    """A row in as many parts as values are given, None: ordinary logits."""
    row, edges = np.empty(n), np.linspace(0, n, len(values) + 1).astype(int)
    for v, a, b in zip(values, edges, edges[1:]):
        row[a:b] = rng.normal(size=b - a) * 3 if v is None else v
    return row


# parts of wavefronts, of workgroups of four and of sixteen wavefronts, and of runs
SHAPES = [(4, 300), (4, 5000), (4, 20000), (130, 33000), (4, 40000), (4, 131073)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_parts_of_a_row_whose_largest_values_are_far_apart(dtype, rows, n):
    """Two kinds of mask in one row, the type's lowest value and another, in wavefronts or runs of their own; the same of large
    positive numbers."""
    rng = np.random.default_rng(n)
    low = LOWEST[TYPES[dtype]]
    kinds = [(low, -2.0 ** 100, None), (low, -2.0 ** 100), (2.0 ** 126, 2e38, None), (-2.0 ** 100, None, low, -np.inf)]
    v = np.stack([blocks(rng, n, *kinds[r % 4]) for r in range(rows)])
    c = Rows(v, rng.integers(0, n, rows), TYPES[dtype])
    c.forward(alternatives=rows < 100)
    if rows > 100 or n <= 5000:         # rows that one launch takes as a whole
        c.train()
        c.train(with_entropy=False, in_place=True)


FAR = {"f32": [1e5, 2.0 ** 20, 3e6, 1e8, 1e9, 1e10, 1e20, 1e30, 9e37, 3e38], "bf16": [1e5, 2.0 ** 20, 3e6, 1e8, 1e9, 1e10, 1e20, 1e30, 9e37, 3e38],
       "f16": [500.0, 30000.0, 65000.0]}


def far_rows(rng, n, sizes):
    """For each size and sign: a row of that number, one spread about it, one that has it among ordinary logits here and there,
    one that is half it and half -inf."""
    rows = []
    for base in [s * sign for s in sizes for sign in (1, -1)]:
        rows += [np.full(n, base), base + rng.normal(size=n) * 3, np.where(rng.random(n) < 0.3, rng.normal(size=n) * 3, base),
                 np.where(np.arange(n) % 2, -np.inf, base)]
    return np.stack(rows)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n", [2, 3, 5, 7, 64, 256, 999, 5000, 20000, 131073])
def test_finite_logits_far_from_zero(dtype, n):
    """Infinities and what is no number come from logits that are so, not from large ones."""
    rng = np.random.default_rng(n)
    v = far_rows(rng, n, FAR[dtype])
    c = Rows(v, 2 * rng.integers(0, (n + 1) // 2, len(v)), TYPES[dtype])
    c.forward(alternatives=n < 1000)
    c.gradient()
    if n <= 5000:                       # rows that one launch takes as a whole
        c.train()
        c.train(with_entropy=False, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_on_many_long_rows_far_from_zero(dtype):
    """Rows that a workgroup of sixteen wavefronts takes as a whole, more than half as many as compute units."""
    rng = np.random.default_rng(1)
    v = np.concatenate([far_rows(rng, 20001, FAR[dtype]), far_rows(rng, 20001, FAR[dtype])])
    c = Rows(v, 2 * rng.integers(0, 10000, len(v)), TYPES[dtype])
    c.train()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,n", [(3, 40000), (30, 20001), (2, 131073), (130, 140000)])
def test_training_in_two_launches_has_the_law_in_all_its_bits(dtype, rows, n):
    """Few long rows, and rows that no workgroup takes as a whole: the same bounds as of those that one does."""
    rng = np.random.default_rng(n)
    base = np.array([0.0, 20.0, -1000.0, 30000.0, -65000.0] if dtype == "f16" else [0.0, -20.0, 100.0, 1000.0, 1e5, -1e7, -1e10, 1e30, 3e38])
    v = rng.normal(size=(rows, n)) * 3 + base[np.arange(rows) % len(base)][:, None]
    v[1::3] = blocks(rng, n, LOWEST[TYPES[dtype]], base[-1])
    v[rows - 1] = LOWEST[TYPES[dtype]]
    c = Rows(v, rng.integers(0, n, rows), TYPES[dtype])
    c.train()
    c.train(with_entropy=False, in_place=True)
    on = lambda x: torch.from_numpy(x).to(DEV)  # noqa: E731
    logp, grad = torch.empty(rows, device=DEV), torch.empty_like(c.x)
    pb.pilc_logprobs_train(c.x, c.t, on(c.a), logp, grad, up_entropy=on(c.b), workspace=c.ws_train)       # lse and entropy not wanted
    want, err = orc.logprobs_grad(c.x64, c.t64, c.a.astype(np.float64), c.b.astype(np.float64), apart=True)
    close(grad, want, err, c.dtype, "training without lse and entropy: gradient")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,n", [(300, 3), (300, 9), (100, 500), (20, 9000), (130, 40000), (4, 150000)])
def test_the_only_symbol_that_can_occur_is_certain(dtype, rows, n):
    """Its power over itself is 1, whatever the logit: ln p is 0 and lse the logit, to the last bit."""
    rng = np.random.default_rng(n)
    v, t = np.full((rows, n), -np.inf), rng.integers(0, n, rows)
    size = np.exp(rng.uniform(-3, 10 if dtype == "f16" else 80, rows))
    v[np.arange(rows), t] = size * rng.choice([-1, 1], rows)
    x, _ = placed(v, TYPES[dtype])
    want = up(x)[np.arange(rows), t]
    ws = torch.empty(pb.pilc_logprobs_workspace_size(rows, n), dtype=torch.uint8, device=DEV)
    logp, entropy, lse, a = (torch.ones(rows, device=DEV) for _ in range(4))
    on = torch.from_numpy(t).to(DEV)
    for k in range(2):
        if k:
            grad = torch.empty_like(x)
            pb.pilc_logprobs_train(x, on, a, logp, grad, entropy=entropy, lse=lse, workspace=ws)
            # a power, a product and a quotient
            assert float(grad.abs().max()) <= 4 * orc.U and int((grad != 0).sum()) <= rows
        else:
            pb.pilc_logprobs(x, on, logp, entropy=entropy, lse=lse, workspace=ws)
        assert (logp == 0).all() and np.array_equal(up(lse), want) and float(entropy.abs().max()) < 16 * orc.U
