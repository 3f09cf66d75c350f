"""pilc_adamw_step and pilc_adamw_values against the references: 64 bits for weights and 32-bit states, the exact codes for
states in 8 bits."""
import numpy as np
import pytest
import torch

from fit_util import TYPES, close, up
from oracle import fit_oracle as orc
from paper_2206_05279_amd import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LR, B1, B2, EPS = 3e-3, 0.9, 0.999, 1e-8


class Tensors:
    """Tensors of the given sizes, each `shift` values into an allocation of its own with a guard behind it."""

    def __init__(self, sizes, ptype, gtype, bits, shift=0, seed=0, decay=0.1):
        rng = np.random.default_rng(seed)
        self.sizes, self.ptype, self.gtype, self.bits = sizes, ptype, gtype, bits
        self.wholes = []

        def put(v, dtype):
            w = torch.full((shift + v.size + 64,), 77, dtype=dtype, device=DEV)
            w[shift:shift + v.size] = torch.from_numpy(v).to(dtype).to(DEV)
            self.wholes.append((w, shift, v.size))
            return w[shift:shift + v.size]

        self.p = [put(rng.normal(size=n) * 0.1, ptype) for n in sizes]
        self.g = [put(rng.normal(size=n) * np.exp(rng.normal(size=n) * 2) * 1e-2, gtype) for n in sizes]
        m = [(rng.normal(size=n) * np.exp(rng.normal(size=n)) * 1e-3).astype(np.float32) for n in sizes]
        v = [((rng.normal(size=n) * np.exp(rng.normal(size=n)) * 1e-2) ** 2).astype(np.float32) for n in sizes]
        self.decay = [decay * (k % 3) for k in range(len(sizes))]
        self.mult = [1.0 + 0.5 * (k % 2) for k in range(len(sizes))]
        self.ms = self.vs = None
        if bits == 32:
            self.m, self.v = [put(t, torch.float32) for t in m], [put(t, torch.float32) for t in v]
        else:
            zero = lambda t: np.zeros(t.size, np.uint32)  # noqa: E731
            pm, pv = [orc.pack(t, zero(t), True) for t in m], [orc.pack(t, zero(t), False) for t in v]
            self.m, self.v = [put(c, torch.uint8) for c, _ in pm], [put(c, torch.uint8) for c, _ in pv]
            self.ms, self.vs = [put(s, torch.uint8) for _, s in pm], [put(s, torch.uint8) for _, s in pv]
        self.list = pb.make_adamw_tensors(self.p, self.g, self.m, self.v, self.ms, self.vs, self.mult, self.decay)

    def state(self):
        """(m, v) of each tensor as they stand, float32."""
        if self.bits == 32:
            return [(a.cpu().numpy(), b.cpu().numpy()) for a, b in zip(self.m, self.v)]
        return [(orc.unpack(a.cpu().numpy(), c.cpu().numpy(), True), orc.unpack(b.cpu().numpy(), d.cpu().numpy(), False))
                for a, b, c, d in zip(self.m, self.v, self.ms, self.vs)]

    def step(self, step, grad_scale=1.0, dither=0):
        before, p, g = self.state(), [up(t) for t in self.p], [up(t) for t in self.g]
        pb.pilc_adamw_step(self.list, LR, B1, B2, EPS, step, grad_scale=grad_scale, dither=dither)
        torch.cuda.synchronize()
        first = 0
        for k, n in enumerate(self.sizes):
            m, v = before[k]
            new, m64, v64, perr, merr, verr = orc.adamw(p[k], g[k], m.astype(np.float64), v.astype(np.float64), LR * self.mult[k], B1, B2, EPS,
                                                        step, self.decay[k], grad_scale)
            close(self.p[k], new, perr, self.ptype, "param %d" % k)
            if self.bits == 32:
                close(self.m[k], m64, merr, torch.float32, "m %d" % k)
                close(self.v[k], v64, verr, torch.float32, "v %d" % k)
            else:
                number = np.arange(n, dtype=np.uint64) + np.uint64(first * 256)
                h = orc.noise(number, dither)
                m32, v32 = orc.moments32(m, v, g[k].astype(np.float32), B1, B2, grad_scale)
                for got, scale, x, bits16, signed in ((self.m[k], self.ms[k], m32, h & 0xFFFF, True), (self.v[k], self.vs[k], v32, h >> 16, False)):
                    codes, scales = orc.pack(x, bits16, signed)
                    assert np.array_equal(scale.cpu().numpy(), scales), (k, signed)
                    assert np.array_equal(got.cpu().numpy(), codes), (k, signed)
            first += -(-n // 256)
        for w, shift, n in self.wholes:
            assert (w[:shift] == 77).all() and (w[shift + n:] == 77).all()


ODD = [1, 2, 255, 256, 257, 1000, 4096, 4097, 12345]


@pytest.mark.parametrize("ptype", list(TYPES))
@pytest.mark.parametrize("gtype", list(TYPES))
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_types_and_places(ptype, gtype, bits, shift):
    t = Tensors(ODD, TYPES[ptype], TYPES[gtype], bits, shift)
    for step in (1, 2, 1000):
        t.step(step, dither=step)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 55, 56, 57, 64, 65, 130, 600])
def test_numbers_of_tensors(bits, count):
    rng = np.random.default_rng(count)
    t = Tensors([int(n) for n in rng.integers(1, 700, count)], torch.float32, torch.float32, bits, seed=count)
    t.step(3, dither=5)


@pytest.mark.parametrize("bits", [32, 8])
def test_large_tensor_among_small_ones(bits):
    t = Tensors([3, 3_000_001, 300, 70_000], torch.bfloat16, torch.bfloat16, bits)
    t.step(10, grad_scale=0.25, dither=123456789)


def test_empty_tensors_take_no_numbers():
    t = Tensors([10, 0, 300, 0], torch.float32, torch.float32, 8)
    t.step(1, dither=1)


def test_states_in_bytes_from_nothing():
    """States begin as zero bytes; gradients of 0 leave them 0 and move the weights by the decay alone."""
    t = Tensors([600, 256], torch.float32, torch.float32, 8)
    for k in (t.m, t.v, t.ms, t.vs):
        for x in k:
            x.zero_()
    t.g[1].zero_()
    for step in (1, 2, 3):
        t.step(step, dither=step)
    assert (t.m[1] == 0).all() and (t.v[1] == 0).all()


def test_denominators_do_not_vanish():
    """Values whose v is far below the largest of their block still have a v."""
    t = Tensors([256], torch.float32, torch.float32, 8)
    for x in (t.m, t.v, t.ms, t.vs):
        x[0].zero_()
    t.g[0].fill_(1e-12)
    t.g[0][0] = 100.0
    before = up(t.p[0])
    t.step(1, dither=9)
    assert (t.v[0] > 0).all()
    t.step(2, dither=10)
    assert np.isfinite(up(t.p[0])).all() and np.abs(up(t.p[0]) - before).max() < 10 * LR * 1.5


@pytest.mark.parametrize("bad", [np.inf, np.nan])
def test_gradients_that_are_not_finite(bad):
    """They spoil their value with states in 32 bits, their block's states in 8."""
    for bits in (32, 8):
        t = Tensors([700], torch.float32, torch.float32, bits)
        t.g[0][300] = bad
        pb.pilc_adamw_step(t.list, LR, B1, B2, EPS, 1)
        p, (m, v) = up(t.p[0]), t.state()[0]
        spoilt = np.arange(700) == 300
        assert np.array_equal(np.isnan(p), spoilt)
        if bits == 32:
            assert np.array_equal(~np.isfinite(m), spoilt) and np.array_equal(~np.isfinite(v), spoilt)
        else:
            assert t.ms[0].cpu().numpy()[1] == 255 and t.vs[0].cpu().numpy()[1] == 255
            block = (np.arange(700) >> 8) == 1
            assert np.array_equal(np.isnan(m), block) and np.array_equal(np.isnan(v), block)


@pytest.mark.parametrize("count", [1, 255, 1000, 70001])
@pytest.mark.parametrize("signed", [True, False])
@pytest.mark.parametrize("shift", [0, 1])
def test_values(count, signed, shift):
    rng = np.random.default_rng(count)
    codes = rng.integers(0, 256, count + shift, dtype=np.uint8)
    scales = rng.integers(0, 256, -(-count // 256), dtype=np.uint8)
    scales[:: 7] = 255
    out = torch.full((count + shift + 3,), 77.0, device=DEV)
    pb.pilc_adamw_values(torch.from_numpy(codes).to(DEV)[shift:], torch.from_numpy(scales).to(DEV), out[shift:shift + count], signed=signed)
    want = orc.unpack(codes[shift:], scales, signed)
    got = out.cpu().numpy()
    assert np.array_equal(got[shift:shift + count], want, equal_nan=True)
    assert (got[:shift] == 77).all() and (got[shift + count:] == 77).all()


def test_tensors_beyond_32_bits():
    """Values beyond the 2^32nd byte of a tensor and beyond the 2^32nd value of the list are moved and numbered right."""
    n = (1 << 32) + 700
    make = lambda d: torch.zeros(n, dtype=d, device=DEV)  # noqa: E731
    p, g, m, v = make(torch.bfloat16), make(torch.bfloat16), make(torch.uint8), make(torch.uint8)
    ms, vs = (torch.zeros(-(-n // 256), dtype=torch.uint8, device=DEV) for _ in range(2))
    tail = 900
    rng = np.random.default_rng(3)
    g[-tail:] = torch.from_numpy(rng.normal(size=tail)).to(torch.bfloat16).to(DEV)
    g64 = up(g[-tail:])
    lst = pb.make_adamw_tensors([p], [g], [m], [v], [ms], [vs])
    pb.pilc_adamw_step(lst, LR, B1, B2, EPS, 1, dither=4)
    zero = np.zeros(tail)
    new, *_, = orc.adamw(zero, g64, zero, zero, LR, B1, B2, EPS, 1, 0.0)
    _, _, _, perr, _, _ = orc.adamw(zero, g64, zero, zero, LR, B1, B2, EPS, 1, 0.0)
    close(p[-tail:], new, perr, torch.bfloat16, "param")
    m32, _ = orc.moments32(zero, zero, g64.astype(np.float32), B1, B2)
    h = orc.noise(np.arange(n - tail, n, dtype=np.uint64), 4)
    whole = (n - tail + 255) // 256 * 256 - (n - tail)          # where the first block that lies in the tail begins
    codes, scales = orc.pack(m32[whole:], (h & 0xFFFF)[whole:], True)
    assert np.array_equal(m[-tail:].cpu().numpy()[whole:], codes)
    assert np.array_equal(ms[-scales.size:].cpu().numpy(), scales)


def test_replays_of_a_graph():
    t = Tensors([5000, 77, 300], torch.float32, torch.bfloat16, 8)
    run = lambda: pb.pilc_adamw_step(t.list, LR, B1, B2, EPS, 5, dither=2)  # noqa: E731
    keep = lambda: [x.clone() for k in (t.p, t.m, t.v, t.ms, t.vs) for x in k]  # noqa: E731

    def back(saved):
        for x, s in zip([x for k in (t.p, t.m, t.v, t.ms, t.vs) for x in k], saved):
            x.copy_(s)

    start = keep()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        run()
    for turn in range(3):
        for x in t.g:
            x.copy_(torch.randn(x.numel(), device=DEV) * 0.01)
        back(start)
        run()
        torch.cuda.synchronize()
        want = keep()
        back(start)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, keep())), turn
