"""pilc_block8_quantize and pilc_block8_values against the reference, whose codes and scales are exact."""
import numpy as np
import pytest
import torch

from block8_util import CODES, DEV, around, holding, room
from fit_util import TYPES, placed, up
from oracle import block8_oracle as orc
from paper_2206_05279_amd import binding as pb

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 127), (2, 128), (3, 129), (128, 128), (127, 5), (129, 257), (5, 1000), (300, 40), (1, 4096), (17, 4100), (260, 384)]


def inputs(rows, width, seed=0):
    rng = np.random.default_rng(rows * 1000 + width + seed)
    x = rng.normal(size=(rows, width)) * np.exp(rng.normal(size=(rows, 1)) * 4)
    x[rng.random(x.shape) < 0.05] = 0.0
    return x


def check(x64, kind, block_rows, codes, scales, what):
    want_codes, want_scales = orc.quantize(x64, kind, block_rows)
    got = scales.cpu().numpy()
    assert np.array_equal(got, want_scales), "%s: scales %s" % (what, np.argwhere(got != want_scales)[:3])
    got = codes.cpu().numpy()
    assert np.array_equal(got, want_codes), "%s: codes at %s" % (what, np.argwhere(got != want_codes)[:3])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width", SIZES)
def test_codes_and_scales(dtype, rows, width):
    turn = rows + width
    kind, other = ("e4m3", "e5m2") if turn % 2 else ("e5m2", "e4m3")
    for block_rows, block_rows_t in ((1, 1), (128, 128), (1, 128)):
        xt, _ = placed(inputs(rows, width), TYPES[dtype], pad=turn % 3, shift=turn % 2)
        out, codes, scales, whole = room(rows, width, kind, block_rows, pad=turn % 5, shift=turn % 4, scale_pad=turn % 2)
        out_t, codes_t, scales_t, whole_t = room(width, rows, other, block_rows_t, pad=turn % 2, shift=turn % 7, scale_pad=turn % 3)
        pb.pilc_block8_quantize(xt, out, out_t)
        check(up(xt), kind, block_rows, codes, scales, "rows")
        check(up(xt).T, other, block_rows_t, codes_t, scales_t, "columns")
        assert around(whole[0], codes) and around(whole[1], scales) and around(whole_t[0], codes_t) and around(whole_t[1], scales_t)
        # one of them alone
        alone, codes, scales, _ = room(rows, width, kind, block_rows)
        pb.pilc_block8_quantize(xt, alone)
        check(up(xt), kind, block_rows, codes, scales, "rows alone")
        alone, codes_t, scales_t, _ = room(width, rows, other, block_rows_t)
        pb.pilc_block8_quantize(xt, None, alone)
        check(up(xt).T, other, block_rows_t, codes_t, scales_t, "columns alone")


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_borders_ties_and_the_smallest(kind):
    """Largest values at, above and below 1.75 times a power of two; values half way between two codes; steps below the type's
    normal ones; blocks of zeros and of the smallest numbers of 32 bits; the largest of 32 bits."""
    most = orc.MOST[kind]
    t = orc.TABLE[kind][np.isfinite(orc.TABLE[kind])]
    rows = [np.concatenate([[most], (t[1:127] + t[:126]) / 2 if kind == "e4m3" else (t[1:124] + t[:123]) / 2])]
    for largest in (most, np.nextafter(np.float32(most), np.float32(np.inf)), np.nextafter(np.float32(most), np.float32(0)), 2 * most, 3.4e38, 2.0 ** -126,
                    2.0 ** -149, 3 * 2.0 ** -140, 448 * 2.0 ** -127, 57344 * 2.0 ** -127):
        rows.append(np.concatenate([[-largest], largest * np.linspace(0, 1, 100)]))
    rows.append(np.zeros(50))
    x = np.zeros((len(rows), 130))
    for i, r in enumerate(rows):
        x[i, : r.size] = r
    xt, _ = placed(x, torch.float32)
    out, codes, scales, _ = room(*x.shape, kind)
    pb.pilc_block8_quantize(xt, out)
    want_codes, want_scales = orc.quantize(up(xt), kind, 1)
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    got = codes.cpu().numpy()
    # a negative value that becomes 0 may keep its sign
    assert np.array_equal(np.where(got == 0x80, 0, got), np.where(want_codes == 0x80, 0, want_codes))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_what_is_not_finite_spoils_its_block(dtype):
    x = inputs(130, 300)
    x = np.clip(x, -1000, 1000)
    x[3, 7], x[5, 299], x[129, 128] = np.nan, np.inf, -np.inf
    xt, _ = placed(x, TYPES[dtype])
    for block_rows in (1, 128):
        out, codes, scales, _ = room(130, 300, "e4m3", block_rows)
        out_t, codes_t, scales_t, _ = room(300, 130, "e5m2", block_rows)
        pb.pilc_block8_quantize(xt, out, out_t)
        check(up(xt), "e4m3", block_rows, codes, scales, "rows")
        check(up(xt).T, "e5m2", block_rows, codes_t, scales_t, "columns")
        back = torch.empty(130, 300, device=DEV)
        pb.pilc_block8_values(out, back)
        bad = np.isnan(up(back))
        assert np.array_equal(bad, np.isnan(orc.powers(scales.cpu().numpy(), (130, 300), block_rows)))


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_values(kind, dtype):
    """Every code under every scale, rounded once to the type."""
    rng = np.random.default_rng(1)
    for rows, width, block_rows, pad in ((256, 131, 1, 3), (256, 256, 128, 0), (1, 15, 1, 0), (7, 16, 128, 1)):
        m, codes, scales, _ = room(rows, width, kind, block_rows, pad=pad, shift=pad)
        c = rng.integers(0, 256, (rows, width)).astype(np.uint8)
        s = rng.integers(0, 256, tuple(scales.shape)).astype(np.uint8)
        if s.size >= 256:
            s.reshape(-1)[:256] = np.arange(256)
        codes.copy_(torch.from_numpy(c))
        scales.copy_(torch.from_numpy(s))
        out, whole = placed(np.full((rows, width), 3.0), TYPES[dtype], pad=pad, shift=pad)
        gaps = torch.isnan(whole)
        pb.pilc_block8_values(m, out)
        assert torch.isnan(whole[gaps]).all()
        with np.errstate(invalid="ignore"):
            want = torch.from_numpy(orc.values(c, s, kind, block_rows)).to(torch.float32).to(TYPES[dtype]).double().numpy()
        assert np.array_equal(up(out), want, equal_nan=True)


def test_nothing_is_no_error():
    x = torch.empty(0, 7, device=DEV)
    pb.pilc_block8_quantize(x, room(0, 7, "e4m3")[0], room(7, 0, "e4m3")[0])
    pb.pilc_block8_values(room(0, 7, "e4m3")[0], x)


def test_rows_beyond_32_bits():
    rows, width = 33000, 70000
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device=DEV)
    some = [0, 30679, 32999]
    x[some] = torch.from_numpy(inputs(3, width)).to(torch.bfloat16).to(DEV)
    codes, scales = torch.full((rows, width), 7, dtype=torch.uint8, device=DEV), torch.full((rows, -(-width // 128)), 7, dtype=torch.uint8, device=DEV)
    held = pb.make_block8(codes.view(CODES["e4m3"]), scales)
    pb.pilc_block8_quantize(x, held)
    check(up(x[some]), "e4m3", 1, codes[some], scales[some], "rows")
    x.fill_(7)
    pb.pilc_block8_values(held, x)
    want = orc.values(codes[some].cpu().numpy(), scales[some].cpu().numpy(), "e4m3", 1)
    assert np.array_equal(up(x[some]), torch.from_numpy(want).to(torch.bfloat16).double().numpy())
    assert (x[1:30679] == 0).all()


def test_on_another_stream_and_in_a_graph():
    x = torch.randn(333, 777, device=DEV)
    out, codes, scales, _ = room(333, 777, "e4m3")
    out_t, codes_t, scales_t, _ = room(777, 333, "e4m3", 128)
    back = torch.empty(777, 333, device=DEV)

    def both(stream=None):
        pb.pilc_block8_quantize(x, out, out_t, stream=stream)
        pb.pilc_block8_values(out_t, back, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    check(up(x), "e4m3", 1, codes, scales, "side")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for _ in range(4):
        x.normal_()
        both()
        torch.cuda.synchronize()
        first = [t.clone() for t in (codes, scales, codes_t, scales_t, back)]
        for t in (codes, scales, codes_t, scales_t, back):
            t.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, (codes, scales, codes_t, scales_t, back)))


def test_a_matrix_of_the_reference_comes_back():
    x = inputs(40, 200)
    m, v = holding(x, "e5m2", 128, pad=3, shift=1)
    out = torch.empty(40, 200, device=DEV)
    pb.pilc_block8_values(m, out)
    assert np.array_equal(up(out), v)
