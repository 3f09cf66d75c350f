"""What the entry points between states and laws refuse, before anything runs on a GPU."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2206_05279_amd import binding as pb

P = 1 << 20          # an address that nothing follows: every call here is refused, or has nothing to do
BIG = 1 << 40
ARG = pb.PILC_E_ARG


def block8(width=100, **k):
    s = dict(code=P, scale=P, stride=width, scale_stride=-(-width // 128), type=0, block_rows=1)
    s.update(k)
    return C.byref(pb.pilc_block8(**s))


BAD_BLOCK8 = [dict(type=2), dict(block_rows=0), dict(block_rows=64), dict(stride=99), dict(stride=1 << 60), dict(scale_stride=0), dict(scale_stride=1 << 60)]


@pytest.mark.parametrize("bad", BAD_BLOCK8 + [dict(code=None), dict(scale=None)])
def test_matrices_in_8_bits(bad):
    L, good, m, ws = pb.lib(), block8(), block8(**bad), P
    assert L.pilc_block8_quantize(4, 100, P, 100, 0, m, None, None) == ARG
    assert L.pilc_block8_quantize(100, 4, P, 4, 0, None, m, None) == ARG
    assert L.pilc_block8_values(4, 100, m, P, 100, 0, None) == ARG
    assert L.pilc_block8_product(4, 5, 100, m, good, P, 5, 0, ws, BIG, None) == ARG
    assert L.pilc_block8_product(4, 5, 100, good, m, P, 5, 0, ws, BIG, None) == ARG
    assert L.pilc_rms_forward(C.byref(rms()), P, None, None, None, None, m, None, None) == ARG


def test_quantize():
    L = pb.lib()

    def call(rows=4, width=100, x=P, stride=100, dtype=0, out=block8(), out_t=block8(4)):
        return L.pilc_block8_quantize(rows, width, x, stride, dtype, out, out_t, None)

    for k in (dict(x=None), dict(x=P + 2), dict(x=P + 1, dtype=1), dict(stride=99), dict(stride=1 << 60), dict(dtype=3), dict(out=None, out_t=None),
              dict(rows=1 << 31), dict(width=1 << 31, stride=1 << 32), dict(out_t=block8(3))):
        assert call(**k) == ARG, k
    assert call(rows=0, x=None) == pb.PILC_OK and call(width=0, x=None) == pb.PILC_OK


def test_values():
    L = pb.lib()

    def call(rows=4, width=100, m=block8(), v=P, stride=100, dtype=0):
        return L.pilc_block8_values(rows, width, m, v, stride, dtype, None)

    for k in (dict(m=None), dict(v=None), dict(v=P + 2), dict(stride=99), dict(stride=1 << 60), dict(dtype=3), dict(rows=1 << 31)):
        assert call(**k) == ARG, k
    assert call(rows=0, v=None) == pb.PILC_OK


def test_product():
    L, n = pb.lib(), C.c_size_t(0)

    def call(rows=4, cols=5, depth=100, a=block8(), b=block8(), c=P, stride=5, dtype=0, ws=P, size=BIG):
        return L.pilc_block8_product(rows, cols, depth, a, b, c, stride, dtype, ws, size, None)

    for k in (dict(a=None), dict(b=None), dict(c=None), dict(c=P + 2), dict(stride=4), dict(stride=1 << 60), dict(dtype=3), dict(ws=None), dict(ws=P + 128),
              dict(rows=1 << 31), dict(cols=1 << 31, stride=1 << 32), dict(depth=1 << 31), dict(depth=101)):
        assert call(**k) == ARG, k
    assert call(size=255) == pb.PILC_E_WORKSPACE
    assert call(rows=0, c=None, ws=None) == pb.PILC_OK and call(cols=0, c=None, ws=None) == pb.PILC_OK
    assert L.pilc_block8_product_workspace_size(4, 5, 6, None) == ARG
    for shape in ((1 << 31, 1, 1), (1, 1 << 31, 1), (1, 1, 1 << 31)):
        assert L.pilc_block8_product_workspace_size(*shape, C.byref(n)) == ARG


def rms(**k):
    s = dict(rows=4, width=100, x_stride=100, add_stride=100, sum_stride=100, y_stride=100, dtype=1, weight_type=1, eps=1e-5)
    s.update(k)
    return pb.pilc_rms_shape(**s)


@pytest.mark.parametrize("bad", [dict(width=0), dict(width=1 << 31, x_stride=1 << 32, add_stride=1 << 32, sum_stride=1 << 32, y_stride=1 << 32), dict(x_stride=99),
                                 dict(add_stride=99), dict(sum_stride=99), dict(y_stride=99), dict(x_stride=1 << 60), dict(dtype=3), dict(weight_type=2),
                                 dict(dtype=0, weight_type=1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))])
def test_shapes_of_norms(bad):
    L, s, n = pb.lib(), rms(**bad), C.c_size_t(0)
    assert L.pilc_rms_forward(C.byref(s), P, P, P, 2 * P, 3 * P, None, P, None) == ARG
    assert L.pilc_rms_backward(C.byref(s), P, P, P, P, P, 2 * P, P, P, BIG, None) == ARG
    if not any(k.endswith("stride") for k in bad):
        assert L.pilc_rms_workspace_size(C.byref(s), C.byref(n)) == ARG


def test_pointers_of_norms():
    L = pb.lib()

    def forward(shape=rms(), x=P, add=2 * P, w=P, s=3 * P, y=4 * P, y8=None, r=P):
        return L.pilc_rms_forward(C.byref(shape) if shape is not None else None, x, add, w, s, y, y8, r, None)

    for k in (dict(shape=None), dict(x=None), dict(s=None, y=None, r=None), dict(x=P + 1), dict(add=P + 1), dict(w=P + 1), dict(s=P + 1), dict(y=P + 1),
              dict(r=P + 2), dict(y=3 * P), dict(y=2 * P), dict(s=P, shape=rms(sum_stride=104)), dict(s=2 * P, shape=rms(sum_stride=104)),
              dict(y=P, shape=rms(y_stride=104)), dict(y8=block8(block_rows=128))):
        assert forward(**k) == ARG, k
    assert forward(shape=rms(rows=0), x=None) == pb.PILC_OK

    def backward(shape=rms(), dy=P, h=2 * P, w=P, r=P, ds=3 * P, dx=4 * P, dw=P, ws=P, size=BIG):
        return L.pilc_rms_backward(C.byref(shape), dy, h, w, r, ds, dx, dw, ws, size, None)

    for k in (dict(dy=None), dict(h=None), dict(r=None), dict(dx=None, dw=None), dict(ws=None), dict(ws=P + 64), dict(dy=P + 1), dict(h=P + 1), dict(ds=P + 1),
              dict(dx=P + 1), dict(dw=P + 1), dict(w=P + 1), dict(r=P + 2), dict(dx=2 * P), dict(dx=P, shape=rms(sum_stride=104)),
              dict(dx=3 * P, shape=rms(sum_stride=104))):
        assert backward(**k) == ARG, k
    assert backward(size=255) == pb.PILC_E_WORKSPACE


def distill(**k):
    s = dict(rows=4, num_sym=100, stride=100, dtype=0, top=8, rest=0, temperature=1.0)
    s.update(k)
    return pb.pilc_distill_shape(**s)


@pytest.mark.parametrize("bad", [dict(num_sym=0), dict(num_sym=1 << 31, stride=1 << 32), dict(stride=99), dict(stride=1 << 60), dict(dtype=3), dict(top=0),
                                 dict(top=129), dict(rest=2), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")),
                                 dict(temperature=float("inf")), dict(temperature=1e-31)])
def test_shapes_of_distillation(bad):
    L, s, n = pb.lib(), distill(**bad), C.c_size_t(0)
    assert L.pilc_distill_workspace_size(C.byref(s), C.byref(n)) == ARG
    assert L.pilc_distill(C.byref(s), P, P, P, P, P, 2 * P, 1 << 32, P, BIG, None) == ARG


def test_pointers_of_distillation():
    L = pb.lib()

    def call(shape=distill(), x=P, sym=P, value=P, up=P, loss=P, g=2 * P, stride=100, ws=P, size=BIG):
        return L.pilc_distill(C.byref(shape) if shape is not None else None, x, sym, value, up, loss, g, stride, ws, size, None)

    for k in (dict(shape=None), dict(x=None), dict(sym=None), dict(value=None), dict(up=None), dict(loss=None), dict(g=None), dict(stride=99), dict(stride=1 << 60),
              dict(ws=None), dict(ws=P + 128), dict(x=P + 2), dict(sym=P + 2), dict(value=P + 1), dict(up=P + 2), dict(loss=P + 2), dict(g=P + 2),
              dict(g=P, stride=104)):
        assert call(**k) == ARG, k
    assert call(size=255) == pb.PILC_E_WORKSPACE
    assert L.pilc_distill(C.byref(distill(rows=0)), None, None, None, None, None, None, 0, None, 0, None) == pb.PILC_OK


def test_numbers_that_a_field_does_not_hold():
    for f in (lambda: pb.pilc_block8_product_workspace_size(1 << 32, 1, 1), lambda: pb.pilc_rms_workspace_size(1 << 32, 4),
              lambda: pb.pilc_distill_workspace_size(1 << 32, 4, 1), lambda: pb.pilc_distill_workspace_size(4, 1 << 40, 1),
              lambda: pb.pilc_block8_product_workspace_size(-1, 1, 1), lambda: pb.pilc_distill_workspace_size(4, 4, -1)):
        with pytest.raises(pb.PilcError):
            f()


@pytest.mark.gpu
def test_tensors_that_the_binding_refuses():
    dev = "cuda:0"
    codes, scales = torch.zeros(4, 300, dtype=torch.float8_e4m3fn, device=dev), torch.zeros(4, 3, dtype=torch.uint8, device=dev)
    held = pb.make_block8(codes, scales)
    for k in (dict(codes=codes.view(torch.uint8)), dict(codes=codes.cpu()), dict(codes=codes.view(-1)), dict(codes=codes.t()), dict(scales=scales[:, :2]),
              dict(scales=scales.int()), dict(scales=scales[:2])):
        with pytest.raises((TypeError, pb.PilcError)):
            pb.make_block8(**{**dict(codes=codes, scales=scales), **k})
    with pytest.raises(pb.PilcError):
        pb.make_block8(codes, scales, block_rows=64)
    x, ws = torch.zeros(4, 300, device=dev), torch.zeros(4096, dtype=torch.uint8, device=dev)
    c, loss, sym, value = torch.zeros(4, 4, device=dev), torch.zeros(4, device=dev), torch.zeros(4, 2, dtype=torch.int32, device=dev), torch.zeros(4, 2, device=dev)
    for f in (lambda: pb.pilc_block8_quantize(x[:, :299], held), lambda: pb.pilc_block8_quantize(x.double(), held), lambda: pb.pilc_block8_quantize(x, None, held),
              lambda: pb.pilc_block8_quantize(x.cpu(), held), lambda: pb.pilc_block8_values(held, x[:3]), lambda: pb.pilc_block8_values(codes, x),
              lambda: pb.pilc_block8_product(held, held, c[:3], workspace=ws), lambda: pb.pilc_block8_product(held, codes, c, workspace=ws),
              lambda: pb.pilc_block8_product(held, held, c, workspace=ws.float()), lambda: pb.pilc_rms_forward(x, None, x[:, :299]),
              lambda: pb.pilc_rms_forward(x, x[0, :299]), lambda: pb.pilc_rms_forward(x, None, x, add=x.half()), lambda: pb.pilc_rms_backward(x[:3], x, None, loss, x, workspace=ws),
              lambda: pb.pilc_distill(x, sym[:3], value, loss, workspace=ws), lambda: pb.pilc_distill(x, sym.long(), value, loss, workspace=ws),
              lambda: pb.pilc_distill(x, sym, value, loss[:3], workspace=ws), lambda: pb.pilc_distill(x, sym, value, loss, up=loss, grad=x.half(), workspace=ws)):
        with pytest.raises(TypeError):
            f()
    for f in (lambda: pb.pilc_rms_forward(x, None), lambda: pb.pilc_distill(x, sym, value, loss, grad=x, workspace=ws),
              lambda: pb.pilc_distill(x, sym, value, loss, temperature=0.0, workspace=ws)):
        with pytest.raises(pb.PilcError):
            f()


def test_the_library_exports_what_the_header_declares_digits_among_the_names():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "pilc.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(pilc_[a-z0-9_]+)\s*\(", text))
    assert names == set(pb.EXPORTS) | set(pb.EXPORTS_WITH_DIGITS)
    for name in names:
        assert hasattr(pb.lib(), name), name
