"""What the entry points that fit laws refuse, before anything runs on a GPU."""
import ctypes as C

import pytest
import torch

from paper_2206_05279_amd import binding as pb

P = 1 << 20          # an address that nothing follows: every call here is refused, or has nothing to do


def logits(**k):
    s = dict(rows=4, num_sym=100, stride=100, dtype=0, target_type=2, top=0)
    s.update(k)
    return pb.pilc_logits_shape(**s)


def norm(**k):
    s = dict(rows=4, width=100, x_stride=100, y_stride=100, dx_stride=100, dtype=1, weight_type=1, eps=1e-5)
    s.update(k)
    return pb.pilc_norm_shape(**s)


BAD_LOGITS = [dict(num_sym=0), dict(num_sym=1 << 31, stride=1 << 32), dict(stride=99), dict(stride=1 << 60), dict(dtype=3), dict(target_type=3),
              dict(top=33)]


@pytest.mark.parametrize("bad", BAD_LOGITS)
def test_shapes_of_logits(bad):
    L, s, n = pb.lib(), logits(**bad), C.c_size_t(0)
    big = 1 << 40
    assert L.pilc_logprobs_workspace_size(C.byref(s), C.byref(n)) == pb.PILC_E_ARG
    assert L.pilc_logprobs(C.byref(s), P, P, P, P, P, P, P, P, big, None) == pb.PILC_E_ARG
    assert L.pilc_logprobs_grad(C.byref(s), P, P, P, P, P, P, 2 * P, 100, None) == pb.PILC_E_ARG
    assert L.pilc_logprobs_train(C.byref(s), P, P, P, P, P, P, P, 2 * P, 100, P, big, None) == pb.PILC_E_ARG


def test_pointers_of_log_probabilities():
    L, big = pb.lib(), 1 << 40
    s, tops = logits(), logits(top=2)

    def forward(shape=s, x=P, t=P, logp=P, h=P, lse=P, sym=P, top=P, ws=P, size=big):
        return L.pilc_logprobs(C.byref(shape) if shape is not None else None, x, t, logp, h, lse, sym, top, ws, size, None)

    for k in (dict(shape=None), dict(x=None), dict(t=None), dict(ws=None), dict(ws=P + 128), dict(x=P + 2), dict(t=P + 4), dict(logp=P + 2),
              dict(h=P + 1), dict(lse=P + 2), dict(shape=tops, sym=None), dict(shape=tops, top=None), dict(shape=tops, top=P + 1)):
        assert forward(**k) == pb.PILC_E_ARG, k
    assert forward(size=0) == pb.PILC_E_WORKSPACE

    def grad(shape=s, x=P, t=P, lse=P, h=P, a=P, b=P, g=2 * P, stride=100):
        return L.pilc_logprobs_grad(C.byref(shape), x, t, lse, h, a, b, g, stride, None)

    for k in (dict(x=None), dict(t=None), dict(lse=None), dict(a=None), dict(h=None), dict(g=None), dict(stride=99), dict(stride=1 << 60),
              dict(g=P, stride=101), dict(g=P + 2), dict(a=P + 1), dict(b=P + 2)):
        assert grad(**k) == pb.PILC_E_ARG, k

    def train(shape=s, x=P, t=P, a=P, b=P, logp=P, h=P, lse=P, g=2 * P, stride=100, ws=P, size=big):
        return L.pilc_logprobs_train(C.byref(shape), x, t, a, b, logp, h, lse, g, stride, ws, size, None)

    for k in (dict(shape=tops), dict(x=None), dict(t=None), dict(a=None), dict(logp=None), dict(g=None), dict(ws=None), dict(stride=99),
              dict(g=P, stride=104), dict(lse=P + 2)):
        assert train(**k) == pb.PILC_E_ARG, k
    assert train(size=0) == pb.PILC_E_WORKSPACE


def test_nothing_to_do_is_no_error():
    L, none = pb.lib(), logits(rows=0)
    assert L.pilc_logprobs(C.byref(none), None, None, None, None, None, None, None, None, 0, None) == pb.PILC_OK
    assert L.pilc_logprobs_grad(C.byref(none), None, None, None, None, None, None, None, 100, None) == pb.PILC_OK
    assert L.pilc_logprobs_train(C.byref(none), None, None, None, None, None, None, None, None, 100, None, 0, None) == pb.PILC_OK
    assert L.pilc_norm_forward(C.byref(norm(rows=0)), None, None, None, None, None, None, None) == pb.PILC_OK
    assert L.pilc_adamw_values(None, None, 0, 1, None, None) == pb.PILC_OK
    par = adamw()
    assert L.pilc_adamw_step(C.byref(par), None, 0, None) == pb.PILC_OK


@pytest.mark.parametrize("bad", [dict(width=0), dict(width=1 << 31, x_stride=1 << 32, y_stride=1 << 32, dx_stride=1 << 32), dict(x_stride=99),
                                 dict(y_stride=99), dict(dtype=3), dict(weight_type=2), dict(dtype=0, weight_type=1), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(eps=float("inf"))])
def test_shapes_of_norms(bad):
    L, s, n = pb.lib(), norm(**bad), C.c_size_t(0)
    assert L.pilc_norm_forward(C.byref(s), P, P, P, 2 * P, P, P, None) == pb.PILC_E_ARG
    assert L.pilc_norm_workspace_size(C.byref(s), C.byref(n)) == pb.PILC_E_ARG
    assert L.pilc_norm_backward(C.byref(s), P, P, P, P, P, 2 * P, P, P, P, 1 << 40, None) == pb.PILC_E_ARG


def test_pointers_of_norms():
    L, s = pb.lib(), norm()

    def forward(x=P, w=P, b=P, y=2 * P, mean=P, rstd=P, shape=s):
        return L.pilc_norm_forward(C.byref(shape) if shape is not None else None, x, w, b, y, mean, rstd, None)

    for k in (dict(shape=None), dict(x=None), dict(y=None), dict(x=P + 1), dict(w=P + 1), dict(b=P + 1), dict(y=P + 1), dict(mean=P + 2),
              dict(rstd=P + 1), dict(y=P, shape=norm(y_stride=104))):
        assert forward(**k) == pb.PILC_E_ARG, k

    def backward(dy=P, x=2 * P, w=P, mean=P, rstd=P, dx=3 * P, dw=P, db=P, ws=P, size=1 << 40, shape=s):
        return L.pilc_norm_backward(C.byref(shape), dy, x, w, mean, rstd, dx, dw, db, ws, size, None)

    for k in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None, dw=None, db=None), dict(ws=None), dict(ws=P + 8),
              dict(dx=P + 1), dict(dw=P + 1), dict(dx=P, shape=norm(dx_stride=104)), dict(shape=norm(dx_stride=99))):
        assert backward(**k) == pb.PILC_E_ARG, k
    assert backward(size=0) == pb.PILC_E_WORKSPACE


def adamw(**k):
    s = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1, param_type=0, grad_type=0, state_bits=32, dither=0)
    s.update(k)
    return pb.pilc_adamw_params(**s)


def tensor(**k):
    s = dict(param=P, grad=P, m=P, v=P, m_scale=P, v_scale=P, count=10, lr_mult=1.0, decay=0.0)
    s.update(k)
    return pb.pilc_adamw_tensor(**s)


NAN = float("nan")


@pytest.mark.parametrize("bad", [dict(lr=-1.0), dict(lr=NAN), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=NAN), dict(eps=-1.0),
                                 dict(eps=float("inf")), dict(grad_scale=NAN), dict(step=0), dict(param_type=3), dict(grad_type=3),
                                 dict(state_bits=16)])
def test_numbers_of_a_step(bad):
    L, par = pb.lib(), adamw(**bad)
    t = (pb.pilc_adamw_tensor * 1)(tensor())
    assert L.pilc_adamw_step(C.byref(par), t, 1, None) == pb.PILC_E_ARG


@pytest.mark.parametrize("bad", [dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param=P + 2), dict(grad=P + 1), dict(m=P + 2),
                                 dict(v=P + 1), dict(lr_mult=NAN), dict(decay=float("inf")), dict(count=1 << 60)])
def test_tensors_of_a_step(bad):
    """The one that is wrong is the second: nothing is done for the first either."""
    L, par = pb.lib(), adamw()
    t = (pb.pilc_adamw_tensor * 2)(tensor(), tensor(**bad))
    assert L.pilc_adamw_step(C.byref(par), t, 2, None) == pb.PILC_E_ARG
    assert L.pilc_adamw_step(None, t, 1, None) == pb.PILC_E_ARG and L.pilc_adamw_step(C.byref(par), None, 1, None) == pb.PILC_E_ARG


def test_states_in_bytes_need_their_scales():
    L, par = pb.lib(), adamw(state_bits=8)
    for bad in (dict(m_scale=None), dict(v_scale=None)):
        t = (pb.pilc_adamw_tensor * 1)(tensor(**bad))
        assert L.pilc_adamw_step(C.byref(par), t, 1, None) == pb.PILC_E_ARG
    for k in ((None, P, 5, 1, P), (P, None, 5, 1, P), (P, P, 5, 1, None), (P, P, 5, 0, P + 2), (P, P, 1 << 60, 0, P)):
        assert L.pilc_adamw_values(*k, None) == pb.PILC_E_ARG


def test_the_binding_refuses_host_tensors():
    x = torch.zeros(3, 5)
    ws = torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(TypeError):
        pb.pilc_logprobs(x, None, None, entropy=torch.zeros(3), workspace=ws)
    with pytest.raises(TypeError):
        pb.pilc_norm_forward(x, None, None, x)
    with pytest.raises(TypeError):
        pb.make_adamw_tensors([x], [x], [x], [x])
    with pytest.raises(TypeError):
        pb.make_adamw_tensors([], [], [], [])


def test_sizes_of_workspaces():
    assert pb.pilc_logprobs_workspace_size(1, 1) >= 256 and pb.pilc_norm_workspace_size(1, 1) >= 256
    with pytest.raises(pb.PilcError):
        pb.pilc_logprobs_workspace_size(1, 0)
    with pytest.raises(pb.PilcError):
        pb.pilc_norm_workspace_size(5, 0)
