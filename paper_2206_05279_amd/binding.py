"""Thin Python binding of libpilc's C ABI: argument marshalling only.

Every step of the path runs in the library's HIP kernels; PyTorch supplies device
memory and streams.  There is no CPU fallback: if the library has not been built, or
no GPU is present, the calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpilc.so")

PILC_OK = 0
PILC_E_ARG = -1
PILC_E_WORKSPACE = -2
PILC_E_CAPACITY = -3
PILC_E_TOO_LARGE = -4
PILC_E_FORMAT = -5
PILC_E_CORRUPT = -6
PILC_E_HIP = -7
PILC_E_TIMEOUT = -8

EXPORTS = [
    "pilc_lane_count", "pilc_workspace_size", "pilc_encode", "pilc_encode_static", "pilc_decode",
    "pilc_symbol_tables",
    "pilc_set_timing", "pilc_set_kernel_policy", "pilc_set_one_pass_wait", "pilc_set_ansai_decode_waves", "pilc_last_timing", "pilc_timing_name", "pilc_strerror",
    "pilc_last_hip_error", "pilc_version",
    "pilc_ansai_table_bytes", "pilc_ansai_build_tables", "pilc_ansai_workspace_size", "pilc_ansai_encode",
    "pilc_ansai_decode", "pilc_ansai_center", "pilc_twar_forward", "pilc_twar_inverse",
    "pilc_mix_encode", "pilc_mix_decode",
    "pilc_logprobs_workspace_size", "pilc_logprobs", "pilc_logprobs_grad", "pilc_logprobs_train",
    "pilc_norm_workspace_size", "pilc_norm_forward", "pilc_norm_backward",
    "pilc_adamw_step", "pilc_adamw_values",
]


class pilc_geom(C.Structure):
    _fields_ = [("n", C.c_uint32), ("h", C.c_uint32), ("w", C.c_uint32), ("prec_bits", C.c_uint32),
                ("lane_mode", C.c_uint32), ("lane_a", C.c_uint32), ("lane_b", C.c_uint32)]


class pilc_params(C.Structure):
    _fields_ = [("mu", C.c_void_p), ("log_scale", C.c_void_p), ("chan_coef", C.c_void_p)]


class pilc_mix_params(C.Structure):
    _fields_ = [("mu", C.c_void_p), ("log_scale", C.c_void_p), ("weight", C.c_void_p),
                ("chan_coef", C.c_void_p), ("num_comp", C.c_uint32)]


class pilc_ansai_shape(C.Structure):
    _fields_ = [("pieces", C.c_uint32), ("count", C.c_uint32), ("prec_bits", C.c_uint32),
                ("num_dist", C.c_uint32), ("num_sym", C.c_uint32)]


class pilc_twar_params(C.Structure):
    _fields_ = [("w", (C.c_int16 * 3) * 3), ("bias", C.c_int32 * 3)]


class pilc_logits_shape(C.Structure):
    _fields_ = [("rows", C.c_uint32), ("num_sym", C.c_uint32), ("stride", C.c_uint64), ("dtype", C.c_uint32),
                ("target_type", C.c_uint32), ("top", C.c_uint32)]


class pilc_norm_shape(C.Structure):
    _fields_ = [("rows", C.c_uint32), ("width", C.c_uint32), ("x_stride", C.c_uint64), ("y_stride", C.c_uint64),
                ("dx_stride", C.c_uint64), ("dtype", C.c_uint32), ("weight_type", C.c_uint32), ("eps", C.c_float)]


class pilc_adamw_tensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("count", C.c_uint64), ("lr_mult", C.c_float),
                ("decay", C.c_float)]


class pilc_adamw_params(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("grad_scale", C.c_double), ("step", C.c_uint64), ("param_type", C.c_uint32), ("grad_type", C.c_uint32),
                ("state_bits", C.c_uint32), ("dither", C.c_uint32)]


class PilcError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().pilc_strerror(code).decode()
        if code == PILC_E_HIP:
            msg += ": " + lib().pilc_last_hip_error().decode()
        super().__init__("%s failed: %s (%d)" % (where, msg, code))


_lib = None


def lib():
    """Loads libpilc.so (building it first only if no built library exists; a library older than
    its sources is loaded with a warning: `python -m paper_2206_05279_amd.build` rebuilds it)."""
    global _lib
    if _lib is None:
        from . import build
        if not os.path.exists(LIB_PATH):
            build.build_lib()
        elif build.built_digest() != build.source_digest():
            import warnings
            warnings.warn("libpilc.so was not built from the current csrc/ and include/pilc.h: "
                          "run `python -m paper_2206_05279_amd.build`", RuntimeWarning, stacklevel=2)
        L = C.CDLL(LIB_PATH)
        gp, pp = C.POINTER(pilc_geom), C.POINTER(pilc_params)
        L.pilc_lane_count.restype = C.c_uint64
        L.pilc_lane_count.argtypes = [gp]
        L.pilc_workspace_size.restype = C.c_int
        L.pilc_workspace_size.argtypes = [gp, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        L.pilc_encode.restype = C.c_int
        L.pilc_encode.argtypes = [gp, C.c_void_p, pp, C.c_void_p, C.c_size_t, C.c_void_p,
                                  C.c_size_t, C.POINTER(C.c_uint64), C.c_void_p]
        L.pilc_encode_static.restype = C.c_int
        L.pilc_encode_static.argtypes = [gp, C.c_void_p, pp, C.c_void_p, C.c_size_t,
                                         C.POINTER(C.c_uint64), C.c_void_p]
        L.pilc_decode.restype = C.c_int
        L.pilc_decode.argtypes = [gp, C.c_void_p, C.c_size_t, pp, C.c_void_p, C.c_size_t,
                                  C.c_void_p, C.c_void_p]
        L.pilc_symbol_tables.restype = C.c_int
        L.pilc_symbol_tables.argtypes = [gp, C.c_void_p, pp, C.c_void_p, C.c_void_p, C.c_void_p]
        L.pilc_set_timing.restype = None
        L.pilc_set_timing.argtypes = [C.c_int]
        L.pilc_set_kernel_policy.restype = C.c_int
        L.pilc_set_kernel_policy.argtypes = [C.c_int]
        L.pilc_set_ansai_decode_waves.restype = C.c_int
        L.pilc_set_ansai_decode_waves.argtypes = [C.c_int]
        L.pilc_set_one_pass_wait.restype = None
        L.pilc_set_one_pass_wait.argtypes = [C.c_uint64, C.c_int]
        L.pilc_last_timing.restype = C.c_int
        L.pilc_last_timing.argtypes = [C.POINTER(C.c_float), C.c_int]
        L.pilc_timing_name.restype = C.c_char_p
        L.pilc_timing_name.argtypes = [C.c_int]
        L.pilc_strerror.restype = C.c_char_p
        L.pilc_strerror.argtypes = [C.c_int]
        L.pilc_last_hip_error.restype = C.c_char_p
        L.pilc_version.restype = C.c_uint32
        sp = C.POINTER(pilc_ansai_shape)
        L.pilc_ansai_table_bytes.restype = C.c_size_t
        L.pilc_ansai_table_bytes.argtypes = [C.c_uint32, C.c_uint32, C.c_uint32]
        L.pilc_ansai_build_tables.restype = C.c_int
        L.pilc_ansai_build_tables.argtypes = [C.c_uint32, C.c_uint32, C.c_uint32, C.c_void_p, C.c_void_p,
                                              C.c_size_t, C.c_void_p]
        L.pilc_ansai_workspace_size.restype = C.c_int
        L.pilc_ansai_workspace_size.argtypes = [sp, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        L.pilc_ansai_encode.restype = C.c_int
        L.pilc_ansai_encode.argtypes = [sp, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                        C.c_void_p, C.c_size_t, C.POINTER(C.c_uint64), C.c_void_p]
        tp = C.POINTER(pilc_twar_params)
        for f in (L.pilc_twar_forward, L.pilc_twar_inverse):
            f.restype = C.c_int
            f.argtypes = [C.c_uint32, C.c_uint32, C.c_uint32, C.c_void_p, tp, C.c_void_p, C.c_void_p]
        L.pilc_ansai_center.restype = C.c_int
        L.pilc_ansai_center.argtypes = [C.c_void_p, C.c_void_p, C.c_uint64, C.c_int, C.c_void_p, C.c_void_p]
        L.pilc_ansai_decode.restype = C.c_int
        L.pilc_ansai_decode.argtypes = [sp, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_size_t, C.c_void_p, C.c_void_p]
        mp = C.POINTER(pilc_mix_params)
        L.pilc_mix_encode.restype = C.c_int
        L.pilc_mix_encode.argtypes = [gp, C.c_void_p, mp, C.c_void_p, C.c_size_t, C.c_void_p,
                                      C.c_size_t, C.POINTER(C.c_uint64), C.c_void_p]
        L.pilc_mix_decode.restype = C.c_int
        L.pilc_mix_decode.argtypes = [gp, C.c_void_p, C.c_size_t, mp, C.c_void_p, C.c_size_t,
                                      C.c_void_p, C.c_void_p]
        V, Z = C.c_void_p, C.c_size_t
        lp, np_ = C.POINTER(pilc_logits_shape), C.POINTER(pilc_norm_shape)
        L.pilc_logprobs_workspace_size.argtypes = [lp, C.POINTER(Z)]
        L.pilc_logprobs.argtypes = [lp, V, V, V, V, V, V, V, V, Z, V]
        L.pilc_logprobs_grad.argtypes = [lp, V, V, V, V, V, V, V, C.c_uint64, V]
        L.pilc_logprobs_train.argtypes = [lp, V, V, V, V, V, V, V, V, C.c_uint64, V, Z, V]
        L.pilc_norm_workspace_size.argtypes = [np_, C.POINTER(Z)]
        L.pilc_norm_forward.argtypes = [np_, V, V, V, V, V, V, V]
        L.pilc_norm_backward.argtypes = [np_, V, V, V, V, V, V, V, V, V, Z, V]
        L.pilc_adamw_step.argtypes = [C.POINTER(pilc_adamw_params), C.POINTER(pilc_adamw_tensor), C.c_uint32, V]
        L.pilc_adamw_values.argtypes = [V, V, C.c_uint64, C.c_int, V, V]
        for f in (L.pilc_logprobs_workspace_size, L.pilc_logprobs, L.pilc_logprobs_grad, L.pilc_logprobs_train,
                  L.pilc_norm_workspace_size, L.pilc_norm_forward, L.pilc_norm_backward, L.pilc_adamw_step,
                  L.pilc_adamw_values):
            f.restype = C.c_int
        _lib = L
    return _lib


def make_geom(n, h, w, prec_bits, lane_mode, lane_a, lane_b=0) -> pilc_geom:
    return pilc_geom(int(n), int(h), int(w), int(prec_bits), int(lane_mode), int(lane_a), int(lane_b))


def _dev_ptr(t: Optional[torch.Tensor], dtype, what: str) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError("%s must be a contiguous %s device tensor" % (what, dtype))
    return t.data_ptr()


def _params(mu, log_scale, chan_coef) -> pilc_params:
    return pilc_params(_dev_ptr(mu, torch.uint16, "mu"), _dev_ptr(log_scale, torch.int16, "log_scale"),
                       _dev_ptr(chan_coef, torch.int16, "chan_coef"))


def _stream_handle(stream: Optional[torch.cuda.Stream]) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def pilc_lane_count(geom: pilc_geom) -> int:
    return int(lib().pilc_lane_count(C.byref(geom)))


def pilc_workspace_size(geom: pilc_geom) -> Tuple[int, int]:
    """Returns (workspace_bytes, max_coded_bytes)."""
    ws, mc = C.c_size_t(0), C.c_size_t(0)
    rc = lib().pilc_workspace_size(C.byref(geom), C.byref(ws), C.byref(mc))
    if rc != PILC_OK:
        raise PilcError(rc, "pilc_workspace_size")
    return int(ws.value), int(mc.value)


def pilc_encode(geom: pilc_geom, img, mu, log_scale, chan_coef, workspace, coded,
                stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> Tuple[int, int]:
    """Runs pilc_encode; returns (rc, coded_bytes).  workspace / coded are uint8 device tensors."""
    nbytes = C.c_uint64(0)
    par = _params(mu, log_scale, chan_coef)
    rc = lib().pilc_encode(C.byref(geom), _dev_ptr(img, torch.uint8, "img"), C.byref(par),
                           _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel(),
                           _dev_ptr(coded, torch.uint8, "coded"), coded.numel(), C.byref(nbytes),
                           _stream_handle(stream))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_encode")
    return rc, int(nbytes.value)


PILC_STATIC_SCRATCH_BYTES = 16 << 20


def pilc_encode_static(geom: pilc_geom, img, mu, log_scale, chan_coef, coded,
                       stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> Tuple[int, int]:
    """Runs pilc_encode_static (the library's own scratch array instead of a workspace)."""
    nbytes = C.c_uint64(0)
    par = _params(mu, log_scale, chan_coef)
    rc = lib().pilc_encode_static(C.byref(geom), _dev_ptr(img, torch.uint8, "img"), C.byref(par),
                                  _dev_ptr(coded, torch.uint8, "coded"), coded.numel(), C.byref(nbytes),
                                  _stream_handle(stream))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_encode_static")
    return rc, int(nbytes.value)


def pilc_decode(geom: pilc_geom, coded, coded_bytes: int, mu, log_scale, chan_coef, workspace,
                img_out, stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    par = _params(mu, log_scale, chan_coef)
    rc = lib().pilc_decode(C.byref(geom), _dev_ptr(coded, torch.uint8, "coded"), int(coded_bytes),
                           C.byref(par), _dev_ptr(workspace, torch.uint8, "workspace"),
                           workspace.numel(), _dev_ptr(img_out, torch.uint8, "img_out"),
                           _stream_handle(stream))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_decode")
    return rc


def pilc_symbol_tables(geom: pilc_geom, img, mu, log_scale, chan_coef, cum_out, freq_out,
                       stream: Optional[torch.cuda.Stream] = None) -> None:
    par = _params(mu, log_scale, chan_coef)
    rc = lib().pilc_symbol_tables(C.byref(geom), _dev_ptr(img, torch.uint8, "img"), C.byref(par),
                                  _dev_ptr(cum_out, torch.uint32, "cum_out"),
                                  _dev_ptr(freq_out, torch.uint32, "freq_out"), _stream_handle(stream))
    if rc != PILC_OK:
        raise PilcError(rc, "pilc_symbol_tables")


def pilc_set_timing(enabled: bool) -> None:
    lib().pilc_set_timing(1 if enabled else 0)


def pilc_set_kernel_policy(policy: int) -> None:
    rc = lib().pilc_set_kernel_policy(int(policy))
    if rc != PILC_OK:
        raise PilcError(rc, "pilc_set_kernel_policy")


def pilc_set_ansai_decode_waves(waves: int) -> None:
    rc = lib().pilc_set_ansai_decode_waves(int(waves))
    if rc != PILC_OK:
        raise PilcError(rc, "pilc_set_ansai_decode_waves")


def pilc_set_one_pass_wait(ticks: int = 0, withhold_first: bool = False) -> None:
    lib().pilc_set_one_pass_wait(int(ticks), int(bool(withhold_first)))


def pilc_last_timing() -> List[Tuple[str, float]]:
    buf = (C.c_float * 16)()
    k = lib().pilc_last_timing(buf, 16)
    return [(lib().pilc_timing_name(i).decode(), float(buf[i])) for i in range(k)]


def pilc_strerror(code: int) -> str:
    return lib().pilc_strerror(int(code)).decode()


def pilc_version() -> int:
    return int(lib().pilc_version())


# ---------------------------------------------------------------- the table-driven coder (ANS-AI)
def make_ansai_shape(pieces, count, prec_bits, num_dist, num_sym=256) -> pilc_ansai_shape:
    return pilc_ansai_shape(int(pieces), int(count), int(prec_bits), int(num_dist), int(num_sym))


def pilc_ansai_table_bytes(prec_bits: int, num_dist: int, num_sym: int = 256) -> int:
    return int(lib().pilc_ansai_table_bytes(int(prec_bits), int(num_dist), int(num_sym)))


def pilc_ansai_build_tables(prec_bits: int, num_dist: int, num_sym: int, mass, tables,
                            stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    """mass: uint32 device tensor [D, X]; tables: uint8 device tensor of pilc_ansai_table_bytes()."""
    rc = lib().pilc_ansai_build_tables(int(prec_bits), int(num_dist), int(num_sym),
                                       _dev_ptr(mass, torch.uint32, "mass"),
                                       _dev_ptr(tables, torch.uint8, "tables"), tables.numel(),
                                       _stream_handle(stream))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_ansai_build_tables")
    return rc


def pilc_ansai_workspace_size(shape: pilc_ansai_shape) -> Tuple[int, int]:
    """Returns (workspace_bytes, max_coded_bytes)."""
    ws, mc = C.c_size_t(0), C.c_size_t(0)
    rc = lib().pilc_ansai_workspace_size(C.byref(shape), C.byref(ws), C.byref(mc))
    if rc != PILC_OK:
        raise PilcError(rc, "pilc_ansai_workspace_size")
    return int(ws.value), int(mc.value)


def pilc_ansai_encode(shape: pilc_ansai_shape, sym, dist, tables, workspace, coded,
                      stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> Tuple[int, int]:
    nbytes = C.c_uint64(0)
    rc = lib().pilc_ansai_encode(C.byref(shape), _dev_ptr(sym, torch.uint8, "sym"),
                                 _dev_ptr(dist, torch.uint8, "dist"), _dev_ptr(tables, torch.uint8, "tables"),
                                 _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel(),
                                 _dev_ptr(coded, torch.uint8, "coded"), coded.numel(), C.byref(nbytes),
                                 _stream_handle(stream))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_ansai_encode")
    return rc, int(nbytes.value)


def pilc_ansai_decode(shape: pilc_ansai_shape, coded, coded_bytes: int, dist, tables, workspace, sym_out,
                      stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    rc = lib().pilc_ansai_decode(C.byref(shape), _dev_ptr(coded, torch.uint8, "coded"), int(coded_bytes),
                                 _dev_ptr(dist, torch.uint8, "dist"), _dev_ptr(tables, torch.uint8, "tables"),
                                 _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel(),
                                 _dev_ptr(sym_out, torch.uint8, "sym_out"), _stream_handle(stream))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_ansai_decode")
    return rc


def pilc_ansai_center(values, mu, out, inverse: bool = False,
                      stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    """out = (values - mu + 128) mod 256, or with inverse (values + mu - 128) mod 256; uint8 tensors."""
    rc = lib().pilc_ansai_center(_dev_ptr(values, torch.uint8, "values"), _dev_ptr(mu, torch.uint8, "mu"),
                                 values.numel(), 1 if inverse else 0, _dev_ptr(out, torch.uint8, "out"),
                                 _stream_handle(stream))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_ansai_center")
    return rc


# ---------------------------------------------------------------- Three-Way AR residual transform
def make_twar_params(weights, bias) -> pilc_twar_params:
    """weights: 3x3 integers (Q2.14), bias: 3 integers (Q8.14)."""
    p = pilc_twar_params()
    for c in range(3):
        for k in range(3):
            p.w[c][k] = int(weights[c][k])
        p.bias[c] = int(bias[c])
    return p


def _twar(fn, name, params, src, dst, stream, check):
    n, h, w, ch = src.shape
    assert ch == 3 and dst.shape == src.shape
    rc = fn(n, h, w, _dev_ptr(src, torch.uint8, "src"), C.byref(params), _dev_ptr(dst, torch.uint8, "dst"),
            _stream_handle(stream))
    if check and rc != PILC_OK:
        raise PilcError(rc, name)
    return rc


def pilc_twar_forward(params: pilc_twar_params, img, res, stream: Optional[torch.cuda.Stream] = None,
                      check: bool = True) -> int:
    return _twar(lib().pilc_twar_forward, "pilc_twar_forward", params, img, res, stream, check)


def pilc_twar_inverse(params: pilc_twar_params, res, img, stream: Optional[torch.cuda.Stream] = None,
                      check: bool = True) -> int:
    return _twar(lib().pilc_twar_inverse, "pilc_twar_inverse", params, res, img, stream, check)


# ---- mixture of K logistic laws per subpixel ------------------------------------------------
def _mix_params(num_comp, mu, log_scale, weight, chan_coef) -> pilc_mix_params:
    return pilc_mix_params(_dev_ptr(mu, torch.uint16, "mu"), _dev_ptr(log_scale, torch.int16, "log_scale"),
                           _dev_ptr(weight, torch.uint16, "weight"),
                           _dev_ptr(chan_coef, torch.int16, "chan_coef"), int(num_comp))


def pilc_mix_encode(geom: pilc_geom, num_comp: int, img, mu, log_scale, weight, chan_coef, workspace,
                    coded, stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> Tuple[int, int]:
    """Runs pilc_mix_encode; returns (rc, coded_bytes)."""
    nbytes = C.c_uint64(0)
    par = _mix_params(num_comp, mu, log_scale, weight, chan_coef)
    rc = lib().pilc_mix_encode(C.byref(geom), _dev_ptr(img, torch.uint8, "img"), C.byref(par),
                               _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel(),
                               _dev_ptr(coded, torch.uint8, "coded"), coded.numel(), C.byref(nbytes),
                               _stream_handle(stream))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_mix_encode")
    return rc, int(nbytes.value)


def pilc_mix_decode(geom: pilc_geom, num_comp: int, coded, coded_bytes: int, mu, log_scale, weight,
                    chan_coef, workspace, img_out, stream: Optional[torch.cuda.Stream] = None,
                    check: bool = True) -> int:
    par = _mix_params(num_comp, mu, log_scale, weight, chan_coef)
    rc = lib().pilc_mix_decode(C.byref(geom), _dev_ptr(coded, torch.uint8, "coded"), int(coded_bytes),
                               C.byref(par), _dev_ptr(workspace, torch.uint8, "workspace"),
                               workspace.numel(), _dev_ptr(img_out, torch.uint8, "img_out"),
                               _stream_handle(stream))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_mix_decode")
    return rc


# ---- fitting the laws ------------------------------------------------------------------------
# These calls enqueue their kernels on the stream and return; see include/pilc.h for what each computes.
_VALUES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_SYMBOLS = {torch.uint8: 0, torch.int32: 1, torch.int64: 2}


def _bad(what: str, wanted: str):
    raise TypeError("%s must be %s on the current device" % (what, wanted))


def _device_of(t: torch.Tensor, what: str) -> int:
    """The number of the current device, which has to hold t."""
    device = t.get_device()
    if device < 0 or device != torch.cuda.current_device():
        _bad(what, "a tensor")
    return device


def _vector(t: Optional[torch.Tensor], dtype, count: int, device: int, what: str) -> Optional[int]:
    """The address of `count` dense values on the device, or None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device or t.numel() != count or not t.is_contiguous():
        _bad(what, "%d contiguous values of %s" % (count, dtype))
    return t.data_ptr()


def _rows(t: torch.Tensor, dtype, rows: int, width: int, device: int, what: str) -> Tuple[int, int]:
    """(address, elements from row to row) of a matrix whose rows are dense and do not overlap."""
    if t.dtype is not dtype or t.get_device() != device or t.dim() != 2 or t.size(0) != rows or t.size(1) != width:
        _bad(what, "%d x %d values of %s" % (rows, width, dtype))
    across, along = t.stride()
    if rows <= 1:
        across = width
    if (along != 1 and width > 1) or across < width:
        _bad(what, "a matrix with dense rows that do not overlap")
    return t.data_ptr(), across


_OVER = 1 << 32     # a field of 32 bits; ctypes would keep the low ones of a larger number without a word


def _logits_shape(rows: int, num_sym: int, stride: int, kind: int, target_kind: int, top: int) -> pilc_logits_shape:
    if not (0 <= rows < _OVER and 0 <= num_sym < _OVER and 0 <= top < _OVER):
        raise PilcError(PILC_E_ARG, "%d rows of %d logits with %d alternatives" % (rows, num_sym, top))
    return pilc_logits_shape(rows, num_sym, stride, kind, target_kind, top)


def _norm_shape(rows: int, width: int, x_stride: int, y_stride: int, dx_stride: int, kind: int, weight_kind: int, eps: float) -> pilc_norm_shape:
    if not (0 <= rows < _OVER and 0 <= width < _OVER):
        raise PilcError(PILC_E_ARG, "%d rows of %d values" % (rows, width))
    return pilc_norm_shape(rows, width, x_stride, y_stride, dx_stride, kind, weight_kind, eps)


def _raw_stream(stream: Optional[torch.cuda.Stream], device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _logits(logits: torch.Tensor, targets: Optional[torch.Tensor], top: int, device: int):
    kind = _VALUES.get(logits.dtype)
    if kind is None or logits.dim() != 2:
        _bad("logits", "a matrix of float32, bfloat16 or float16")
    rows, num_sym = logits.shape
    ptr, stride = _rows(logits, logits.dtype, rows, num_sym, device, "logits")
    if targets is None:
        return _logits_shape(rows, num_sym, stride, kind, 0, top), ptr, None
    t_kind = _SYMBOLS.get(targets.dtype)
    if t_kind is None:
        _bad("targets", "uint8, int32 or int64")
    return (_logits_shape(rows, num_sym, stride, kind, t_kind, top), ptr,
            _vector(targets, targets.dtype, rows, device, "targets"))


def _workspace(workspace: torch.Tensor, device: int) -> Tuple[int, int]:
    n = workspace.numel()
    return _vector(workspace, torch.uint8, n, device, "workspace"), n


def pilc_logprobs_workspace_size(rows: int, num_sym: int, top: int = 0) -> int:
    """Bytes of workspace that pilc_logprobs and pilc_logprobs_train need for any type of logits."""
    n = C.c_size_t(0)
    shape = _logits_shape(int(rows), int(num_sym), int(num_sym), 0, 0, int(top))
    rc = lib().pilc_logprobs_workspace_size(C.byref(shape), C.byref(n))
    if rc != PILC_OK:
        raise PilcError(rc, "pilc_logprobs_workspace_size")
    return int(n.value)


def pilc_logprobs(logits, targets=None, logp=None, entropy=None, lse=None, top_sym=None, top_logp=None, *, workspace,
                  stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    """ln p of the targets, entropy, ln of the sum and the most likely symbols of each row; what is None is not wanted.
    logits [rows, num_sym], its rows dense; top_sym int32 and top_logp float32 [rows, top]; the rest [rows]."""
    dev, f32 = _device_of(logits, "logits"), torch.float32
    top = 0 if top_sym is None else top_sym.shape[-1]
    shape, x, t = _logits(logits, targets, top, dev)
    rows = shape.rows
    rc = lib().pilc_logprobs(C.byref(shape), x, t, _vector(logp, f32, rows, dev, "logp"), _vector(entropy, f32, rows, dev, "entropy"),
                             _vector(lse, f32, rows, dev, "lse"), _vector(top_sym, torch.int32, rows * top, dev, "top_sym"),
                             _vector(top_logp, f32, rows * top, dev, "top_logp"), *_workspace(workspace, dev), _raw_stream(stream, dev))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_logprobs")
    return rc


def pilc_logprobs_grad(logits, targets, lse, up_logp, grad, entropy=None, up_entropy=None,
                       stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    """grad = gradient of sum(up_logp * logp) + sum(up_entropy * entropy) by the logits; grad may be the logits."""
    dev, f32 = _device_of(logits, "logits"), torch.float32
    shape, x, t = _logits(logits, targets, 0, dev)
    rows = shape.rows
    g, g_stride = _rows(grad, logits.dtype, rows, shape.num_sym, dev, "grad")
    rc = lib().pilc_logprobs_grad(C.byref(shape), x, t, _vector(lse, f32, rows, dev, "lse"), _vector(entropy, f32, rows, dev, "entropy"),
                                  _vector(up_logp, f32, rows, dev, "up_logp"), _vector(up_entropy, f32, rows, dev, "up_entropy"), g,
                                  g_stride, _raw_stream(stream, dev))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_logprobs_grad")
    return rc


def pilc_logprobs_train(logits, targets, up_logp, logp, grad, entropy=None, lse=None, up_entropy=None, *, workspace,
                        stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    """pilc_logprobs (without alternatives) and pilc_logprobs_grad in one call."""
    dev, f32 = _device_of(logits, "logits"), torch.float32
    shape, x, t = _logits(logits, targets, 0, dev)
    rows = shape.rows
    g, g_stride = _rows(grad, logits.dtype, rows, shape.num_sym, dev, "grad")
    rc = lib().pilc_logprobs_train(C.byref(shape), x, t, _vector(up_logp, f32, rows, dev, "up_logp"),
                                   _vector(up_entropy, f32, rows, dev, "up_entropy"), _vector(logp, f32, rows, dev, "logp"),
                                   _vector(entropy, f32, rows, dev, "entropy"), _vector(lse, f32, rows, dev, "lse"), g, g_stride,
                                   *_workspace(workspace, dev), _raw_stream(stream, dev))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_logprobs_train")
    return rc


def _norm_types(x, *weights):
    """The type of x's values, and the one its weights share."""
    kind = None
    for w in weights:
        if w is not None:
            if kind is not None and w.dtype is not kind:
                _bad("weights", "of one type")
            kind = w.dtype
    if kind is None:
        kind = x.dtype
    if x.dim() != 2 or x.dtype not in _VALUES or (kind is not x.dtype and kind is not torch.float32):
        _bad("x", "a matrix of float32, bfloat16 or float16, its weights of its type or float32,")
    return x.dtype, kind


def pilc_norm_forward(x, weight, bias, y, mean=None, rstd=None, eps: float = 1e-5,
                      stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    """y = (x - mean) * rstd * weight + bias over each row of x [rows, width]; weight, bias None: 1 and 0."""
    dev, f32 = _device_of(x, "x"), torch.float32
    own, kind = _norm_types(x, weight, bias)
    rows, width = x.shape
    xp, xs = _rows(x, own, rows, width, dev, "x")
    yp, ys = _rows(y, own, rows, width, dev, "y")
    shape = _norm_shape(rows, width, xs, ys, 0, _VALUES[own], _VALUES[kind], eps)
    rc = lib().pilc_norm_forward(C.byref(shape), xp, _vector(weight, kind, width, dev, "weight"), _vector(bias, kind, width, dev, "bias"),
                                 yp, _vector(mean, f32, rows, dev, "mean"), _vector(rstd, f32, rows, dev, "rstd"),
                                 _raw_stream(stream, dev))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_norm_forward")
    return rc


def pilc_norm_workspace_size(rows: int, width: int) -> int:
    """Bytes of workspace that pilc_norm_backward needs for any types."""
    n = C.c_size_t(0)
    shape = _norm_shape(int(rows), int(width), int(width), int(width), int(width), 0, 0, 0.0)
    rc = lib().pilc_norm_workspace_size(C.byref(shape), C.byref(n))
    if rc != PILC_OK:
        raise PilcError(rc, "pilc_norm_workspace_size")
    return int(n.value)


def pilc_norm_backward(dy, x, weight, mean, rstd, dx=None, dweight=None, dbias=None, *, workspace,
                       stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    """Gradients of pilc_norm_forward by x, weight and bias; what is None is not wanted.  dx may be dy."""
    dev, f32 = _device_of(x, "x"), torch.float32
    own, kind = _norm_types(x, weight, dweight, dbias)
    rows, width = x.shape
    xp, xs = _rows(x, own, rows, width, dev, "x")
    dyp, dys = _rows(dy, own, rows, width, dev, "dy")
    dxp, dxs = _rows(dx, own, rows, width, dev, "dx") if dx is not None else (None, width)
    shape = _norm_shape(rows, width, xs, dys, dxs, _VALUES[own], _VALUES[kind], 0.0)
    rc = lib().pilc_norm_backward(C.byref(shape), dyp, xp, _vector(weight, kind, width, dev, "weight"),
                                  _vector(mean, f32, rows, dev, "mean"), _vector(rstd, f32, rows, dev, "rstd"), dxp,
                                  _vector(dweight, kind, width, dev, "dweight"), _vector(dbias, kind, width, dev, "dbias"),
                                  *_workspace(workspace, dev), _raw_stream(stream, dev))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_norm_backward")
    return rc


class AdamwTensors:
    """The tensors of an AdamW step as pilc_adamw_step takes them; holds them, so that they stay where they are."""

    def __init__(self, records, param_type: int, grad_type: int, state_bits: int, device: int, held):
        self.records, self.held = records, held
        self.param_type, self.grad_type, self.state_bits, self.device = param_type, grad_type, state_bits, device


def make_adamw_tensors(params, grads, ms, vs, m_scales=None, v_scales=None, lr_mults=None, decay=0.0) -> AdamwTensors:
    """Lists of dense device tensors, one entry a tensor.  Parameters share a type, gradients too.  ms and vs are float32,
    or uint8 codes with m_scales and v_scales (uint8, one for each 256 values, the last ones maybe fewer).  decay: one
    number or one a tensor.  Made once and used for every step as long as the tensors stay the same ones: looking at them takes
    1.8 us a tensor, 2.6 with scales (24 tensors 44 us, 291 with scales 758; the step's call 5 and 22), so gradients are better
    written where they were than allocated anew."""
    n = len(params)
    state = torch.float32 if m_scales is None else torch.uint8
    lists = [params, grads, ms, vs] + ([] if m_scales is None and v_scales is None else [m_scales, v_scales])
    if n == 0 or any(k is None or len(k) != n for k in lists):
        raise TypeError("as many gradients and states as parameters, one at least")
    p_type, g_type = params[0].dtype, grads[0].dtype
    if p_type not in _VALUES or g_type not in _VALUES:
        raise TypeError("parameters and gradients must be float32, bfloat16 or float16")
    decays = [float(decay)] * n if isinstance(decay, (int, float)) else [float(d) for d in decay]
    mults = [1.0] * n if lr_mults is None else [float(m) for m in lr_mults]
    if len(decays) != n or len(mults) != n:
        raise TypeError("one decay and one lr_mult a tensor")
    records, dev = (pilc_adamw_tensor * n)(), _device_of(params[0], "params")
    for i in range(n):
        count = params[i].numel()
        scales = [None, None] if m_scales is None else [
            _vector(s[i], torch.uint8, -(-count // 256), dev, "scales") for s in (m_scales, v_scales)]
        records[i] = pilc_adamw_tensor(_vector(params[i], p_type, count, dev, "params"), _vector(grads[i], g_type, count, dev, "grads"),
                                       _vector(ms[i], state, count, dev, "ms"), _vector(vs[i], state, count, dev, "vs"), *scales, count,
                                       mults[i], decays[i])
    return AdamwTensors(records, _VALUES[p_type], _VALUES[g_type], 32 if m_scales is None else 8, dev, [list(k) for k in lists])


def pilc_adamw_step(tensors: AdamwTensors, lr: float, beta1: float, beta2: float, eps: float, step: int,
                    grad_scale: float = 1.0, dither: int = 0, stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    """One AdamW step, in place.  dither: with states in 8 bits another number every step, say the step's own."""
    dev = tensors.device
    if dev != torch.cuda.current_device():
        _bad("tensors", "those of a list made")
    if not 0 <= step < 1 << 64:
        raise PilcError(PILC_E_ARG, "step %d" % step)
    par = pilc_adamw_params(lr, beta1, beta2, eps, grad_scale, step, tensors.param_type, tensors.grad_type, tensors.state_bits,
                            dither & 0xFFFFFFFF)
    rc = lib().pilc_adamw_step(C.byref(par), tensors.records, len(tensors.records), _raw_stream(stream, dev))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_adamw_step")
    return rc


def pilc_adamw_values(codes, scales, values, signed: bool, stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    """values (float32) = what the codes of an 8-bit state stand for; signed for m, not for v."""
    dev, n = _device_of(codes, "codes"), codes.numel()
    rc = lib().pilc_adamw_values(_vector(codes, torch.uint8, n, dev, "codes"), _vector(scales, torch.uint8, -(-n // 256), dev, "scales"),
                                 n, 1 if signed else 0, _vector(values, torch.float32, n, dev, "values"), _raw_stream(stream, dev))
    if check and rc != PILC_OK:
        raise PilcError(rc, "pilc_adamw_values")
    return rc
