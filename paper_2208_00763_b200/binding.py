"""ctypes binding of ``libhikonv.so``: same names as the C interface, argument marshalling only.

PyTorch is used for device memory and streams; every arithmetic step runs in the CUDA
library.  Loading fails loudly when the library has not been built: there is no fallback.

The calls of every step (``conv1d``, ``conv1d_dense``, ``pack``, ``conv2d``, ``conv2d_dense`` without tuning record and
explicit stream, ``quantize_rows``, ``linear``, ``grouped_linear`` and the calls of a mixture of experts without explicit stream) go through the extension module ``_fast`` first, which makes the same checks on the tensors natively and
returns None where anything is amiss; the Python code below then raises the error.

No call records gradients: what it returns does not require one, whether its inputs do or not.  ``rows_from_experts`` has its gradient in
``rows_from_experts_grad``, ``rows_to_experts`` in ``rows_from_experts``.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhikonv.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_NO_FIT, ERR_WORKSPACE, ERR_CUDA, ERR_TOO_LARGE, ERR_RANGE = range(8)
STATIC_SCRATCH_BYTES = 4 << 20
ALGO_PACKED32, ALGO_PACKED64EMU, ALGO_UNPACKED_IMAD, ALGO_DP4A = 0, 1, 2, 3
FORM_TWO_LAUNCHES, FORM_ONE_LAUNCH, FORM_FILTERS, FORM_UNPACKED = 0, 1, 2, 3
GB_SINGLE, GB_1D, GB_DNN = 0, 1, 2
OUT_SUMS, OUT_CODES, OUT_F32, OUT_F16, OUT_BF16 = range(5)
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = range(4)
MAX_GROUPS = 1024
F8_E4M3, F8_E5M2 = range(2)
PIPE_KINDS = {"mad_wide_u32": 0, "mad_wide_s32": 1, "mad_lo_s32": 2, "logic": 3, "shift": 4, "prmt": 5,
              "mad_wide_with_logic": 6, "fma_f64": 7}


class HikonvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (where, status_string(status), status))


class PlanT(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("N", "K", "S", "Gb", "ops")]


class LayoutT(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("N", "S", "Kc", "J", "segments", "top_bits", "M", "signed_prod", "S_paper", "carry_bits")]


class TuningT(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("N", "S", "M", "tile")]


class Conv2dFormT(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("form", "launches", "cluster", "words", "groups", "step_channels", "ctas", "tiles", "segments")]
                + [(n, ctypes.c_double) for n in ("multiplies", "double_multiplies")])


class EpilogueT(ctypes.Structure):
    _fields_ = [("out_type", ctypes.c_int), ("activation", ctypes.c_int), ("d_x_scale", ctypes.c_void_p), ("d_w_scale", ctypes.c_void_p),
                ("d_bias", ctypes.c_void_p), ("d_residual", ctypes.c_void_p), ("residual_row_stride", ctypes.c_longlong),
                ("shift", ctypes.c_int), ("lo", ctypes.c_int), ("hi", ctypes.c_int)]


_lib = None
_fast = None          # the extension module, its entry points bound to the library's

_vp, _sz, _i, _d, _ll = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_double, ctypes.c_longlong

_SIGNATURES = {
    "hikonv_plan": (_i, [_i] * 7 + [ctypes.POINTER(PlanT)]),
    "hikonv_layout": (_i, [_i] * 7 + [ctypes.POINTER(TuningT), ctypes.POINTER(LayoutT)]),
    "hikonv_layout_emu64": (_i, [_i] * 5 + [ctypes.POINTER(TuningT), ctypes.POINTER(LayoutT)]),
    "hikonv_pack": (_i, [_vp, _sz, _i, _i, _i, _i, _i, _vp, _vp]),
    "hikonv_check_range": (_i, [_vp, _sz, _i, _i, _vp, ctypes.POINTER(ctypes.c_ulonglong), _vp]),
    "hikonv_conv1d": (_i, [_vp, _sz, _vp, _i, _i, _i, _i, _i, _vp, _i, ctypes.POINTER(TuningT), _vp]),
    "hikonv_conv1d_layout": (_i, [_i] * 5 + [ctypes.POINTER(TuningT), ctypes.POINTER(LayoutT)]),
    "hikonv_conv1d_dense": (_i, [_vp, _sz, _vp, _i, _i, _i, _i, _i, _vp, ctypes.POINTER(TuningT), _vp]),
    "hikonv_conv1d_host_workspace_bytes": (_sz, [_sz, _i]),
    "hikonv_conv1d_host": (_i, [_vp, _sz, _vp, _i, _i, _i, _i, _i, _vp, _vp, _sz, _i, ctypes.POINTER(TuningT), _vp]),
    "hikonv_conv2d": (_i, [_vp, _i, _i, _i, _i, _vp, _i, _i, _i, _i, _i, _i, _i, _i, _vp, _i, _i, _i, _i, _vp, _sz, _i,
                           ctypes.POINTER(TuningT), _vp]),
    "hikonv_conv2d_dense": (_i, [_vp, _i, _i, _i, _i, _i, _vp, _i, _i, _i, _i, _i, _i, _i, _i, _i, _vp, _i, _i, _i, _i, _i, _i, _vp, _sz,
                                 _i, ctypes.POINTER(TuningT), _vp]),
    "hikonv_conv2d_tune": (_i, [_vp, _i, _i, _i, _i, _i, _vp, _i, _i, _i, _i, _i, _i, _i, _i, _i, _vp, _i, _i, _i, _i, _i, _i, _vp, _sz,
                                _i, _i, ctypes.POINTER(_i), ctypes.POINTER(_d), ctypes.POINTER(_d), _vp]),
    "hikonv_conv2d_workspace_bytes": (_sz, [_i] * 7),
    "hikonv_conv2d_launches": (_i, [_i] * 13 + [ctypes.POINTER(TuningT), ctypes.POINTER(_i), ctypes.POINTER(_i)]),
    "hikonv_conv2d_form": (_i, [_i] * 14 + [ctypes.POINTER(TuningT), ctypes.POINTER(Conv2dFormT)]),
    "hikonv_conv2d_wait_timeouts": (_i, [_vp]),
    "hikonv_conv2d_wait_check": (_i, [ctypes.c_longlong, _vp]),
    "hikonv_conv2d_static_scratch": (_i, [_vp, _i, _i, _i, _i, _vp, _i, _i, _i, _i, _i, _i, _i, _i, _vp, _i, _i, _i, _i, _i,
                                          ctypes.POINTER(TuningT), _vp]),
    "hikonv_conv2d_host_workspace_bytes": (_sz, [_i] * 8),
    "hikonv_conv2d_host": (_i, [_vp, _i, _i, _i, _i, _vp, _i, _i, _i, _i, _i, _i, _i, _i, _vp, _i, _i, _i, _i, _vp, _sz,
                                _i, ctypes.POINTER(TuningT), _vp]),
    "hikonv_maxpool2x2_i8": (_i, [_vp, _i, _i, _i, _i, _i, _vp, _vp]),
    "hikonv_conv1d_multiplies": (_d, [_sz, _i, _i, _i, _i, _i, _i, ctypes.POINTER(TuningT)]),
    "hikonv_conv2d_multiplies": (_d, [_i] * 12 + [ctypes.POINTER(TuningT)]),
    "hikonv_conv2d_layout": (_i, [_i] * 11 + [ctypes.POINTER(TuningT), ctypes.POINTER(LayoutT), ctypes.POINTER(_i)]),
    "hikonv_pipe_rate": (_i, [_i, _i, _vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), _vp]),
    "hikonv_quantize_rows": (_i, [_vp, _i, _ll, _i, _i, _i, _i, _vp, _vp, _vp]),
    "hikonv_linear": (_i, [_vp, _ll, _vp] + [_i] * 8 + [_vp, _ll, ctypes.POINTER(EpilogueT), _vp, _sz, _vp]),
    "hikonv_grouped_linear": (_i, [_vp, _ll, _vp, _i, _vp] + [_i] * 8 + [_vp, _ll, ctypes.POINTER(EpilogueT), _vp, _sz, _vp]),
    "hikonv_linear_workspace_bytes": (_sz, [_vp, _ll, _vp] + [_i] * 5),
    "hikonv_linear_wait_timeouts": (_i, [_vp]),
    "hikonv_linear_wait_check": (_i, [_ll, _vp]),
    "hikonv_linear_f8_wait_check": (_i, [_ll, _vp]),
    "hikonv_sort_by_expert": (_i, [_vp, _i, _ll, _i, _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "hikonv_sort_by_expert_workspace_bytes": (_sz, [_i, _i, _i]),
    "hikonv_rows_to_experts": (_i, [_vp, _i, _ll, _vp, _i, _i, _i, _vp, _ll, _i, _vp]),
    "hikonv_rows_from_experts": (_i, [_vp, _i, _ll, _i, _vp, _vp, _i, _i, _i, _vp, _ll, _vp, _ll, _vp]),
    "hikonv_rows_from_experts_grad": (_i, [_vp, _i, _ll, _vp, _ll, _i, _vp, _vp, _i, _i, _i, _vp, _ll, _vp, _vp]),
    "hikonv_zero_other_rows": (_i, [_vp, _i, _i, _vp, _i, _ll, _i, _i, _vp, _sz, _vp]),
    "hikonv_quantize_blocks": (_i, [_vp, _i, _ll, _i, _i, _i, _vp, _i, _i, _vp, _ll, _vp, _ll, _vp]),
    "hikonv_quantize_tiles": (_i, [_vp, _i, _ll, _i, _i, _i, _i, _vp, _ll, _vp, _vp]),
    "hikonv_linear_f8": (_i, [_vp, _i, _ll, _vp, _i, _ll, _i, _i, _i, _vp, _ll, _vp, _vp, _ll, ctypes.POINTER(EpilogueT), _vp]),
    "hikonv_grouped_linear_f8": (_i, [_vp, _i, _ll, _vp, _i, _ll, _vp, _i, _i, _i, _i, _vp, _ll, _vp, _vp, _ll, ctypes.POINTER(EpilogueT), _vp]),
    "hikonv_status_string": (ctypes.c_char_p, [_i]),
}


_FAST_ENTRY_POINTS = ("hikonv_conv1d", "hikonv_conv1d_dense", "hikonv_pack", "hikonv_conv2d", "hikonv_conv2d_dense",
                      "hikonv_conv2d_workspace_bytes", "hikonv_quantize_rows", "hikonv_linear", "hikonv_grouped_linear",
                      "hikonv_linear_workspace_bytes", "hikonv_sort_by_expert", "hikonv_sort_by_expert_workspace_bytes",
                      "hikonv_rows_to_experts", "hikonv_rows_from_experts", "hikonv_rows_from_experts_grad", "hikonv_zero_other_rows",
                      "hikonv_quantize_blocks",
                      "hikonv_linear_f8", "hikonv_grouped_linear_f8")


def exported_names():
    return sorted(_SIGNATURES)


def lib():
    """The loaded CUDA library.  Raises if it has not been built (no CPU fallback exists)."""
    global _lib, _fast
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "CUDA library %s is missing: run `python -m paper_2208_00763_b200.build` "
                "(or __graft_entry__.build()) first; there is no CPU fallback" % LIB_PATH)
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        try:
            from . import _fast as ext
        except ImportError as err:
            raise RuntimeError("the binding's extension module is missing or does not load (%s): run "
                               "`python -m paper_2208_00763_b200.build` first" % err) from err
        for name in _FAST_ENTRY_POINTS:
            ext.bind(name, ctypes.cast(getattr(handle, name), ctypes.c_void_p).value)
        _lib, _fast = handle, ext
    return _lib


def _load_fast():
    lib()
    return _fast


def status_string(status: int) -> str:
    return lib().hikonv_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != OK:
        raise HikonvError(status, where)


def _tune(tune: Optional[dict]):
    if not tune:
        return None
    t = TuningT(int(tune.get("N", 0)), int(tune.get("S", 0)), int(tune.get("M", 0)), int(tune.get("tile", 0)))
    return ctypes.byref(t)


# The current stream as a plain address, without building a torch.cuda.Stream around it (0.1 against 3.1 us; a short 1-D
# call takes 9 us in all): only called with CUDA tensors at hand, so CUDA is initialised.
_raw_stream, _current_device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))


def _stream(stream) -> int:
    return _raw_stream(_current_device()) if stream is None else int(stream.cuda_stream)


_CODE_DTYPES = (torch.int8, torch.uint8)
_INT32 = (torch.int32,)


def _dev_i8(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda or t.dtype not in _CODE_DTYPES or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA int8/uint8 tensor" % name)
    return t.data_ptr()


def _dev_out(t: torch.Tensor, name: str, numel: int, dtypes, like: torch.Tensor) -> int:
    """Checks a caller-supplied output tensor before its address goes to a kernel: the library writes `numel`
    elements of one of `dtypes` there and cannot see the tensor's size, type, layout or device."""
    if not getattr(t, "is_cuda", False):
        raise ValueError("%s must be a CUDA tensor" % name)
    if t.device != like.device:
        raise ValueError("%s is on %s, the inputs are on %s" % (name, t.device, like.device))
    if t.dtype not in dtypes:
        raise ValueError("%s must have dtype %s, not %s" % (name, " or ".join(str(d) for d in dtypes), t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.numel() != numel:
        raise ValueError("%s holds %d elements, the call writes %d" % (name, t.numel(), numel))
    return t.data_ptr()


# ------------------------------------------------------------------ host-only planning

def plan(p, q, LA=32, LB=32, mode=GB_SINGLE, M=1, K_fixed=0) -> dict:
    out = PlanT()
    _check(lib().hikonv_plan(p, q, LA, LB, mode, M, K_fixed, ctypes.byref(out)), "hikonv_plan")
    return {n: getattr(out, n) for n, _ in PlanT._fields_}


def layout(p, q, f_signed, g_signed, K, dims, total_terms=0, tune=None) -> dict:
    out = LayoutT()
    _check(lib().hikonv_layout(p, q, int(f_signed), int(g_signed), K, dims, total_terms, _tune(tune), ctypes.byref(out)),
           "hikonv_layout")
    return {n: getattr(out, n) for n, _ in LayoutT._fields_}


def layout_emu64(p, q, f_signed, g_signed, K, tune=None) -> dict:
    out = LayoutT()
    _check(lib().hikonv_layout_emu64(p, q, int(f_signed), int(g_signed), K, _tune(tune), ctypes.byref(out)),
           "hikonv_layout_emu64")
    return {n: getattr(out, n) for n, _ in LayoutT._fields_}


def conv1d_layout(p, q, f_signed, g_signed, K, tune=None) -> dict:
    """The layout ``conv1d`` (packed algorithm, one code per byte) runs with."""
    out = LayoutT()
    _check(lib().hikonv_conv1d_layout(p, q, int(f_signed), int(g_signed), K, _tune(tune), ctypes.byref(out)),
           "hikonv_conv1d_layout")
    return {n: getattr(out, n) for n, _ in LayoutT._fields_}


def conv2d_layout(B, Ci, H, W, Co, K, pad, p, q, x_signed, w_signed, tune=None) -> dict:
    """The layout ``conv2d`` (packed algorithm) runs this layer with, plus ``x_shift``: 0, or 2^(p-1) when the layer
    runs its unsigned activations as signed codes shifted by that much."""
    out, shift = LayoutT(), ctypes.c_int(0)
    _check(lib().hikonv_conv2d_layout(B, Ci, H, W, Co, K, pad, p, q, int(x_signed), int(w_signed), _tune(tune), ctypes.byref(out),
                                      ctypes.byref(shift)), "hikonv_conv2d_layout")
    d = {n: getattr(out, n) for n, _ in LayoutT._fields_}
    d["x_shift"] = shift.value
    return d


def conv2d_launches(B, Ci, H, W, Co, K, pad, p, q, x_signed, w_signed, requant=False, pool=False, tune=None) -> tuple:
    """(kernels a layer runs in, CTAs that share a tile's input channels in a single one or 0)."""
    launches, cluster = ctypes.c_int(0), ctypes.c_int(0)
    _check(lib().hikonv_conv2d_launches(B, Ci, H, W, Co, K, pad, p, q, int(x_signed), int(w_signed), int(bool(requant)), int(pool),
                                        _tune(tune), ctypes.byref(launches), ctypes.byref(cluster)), "hikonv_conv2d_launches")
    return launches.value, cluster.value


def conv2d_form(B, Ci, H, W, Co, K, pad, p, q, x_signed, w_signed, requant=False, pool=False, algo=ALGO_PACKED32, tune=None) -> dict:
    """The form a layer on one code per byte runs in (``FORM_*``), its launches, its tile and the multiplies it executes."""
    out = Conv2dFormT()
    _check(lib().hikonv_conv2d_form(B, Ci, H, W, Co, K, pad, p, q, int(x_signed), int(w_signed), int(bool(requant)), int(pool), algo,
                                    _tune(tune), ctypes.byref(out)), "hikonv_conv2d_form")
    return {n: getattr(out, n) for n, _ in Conv2dFormT._fields_}


# ------------------------------------------------------------------ device entry points

def pack(d_in: torch.Tensor, bits: int, is_signed: bool, S: int, N: int, word_bits: int = 32, stream=None) -> torch.Tensor:
    if stream is None:
        done = (_fast or _load_fast()).pack(d_in, bits, is_signed, S, N, word_bits)
        if done is not None:
            return done
    n = d_in.numel()
    n_words = (n + N - 1) // N
    out = torch.empty(n_words, dtype=torch.int32 if word_bits == 32 else torch.int64, device=d_in.device)
    _check(lib().hikonv_pack(_dev_i8(d_in, "d_in"), n, bits, int(is_signed), S, N, word_bits, out.data_ptr(), _stream(stream)),
           "hikonv_pack")
    return out


def check_range(d_in: torch.Tensor, bits: int, is_signed: bool, stream=None) -> int:
    """Number of stored codes outside their range (0 = all valid).  Synchronises the stream."""
    d_count = torch.empty(1, dtype=torch.int64, device=d_in.device)
    found = ctypes.c_ulonglong(0)
    rc = lib().hikonv_check_range(_dev_i8(d_in, "d_in"), d_in.numel(), bits, int(is_signed), d_count.data_ptr(),
                                  ctypes.byref(found), _stream(stream))
    if rc not in (OK, ERR_RANGE):
        _check(rc, "hikonv_check_range")
    assert (rc == ERR_RANGE) == (found.value > 0)
    return int(found.value)


def conv2d_wait_timeouts() -> int:
    """Waits of 2-D layer kernels on the current device that ran out since the last call (0 on a healthy device).  Synchronises."""
    count = ctypes.c_uint(0)
    _check(lib().hikonv_conv2d_wait_timeouts(ctypes.byref(count)), "hikonv_conv2d_wait_timeouts")
    return int(count.value)


def conv2d_wait_check(cycles: int, stream=None) -> None:
    """One thread waits `cycles` for a barrier that nothing completes, gives up and is counted."""
    _check(lib().hikonv_conv2d_wait_check(int(cycles), _stream(stream)), "hikonv_conv2d_wait_check")


def conv1d(d_f: torch.Tensor, d_g: torch.Tensor, p: int, q: int, f_signed: bool, g_signed: bool,
           algo: int = ALGO_PACKED32, tune=None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    if tune is None and stream is None:
        done = (_fast or _load_fast()).conv1d(d_f, d_g, p, q, f_signed, g_signed, algo, out)
        if done is not None:
            return done
    n, K = d_f.numel(), d_g.numel()
    if out is None:
        out = torch.empty(n + K - 1, dtype=torch.int32, device=d_f.device)
    _check(lib().hikonv_conv1d(_dev_i8(d_f, "d_f"), n, _dev_i8(d_g, "d_g"), K, p, q, int(f_signed), int(g_signed),
                               _dev_out(out, "out", n + K - 1, _INT32, d_f), algo, _tune(tune), _stream(stream)),
           "hikonv_conv1d")
    return out


def conv1d_dense(d_f_dense: torch.Tensor, n: int, d_g: torch.Tensor, p: int, q: int, f_signed: bool, g_signed: bool,
                 tune=None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """`d_f_dense`: uint8 tensor holding `n` codes of p bits, 8 / p per byte."""
    if tune is None and stream is None:
        done = (_fast or _load_fast()).conv1d_dense(d_f_dense, n, d_g, p, q, f_signed, g_signed, out)
        if done is not None:
            return done
    K = d_g.numel()
    if d_f_dense.dtype != torch.uint8 or not d_f_dense.is_cuda or not d_f_dense.is_contiguous():
        raise ValueError("d_f_dense must be a contiguous CUDA uint8 tensor")
    if d_f_dense.numel() * 8 < n * p:
        raise ValueError("d_f_dense holds fewer than n codes")
    if out is None:
        out = torch.empty(n + K - 1, dtype=torch.int32, device=d_f_dense.device)
    _check(lib().hikonv_conv1d_dense(d_f_dense.data_ptr(), n, _dev_i8(d_g, "d_g"), K, p, q, int(f_signed), int(g_signed),
                                     _dev_out(out, "out", n + K - 1, _INT32, d_f_dense), _tune(tune), _stream(stream)),
           "hikonv_conv1d_dense")
    return out


def conv1d_host_workspace_bytes(n: int, K: int) -> int:
    return int(lib().hikonv_conv1d_host_workspace_bytes(n, K))


def conv1d_host(h_f: torch.Tensor, h_g: torch.Tensor, p, q, f_signed, g_signed, h_y: torch.Tensor,
                d_workspace: torch.Tensor, algo: int = ALGO_PACKED32, tune=None, stream=None) -> None:
    """Host buffers in, host buffer out (pinned tensors make the copies asynchronous)."""
    n, K = h_f.numel(), h_g.numel()
    _check(lib().hikonv_conv1d_host(h_f.data_ptr(), n, h_g.data_ptr(), K, p, q, int(f_signed), int(g_signed),
                                    h_y.data_ptr(), d_workspace.data_ptr(), d_workspace.numel() * d_workspace.element_size(),
                                    algo, _tune(tune), _stream(stream)), "hikonv_conv1d_host")


def conv2d_workspace_bytes(B: int, Ci: int, H: int, W: int, Co: int, K: int, pad: int) -> int:
    return int(lib().hikonv_conv2d_workspace_bytes(B, Ci, H, W, Co, K, pad))


def conv2d(d_x: torch.Tensor, d_w: torch.Tensor, pad: int, p: int, q: int, x_signed: bool, w_signed: bool,
           requant: Optional[tuple] = None, algo: int = ALGO_PACKED32, tune=None, workspace: Optional[torch.Tensor] = None,
           out: Optional[torch.Tensor] = None, stride: int = 1, stream=None) -> torch.Tensor:
    """requant = (shift, lo, hi) selects int8 output, None the exact int32 sums."""
    if tune is None and stream is None:
        done = (_fast or _load_fast()).conv2d(d_x, d_w, pad, p, q, x_signed, w_signed, requant, algo, workspace, out, stride)
        if done is not None:
            return done
    B, Ci, H, W = d_x.shape
    Co, Ci2, K, K2 = d_w.shape
    if Ci != Ci2 or K != K2:
        raise ValueError("weight shape does not match the input")
    Ho, Wo = H + 2 * pad - K + 1, W + 2 * pad - K + 1
    if workspace is None:
        workspace = torch.empty(conv2d_workspace_bytes(B, Ci, H, W, Co, K, pad), dtype=torch.uint8, device=d_x.device)
    if out is None:
        out = torch.empty((B, Co, max(Ho, 0), max(Wo, 0)), dtype=torch.int8 if requant else torch.int32, device=d_x.device)
    shift, lo, hi = requant if requant else (0, 0, 0)
    out_ptr = _dev_out(out, "out", B * Co * max(Ho, 0) * max(Wo, 0), _CODE_DTYPES if requant else _INT32, d_x)
    if not workspace.is_cuda or workspace.device != d_x.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA tensor on the inputs' device")
    _check(lib().hikonv_conv2d(_dev_i8(d_x, "d_x"), B, Ci, H, W, _dev_i8(d_w, "d_w"), Co, K, stride, pad, p, q,
                               int(x_signed), int(w_signed), out_ptr, 1 if requant else 0, shift, lo, hi,
                               workspace.data_ptr(), workspace.numel() * workspace.element_size(), algo, _tune(tune),
                               _stream(stream)), "hikonv_conv2d")
    return out


def conv2d_tune(d_x: torch.Tensor, x_shape, x_store_bits: int, d_w: torch.Tensor, w_shape, w_store_bits: int, pad: int, p: int,
                q: int, x_signed: bool, w_signed: bool, requant: Optional[tuple] = None, out_store_bits: int = 8,
                pool: bool = False, algo: int = ALGO_PACKED32, workspace: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, stride: int = 1, stream=None, repeats: int = 3) -> dict:
    """Times the tile shapes of this layer on the device (``hikonv_conv2d_tune``; arguments as for ``conv2d_dense``).
    Returns ``{"tune": {"tile": t} or None, "us": best, "default_us": the automatic choice's, "out": the layer's output}``;
    pass ``tune`` to later calls on this shape.  Synchronises."""
    return conv2d_dense(d_x, x_shape, x_store_bits, d_w, w_shape, w_store_bits, pad, p, q, x_signed, w_signed, requant, out_store_bits,
                        pool, algo, None, workspace, out, stride, stream, _tuner_repeats=int(repeats))


def conv2d_dense(d_x: torch.Tensor, x_shape, x_store_bits: int, d_w: torch.Tensor, w_shape, w_store_bits: int, pad: int, p: int,
                 q: int, x_signed: bool, w_signed: bool, requant: Optional[tuple] = None, out_store_bits: int = 8,
                 pool: bool = False, algo: int = ALGO_PACKED32, tune=None, workspace: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None, stride: int = 1, stream=None, _tuner_repeats: Optional[int] = None):
    """``conv2d`` on densely stored tensors.  ``d_x`` / ``d_w`` are flat uint8 (dense) or int8 (one code per byte)
    tensors holding the codes of ``x_shape`` = (B, Ci, H, W) / ``w_shape`` = (Co, Ci, K, K).  Returns int32
    [B, Co, Ho, Wo] without ``requant``; with it a flat uint8 tensor of the (optionally pooled) output codes,
    ``out_store_bits`` per code (8: shaped [B, Co, Ho', Wo'] int8)."""
    if tune is None and stream is None and _tuner_repeats is None:
        done = (_fast or _load_fast()).conv2d_dense(d_x, x_shape, x_store_bits, d_w, w_shape, w_store_bits, pad, p, q, x_signed, w_signed,
                                                    requant, out_store_bits, pool, algo, workspace, out, stride)
        if done is not None:
            return done
    B, Ci, H, W = x_shape
    Co, Ci2, K, K2 = w_shape
    if Ci != Ci2 or K != K2:
        raise ValueError("weight shape does not match the input")
    for t, n, bits, name in ((d_x, B * Ci * H * W, x_store_bits, "d_x"), (d_w, Co * Ci * K * K, w_store_bits, "d_w")):
        if not t.is_cuda or not t.is_contiguous() or t.dtype not in _CODE_DTYPES or t.numel() * 8 < n * bits:
            raise ValueError("%s must be a contiguous CUDA byte tensor holding all codes" % name)
    Ho, Wo = H + 2 * pad - K + 1, W + 2 * pad - K + 1
    Hq, Wq = (Ho // 2, Wo // 2) if pool else (Ho, Wo)
    count = B * Co * max(Hq, 0) * max(Wq, 0)
    if workspace is None:
        workspace = torch.empty(conv2d_workspace_bytes(B, Ci, H, W, Co, K, pad), dtype=torch.uint8, device=d_x.device)
    if not requant:
        if out is None:
            out = torch.empty((B, Co, max(Ho, 0), max(Wo, 0)), dtype=torch.int32, device=d_x.device)
        out_ptr, store = _dev_out(out, "out", B * Co * max(Ho, 0) * max(Wo, 0), _INT32, d_x), 32
    else:
        nbytes = (count * out_store_bits + 7) // 8
        if out is None:
            out = (torch.empty((B, Co, Hq, Wq), dtype=torch.int8, device=d_x.device) if out_store_bits == 8
                   else torch.empty(nbytes, dtype=torch.uint8, device=d_x.device))
        out_ptr, store = _dev_out(out, "out", nbytes, _CODE_DTYPES, d_x), out_store_bits
    shift, lo, hi = requant if requant else (0, 0, 0)
    if _tuner_repeats is not None:
        tile, us, default_us = ctypes.c_int(0), ctypes.c_double(0.0), ctypes.c_double(0.0)
        with torch.cuda.device(d_x.device):
            _check(lib().hikonv_conv2d_tune(d_x.data_ptr(), x_store_bits, B, Ci, H, W, d_w.data_ptr(), w_store_bits, Co, K, stride, pad,
                                            p, q, int(x_signed), int(w_signed), out_ptr, store, 1 if requant else 0, shift, lo, hi,
                                            1 if pool else 0, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                            algo, _tuner_repeats, ctypes.byref(tile), ctypes.byref(us), ctypes.byref(default_us),
                                            _stream(stream)), "hikonv_conv2d_tune")
        return {"tune": {"tile": tile.value} if tile.value else None, "us": us.value, "default_us": default_us.value, "out": out}
    _check(lib().hikonv_conv2d_dense(d_x.data_ptr(), x_store_bits, B, Ci, H, W, d_w.data_ptr(), w_store_bits, Co, K, stride, pad, p, q,
                                     int(x_signed), int(w_signed), out_ptr, store, 1 if requant else 0, shift, lo, hi,
                                     1 if pool else 0, workspace.data_ptr(), workspace.numel() * workspace.element_size(), algo,
                                     _tune(tune), _stream(stream)), "hikonv_conv2d_dense")
    return out


def conv2d_static_scratch(d_x: torch.Tensor, d_w: torch.Tensor, pad: int, p: int, q: int, x_signed: bool, w_signed: bool,
                          out: torch.Tensor, requant: Optional[tuple] = None, algo: int = ALGO_PACKED32, tune=None,
                          stride: int = 1, stream=None) -> torch.Tensor:
    """``conv2d`` without a workspace: the packed kernel and activation rows go to the library's built-in device buffer.

    For callers that may not allocate device memory when the layer runs (they own only the input and
    output tensors, or allocation is forbidden after start-up).  ``out`` must be preallocated by the
    caller.  Layers whose packed rows exceed ``STATIC_SCRATCH_BYTES`` raise ``ERR_TOO_LARGE``; calls
    that may overlap on the GPU must be ordered by the caller, since they share the buffer.
    """
    B, Ci, H, W = d_x.shape
    Co, Ci2, K, K2 = d_w.shape
    if Ci != Ci2 or K != K2:
        raise ValueError("weight shape does not match the input")
    shift, lo, hi = requant if requant else (0, 0, 0)
    Ho, Wo = H + 2 * pad - K + 1, W + 2 * pad - K + 1
    out_ptr = _dev_out(out, "out", B * Co * max(Ho, 0) * max(Wo, 0), _CODE_DTYPES if requant else _INT32, d_x)
    if d_w.device != d_x.device:
        raise ValueError("d_w is on %s, d_x on %s" % (d_w.device, d_x.device))
    with torch.cuda.device(d_x.device):      # the built-in buffer that is used is the current device's
        _check(lib().hikonv_conv2d_static_scratch(_dev_i8(d_x, "d_x"), B, Ci, H, W, _dev_i8(d_w, "d_w"), Co, K, stride, pad, p, q,
                                                  int(x_signed), int(w_signed), out_ptr, 1 if requant else 0, shift, lo, hi,
                                                  algo, _tune(tune), _stream(stream)), "hikonv_conv2d_static_scratch")
    return out


def conv2d_host_workspace_bytes(B, Ci, H, W, Co, K, pad, requant) -> int:
    return int(lib().hikonv_conv2d_host_workspace_bytes(B, Ci, H, W, Co, K, pad, 1 if requant else 0))


def conv2d_host(h_x: torch.Tensor, h_w: torch.Tensor, pad, p, q, x_signed, w_signed, h_out: torch.Tensor,
                d_workspace: torch.Tensor, requant: Optional[tuple] = None, algo: int = ALGO_PACKED32, tune=None,
                stride: int = 1, stream=None) -> None:
    B, Ci, H, W = h_x.shape
    Co, _, K, _ = h_w.shape
    shift, lo, hi = requant if requant else (0, 0, 0)
    _check(lib().hikonv_conv2d_host(h_x.data_ptr(), B, Ci, H, W, h_w.data_ptr(), Co, K, stride, pad, p, q, int(x_signed),
                                    int(w_signed), h_out.data_ptr(), 1 if requant else 0, shift, lo, hi,
                                    d_workspace.data_ptr(), d_workspace.numel() * d_workspace.element_size(), algo,
                                    _tune(tune), _stream(stream)), "hikonv_conv2d_host")


def maxpool2x2_i8(d_in: torch.Tensor, is_signed: bool, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    B, C, H, W = d_in.shape
    if out is None:
        out = torch.empty((B, C, H // 2, W // 2), dtype=d_in.dtype, device=d_in.device)
    _check(lib().hikonv_maxpool2x2_i8(_dev_i8(d_in, "d_in"), B, C, H, W, int(is_signed),
                                      _dev_out(out, "out", B * C * (H // 2) * (W // 2), _CODE_DTYPES, d_in), _stream(stream)),
           "hikonv_maxpool2x2_i8")
    return out


def conv1d_multiplies(n, K, p, q, f_signed, g_signed, algo=ALGO_PACKED32, tune=None) -> float:
    return float(lib().hikonv_conv1d_multiplies(n, K, p, q, int(f_signed), int(g_signed), algo, _tune(tune)))


def conv2d_multiplies(B, Ci, H, W, Co, K, pad, p, q, x_signed, w_signed, algo=ALGO_PACKED32, tune=None) -> float:
    return float(lib().hikonv_conv2d_multiplies(B, Ci, H, W, Co, K, pad, p, q, int(x_signed), int(w_signed), algo, _tune(tune)))


# ------------------------------------------------------------------ linear layers

_FLOAT_TYPES = {torch.float32: OUT_F32, torch.float16: OUT_F16, torch.bfloat16: OUT_BF16}


def _fits(name: str, *sizes: int) -> None:
    """The library takes sizes as 32-bit integers, which ctypes makes of larger ones without a word."""
    if max(sizes) > 0x7FFFFFFF:
        raise ValueError("%s: a size of %d, above 2^31 - 1" % (name, max(sizes)))


def _rows(t: torch.Tensor, name: str, dtypes, like: Optional[torch.Tensor] = None, shape=None) -> int:
    """Checks a matrix whose rows may lie apart; returns the elements from one row to the next."""
    if not getattr(t, "is_cuda", False) or t.layout != torch.strided or t.dim() != 2:
        raise ValueError("%s must be a CUDA matrix" % name)
    if t.dtype not in dtypes:
        raise ValueError("%s must have dtype %s, not %s" % (name, " or ".join(str(d) for d in dtypes), t.dtype))
    if like is not None and t.device != like.device:
        raise ValueError("%s is on %s, x is on %s" % (name, t.device, like.device))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, the call needs %s" % (name, tuple(t.shape), tuple(shape)))
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError("%s must have contiguous rows" % name)
    _fits(name, *t.shape)
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _vector(t: Optional[torch.Tensor], name: str, dtype, shape, like: torch.Tensor):
    """Checks a contiguous tensor of scales, biases or offsets; returns its address, None for None."""
    if t is None:
        return None
    if not getattr(t, "is_cuda", False) or t.device != like.device or t.dtype != dtype or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor on %s" % (name, dtype, like.device))
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, the call needs %s" % (name, tuple(t.shape), tuple(shape)))
    return t.data_ptr()


def _stream_of(t: torch.Tensor, stream) -> int:
    """The given stream, or the current one of the tensor's device."""
    return _raw_stream(t.device.index) if stream is None else int(stream.cuda_stream)


def _empty(shape, dtype, like: torch.Tensor, stream, make=torch.empty) -> torch.Tensor:
    """Memory that a call on `stream` may write at once: the allocator's for that stream, which nothing on another one still uses."""
    if stream is None:
        return make(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype, device=like.device)


def quantize_rows(x: torch.Tensor, bits: int, is_signed: bool = True, codes: Optional[torch.Tensor] = None,
                  scale: Optional[torch.Tensor] = None, stream=None) -> tuple:
    """Codes of ``bits`` bits, one per byte, and one float scale per row of the matrix ``x`` (float32, float16 or bfloat16; its rows
    may lie apart, or be one): ``x`` is ``codes * scale`` up to half a step.  Signed codes use the range symmetric around zero,
    unsigned ones leave out what is negative.  Returns (codes, scale)."""
    if stream is None:
        done = (_fast or _load_fast()).quantize_rows(x, bits, is_signed, codes, scale)
        if done is not None:
            return done
    if getattr(x, "dtype", None) not in _FLOAT_TYPES:
        raise ValueError("x must be a float32, float16 or bfloat16 matrix")
    x_row = _rows(x, "x", (x.dtype,))
    M, K = x.shape
    if codes is None:
        codes = _empty((M, K), torch.int8 if is_signed else torch.uint8, x, stream)
    if scale is None:
        scale = _empty(M, torch.float32, x, stream)
    if tuple(codes.shape) != (M, K):
        raise ValueError("codes has shape %s, the call needs %s" % (tuple(codes.shape), (M, K)))
    with torch.cuda.device(x.device):
        _check(lib().hikonv_quantize_rows(x.data_ptr(), _FLOAT_TYPES[x.dtype], x_row, M, K, bits, int(is_signed),
                                          _dev_out(codes, "codes", M * K, _CODE_DTYPES, x),
                                          _vector(scale, "scale", torch.float32, (M,), x), _stream_of(x, stream)), "hikonv_quantize_rows")
    return codes, scale


def linear(x: torch.Tensor, w: torch.Tensor, p: int, q: int, x_signed: bool, w_signed: bool, w_store_bits: int = 8,
           x_scale: Optional[torch.Tensor] = None, w_scale: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
           activation: int = ACT_NONE, residual: Optional[torch.Tensor] = None, requant: Optional[tuple] = None,
           out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
           stream=None) -> torch.Tensor:
    """Matrix product of codes, ``x`` [M, K] with ``w`` [N, K] (``w_store_bits`` 1, 2 or 4: dense bytes [N, K * q / 8], which
    ``inputs.to_dense`` packs on the host, once).

    requant = (shift, lo, hi): codes, one per byte, of the sums plus an int32 ``bias``.  Scales, or a float ``out_dtype`` or ``out``:
    ``act(sum * x_scale[m] * w_scale[n] + bias[n]) + residual[m, n]`` (bfloat16 unless ``out_dtype`` or ``out`` says
    otherwise; scales and bias float32, residual of the output's type, which may be ``out`` itself).  Else: the exact int32 sums.
    Rows of ``x``, ``residual`` and ``out`` may lie apart, and be columns of one buffer if they are equally many bytes apart.  Rows of
    ``x`` and ``w`` that do not start on 16-byte boundaries may be copied to such first, into ``workspace`` (``linear_workspace_bytes``;
    made by the call when it is not given)."""
    return _linear("hikonv_linear", x, w, None, p, q, x_signed, w_signed, w_store_bits, x_scale, w_scale, bias, activation, residual,
                   requant, out_dtype, out, workspace, stream)


def linear_workspace_bytes(x: torch.Tensor, w: torch.Tensor, w_store_bits: int = 8) -> int:
    """Bytes that ``linear`` (``w`` [N, K]) or ``grouped_linear`` (``w`` [E, N, K]) needs to copy rows of these operands: 0 for most."""
    M, K = x.shape
    groups = w.shape[0] if w.dim() == 3 else 0
    return int(lib().hikonv_linear_workspace_bytes(x.data_ptr(), x.stride(0), w.data_ptr(), w_store_bits, groups, M, w.shape[-2], K))


def grouped_linear(x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, p: int, q: int, x_signed: bool, w_signed: bool,
                   w_store_bits: int = 8, x_scale: Optional[torch.Tensor] = None, w_scale: Optional[torch.Tensor] = None,
                   bias: Optional[torch.Tensor] = None, activation: int = ACT_NONE, residual: Optional[torch.Tensor] = None,
                   requant: Optional[tuple] = None, out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """``linear`` with a matrix of weights per group of rows: ``w`` [E, N, K], ``w_scale`` and ``bias`` [E, N]; rows
    ``offsets[e]`` to ``offsets[e + 1] - 1`` (int32 [E + 1], on the device) belong to matrix e.  Rows of no group are left as they
    were in ``out`` (undefined when the call makes it)."""
    return _linear("hikonv_grouped_linear", x, w, offsets, p, q, x_signed, w_signed, w_store_bits, x_scale, w_scale, bias, activation,
                   residual, requant, out_dtype, out, workspace, stream)


def _linear(name, x, w, offsets, p, q, x_signed, w_signed, w_store_bits, x_scale, w_scale, bias, activation, residual, requant, out_dtype,
            out, workspace, stream):
    grouped = name == "hikonv_grouped_linear"
    if stream is None and grouped == (offsets is not None):
        done = (_fast or _load_fast()).linear(x, w, offsets, p, q, x_signed, w_signed, w_store_bits, x_scale, w_scale, bias, activation,
                                              residual, requant, out_dtype, out, workspace)
        if done is not None:
            return done
    x_row = _rows(x, "x", _CODE_DTYPES)
    M, K = x.shape
    if not getattr(w, "is_cuda", False) or w.dtype not in _CODE_DTYPES or not w.is_contiguous() or w.dim() != (3 if grouped else 2):
        raise ValueError("w must be a contiguous CUDA int8/uint8 tensor of %s" % ("[E, N, K]" if grouped else "[N, K]"))
    if w.device != x.device:
        raise ValueError("w is on %s, x is on %s" % (w.device, x.device))
    lead, N = tuple(w.shape[:-2]), w.shape[-2]
    if w_store_bits not in (1, 2, 4, 8) or w.shape[-1] * 8 != K * w_store_bits:
        raise ValueError("w has %d bytes per row, %d codes of %s bits need %s" % (w.shape[-1], K, w_store_bits, K * w_store_bits / 8))
    if requant is not None and (x_scale is not None or w_scale is not None or out_dtype in _FLOAT_TYPES):
        raise ValueError("requantised codes take no scales and no float type")
    if out_dtype is None and out is not None:
        out_dtype = out.dtype
    if requant is not None:
        kind, dtypes = OUT_CODES, _CODE_DTYPES
        if out_dtype not in (None, torch.int8, torch.uint8):
            raise ValueError("requantised codes are int8 or uint8, not %s" % out_dtype)
    elif x_scale is not None or w_scale is not None or out_dtype in _FLOAT_TYPES:
        out_dtype = out_dtype or torch.bfloat16
        if out_dtype not in _FLOAT_TYPES:
            raise ValueError("scaled sums are float32, float16 or bfloat16, not %s" % out_dtype)
        kind, dtypes = _FLOAT_TYPES[out_dtype], (out_dtype,)
    else:
        kind, dtypes = OUT_SUMS, _INT32
        if out_dtype not in (None, torch.int32):
            raise ValueError("sums are int32, not %s" % out_dtype)
    if out is None:
        out = _empty((M, N), out_dtype or (torch.int8 if kind == OUT_CODES else torch.int32), x, stream)
    ep = EpilogueT(out_type=kind, activation=int(activation))
    out_row = _rows(out, "out", dtypes, x, (M, N))
    ep.d_x_scale = _vector(x_scale, "x_scale", torch.float32, (M,), x)
    ep.d_w_scale = _vector(w_scale, "w_scale", torch.float32, lead + (N,), x)
    ep.d_bias = _vector(bias, "bias", torch.int32 if kind == OUT_CODES else torch.float32, lead + (N,), x)
    if residual is not None:
        ep.residual_row_stride = _rows(residual, "residual", dtypes, x, (M, N))
        ep.d_residual = residual.data_ptr()
    if requant is not None:
        ep.shift, ep.lo, ep.hi = (int(v) for v in requant)
    groups = ()
    if grouped:
        groups = (_vector(offsets, "offsets", torch.int32, (lead[0] + 1,), x), lead[0])
    with torch.cuda.device(x.device):
        need = int(lib().hikonv_linear_workspace_bytes(x.data_ptr(), x_row, w.data_ptr(), w_store_bits, lead[0] if grouped else 0, M, N, K))
        if need and workspace is None:
            workspace = _empty(need, torch.uint8, x, stream)
        if workspace is not None and (not workspace.is_cuda or workspace.device != x.device or not workspace.is_contiguous()):
            raise ValueError("workspace must be a contiguous CUDA tensor on x's device")
        space = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
        _check(getattr(lib(), name)(x.data_ptr(), x_row, w.data_ptr(), w_store_bits, *groups, M, N, K, p, q, int(x_signed),
                                    int(w_signed), out.data_ptr(), out_row, ctypes.byref(ep), *space, _stream_of(x, stream)), name)
    return out


def linear_wait_timeouts() -> int:
    """Waits of linear-layer kernels on the current device that ran out since the last call (0 on a healthy device).  Synchronises."""
    count = ctypes.c_uint(0)
    _check(lib().hikonv_linear_wait_timeouts(ctypes.byref(count)), "hikonv_linear_wait_timeouts")
    return int(count.value)


def linear_wait_check(cycles: int, stream=None) -> None:
    """One thread waits `cycles` for a barrier that nothing completes, gives up and is counted."""
    _check(lib().hikonv_linear_wait_check(int(cycles), _stream(stream)), "hikonv_linear_wait_check")


def linear_f8_wait_check(cycles: int, stream=None) -> None:
    """The same for the products of 8-bit floating point numbers, whose waits that ran out ``linear_wait_timeouts`` counts, too."""
    _check(lib().hikonv_linear_f8_wait_check(int(cycles), _stream(stream)), "hikonv_linear_f8_wait_check")


# ------------------------------------------------------------------ a mixture of experts

_F8_TYPES = {torch.float8_e4m3fn: F8_E4M3, torch.float8_e5m2: F8_E5M2}
_INDEX_TYPES = {torch.int32: 4, torch.int64: 8}


def _slots(slots: torch.Tensor, like: torch.Tensor, rows: Optional[int] = None) -> tuple:
    """Checks the places of pairs; returns (address, T, k)."""
    if getattr(slots, "dim", lambda: 0)() != 2:
        raise ValueError("slots must be a matrix, a row per token")
    T, k = slots.shape
    if rows is not None and T != rows:
        raise ValueError("slots has %d rows, there are %d tokens" % (T, rows))
    _fits("slots", T, k)
    return _vector(slots, "slots", torch.int32, (T, k), like), T, k


def sort_by_expert(experts: torch.Tensor, n_experts: int, offsets: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> tuple:
    """Places of (token, choice) pairs in the order of their experts: ``experts`` [T, k] int32 or int64, as ``torch.topk`` gives them (its
    rows may lie apart).  Returns (offsets, slots), int32: the pairs of expert e have the places ``offsets[e]`` to ``offsets[e + 1] - 1``
    (what ``grouped_linear`` and ``grouped_linear_f8`` take), ``slots`` [T, k] the place of each pair, equal experts in the pairs' order.
    Experts outside 0 .. n_experts - 1 mean none: such a pair's slot is -2 - place, with places behind ``offsets[-1]``."""
    if stream is None:
        done = (_fast or _load_fast()).sort_by_expert(experts, n_experts, offsets, slots, workspace)
        if done is not None:
            return done
    if getattr(experts, "dtype", None) not in _INDEX_TYPES:
        raise ValueError("experts must be an int32 or int64 matrix")
    row = _rows(experts, "experts", (experts.dtype,))
    _fits("n_experts", n_experts)
    T, k = experts.shape
    if offsets is None:
        offsets = _empty(n_experts + 1, torch.int32, experts, stream)
    if slots is None:
        slots = _empty((T, k), torch.int32, experts, stream)
    with torch.cuda.device(experts.device):
        need = int(lib().hikonv_sort_by_expert_workspace_bytes(T, k, n_experts))
        if need and workspace is None:
            workspace = _empty(need, torch.uint8, experts, stream)
        if workspace is not None and (not workspace.is_cuda or workspace.device != experts.device or not workspace.is_contiguous()):
            raise ValueError("workspace must be a contiguous CUDA tensor on experts' device")
        space = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
        _check(lib().hikonv_sort_by_expert(experts.data_ptr(), _INDEX_TYPES[experts.dtype], row, T, k, n_experts,
                                           _vector(offsets, "offsets", torch.int32, (n_experts + 1,), experts),
                                           _vector(slots, "slots", torch.int32, (T, k), experts), *space, _stream_of(experts, stream)),
               "hikonv_sort_by_expert")
    return offsets, slots


def sort_by_expert_workspace_bytes(tokens: int, choices: int, n_experts: int) -> int:
    """Bytes that ``sort_by_expert`` needs between its launches: 0 for up to 4096 pairs."""
    _fits("sort_by_expert", tokens, choices, n_experts)
    return int(lib().hikonv_sort_by_expert_workspace_bytes(tokens, choices, n_experts))


def rows_to_experts(x: torch.Tensor, slots: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Rows of tokens to the places of their pairs: ``out[slots[t, j]] = x[t]``, for any type of 1, 2 or 4 bytes.  ``out`` [T k, H] unless it
    is given (with as many rows as wanted); rows that no slot names are left as they were (undefined when the call makes it).  Its gradient
    is ``rows_from_experts`` without weights."""
    if stream is None:
        done = (_fast or _load_fast()).rows_to_experts(x, slots, out)
        if done is not None:
            return done
    if getattr(x, "dtype", None) is None or x.dtype.itemsize not in (1, 2, 4) or x.dtype.is_complex:
        raise ValueError("x must be a matrix of 1-, 2- or 4-byte elements")
    x_row = _rows(x, "x", (x.dtype,))
    H = x.shape[1]
    places, T, k = _slots(slots, x, x.shape[0])
    if out is None:
        out = _empty((T * k, H), x.dtype, x, stream)
    out_row = _rows(out, "out", (x.dtype,), x, (out.shape[0], H) if out.dim() == 2 else (T * k, H))
    with torch.cuda.device(x.device):
        _check(lib().hikonv_rows_to_experts(x.data_ptr(), x.dtype.itemsize, x_row, places, T, k, H, out.data_ptr(), out_row, out.shape[0],
                                            _stream_of(x, stream)), "hikonv_rows_to_experts")
    return out


def rows_from_experts(y: torch.Tensor, slots: torch.Tensor, weights: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Rows of experts back to their tokens: ``out[t] = residual[t] + sum_j weights[t, j] * y[slots[t, j]]`` in 32-bit arithmetic, rounded
    once.  ``y`` [rows, H] float32, float16 or bfloat16, ``weights`` [T, k] float32 (None: ones), ``residual`` of y's type, which may be
    ``out`` itself.  Pairs without a place add nothing, whatever their weight."""
    if stream is None:
        done = (_fast or _load_fast()).rows_from_experts(y, slots, weights, residual, out)
        if done is not None:
            return done
    if getattr(y, "dtype", None) not in _FLOAT_TYPES:
        raise ValueError("y must be a float32, float16 or bfloat16 matrix")
    y_row = _rows(y, "y", (y.dtype,))
    R, H = y.shape
    places, T, k = _slots(slots, y)
    if out is None:
        out = _empty((T, H), y.dtype, y, stream)
    out_row = _rows(out, "out", (y.dtype,), y, (T, H))
    res_row = H if residual is None else _rows(residual, "residual", (y.dtype,), y, (T, H))
    with torch.cuda.device(y.device):
        _check(lib().hikonv_rows_from_experts(y.data_ptr(), _FLOAT_TYPES[y.dtype], y_row, R, places,
                                              _vector(weights, "weights", torch.float32, (T, k), y), T, k, H,
                                              None if residual is None else residual.data_ptr(), res_row, out.data_ptr(), out_row,
                                              _stream_of(y, stream)), "hikonv_rows_from_experts")
    return out


# As in pyext/fast.cpp.  Zeros to 8 MB take 3 us, to 256 MB 70; finding the rows that no slot names 5.
_ZERO_ALL_BYTES = 8 << 20


def rows_from_experts_grad(grad: torch.Tensor, y: Optional[torch.Tensor], slots: torch.Tensor, weights: Optional[torch.Tensor] = None,
                           grad_y: Optional[torch.Tensor] = None, grad_weights: Optional[torch.Tensor] = None, stream=None) -> tuple:
    """The gradient of ``rows_from_experts``, from the one for its output: (grad_y, grad_weights).  ``grad_y[slots[t, j]]`` is
    ``weights[t, j] * grad[t]``, zeros in the places of pairs without expert; ``grad_weights[t, j]`` the product of ``grad[t]`` with the
    pair's row of ``y``, 0 without one.  Without weights ``y`` is not read (it may be None) and there is no grad_weights.  ``grad_y`` has the rows of
    ``y``, or one for each pair without it, and zeros where no slot names a row (padding of ``y``, a row whose pair was dropped by a slot of
    -1).  In a ``grad_y`` that is given such rows are left as they were: with the slots of ``sort_by_expert`` there are none among T k rows.  The
    residual's gradient is ``grad`` itself."""
    if stream is None:
        done = (_fast or _load_fast()).rows_from_experts_grad(grad, y, slots, weights, grad_y, grad_weights)
        if done is not None:
            return done
    if getattr(grad, "dtype", None) not in _FLOAT_TYPES:
        raise ValueError("grad must be a float32, float16 or bfloat16 matrix")
    grad_row = _rows(grad, "grad", (grad.dtype,))
    H = grad.shape[1]
    places, T, k = _slots(slots, grad, grad.shape[0])
    if weights is None and grad_weights is not None:
        raise ValueError("grad_weights without weights")
    if weights is not None and y is None:
        raise ValueError("the gradient of weights needs y")
    others = None
    if grad_y is None:
        # rows that no slot names are zeros: all rows beforehand where that is cheap, else those alone
        rows = T * k if y is None else y.shape[0]
        small = rows * H * grad.element_size() <= _ZERO_ALL_BYTES
        grad_y = _empty((rows, H), grad.dtype, grad, stream, torch.zeros if small else torch.empty)
        others = None if small else _empty(rows, torch.uint8, grad, stream)
    grad_y_row = _rows(grad_y, "grad_y", (grad.dtype,), grad, (grad_y.shape[0] if grad_y.dim() == 2 else T * k, H))
    R = grad_y.shape[0]
    y_row = H if weights is None else _rows(y, "y", (grad.dtype,), grad, (R, H))
    if weights is not None and grad_weights is None:
        grad_weights = _empty((T, k), torch.float32, grad, stream)
    with torch.cuda.device(grad.device):
        if others is not None:
            _check(lib().hikonv_zero_other_rows(places, T, k, grad_y.data_ptr(), grad.element_size(), grad_y_row, R, H, others.data_ptr(), R,
                                                _stream_of(grad, stream)), "hikonv_zero_other_rows")
        _check(lib().hikonv_rows_from_experts_grad(grad.data_ptr(), _FLOAT_TYPES[grad.dtype], grad_row, None if weights is None else y.data_ptr(),
                                                   y_row, R, places, _vector(weights, "weights", torch.float32, (T, k), grad), T, k, H,
                                                   grad_y.data_ptr(), grad_y_row,
                                                   _vector(grad_weights, "grad_weights", torch.float32, (T, k), grad), _stream_of(grad, stream)),
               "hikonv_rows_from_experts_grad")
    return grad_y, grad_weights


# ------------------------------------------------------------------ blocks of 8-bit floating point numbers

def _f8_rows(rows: tuple, K: int, dtype: torch.dtype, like: torch.Tensor, stream) -> torch.Tensor:
    """A tensor [*rows, K] whose rows begin on 16-byte boundaries."""
    return _empty((*rows, (K + 15) // 16 * 16), dtype, like, stream)[..., :K]


def quantize_blocks(x: torch.Tensor, dtype: torch.dtype = torch.float8_e4m3fn, slots: Optional[torch.Tensor] = None,
                    values: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None, stream=None) -> tuple:
    """Rows of floats to 8-bit floating point numbers with a scale for each block of 128: (values [M, K], scale [ceil(K / 128), M]), with
    ``x[m, k]`` about ``values[m, k] * scale[k // 128, m]``.  With ``slots`` [M, k] (of ``sort_by_expert``) row m goes to the rows
    ``slots[m, j]`` instead: values [M k, K] unless given; rows that no slot names are left as they were.  Rows of values begin on 16-byte
    boundaries (the call's own are so far apart)."""
    if stream is None:
        done = (_fast or _load_fast()).quantize_blocks(x, dtype, slots, values, scale)
        if done is not None:
            return done
    if getattr(x, "dtype", None) not in _FLOAT_TYPES:
        raise ValueError("x must be a float32, float16 or bfloat16 matrix")
    if dtype not in _F8_TYPES:
        raise ValueError("values are float8_e4m3fn or float8_e5m2, not %s" % dtype)
    x_row = _rows(x, "x", (x.dtype,))
    M, K = x.shape
    places, k = None, 0
    if slots is not None:
        places, _, k = _slots(slots, x, M)
    rows = values.shape[0] if values is not None and values.dim() == 2 else M * k if slots is not None else M
    if values is None:
        values = _f8_rows((rows,), K, dtype, x, stream)
    values_row = _rows(values, "values", (dtype,), x, (rows if slots is not None else M, K))
    blocks = (K + 127) // 128
    if scale is None:
        scale = _empty((blocks, rows), torch.float32, x, stream)
    scale_row = _rows(scale, "scale", (torch.float32,), x, (blocks, rows))
    with torch.cuda.device(x.device):
        _check(lib().hikonv_quantize_blocks(x.data_ptr(), _FLOAT_TYPES[x.dtype], x_row, M, K, _F8_TYPES[dtype], places, k,
                                            rows if slots is not None else 0, values.data_ptr(), values_row, scale.data_ptr(), scale_row,
                                            _stream_of(x, stream)), "hikonv_quantize_blocks")
    return values, scale


def quantize_tiles(w: torch.Tensor, dtype: torch.dtype = torch.float8_e4m3fn, values: Optional[torch.Tensor] = None,
                   scale: Optional[torch.Tensor] = None, stream=None) -> tuple:
    """Weights [N, K] or [E, N, K] to 8-bit floating point numbers with a scale for each tile of 128 x 128: (values, scale
    [.., ceil(N / 128), ceil(K / 128)]).  Done once, when weights are loaded."""
    if getattr(w, "dtype", None) not in _FLOAT_TYPES:
        raise ValueError("w must be float32, float16 or bfloat16")
    if dtype not in _F8_TYPES:
        raise ValueError("values are float8_e4m3fn or float8_e5m2, not %s" % dtype)
    w_row = _weight_rows(w, "w", (w.dtype,))
    lead, N, K = tuple(w.shape[:-2]), w.shape[-2], w.shape[-1]
    if values is None:
        values = _f8_rows((*lead, N), K, dtype, w, stream)
    values_row = _weight_rows(values, "values", (dtype,), w, w.shape)
    tiles = lead + ((N + 127) // 128, (K + 127) // 128)
    if scale is None:
        scale = _empty(tiles, torch.float32, w, stream)
    with torch.cuda.device(w.device):
        _check(lib().hikonv_quantize_tiles(w.data_ptr(), _FLOAT_TYPES[w.dtype], w_row, lead[0] if lead else 1, N, K, _F8_TYPES[dtype],
                                           values.data_ptr(), values_row, _vector(scale, "scale", torch.float32, tiles, w),
                                           _stream_of(w, stream)), "hikonv_quantize_tiles")
    return values, scale


def _weight_rows(w: torch.Tensor, name: str, dtypes, like: Optional[torch.Tensor] = None, shape=None) -> int:
    """Checks a matrix of weights, or one per expert, whose rows are equally far apart throughout; returns that distance in elements."""
    if not getattr(w, "is_cuda", False) or w.layout != torch.strided or w.dim() not in (2, 3):
        raise ValueError("%s must be a CUDA tensor of [N, K] or [E, N, K]" % name)
    if w.dtype not in dtypes:
        raise ValueError("%s must have dtype %s, not %s" % (name, " or ".join(str(d) for d in dtypes), w.dtype))
    if like is not None and w.device != like.device:
        raise ValueError("%s is on %s, not on %s" % (name, w.device, like.device))
    if shape is not None and tuple(w.shape) != tuple(shape):
        raise ValueError("%s has shape %s, the call needs %s" % (name, tuple(w.shape), tuple(shape)))
    N, K = w.shape[-2:]
    if K > 1 and w.stride(-1) != 1:
        raise ValueError("%s must have contiguous rows" % name)
    row = w.stride(-2) if N > 1 else w.stride(0) if w.dim() == 3 and w.shape[0] > 1 else K
    if w.dim() == 3 and w.shape[0] > 1 and w.stride(0) != N * row:
        raise ValueError("%s must have its matrices one behind the other" % name)
    _fits(name, *w.shape)
    return row


def linear_f8(x: torch.Tensor, w: torch.Tensor, x_scale: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
              activation: int = ACT_NONE, residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
              out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Matrix product of 8-bit floating point numbers with a scale for each block of 128: ``x`` [M, K] and ``x_scale`` [ceil(K / 128), M] as
    ``quantize_blocks`` gives them, ``w`` [N, K] and ``w_scale`` [ceil(N / 128), ceil(K / 128)] as ``quantize_tiles`` does:
    ``act(sum + bias[n]) + residual[m, n]`` in bfloat16 unless ``out_dtype`` or ``out`` says otherwise (float32, float16).  Either operand
    is float8_e4m3fn or float8_e5m2, with rows on 16-byte boundaries; bias float32; residual of the output's type, which may be ``out``."""
    return _linear_f8("hikonv_linear_f8", x, w, None, x_scale, w_scale, bias, activation, residual, out_dtype, out, stream)


def grouped_linear_f8(x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, x_scale: torch.Tensor, w_scale: torch.Tensor,
                      bias: Optional[torch.Tensor] = None, activation: int = ACT_NONE, residual: Optional[torch.Tensor] = None,
                      out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """``linear_f8`` with a matrix of weights per group of rows: ``w`` [E, N, K], ``w_scale`` [E, ..], ``bias`` [E, N]; rows
    ``offsets[e]`` to ``offsets[e + 1] - 1`` (int32 [E + 1], on the device) belong to matrix e.  Rows of no group are left as they
    were in ``out`` (undefined when the call makes it)."""
    return _linear_f8("hikonv_grouped_linear_f8", x, w, offsets, x_scale, w_scale, bias, activation, residual, out_dtype, out, stream)


def _linear_f8(name, x, w, offsets, x_scale, w_scale, bias, activation, residual, out_dtype, out, stream):
    grouped = name == "hikonv_grouped_linear_f8"
    if stream is None and grouped == (offsets is not None):
        done = (_fast or _load_fast()).linear_f8(x, w, offsets, x_scale, w_scale, bias, activation, residual, out_dtype, out)
        if done is not None:
            return done
    x_row = _rows(x, "x", tuple(_F8_TYPES))
    M, K = x.shape
    w_row = _weight_rows(w, "w", tuple(_F8_TYPES), x)
    if w.dim() != (3 if grouped else 2) or w.shape[-1] != K:
        raise ValueError("w has shape %s, the call needs %s of depth %d" % (tuple(w.shape), "[E, N, K]" if grouped else "[N, K]", K))
    lead, N = tuple(w.shape[:-2]), w.shape[-2]
    blocks = (K + 127) // 128
    scale_row = _rows(x_scale, "x_scale", (torch.float32,), x, (blocks, M))
    if out_dtype is None:
        out_dtype = torch.bfloat16 if out is None else out.dtype
    if out_dtype not in _FLOAT_TYPES:
        raise ValueError("the output is float32, float16 or bfloat16, not %s" % out_dtype)
    if out is None:
        out = _empty((M, N), out_dtype, x, stream)
    ep = EpilogueT(out_type=_FLOAT_TYPES[out_dtype], activation=int(activation))
    out_row = _rows(out, "out", (out_dtype,), x, (M, N))
    ep.d_bias = _vector(bias, "bias", torch.float32, lead + (N,), x)
    if residual is not None:
        ep.residual_row_stride = _rows(residual, "residual", (out_dtype,), x, (M, N))
        ep.d_residual = residual.data_ptr()
    w_scales = _vector(w_scale, "w_scale", torch.float32, lead + ((N + 127) // 128, blocks), x)
    groups = (_vector(offsets, "offsets", torch.int32, (lead[0] + 1,), x), lead[0]) if grouped else ()
    with torch.cuda.device(x.device):
        _check(getattr(lib(), name)(x.data_ptr(), _F8_TYPES[x.dtype], x_row, w.data_ptr(), _F8_TYPES[w.dtype], w_row, *groups, M, N, K,
                                    x_scale.data_ptr(), scale_row, w_scales, out.data_ptr(), out_row, ctypes.byref(ep), _stream_of(x, stream)),
               name)
    return out


def pipe_rate(kind: str, iters: int = 2048, device=None, stream=None) -> dict:
    """Measured rate of one instruction (see ``PIPE_KINDS``): operations per second (instructions x 32
    lanes) and lanes per clock per SM at the device's maximum SM clock.  Synchronises."""
    word = torch.zeros(1, dtype=torch.int32, device=device or "cuda")
    ops, lanes = ctypes.c_double(0.0), ctypes.c_double(0.0)
    with torch.cuda.device(word.device):
        _check(lib().hikonv_pipe_rate(PIPE_KINDS[kind], int(iters), word.data_ptr(), ctypes.byref(ops), ctypes.byref(lanes),
                                      _stream(stream)), "hikonv_pipe_rate")
    return {"ops_per_second": ops.value, "lanes_per_clock_per_sm": lanes.value}
