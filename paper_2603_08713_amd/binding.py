"""Binding of ``libmx4.so`` (C ABI in ``include/mx4.h``), same names as the C entry points.

Marshalling only: tensors in, ``data_ptr()`` + sizes + the current HIP stream out.  Output tensors
are allocated with torch when the caller does not pass them.  Nothing is computed here.  Calls that bring plain CUDA
tensors and all outputs are marshalled natively (csrc_host/marshal.cpp); what that declines goes through ctypes below.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import threading
from typing import Optional, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libmx4.so")
_MARSHAL_PATH = os.path.join(_HERE, "_marshal.so")

MX_RULE_OCP, MX_RULE_FLOOR, MX_RULE_OAS = 0, 1, 2
MX_OUT_F32, MX_OUT_BF16 = 0, 1
MX_ELEM_E2M1, MX_ELEM_E4M3, MX_ELEM_E5M2, MX_ELEM_E2M3, MX_ELEM_E3M2 = 0, 1, 2, 3, 4
_ELEMS = {"e2m1": MX_ELEM_E2M1, "e4m3": MX_ELEM_E4M3, "e5m2": MX_ELEM_E5M2, "e2m3": MX_ELEM_E2M3, "e3m2": MX_ELEM_E3M2}
_RULES = {"ocp": MX_RULE_OCP, "floor": MX_RULE_FLOOR, "oas": MX_RULE_OAS}

_lib: Optional[ctypes.CDLL] = None


class MxError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, mx_status_string(status), status))


def load_library() -> ctypes.CDLL:
    """Load the in-tree HIP library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            "libmx4.so is missing: build it with `python -m paper_2603_08713_amd.build` "
            "(or __graft_entry__.build()); this package has no CPU fallback")
    L = ctypes.CDLL(_LIB_PATH)
    i64, i32, vp, ci = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int
    L.mx_quantize.restype = ci
    L.mx_quantize.argtypes = [vp, i64, i64, i64, ci, vp, vp, vp]
    L.mx_quantize_oas.restype = ci
    L.mx_quantize_oas.argtypes = [vp, i64, i64, i64, vp, vp, vp]
    L.mx_quantize_mbs.restype = ci
    L.mx_quantize_mbs.argtypes = [vp, i64, i64, i64, ci, vp, vp, vp, vp]
    L.mx_quantize_mbs_pair.restype = ci
    L.mx_quantize_mbs_pair.argtypes = [vp, i64, i64, vp, vp, vp, vp, i64, i64, vp, vp, vp, i64, ci, vp]
    L.mx_gemm_mbs_quantize_a.restype = ci
    L.mx_gemm_mbs_quantize_a.argtypes = [vp, i64, ci, ci, vp, vp, vp, i64, i64, i64, ci, vp, i64, vp]
    L.mx_quantize_mbs_dynamic.restype = ci
    L.mx_quantize_mbs_dynamic.argtypes = [vp, i64, i64, i64, ci, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                          vp, vp, vp, vp]
    L.mx_mbs_lut_build.restype = ci
    L.mx_mbs_lut_build.argtypes = [vp, vp]
    L.mx_quantize_mbs_dynamic_lut.restype = ci
    L.mx_quantize_mbs_dynamic_lut.argtypes = [vp, i64, i64, i64, ci, vp, ci, vp, vp, vp, vp]
    L.mx_quantize_mbs_dynamic_lut_static.restype = ci
    L.mx_quantize_mbs_dynamic_lut_static.argtypes = [vp, i64, i64, i64, ci, ci, vp, vp, vp, vp]
    L.mx_dequantize.restype = ci
    L.mx_dequantize.argtypes = [vp, vp, vp, i64, i64, ci, vp, i64, vp]
    L.mx_gemm.restype = ci
    L.mx_gemm.argtypes = [vp, vp, vp, vp, i64, i64, i64, ci, vp, i64, vp]
    L.mx_gemm_mbs.restype = ci
    L.mx_gemm_mbs.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, ci, vp, i64, vp]
    L.mx_gemm_mbs_grouped.restype = ci
    L.mx_gemm_mbs_grouped.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp, i64, i64, i64, ci, vp, i64, vp]
    L.mx_quantize_elem.restype = ci
    L.mx_quantize_elem.argtypes = [ci, vp, i64, i64, i64, ci, ci, vp, vp, vp, vp]
    L.mx_dequantize_elem.restype = ci
    L.mx_dequantize_elem.argtypes = [ci, vp, vp, vp, i64, i64, ci, vp, i64, vp]
    L.mx_gemm_mbs_elem.restype = ci
    L.mx_gemm_mbs_elem.argtypes = [ci, vp, vp, vp, ci, vp, vp, vp, i64, i64, i64, ci, vp, i64, vp]
    L.mx_status_string.restype = ctypes.c_char_p
    L.mx_status_string.argtypes = [ci]
    L.mx_version.restype = ci
    L.mx_version.argtypes = []
    L.mx_internal_quantize.restype = ci
    L.mx_internal_quantize.argtypes = [vp, i64, i64, i64, ci, ci, ci, vp, vp, vp, vp]
    L.mx_internal_quantize_elem.restype = ci
    L.mx_internal_quantize_elem.argtypes = [ci, vp, i64, i64, i64, ci, ci, ci, vp, vp, vp, vp]
    L.mx_internal_gemm.restype = ci
    L.mx_internal_gemm.argtypes = [vp, vp, vp, vp, vp, vp, ci, i32, vp, i64, i64, i64, ci, vp, i64, ci, ci, vp]
    L.mx_internal_gemm_plan.restype = ci
    L.mx_internal_gemm_plan.argtypes = [i64, i64, i64, ci, ci, ci, ctypes.c_char_p, ci]
    L.mx_quantize_elem_mbs_dynamic.restype = ci
    L.mx_quantize_elem_mbs_dynamic.argtypes = [ci, vp, i64, i64, i64, ci, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                               vp, vp, vp, vp]
    L.mx_gemm_mbs_elem_grouped.restype = ci
    L.mx_gemm_mbs_elem_grouped.argtypes = [ci, vp, vp, vp, ci, vp, vp, vp, ctypes.c_int32, vp, i64, i64, i64, ci, vp, i64, vp]
    L.mx_internal_gemm_elem.restype = ci
    L.mx_internal_gemm_elem.argtypes = [ci, vp, vp, vp, ci, vp, vp, vp, i64, i64, i64, ci, vp, i64, ci, vp]
    ip, d, f = vp, ctypes.c_double, ctypes.c_float
    L.mx_kv_plan.restype = ci
    L.mx_kv_plan.argtypes = [ip, ip, i64, i64, ip, i64, ip, i64, ip, i64, vp, ip, vp, ip, ip, vp]
    L.mx_qk_norm_rope.restype = ci
    L.mx_qk_norm_rope.argtypes = [vp, i64, vp, i64, ip, vp, i64, vp, vp, d, ci, i64, i64, i64, i64, i64, vp, i64, vp, i64, vp]
    L.mx_kv_write.restype = ci
    L.mx_kv_write.argtypes = [vp, i64, vp, i64, vp, ci, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, vp]
    L.mx_qk_norm_rope_kv_write.restype = ci
    L.mx_qk_norm_rope_kv_write.argtypes = [vp, i64, vp, i64, vp, i64, ip, vp, i64, vp, vp, d, ci, vp, ci, vp, vp, vp, vp, vp, vp,
                                           i64, i64, i64, i64, i64, i64, i64, vp, i64, vp]
    L.mx_kv_read.restype = ci
    L.mx_kv_read.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, ci, vp, i64, vp, i64, vp]
    L.mx_attention_kv.restype = ci
    L.mx_attention_kv.argtypes = [vp, i64, vp, ip, ip, i64, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i64, f, ci, i64, vp, i64, vp,
                                  vp, i64, vp]
    L.mx_internal_attention_kv.restype = ci
    L.mx_internal_attention_kv.argtypes = [ci] + L.mx_attention_kv.argtypes
    L.mx_internal_attention_kv_workspace.restype = i64
    L.mx_internal_attention_kv_workspace.argtypes = [ci, i64, i64, i64, i64, i64]
    L.mx_attention_kv_workspace.restype = i64
    L.mx_attention_kv_workspace.argtypes = [i64, i64, i64, i64, i64]
    _lib = L
    return L


def mx_status_string(status: int) -> str:
    return load_library().mx_status_string(int(status)).decode()


def mx_version() -> int:
    return load_library().mx_version()


# ---- development routing (tests only) ----------------------------------------------------------------
# The library keeps no switches.  Its development entry points (csrc/mx_internal.h) take the choice of
# implementation as one more argument of the call; `forced(...)` makes the functions below pass such a
# choice, for the calling thread, while the block runs.
_dev = threading.local()


@contextlib.contextmanager
def forced(**choices):
    """quantize_hw / quantize_elem_hw = 0 or 1 (rounding implementation), gemm_shape = a kernel form and
    tile shape code of mx_gemm.hip, gemm_elem = which kernel takes an 8-/6-bit GEMM (1 = the main kernel's general
    form, 2 = the main kernel in the form the problem allows, 3 = the few-row kernel, 16 / 17 / 18 = the main kernel on 256 x 128 /
    128 x 128 / 64 x 128 tiles, the last two for K >= 512), attention = 1 or 2 (the kernel for few or for many rows)."""
    allowed = {"quantize_hw", "quantize_elem_hw", "gemm_shape", "gemm_elem", "attention"}
    if set(choices) - allowed:
        raise TypeError("unknown choice: %s" % sorted(set(choices) - allowed))
    old = getattr(_dev, "choices", {})
    _dev.choices = dict(old, **choices)
    try:
        yield
    finally:
        _dev.choices = old


def _forced(name):
    choices = getattr(_dev, "choices", None)
    return choices.get(name) if choices else None


def gemm_plan(M: int, N: int, K: int, a_has_mbs: bool = True, b_has_mbs: bool = True, grouped: bool = False,
              num_groups: int = 1) -> str:
    """The kernel the dispatcher of mx_gemm / mx_gemm_mbs / mx_gemm_mbs_grouped (of num_groups groups) picks for a problem
    with aligned arrays (host only; reported by the benchmark beside its timings)."""
    buf = ctypes.create_string_buffer(512)
    _check((_lib or load_library()).mx_internal_gemm_plan(M, N, K, int(a_has_mbs), int(b_has_mbs), int(num_groups) if grouped else 0, buf, 512),
           "mx_internal_gemm_plan")
    return buf.value.decode()


def _quantize_forced(where, hw, x, rows, K, ldx, rule, use_mbs, codes, scales, mbs):
    _check((_lib or load_library()).mx_internal_quantize(_ptr(x), rows, K, ldx, rule, int(use_mbs), int(hw), _ptr(codes),
                                               _ptr(scales), _ptr(mbs), _stream()), where + " (mx_internal_quantize)")


def _gemm_forced(where, shape, a, b, grouped, num_groups, row_offsets, M, N, K, code, out, ldc, mbs_entry):
    _check((_lib or load_library()).mx_internal_gemm(_ptr(a[0]), _ptr(a[1]), _ptr(a[2]), _ptr(b[0]), _ptr(b[1]), _ptr(b[2]),
                                           int(grouped), int(num_groups), _ptr(row_offsets), M, N, K, code, _ptr(out),
                                           ldc, int(mbs_entry), int(shape), _stream()), where + " (mx_internal_gemm)")


# ---- helpers ---------------------------------------------------------------------------------------
# The marshalling stands in front of kernels of a few microseconds, so it is kept short: natively a call costs about 3.3 us of host
# time, nearly all of it the launch; through ctypes and the checks below 5.5 (quantizer and GEMM in a row 7.2 and 13.7).
_torch_module = None
_stream_handle = _stream_device = None  # torch's calls for the current stream's handle and the current device, if it has them
_native = None                          # the native marshaller, once torch is there
_out_dtypes = {}                        # what a caller may pass as an output type -> (type code, torch dtype)


def _torch():
    global _torch_module, _stream_handle, _stream_device, _native
    if _torch_module is None:
        import torch

        _stream_handle = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _stream_device = getattr(torch._C, "_cuda_getDevice", None)
        for names, value in (((MX_OUT_F32, "f32", "fp32", torch.float32), (MX_OUT_F32, torch.float32)),
                             ((MX_OUT_BF16, "bf16", torch.bfloat16), (MX_OUT_BF16, torch.bfloat16))):
            _out_dtypes.update((name, value) for name in names)
        _native = _load_native(torch)
        _torch_module = torch
    return _torch_module


# (in the order in which csrc_host/marshal.cpp keeps the addresses)
_NATIVE_CALLS = ("mx_quantize", "mx_quantize_mbs", "mx_quantize_mbs_pair", "mx_quantize_mbs_dynamic", "mx_quantize_elem", "mx_dequantize", "mx_gemm",
                 "mx_gemm_mbs", "mx_gemm_mbs_grouped", "mx_gemm_mbs_quantize_a", "mx_gemm_mbs_elem", "mx_gemm_mbs_elem_grouped", "mx_kv_plan",
                 "mx_qk_norm_rope", "mx_kv_write", "mx_qk_norm_rope_kv_write", "mx_kv_read", "mx_attention_kv", "mx_attention_kv_workspace")


def marshal_tag(torch) -> str:
    """What a native marshaller has to have been compiled against to be loaded here: this interpreter and this torch."""
    import sysconfig

    return "%s torch-%s" % (sysconfig.get_config_var("SOABI"), torch.__version__)


def _load_native(torch):
    """The native marshaller (the build step makes it beside libmx4.so).  Without one, or with one made for another torch or
    interpreter, every call goes through ctypes."""
    if not os.path.exists(_MARSHAL_PATH):
        return None
    import importlib.machinery
    import importlib.util
    import warnings

    L = load_library()
    loader = importlib.machinery.ExtensionFileLoader("_marshal", _MARSHAL_PATH)
    try:
        module = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_marshal", _MARSHAL_PATH, loader=loader))
        loader.exec_module(module)
        built_for = module.built_for()
    except (ImportError, AttributeError) as e:
        warnings.warn("%s does not load, calls go through ctypes: %s" % (_MARSHAL_PATH, e))
        return None
    if built_for != marshal_tag(torch):
        warnings.warn("%s was built for %s, not for %s: calls go through ctypes" % (_MARSHAL_PATH, built_for, marshal_tag(torch)))
        return None
    module.use(*(ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in _NATIVE_CALLS))
    return module


def _done(status, where: str) -> bool:
    """Whether the native marshaller has made the call (None: it declined)."""
    if status is None:
        return False
    _check(status, where)
    return True


def _rule(rule) -> int:
    return _RULES[rule] if isinstance(rule, str) else int(rule)


def _elem(elem) -> int:
    return _ELEMS[elem] if isinstance(elem, str) else int(elem)


def _stream() -> int:
    torch = _torch_module or _torch()
    if _stream_handle is None or _stream_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _stream_handle(_stream_device())


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _check(status: int, where: str):
    if status != 0:
        raise MxError(status, where)


def _rows_ld(x):
    torch = _torch_module or _torch()
    if x.dtype is not torch.bfloat16 or x.dim() != 2 or not x.is_cuda:
        raise TypeError("expected a 2-D bf16 CUDA tensor")
    rows, K = x.shape
    ld, inner = x.stride()
    if inner != 1 and K > 1:
        raise ValueError("innermost dimension must be contiguous")
    return rows, K, (ld if rows > 1 else max(ld, K))


def _u8(t, shape, name):
    if t.dtype is not _torch_module.uint8 or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        raise TypeError("%s must be a contiguous uint8 CUDA tensor of shape %s" % (name, shape))
    return t


def _outputs(x, rows, K, code_bytes, codes, scales, mbs, want_mbs):
    torch = _torch_module
    shape = (rows, code_bytes)
    if codes is None:
        codes = torch.empty(shape, dtype=torch.uint8, device=x.device)
    else:
        _u8(codes, shape, "codes")
    shape = (rows, K // 32)
    if scales is None:
        scales = torch.empty(shape, dtype=torch.uint8, device=x.device)
    else:
        _u8(scales, shape, "scales")
    if want_mbs:
        shape = (rows, (K + 127) // 128)
        if mbs is None:
            mbs = torch.empty(shape, dtype=torch.uint8, device=x.device)
        else:
            _u8(mbs, shape, "mbs")
    return codes, scales, mbs


def _alloc_outputs(x, rows, K, codes, scales, mbs, want_mbs):
    return _outputs(x, rows, K, K // 2, codes, scales, mbs, want_mbs)


# ---- entry points ----------------------------------------------------------------------------------
def mx_quantize(x, rule="ocp", codes=None, scales=None):
    """bf16 [rows, K] -> (codes uint8 [rows, K/2], scales uint8 [rows, K/32]) with `rule`, no MBS."""
    if _native is not None and scales is not None and not getattr(_dev, "choices", None) and _done(
            _native.quantize(x, rule, codes, scales), "mx_quantize"):
        return codes, scales
    rows, K, ldx = _rows_ld(x)
    codes, scales, _ = _alloc_outputs(x, rows, K, codes, scales, None, False)
    hw = _forced("quantize_hw")
    if hw is not None:
        _quantize_forced("mx_quantize", hw, x, rows, K, ldx, _rule(rule), False, codes, scales, None)
    else:
        _check((_lib or load_library()).mx_quantize(x.data_ptr(), rows, K, ldx, _rule(rule), codes.data_ptr(),
                                                    scales.data_ptr(), _stream()), "mx_quantize")
    return codes, scales


def mx_quantize_oas(x, codes=None, scales=None):
    rows, K, ldx = _rows_ld(x)
    codes, scales, _ = _alloc_outputs(x, rows, K, codes, scales, None, False)
    hw = _forced("quantize_hw")
    if hw is not None:
        _quantize_forced("mx_quantize_oas", hw, x, rows, K, ldx, MX_RULE_OAS, False, codes, scales, None)
    else:
        _check((_lib or load_library()).mx_quantize_oas(x.data_ptr(), rows, K, ldx, codes.data_ptr(), scales.data_ptr(),
                                                        _stream()), "mx_quantize_oas")
    return codes, scales


def mx_quantize_mbs(x, rule="oas", codes=None, scales=None, mbs=None):
    """MBS-Static quantization -> (codes, scales, mbs uint8 [rows, ceil(K/128)])."""
    if _native is not None and mbs is not None and not getattr(_dev, "choices", None) and _done(
            _native.quantize_mbs(x, rule, codes, scales, mbs), "mx_quantize_mbs"):
        return codes, scales, mbs
    rows, K, ldx = _rows_ld(x)
    codes, scales, mbs = _alloc_outputs(x, rows, K, codes, scales, mbs, True)
    hw = _forced("quantize_hw")
    if hw is not None:
        _quantize_forced("mx_quantize_mbs", hw, x, rows, K, ldx, _rule(rule), True, codes, scales, mbs)
    else:
        _check((_lib or load_library()).mx_quantize_mbs(x.data_ptr(), rows, K, ldx, _rule(rule), codes.data_ptr(),
                                                        scales.data_ptr(), mbs.data_ptr(), _stream()), "mx_quantize_mbs")
    return codes, scales, mbs


def mx_quantize_mbs_pair(x0, x1, rule="oas", out0=None, out1=None):
    """MBS-Static quantization of two tensors with the same K in one launch -> ((codes, scales, mbs), (...))."""
    if _native is not None and type(out0) is tuple and type(out1) is tuple and len(out0) == len(out1) == 3 and _done(
            _native.quantize_mbs_pair(x0, x1, rule, *out0, *out1), "mx_quantize_mbs_pair"):
        return out0, out1
    rows0, K, ld0 = _rows_ld(x0)
    rows1, K1, ld1 = _rows_ld(x1)
    if K != K1:
        raise ValueError("the two tensors must share K")
    o0 = _alloc_outputs(x0, rows0, K, *(out0 or (None, None, None)), True)
    o1 = _alloc_outputs(x1, rows1, K, *(out1 or (None, None, None)), True)
    _check((_lib or load_library()).mx_quantize_mbs_pair(_ptr(x0), rows0, ld0, _ptr(o0[0]), _ptr(o0[1]), _ptr(o0[2]),
                                               _ptr(x1), rows1, ld1, _ptr(o1[0]), _ptr(o1[1]), _ptr(o1[2]),
                                               K, _rule(rule), _stream()), "mx_quantize_mbs_pair")
    return o0, o1


def mx_quantize_mbs_dynamic(x, rule="oas", cand_first=0, cand_count=16, cand_stride=16, codes=None, scales=None,
                            mbs=None):
    """MBS-Dynamic quantization (searched word per 1x128 window) -> (codes, scales, mbs)."""
    if _native is not None and mbs is not None and not getattr(_dev, "choices", None) and _done(
            _native.quantize_mbs_dynamic(x, rule, cand_first, cand_count, cand_stride, codes, scales, mbs), "mx_quantize_mbs_dynamic"):
        return codes, scales, mbs
    rows, K, ldx = _rows_ld(x)
    codes, scales, mbs = _alloc_outputs(x, rows, K, codes, scales, mbs, True)
    _check((_lib or load_library()).mx_quantize_mbs_dynamic(_ptr(x), rows, K, ldx, _rule(rule), int(cand_first),
                                                  int(cand_count), int(cand_stride), _ptr(codes), _ptr(scales),
                                                  _ptr(mbs), _stream()), "mx_quantize_mbs_dynamic")
    return codes, scales, mbs


def mx_mbs_lut_build(lut=None):
    """The table of squared relative errors MBS-Dynamic reads (2 x 64 points x 16 slots, fp16 bit patterns as int16)."""
    torch = _torch()
    if lut is None:
        lut = torch.empty((2, 64, 16), dtype=torch.int16, device="cuda")
    if lut.dtype != torch.int16 or not lut.is_cuda or not lut.is_contiguous() or lut.numel() != 2048:
        raise TypeError("lut must be a contiguous int16 CUDA tensor of 2048 elements")
    _check((_lib or load_library()).mx_mbs_lut_build(_ptr(lut), _stream()), "mx_mbs_lut_build")
    return lut


def mx_quantize_mbs_dynamic_lut(x, lut, rule="oas", keep_static=True, codes=None, scales=None, mbs=None):
    """MBS-Dynamic quantization through the table (word 16 j* of least tabulated cost per 1x128 window) -> (codes, scales, mbs)."""
    torch = _torch()
    rows, K, ldx = _rows_ld(x)
    if lut.dtype != torch.int16 or not lut.is_cuda or not lut.is_contiguous() or lut.numel() != 2048:
        raise TypeError("lut must be a contiguous int16 CUDA tensor of 2048 elements")
    codes, scales, mbs = _alloc_outputs(x, rows, K, codes, scales, mbs, True)
    _check((_lib or load_library()).mx_quantize_mbs_dynamic_lut(_ptr(x), rows, K, ldx, _rule(rule), _ptr(lut), int(bool(keep_static)),
                                                      _ptr(codes), _ptr(scales), _ptr(mbs), _stream()),
           "mx_quantize_mbs_dynamic_lut")
    return codes, scales, mbs


def mx_quantize_mbs_dynamic_lut_static(x, codes, scales, mbs, rule="oas", keep_static=True):
    """mx_quantize_mbs_dynamic_lut on the table the library keeps per GPU; the call allocates nothing, so the
    caller passes the three output tensors ([rows, K/2], [rows, K/32], [rows, ceil(K/128)], uint8)."""
    rows, K, ldx = _rows_ld(x)
    _alloc_outputs(x, rows, K, codes, scales, mbs, True)  # given all three, this only checks them
    _check((_lib or load_library()).mx_quantize_mbs_dynamic_lut_static(_ptr(x), rows, K, ldx, _rule(rule), int(bool(keep_static)),
                                                             _ptr(codes), _ptr(scales), _ptr(mbs), _stream()),
           "mx_quantize_mbs_dynamic_lut_static")
    return codes, scales, mbs


def _out_dtype(dtype) -> Tuple[int, object]:
    if _torch_module is None:
        _torch()
    try:
        return _out_dtypes[dtype]
    except (KeyError, TypeError):  # what is equal to one of the names without hashing like it (a 0-d array or tensor)
        for name, value in _out_dtypes.items():
            if dtype == name:
                return value
    raise ValueError("output dtype must be fp32 or bf16")


def _matrix(rows, cols, out_dtype, out, device, what):
    """The output matrix (allocated if not given), its type code and its leading dimension."""
    code, tdt = _out_dtype(out_dtype)
    if out is None:
        out = _torch_module.empty((rows, cols), dtype=tdt, device=device)
    if out.dtype is not tdt or out.shape != (rows, cols):
        raise TypeError(what)
    ld, inner = out.stride()
    if inner != 1 and cols > 1:
        raise TypeError(what)
    return code, out, (ld if rows > 1 else max(ld, cols))


def mx_dequantize(codes, scales, mbs=None, out_dtype="f32", out=None):
    if _native is not None and out is not None and _done(_native.dequantize(codes, scales, mbs, out_dtype, out), "mx_dequantize"):
        return out
    shape = codes.shape
    rows, K = shape[0], shape[1] * 2
    code, out, ldo = _matrix(rows, K, out_dtype, out, codes.device,
                             "out must be [rows, K] of the requested dtype with a contiguous last dimension")
    _check((_lib or load_library()).mx_dequantize(codes.data_ptr(), _ptr(scales), _ptr(mbs), rows, K, code,
                                                  out.data_ptr(), ldo, _stream()), "mx_dequantize")
    return out


def _c_tensor(M, N, out_dtype, out, device):
    return _matrix(M, N, out_dtype, out, device, "C must be [M, N] of the requested dtype with a contiguous last dimension")


def mx_gemm(a_codes, a_scales, b_codes, b_scales, out_dtype="f32", out=None):
    """Plain MXFP4 GEMM: C[M,N] = A[M,K] . B[N,K]^T."""
    if _native is not None and out is not None and not getattr(_dev, "choices", None) and _done(
            _native.gemm(a_codes, a_scales, b_codes, b_scales, out_dtype, out), "mx_gemm"):
        return out
    a_shape, b_shape = a_codes.shape, b_codes.shape
    M, half, N = a_shape[0], a_shape[1], b_shape[0]
    if b_shape[1] != half:
        raise ValueError("A and B disagree on K")
    code, out, ldc = _c_tensor(M, N, out_dtype, out, a_codes.device)
    shape = _forced("gemm_shape")
    if shape is not None:
        _gemm_forced("mx_gemm", shape, (a_codes, a_scales, None), (b_codes, b_scales, None), False, 0, None, M, N, 2 * half,
                     code, out, ldc, False)
    else:
        _check((_lib or load_library()).mx_gemm(a_codes.data_ptr(), _ptr(a_scales), b_codes.data_ptr(), _ptr(b_scales),
                                                M, N, 2 * half, code, out.data_ptr(), ldc, _stream()), "mx_gemm")
    return out


def mx_gemm_mbs(a_codes, a_scales, a_mbs, b_codes, b_scales, b_mbs, out_dtype="f32", out=None):
    """GEMM with the per-macro-block MBS correction; a_mbs / b_mbs may be None."""
    if _native is not None and out is not None and not getattr(_dev, "choices", None) and _done(
            _native.gemm_mbs(a_codes, a_scales, a_mbs, b_codes, b_scales, b_mbs, out_dtype, out), "mx_gemm_mbs"):
        return out
    a_shape, b_shape = a_codes.shape, b_codes.shape
    M, half, N = a_shape[0], a_shape[1], b_shape[0]
    if b_shape[1] != half:
        raise ValueError("A and B disagree on K")
    code, out, ldc = _c_tensor(M, N, out_dtype, out, a_codes.device)
    shape = _forced("gemm_shape")
    if shape is not None:
        _gemm_forced("mx_gemm_mbs", shape, (a_codes, a_scales, a_mbs), (b_codes, b_scales, b_mbs), False, 0, None, M, N,
                     2 * half, code, out, ldc, True)
    else:
        _check((_lib or load_library()).mx_gemm_mbs(a_codes.data_ptr(), _ptr(a_scales), _ptr(a_mbs), b_codes.data_ptr(),
                                                    _ptr(b_scales), _ptr(b_mbs), M, N, 2 * half, code, out.data_ptr(),
                                                    ldc, _stream()), "mx_gemm_mbs")
    return out


def elem_code_bytes(elem, K: int) -> int:
    """Bytes of a row of K codes: one per element for the 8-bit formats, 6-bit codes packed for E2M3 / E3M2."""
    return K * 3 // 4 if _elem(elem) in (MX_ELEM_E2M3, MX_ELEM_E3M2) else K


def mx_quantize_elem(x, elem="e4m3", rule="oas", use_mbs=True, codes=None, scales=None, mbs=None):
    """Quantize into an 8-bit (codes one per byte) or 6-bit (packed) MX element format, with or without MBS words."""
    if _native is not None and scales is not None and not getattr(_dev, "choices", None) and _done(
            _native.quantize_elem(x, elem, rule, use_mbs, codes, scales, mbs), "mx_quantize_elem"):
        return codes, scales, (mbs if use_mbs else None)
    rows, K, ldx = _rows_ld(x)
    codes, scales, mbs = _outputs(x, rows, K, elem_code_bytes(elem, K), codes, scales, mbs, use_mbs)
    hw = _forced("quantize_elem_hw")
    if hw is None:
        _check((_lib or load_library()).mx_quantize_elem(_elem(elem), _ptr(x), rows, K, ldx, _rule(rule), int(bool(use_mbs)),
                                               _ptr(codes), _ptr(scales), _ptr(mbs) if use_mbs else None, _stream()),
               "mx_quantize_elem")
    else:
        _check((_lib or load_library()).mx_internal_quantize_elem(_elem(elem), _ptr(x), rows, K, ldx, _rule(rule), int(bool(use_mbs)),
                                                        int(hw), _ptr(codes), _ptr(scales), _ptr(mbs) if use_mbs else None,
                                                        _stream()), "mx_quantize_elem (mx_internal_quantize_elem)")
    return codes, scales, (mbs if use_mbs else None)


def mx_quantize_elem_mbs_dynamic(x, elem, rule="oas", cand_first=0, cand_count=16, cand_stride=16, codes=None, scales=None,
                                 mbs=None):
    """MBS-Dynamic into an 8-bit or 6-bit element format: the word of every 1x128 window searched among the static
    word and cand_count candidates for the least squared error.  Returns (codes, scales, mbs)."""
    rows, K, ldx = _rows_ld(x)
    codes, scales, mbs = _outputs(x, rows, K, elem_code_bytes(elem, K), codes, scales, mbs, True)
    _check((_lib or load_library()).mx_quantize_elem_mbs_dynamic(_elem(elem), _ptr(x), rows, K, ldx, _rule(rule), int(cand_first),
                                                       int(cand_count), int(cand_stride), _ptr(codes), _ptr(scales),
                                                       _ptr(mbs), _stream()), "mx_quantize_elem_mbs_dynamic")
    return codes, scales, mbs


def mx_dequantize_elem(elem, codes, scales, mbs=None, out_dtype="f32", out=None):
    """Dequantize codes of an 8-bit (one per byte) or 6-bit (packed) MX element format to fp32 or bf16.  K is taken
    from the scale array."""
    rows, K = codes.shape[0], scales.shape[1] * 32
    if codes.shape[1] != elem_code_bytes(elem, K):
        raise ValueError("the code array does not have the row length of its format")
    code, out, ldo = _matrix(rows, K, out_dtype, out, codes.device,
                             "out must be [rows, K] of the requested dtype with a contiguous last dimension")
    _check((_lib or load_library()).mx_dequantize_elem(_elem(elem), _ptr(codes), _ptr(scales), _ptr(mbs), rows, K, code, _ptr(out),
                                             ldo, _stream()), "mx_dequantize_elem")
    return out


def mx_gemm_mbs_elem(a_elem, a_codes, a_scales, a_mbs, b_elem, b_codes, b_scales, b_mbs, out_dtype="f32", out=None):
    """GEMM with the MBS correction for operands in 8-bit or (packed) 6-bit MX element formats; a_mbs / b_mbs may
    be None.  K is taken from the scale arrays."""
    if _native is not None and out is not None and not getattr(_dev, "choices", None) and _done(
            _native.gemm_mbs_elem(a_elem, a_codes, a_scales, a_mbs, b_elem, b_codes, b_scales, b_mbs, out_dtype, out), "mx_gemm_mbs_elem"):
        return out
    M, N, K = a_codes.shape[0], b_codes.shape[0], a_scales.shape[1] * 32
    if b_scales.shape[1] * 32 != K or a_codes.shape[1] != elem_code_bytes(a_elem, K) or b_codes.shape[1] != elem_code_bytes(b_elem, K):
        raise ValueError("A and B disagree on K, or a code array does not have the row length of its format")
    code, out, ldc = _c_tensor(M, N, out_dtype, out, a_codes.device)
    force = _forced("gemm_elem")
    if force:
        _check((_lib or load_library()).mx_internal_gemm_elem(_elem(a_elem), _ptr(a_codes), _ptr(a_scales), _ptr(a_mbs), _elem(b_elem),
                                                    _ptr(b_codes), _ptr(b_scales), _ptr(b_mbs), M, N, K, code, _ptr(out),
                                                    ldc, int(force), _stream()),
               "mx_gemm_mbs_elem (mx_internal_gemm_elem)")
    else:
        _check((_lib or load_library()).mx_gemm_mbs_elem(_elem(a_elem), _ptr(a_codes), _ptr(a_scales), _ptr(a_mbs), _elem(b_elem),
                                               _ptr(b_codes), _ptr(b_scales), _ptr(b_mbs), M, N, K, code, _ptr(out), ldc,
                                               _stream()), "mx_gemm_mbs_elem")
    return out


def mx_gemm_mbs_elem_grouped(a_elem, a_codes, a_scales, a_mbs, b_elem, b_codes, b_scales, b_mbs, row_offsets, N,
                             out_dtype="f32", out=None):
    """Grouped GEMM for operands in 8-bit or 6-bit element formats: rows row_offsets[e]..row_offsets[e+1]-1 of A
    times B_e^T, B stacked [G*N, ...]."""
    if _native is not None and out is not None and not getattr(_dev, "choices", None) and _done(
            _native.gemm_mbs_elem_grouped(a_elem, a_codes, a_scales, a_mbs, b_elem, b_codes, b_scales, b_mbs, row_offsets, N, out_dtype, out), "mx_gemm_mbs_elem_grouped"):
        return out
    torch = _torch_module or _torch()
    M, K = a_codes.shape[0], a_scales.shape[1] * 32
    if row_offsets.dtype != torch.int64 or not row_offsets.is_cuda or not row_offsets.is_contiguous():
        raise TypeError("row_offsets must be a contiguous int64 CUDA tensor")
    G = row_offsets.numel() - 1
    if (b_codes.shape[0] != G * N or b_scales.shape[1] * 32 != K or a_codes.shape[1] != elem_code_bytes(a_elem, K)
            or b_codes.shape[1] != elem_code_bytes(b_elem, K)):
        raise ValueError("B must hold num_groups stacked [N, K] weights in its format's row length")
    code, out, ldc = _c_tensor(M, N, out_dtype, out, a_codes.device)
    _check((_lib or load_library()).mx_gemm_mbs_elem_grouped(_elem(a_elem), _ptr(a_codes), _ptr(a_scales), _ptr(a_mbs), _elem(b_elem),
                                                   _ptr(b_codes), _ptr(b_scales), _ptr(b_mbs), G, _ptr(row_offsets), M, N, K,
                                                   code, _ptr(out), ldc, _stream()), "mx_gemm_mbs_elem_grouped")
    return out


def mx_gemm_mbs_quantize_a(a, rule, b_codes, b_scales, b_mbs, out_dtype="f32", out=None, a_use_mbs=True):
    """Few-row GEMM with the bf16 activations `a` [M, K] quantized inside the kernel (M <= 64)."""
    if _native is not None and out is not None and not getattr(_dev, "choices", None) and _done(
            _native.gemm_mbs_quantize_a(a, rule, a_use_mbs, b_codes, b_scales, b_mbs, out_dtype, out), "mx_gemm_mbs_quantize_a"):
        return out
    M, K, lda = _rows_ld(a)
    N = b_codes.shape[0]
    if b_codes.shape[1] * 2 != K:
        raise ValueError("A and B disagree on K")
    code, out, ldc = _c_tensor(M, N, out_dtype, out, a.device)
    _check((_lib or load_library()).mx_gemm_mbs_quantize_a(_ptr(a), lda, _rule(rule), int(bool(a_use_mbs)), _ptr(b_codes),
                                                 _ptr(b_scales), _ptr(b_mbs), M, N, K, code, _ptr(out), ldc,
                                                 _stream()), "mx_gemm_mbs_quantize_a")
    return out


def mx_gemm_mbs_grouped(a_codes, a_scales, a_mbs, b_codes, b_scales, b_mbs, row_offsets, N, out_dtype="f32",
                        out=None):
    """Grouped GEMM: rows row_offsets[e]..row_offsets[e+1]-1 of A times B_e^T, B stacked [G*N, K]."""
    if _native is not None and out is not None and not getattr(_dev, "choices", None) and _done(
            _native.gemm_mbs_grouped(a_codes, a_scales, a_mbs, b_codes, b_scales, b_mbs, row_offsets, N, out_dtype, out), "mx_gemm_mbs_grouped"):
        return out
    torch = _torch_module or _torch()
    M, K = a_codes.shape[0], a_codes.shape[1] * 2
    if row_offsets.dtype != torch.int64 or not row_offsets.is_cuda or not row_offsets.is_contiguous():
        raise TypeError("row_offsets must be a contiguous int64 CUDA tensor")
    G = row_offsets.numel() - 1
    if b_codes.shape[0] != G * N or b_codes.shape[1] * 2 != K:
        raise ValueError("B must hold num_groups stacked [N, K] weights")
    code, out, ldc = _c_tensor(M, N, out_dtype, out, a_codes.device)
    shape = _forced("gemm_shape")
    if shape is not None:
        _gemm_forced("mx_gemm_mbs_grouped", shape, (a_codes, a_scales, a_mbs), (b_codes, b_scales, b_mbs), True, G, row_offsets,
                     M, N, K, code, out, ldc, True)
    else:
        _check((_lib or load_library()).mx_gemm_mbs_grouped(a_codes.data_ptr(), _ptr(a_scales), _ptr(a_mbs),
                                                            b_codes.data_ptr(), _ptr(b_scales), _ptr(b_mbs), G,
                                                            row_offsets.data_ptr(), M, N, K, code, out.data_ptr(), ldc,
                                                            _stream()), "mx_gemm_mbs_grouped")
    return out


# ---- the paged MXFP4 key/value cache --------------------------------------------------------------------
_STYLES = {"half": 0, "pairs": 1}


def _here(t, dtype, name, dims=None):
    """A CUDA tensor of that type (and rank) on the current device: the launch goes to the current device's stream."""
    torch = _torch_module or _torch()
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or not t.is_cuda or (dims is not None and t.dim() != dims):
        raise TypeError("%s must be a %s CUDA tensor%s" % (name, dtype, "" if dims is None else " of %d dimensions" % dims))
    if t.device.index != torch.cuda.current_device():
        raise ValueError("%s is on %s, the current device is %d" % (name, t.device, torch.cuda.current_device()))
    return t


def _flat(t, dtype, shape, name):
    _here(t, dtype, name)
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise TypeError("%s must be contiguous of shape %s" % (name, tuple(shape)))
    return t


def _rows_of_heads(t, dtype, name, shape=None):
    """[T, heads, D] with a token's heads next to each other -> elements from one token to the next."""
    _here(t, dtype, name, 3)
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise TypeError("%s must have the shape %s" % (name, tuple(shape)))
    T, H, D = t.shape
    ld, between, inner = t.stride()
    if T and H and ((inner != 1 and D > 1) or (between != D and H > 1)):
        raise ValueError("the heads of a token of %s must lie next to each other" % name)
    return ld if T > 1 else max(ld, H * D)


def _cache_arrays(k_cache, v_cache):
    """((codes, scales, mbs or None), the same for V) -> pointers in the order of the C calls, pages, heads, page size, D."""
    torch = _torch_module or _torch()
    (kc, ks, km), (vc, vs, vm) = k_cache, v_cache
    _here(kc, torch.uint8, "k codes", 5)
    pages, heads, blocks, page, _ = kc.shape
    D = 32 * blocks
    _flat(kc, torch.uint8, (pages, heads, blocks, page, 16), "k codes")
    _flat(vc, torch.uint8, (pages, heads, page // 4, D // 8, 4, 4), "v codes")
    _flat(ks, torch.uint8, (pages, heads, blocks, page), "k scales")
    _flat(vs, torch.uint8, (pages, heads, blocks, page), "v scales")
    if (km is None) != (vm is None):
        raise ValueError("MBS words for both keys and values, or for neither")
    if km is not None:
        _flat(km, torch.uint8, (pages, heads, (D + 127) // 128, page), "k mbs")
        _flat(vm, torch.uint8, (pages, heads, (D + 127) // 128, page), "v mbs")
    return (_ptr(kc), _ptr(ks), _ptr(km), _ptr(vc), _ptr(vs), _ptr(vm)), pages, heads, page, D


def mx_kv_cache(num_pages, heads, head_dim, page_size=64, use_mbs=True, device="cuda"):
    """The zeroed arrays of a cache: (k_cache, v_cache), each (codes, scales, mbs or None), in the layout of include/mx4.h."""
    torch = _torch_module or _torch()

    def array(*shape):
        return torch.zeros(shape, dtype=torch.uint8, device=device)

    words, blocks = (head_dim + 127) // 128, head_dim // 32
    return tuple((array(*codes), array(num_pages, heads, blocks, page_size), array(num_pages, heads, words, page_size) if use_mbs else None)
                 for codes in ((num_pages, heads, blocks, page_size, 16), (num_pages, heads, page_size // 4, head_dim // 8, 4, 4)))


def mx_kv_plan(ctx_lens, new_lens, page_size, block_table, free_pages, free_start, total_tokens, row_offsets=None, kv_lens=None, slots=None,
               positions=None, free_next=None):
    """Pages, slots, positions and offsets of a step whose requests have ctx_lens tokens and bring new_lens; block_table is extended in place.
    Returns (row_offsets, kv_lens, slots, positions, free_next)."""
    if _native is not None and free_next is not None and _done(_native.kv_plan(ctx_lens, new_lens, page_size, block_table, free_pages, free_start,
                                                                               total_tokens, row_offsets, kv_lens, slots, positions, free_next), "mx_kv_plan"):
        return row_offsets, kv_lens, slots, positions, free_next
    torch = _torch_module or _torch()
    i32, i64 = torch.int32, torch.int64
    S = _here(ctx_lens, i32, "ctx_lens", 1).shape[0]
    _flat(ctx_lens, i32, (S,), "ctx_lens")
    _flat(new_lens, i32, (S,), "new_lens")
    _here(block_table, i32, "block_table", 2)
    _flat(block_table, i32, (S, block_table.shape[1]), "block_table")
    _here(free_pages, i32, "free_pages", 1)
    _flat(free_pages, i32, free_pages.shape, "free_pages")
    _flat(free_start, i32, (1,), "free_start")

    def output(t, dtype, n, name):
        return torch.empty(n, dtype=dtype, device=ctx_lens.device) if t is None else _flat(t, dtype, (n,), name)

    T = int(total_tokens)
    row_offsets, kv_lens = output(row_offsets, i64, S + 1, "row_offsets"), output(kv_lens, i32, S, "kv_lens")
    slots, positions = output(slots, i64, T, "slots"), output(positions, i32, T, "positions")
    free_next = output(free_next, i32, 1, "free_next")
    _check((_lib or load_library()).mx_kv_plan(_ptr(ctx_lens), _ptr(new_lens), S, int(page_size), _ptr(block_table), block_table.shape[1],
                                               _ptr(free_pages), free_pages.shape[0], _ptr(free_start), T, _ptr(row_offsets), _ptr(kv_lens),
                                               _ptr(slots), _ptr(positions), _ptr(free_next), _stream()), "mx_kv_plan")
    return row_offsets, kv_lens, slots, positions, free_next


def _turn_arguments(q, k, positions, cos_sin, q_weight, k_weight, style):
    """What mx_qk_norm_rope and its form with the cache pass alike."""
    torch = _torch_module or _torch()
    bf16 = torch.bfloat16
    ldq, ldk = _rows_of_heads(q, bf16, "q"), _rows_of_heads(k, bf16, "k")
    T, Hq, D = q.shape
    if k.shape[0] != T or k.shape[2] != D:
        raise ValueError("q and k disagree on the tokens or on the head size")
    table, R = 0, 0
    if cos_sin is not None:
        table, R = _here(cos_sin, torch.float32, "cos_sin", 2).shape
        _flat(cos_sin, torch.float32, (table, R), "cos_sin")
        _flat(positions, torch.int32, (T,), "positions")
    for weight, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if weight is not None:
            _flat(weight, bf16, (D,), name)
    return T, Hq, k.shape[1], D, R, table, ldq, ldk, _STYLES[style] if isinstance(style, str) else int(style)


def mx_qk_norm_rope(q, k, positions, cos_sin, q_weight=None, k_weight=None, eps=1e-6, style="half", q_out=None, k_out=None):
    """RMS norm (where there is a weight) and rotation (where there is a table) of the heads of q [T, Hq, D] and k [T, Hkv, D], bf16.
    cos_sin fp32 [positions, R]: R/2 cosines, then R/2 sines.  Outputs may be the inputs.  Returns (q_out, k_out)."""
    if _native is not None and k_out is not None and _done(
            _native.qk_norm_rope(q, k, positions, cos_sin, q_weight, k_weight, eps, style, q_out, k_out), "mx_qk_norm_rope"):
        return q_out, k_out
    torch = _torch_module or _torch()
    T, Hq, Hkv, D, R, table, ldq, ldk, code = _turn_arguments(q, k, positions, cos_sin, q_weight, k_weight, style)
    q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None else q_out
    k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device) if k_out is None else k_out
    ldqo, ldko = _rows_of_heads(q_out, q.dtype, "q_out", q.shape), _rows_of_heads(k_out, k.dtype, "k_out", k.shape)
    _check((_lib or load_library()).mx_qk_norm_rope(_ptr(q), ldq, _ptr(k), ldk, _ptr(positions), _ptr(cos_sin), table, _ptr(q_weight),
                                                    _ptr(k_weight), eps, code, T, Hq, Hkv, D, R, _ptr(q_out), ldqo, _ptr(k_out), ldko, _stream()),
           "mx_qk_norm_rope")
    return q_out, k_out


def mx_kv_write(k, v, slots, k_cache, v_cache, rule="oas"):
    """Quantizes k, v [T, Hkv, D] (bf16) into the places `slots` (int64 [T], distinct) of the cache."""
    if _native is not None and _done(_native.kv_write(k, v, slots, *k_cache, *v_cache, rule), "mx_kv_write"):
        return
    torch = _torch_module or _torch()
    pointers, pages, heads, page, D = _cache_arrays(k_cache, v_cache)
    ldk = _rows_of_heads(k, torch.bfloat16, "k")
    T = k.shape[0]
    if tuple(k.shape) != (T, heads, D):
        raise ValueError("k and the cache disagree on heads or head size")
    ldv = _rows_of_heads(v, torch.bfloat16, "v", k.shape)
    _flat(slots, torch.int64, (T,), "slots")
    _check((_lib or load_library()).mx_kv_write(_ptr(k), ldk, _ptr(v), ldv, _ptr(slots), _rule(rule), *pointers, pages, page, T, heads, D, _stream()),
           "mx_kv_write")


def mx_qk_norm_rope_kv_write(q, k, v, positions, slots, cos_sin, k_cache, v_cache, q_weight=None, k_weight=None, eps=1e-6, style="half", rule="oas",
                             q_out=None):
    """mx_qk_norm_rope, then mx_kv_write of the rotated keys and the values, in one launch and with the same bits.  Returns q_out."""
    if _native is not None and q_out is not None and _done(
            _native.qk_norm_rope_kv_write(q, k, v, positions, slots, cos_sin, *k_cache, *v_cache, q_weight, k_weight, eps, style, rule, q_out),
            "mx_qk_norm_rope_kv_write"):
        return q_out
    torch = _torch_module or _torch()
    pointers, pages, heads, page, head_dim = _cache_arrays(k_cache, v_cache)
    T, Hq, Hkv, D, R, table, ldq, ldk, code = _turn_arguments(q, k, positions, cos_sin, q_weight, k_weight, style)
    if (Hkv, D) != (heads, head_dim):
        raise ValueError("k and the cache disagree on heads or head size")
    ldv = _rows_of_heads(v, torch.bfloat16, "v", k.shape)
    _flat(slots, torch.int64, (T,), "slots")
    q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None else q_out
    ldqo = _rows_of_heads(q_out, q.dtype, "q_out", q.shape)
    _check((_lib or load_library()).mx_qk_norm_rope_kv_write(_ptr(q), ldq, _ptr(k), ldk, _ptr(v), ldv, _ptr(positions), _ptr(cos_sin), table,
                                                             _ptr(q_weight), _ptr(k_weight), eps, code, _ptr(slots), _rule(rule), *pointers, pages,
                                                             page, T, Hq, Hkv, D, R, _ptr(q_out), ldqo, _stream()), "mx_qk_norm_rope_kv_write")
    return q_out


def mx_kv_read(slots, k_cache, v_cache, out_dtype="bf16", k_out=None, v_out=None):
    """Rows of the cache by slot, rounded as by mx_dequantize.  Returns (k_out, v_out) [T, Hkv, D]."""
    if _native is not None and v_out is not None and _done(_native.kv_read(slots, *k_cache, *v_cache, out_dtype, k_out, v_out), "mx_kv_read"):
        return k_out, v_out
    torch = _torch_module or _torch()
    pointers, pages, heads, page, D = _cache_arrays(k_cache, v_cache)
    T = _here(slots, torch.int64, "slots", 1).shape[0]
    _flat(slots, torch.int64, (T,), "slots")
    code, dtype = _out_dtypes[out_dtype]
    k_out = torch.empty((T, heads, D), dtype=dtype, device=slots.device) if k_out is None else k_out
    v_out = torch.empty((T, heads, D), dtype=dtype, device=slots.device) if v_out is None else v_out
    ldk, ldv = _rows_of_heads(k_out, dtype, "k_out", (T, heads, D)), _rows_of_heads(v_out, dtype, "v_out", (T, heads, D))
    _check((_lib or load_library()).mx_kv_read(_ptr(slots), *pointers, pages, page, T, heads, D, code, _ptr(k_out), ldk, _ptr(v_out), ldv, _stream()),
           "mx_kv_read")
    return k_out, v_out


def mx_attention_kv_workspace(num_seqs, total_tokens, q_heads, kv_heads, head_dim) -> int:
    """Bytes of workspace that mx_attention_kv wants for these sizes, whatever the lengths."""
    need = (_lib or load_library()).mx_internal_attention_kv_workspace(_forced("attention") or 0, num_seqs, total_tokens, q_heads, kv_heads, head_dim)
    _check(min(need, 0), "mx_attention_kv_workspace")
    return need


def mx_attention_kv(q, row_offsets, kv_lens, block_table, k_cache, v_cache, scale=None, causal=True, window=0, out=None, lse=None, workspace=None):
    """Attention of q [T, Hq, D] (bf16; request s has the rows row_offsets[s] .. row_offsets[s+1]-1) over the cache: request s has kv_lens[s]
    keys in the pages block_table[s].  scale: 1 / sqrt(D) if None.  lse: fp32 [T, Hq], filled if given.  workspace: uint8, if the caller keeps
    one (calls that can run at the same time need one each); else it comes from the allocator.  Returns out, bf16 [T, Hq, D].
    Single tokens and prompts of one step are faster as two calls, the k single tokens first: q[:k], row_offsets[:k + 1], kv_lens[:k], block_table[:k],
    out=out[:k], and q, row_offsets[k:], kv_lens[k:], block_table[k:], out=out."""
    if _native is not None and out is not None and not getattr(_dev, "choices", None) and _done(
            _native.attention_kv(q, row_offsets, kv_lens, block_table, *k_cache, *v_cache, q.shape[-1] ** -0.5 if scale is None else scale, causal, window, out,
                                 lse, workspace), "mx_attention_kv"):
        return out
    torch = _torch_module or _torch()
    pointers, pages, heads, page, D = _cache_arrays(k_cache, v_cache)
    ldq = _rows_of_heads(q, torch.bfloat16, "q")
    T, Hq, _ = q.shape
    if q.shape[2] != D or not heads or Hq % heads:
        raise ValueError("q and the cache disagree on the head size, or the key heads do not divide the query heads")
    S = _here(kv_lens, torch.int32, "kv_lens", 1).shape[0]
    _flat(kv_lens, torch.int32, (S,), "kv_lens")
    _flat(row_offsets, torch.int64, (S + 1,), "row_offsets")
    _here(block_table, torch.int32, "block_table", 2)
    _flat(block_table, torch.int32, (S, block_table.shape[1]), "block_table")
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
    ldo = _rows_of_heads(out, q.dtype, "out", q.shape)
    if lse is not None:
        _flat(lse, torch.float32, (T, Hq), "lse")
    if workspace is None:
        workspace = torch.empty(mx_attention_kv_workspace(S, T, Hq, heads, D), dtype=torch.uint8, device=q.device)
    else:
        _here(workspace, torch.uint8, "workspace", 1)
        _flat(workspace, torch.uint8, workspace.shape, "workspace")
    arguments = (_ptr(q), ldq, _ptr(row_offsets), _ptr(kv_lens), _ptr(block_table), block_table.shape[1], *pointers, pages, page, S, T, Hq, heads, D,
                 D ** -0.5 if scale is None else scale, int(bool(causal)), int(window), _ptr(out), ldo, _ptr(lse), _ptr(workspace), workspace.numel(), _stream())
    force = _forced("attention")
    if force:
        _check((_lib or load_library()).mx_internal_attention_kv(int(force), *arguments), "mx_attention_kv (mx_internal_attention_kv)")
    else:
        _check((_lib or load_library()).mx_attention_kv(*arguments), "mx_attention_kv")
    return out
