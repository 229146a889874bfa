"""Thin ctypes binding over libqqq.so (the C ABI declared in include/qqq.h; the offline stage in include/qqq_calib.h, what lies
between a decoder layer's linear calls in include/qqq_layer.h, tuning and diagnostic controls in include/qqq_tuning.h).

Argument marshalling only: every step of the path runs in the library's HIP kernels.  PyTorch
supplies device memory and the stream.  There is no CPU fallback: if the library is missing or a
tensor is not on the GPU the call raises.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import typing
import warnings

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# QQQ_LIB_PATH: load another build of the same library (the host-sanitizer build of the CPU tests)
LIB_PATH = os.environ.get("QQQ_LIB_PATH") or os.path.join(_HERE, "libqqq.so")
GROUP = 128
SG_SYMMETRIC_CODES = 0x100   # QQQ_SG_SYMMETRIC_CODES of include/qqq.h, or-ed into sg_max

SYMBOLS = [
    "qqq_version", "qqq_last_error", "qqq_quant_act", "qqq_packed_w4_bytes", "qqq_pack_w4",
    "qqq_unpack_w4", "qqq_gemm_workspace_bytes", "qqq_gemm_w4a8_perchannel",
    "qqq_gemm_w4a8_pergroup", "qqq_gemm_w4a8_pergroup_f16scale", "qqq_linear_workspace_bytes", "qqq_linear_w4a8_perchannel",
    "qqq_linear_w4a8_pergroup", "qqq_set_fused_quant", "qqq_set_kernel_override",
    "qqq_set_group_mode_override", "qqq_set_skinny_tuning", "qqq_set_prefill_tuning",
    "qqq_quantize_w4_perchannel", "qqq_quantize_w4_pergroup", "qqq_set_prefill_ksplit",
    "qqq_gemm_workspace_zero_bytes", "qqq_linear_w4a8_perchannel_static", "qqq_last_route",
    "qqq_debug_count_sg_violations", "qqq_probe_stream_read", "qqq_probe_mfma_i8", "qqq_probe_prefill_loop",
    "qqq_smoothing_workspace_bytes", "qqq_adaptive_smoothing", "qqq_channel_absmax", "qqq_smooth_apply",
    "qqq_fp16_gemm_nt", "qqq_hessian", "qqq_gptq_workspace_bytes", "qqq_gptq_quantize_w4_perchannel",
    "qqq_gptq_quantize_w4_pergroup", "qqq_set_factor_workgroups",
]

# the entry points of include/qqq_layer.h
LAYER_SYMBOLS = [
    "qqq_add_rmsnorm", "qqq_add_rmsnorm_quant", "qqq_gated_act_quant", "qqq_kv8_append", "qqq_kv8_read",
    "qqq_attention_kv8_workspace_bytes", "qqq_attention_kv8",
]

_lib = None
_F16, _I8, _U8, _I32 = torch.float16, torch.int8, torch.uint8, torch.int32


class QQQError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("libqqq error %d: %s" % (code, msg))
        self.code = code


def _no_native(*args):
    return None


_native_linear = _native_rmsnorm = _native_gated = _native_append = _native_read = _native_attention = _no_native


def _call_path():
    from .build import call_path
    return call_path()


def _load_native(library):
    """The extension that takes the linear calls and those of include/qqq_layer.h from tensors to the library (csrc/qqq_torch_call.cpp).  Without
    it they are marshalled here."""
    global _native_linear, _native_rmsnorm, _native_gated, _native_append, _native_read, _native_attention
    path = _call_path()
    try:
        spec = importlib.util.spec_from_file_location("_qqq_call", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError as e:
        warnings.warn("linear calls are marshalled in Python, a microsecond slower each: build.py has not built %s for this torch and interpreter (%s)"
                      % (os.path.basename(path), e), RuntimeWarning, stacklevel=3)
        return
    module.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (library.qqq_linear_w4a8_perchannel, library.qqq_linear_w4a8_pergroup)))
    module.bind_layer(*(ctypes.cast(getattr(library, n), ctypes.c_void_p).value for n in LAYER_SYMBOLS))
    _native_linear, _native_rmsnorm, _native_gated = module.linear, module.rmsnorm, module.gated
    _native_append, _native_read, _native_attention = module.append, module.read, module.attention


def lib():
    """Loads the built library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libqqq.so is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                "(or python paper_2406_09904_amd/build.py) first")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, sz, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
        L.qqq_version.restype = ci
        L.qqq_last_error.restype = ctypes.c_char_p
        L.qqq_last_route.restype = ctypes.c_char_p
        L.qqq_debug_count_sg_violations.argtypes = [vp, i64, i64, ci, vp, vp]
        L.qqq_smoothing_workspace_bytes.argtypes = [i64, i64, i64]
        L.qqq_smoothing_workspace_bytes.restype = sz
        L.qqq_adaptive_smoothing.argtypes = [vp, vp, i64, i64, i64, ci, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.qqq_channel_absmax.argtypes = [vp, i64, i64, vp, vp]
        L.qqq_smooth_apply.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, vp, vp, vp]
        L.qqq_fp16_gemm_nt.argtypes = [vp, vp, i64, i64, i64, vp, vp]
        L.qqq_hessian.argtypes = [vp, i64, i64, vp, vp]
        L.qqq_gptq_workspace_bytes.argtypes = [i64, i64]
        L.qqq_gptq_workspace_bytes.restype = sz
        L.qqq_gptq_quantize_w4_perchannel.argtypes = [vp, vp, i64, i64, ctypes.c_double, vp, vp, vp, sz, vp]
        L.qqq_gptq_quantize_w4_pergroup.argtypes = [vp, vp, i64, i64, ci, ctypes.c_double, vp, vp, vp, vp, vp, vp, sz, vp]
        L.qqq_probe_stream_read.argtypes = [vp, sz, ci, vp, vp]
        L.qqq_probe_mfma_i8.argtypes = [vp, vp, ci, ci, vp, vp]
        L.qqq_probe_prefill_loop.argtypes = [vp, sz, ci, ci, ci, vp, vp]
        L.qqq_quant_act.argtypes = [vp, i64, i64, i64, vp, vp, vp]
        L.qqq_packed_w4_bytes.argtypes = [i64, i64]
        L.qqq_packed_w4_bytes.restype = sz
        L.qqq_pack_w4.argtypes = [vp, i64, i64, vp, vp]
        L.qqq_unpack_w4.argtypes = [vp, i64, i64, vp, vp]
        L.qqq_gemm_workspace_bytes.argtypes = [i64, i64, i64]
        L.qqq_gemm_workspace_bytes.restype = sz
        L.qqq_gemm_workspace_zero_bytes.argtypes = [i64, i64, i64]
        L.qqq_gemm_workspace_zero_bytes.restype = sz
        L.qqq_gemm_w4a8_perchannel.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, vp, sz, vp]
        L.qqq_gemm_w4a8_pergroup.argtypes = [vp, vp, vp, vp, vp, ci, ci, vp, vp, i64, i64, i64,
                                             vp, sz, vp]
        L.qqq_gemm_w4a8_pergroup_f16scale.argtypes = [vp, vp, vp, vp, vp, ci, vp, vp, i64, i64, i64,
                                                      vp, sz, vp]
        L.qqq_linear_workspace_bytes.argtypes = [i64, i64, i64]
        L.qqq_linear_workspace_bytes.restype = sz
        L.qqq_linear_w4a8_perchannel.argtypes = [vp, i64, vp, vp, vp, vp, i64, i64, i64, vp, sz, vp]
        L.qqq_linear_w4a8_pergroup.argtypes = [vp, i64, vp, vp, vp, ci, ci, vp, vp, i64, i64, i64,
                                               vp, sz, vp]
        L.qqq_linear_w4a8_perchannel_static.argtypes = [vp, i64, vp, vp, vp, vp, i64, i64, i64, vp]
        L.qqq_quantize_w4_perchannel.argtypes = [vp, i64, i64, i64, vp, vp, vp]
        L.qqq_quantize_w4_pergroup.argtypes = [vp, i64, i64, i64, ci, vp, vp, vp, vp, vp, vp]
        L.qqq_set_fused_quant.argtypes = [ci]
        L.qqq_set_kernel_override.argtypes = [ci]
        L.qqq_set_group_mode_override.argtypes = [ci]
        L.qqq_set_skinny_tuning.argtypes = [ci, ci, ci, ci]
        L.qqq_set_prefill_tuning.argtypes = [ci]
        L.qqq_set_prefill_ksplit.argtypes = [ci]
        L.qqq_set_factor_workgroups.argtypes = [ci]
        cf = ctypes.c_float
        L.qqq_add_rmsnorm.argtypes = [vp, i64, vp, i64, ci, vp, cf, i64, i64, vp, i64, vp, vp]
        L.qqq_add_rmsnorm_quant.argtypes = [vp, i64, vp, i64, ci, vp, cf, i64, i64, vp, i64, vp, vp, vp]
        L.qqq_gated_act_quant.argtypes = [vp, i64, vp, i64, ci, i64, i64, vp, vp, vp]
        L.qqq_kv8_append.argtypes = [vp, vp, vp, i64, i64, vp, i64, i64, i64, vp]
        L.qqq_kv8_read.argtypes = [vp, vp, vp, vp, i64, vp]
        L.qqq_attention_kv8_workspace_bytes.argtypes = [vp, vp, ci, i64]
        L.qqq_attention_kv8_workspace_bytes.restype = sz
        L.qqq_attention_kv8.argtypes = [vp, vp, vp, i64, i64, ci, i64, cf, ci, ci, vp, vp, vp, sz, vp]
        _load_native(L)
        _lib = L
    return _lib


def _check(rc):
    if rc:
        raise QQQError(rc, lib().qqq_last_error().decode())


def _ptr(t, dtype=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libqqq takes device tensors only")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError("expected %s, got %s" % (dtype, t.dtype))
    return t.data_ptr()


# The calling thread's current stream on its current device as the plain handle.  torch.cuda.current_stream() builds a Stream
# object around the same handle, at a tenth of what a whole one-row linear call takes on the host.  Both names are torch's own
# business: where one is missing, the public way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)
if _raw_stream is None or _device is None:
    _device = torch.cuda.current_device

    def _raw_stream(device):
        return torch.cuda.current_stream(device).cuda_stream


def _stream():
    return _raw_stream(_device())


def qqq_quant_act(a_fp16: torch.Tensor, a_q: torch.Tensor = None, s_a: torch.Tensor = None):
    """a_fp16 [M,K] fp16 (row stride allowed) -> (a_q int8 [M,K], s_a fp32 [M])."""
    if a_fp16.dtype != torch.float16 or a_fp16.dim() != 2 or a_fp16.stride(1) != 1:
        raise ValueError("a_fp16 must be a 2-D fp16 tensor with unit inner stride")
    M, K = a_fp16.shape
    lda = a_fp16.stride(0) if M > 1 else max(K, a_fp16.stride(0))
    if a_q is None:
        a_q = torch.empty((M, K), dtype=torch.int8, device=a_fp16.device)
    if s_a is None:
        s_a = torch.empty((M,), dtype=torch.float32, device=a_fp16.device)
    if not a_fp16.is_cuda:
        raise ValueError("libqqq takes device tensors only")
    _check(lib().qqq_quant_act(ctypes.c_void_p(a_fp16.data_ptr()), M, K, lda,
                               _ptr(a_q, torch.int8), _ptr(s_a, torch.float32), _stream()))
    return a_q, s_a


def _weights_arg(w_fp16):
    if w_fp16.dtype != torch.float16 or w_fp16.dim() != 2 or w_fp16.stride(1) != 1 or not w_fp16.is_cuda:
        raise ValueError("w_fp16 must be a 2-D fp16 device tensor with unit inner stride")
    N, K = w_fp16.shape
    return N, K, (w_fp16.stride(0) if N > 1 else max(K, w_fp16.stride(0)))


def qqq_quantize_w4_perchannel(w_fp16: torch.Tensor, out=None):
    """fp16 weights [N,K] -> (w_nat int32 [N,K/8] natural nibble words, s_w fp16 [N]); out = a
    previous result to write into."""
    N, K, ldw = _weights_arg(w_fp16)
    if out is not None:
        w_nat, s_w = out
    else:
        w_nat = torch.empty((N, K // 8), dtype=torch.int32, device=w_fp16.device)
        s_w = torch.empty((N,), dtype=torch.float16, device=w_fp16.device)
    _check(lib().qqq_quantize_w4_perchannel(ctypes.c_void_p(w_fp16.data_ptr()), N, K, ldw,
                                            _ptr(w_nat, torch.int32), _ptr(s_w, torch.float16), _stream()))
    return w_nat, s_w


def qqq_quantize_w4_pergroup(w_fp16: torch.Tensor, group: int = 128, want_int: bool = True,
                             want_wg: bool = True, out=None):
    """fp16 weights [N,K] -> (w_nat, s_star fp16 [K/128,N], s_int int8 [K/128,N] or None, s_wc fp16 [N],
    s_wg fp16 [K/128,N] or None); out = a previous result to write into."""
    N, K, ldw = _weights_arg(w_fp16)
    dev = w_fp16.device
    G = K // group if group > 0 else 0
    if out is not None:
        w_nat, s_star, s_int, s_wc, s_wg = out
    else:
        w_nat = torch.empty((N, K // 8), dtype=torch.int32, device=dev)
        s_star = torch.empty((G, N), dtype=torch.float16, device=dev)
        s_int = torch.empty((G, N), dtype=torch.int8, device=dev) if want_int else None
        s_wg = torch.empty((G, N), dtype=torch.float16, device=dev) if want_wg else None
        s_wc = torch.empty((N,), dtype=torch.float16, device=dev)
    _check(lib().qqq_quantize_w4_pergroup(ctypes.c_void_p(w_fp16.data_ptr()), N, K, ldw, group,
                                          _ptr(w_nat, torch.int32), _ptr(s_star, torch.float16),
                                          _ptr(s_int, torch.int8), _ptr(s_wc, torch.float16),
                                          _ptr(s_wg, torch.float16), _stream()))
    return w_nat, s_star, s_int, s_wc, s_wg


def qqq_packed_w4_bytes(N: int, K: int) -> int:
    return int(lib().qqq_packed_w4_bytes(N, K))


def qqq_pack_w4(w_nat: torch.Tensor, K: int, out: torch.Tensor = None) -> torch.Tensor:
    """w_nat [N,K/8] int32 (bit pattern of the uint32 natural words) -> opaque packed uint8 [N*K/2]."""
    N = w_nat.shape[0]
    nbytes = qqq_packed_w4_bytes(N, K)
    if nbytes == 0 or w_nat.shape[1] * 8 != K:
        raise QQQError(2, "pack: unsupported N=%d K=%d" % (N, K))
    if out is None:
        out = torch.empty((nbytes,), dtype=torch.uint8, device=w_nat.device)
    _check(lib().qqq_pack_w4(_ptr(w_nat, torch.int32), N, K, _ptr(out, torch.uint8), _stream()))
    return out


def qqq_unpack_w4(w_packed: torch.Tensor, N: int, K: int) -> torch.Tensor:
    out = torch.empty((N, K // 8), dtype=torch.int32, device=w_packed.device)
    _check(lib().qqq_unpack_w4(_ptr(w_packed, torch.uint8), N, K, _ptr(out, torch.int32), _stream()))
    return out


def qqq_gemm_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().qqq_gemm_workspace_bytes(M, N, K))


def qqq_gemm_workspace_zero_bytes(M: int, N: int, K: int) -> int:
    return int(lib().qqq_gemm_workspace_zero_bytes(M, N, K))


def split_k_part(workspace: torch.Tensor, M: int, N: int, K: int) -> torch.Tensor:
    """The part of a GEMM workspace that every call leaves zero (arrival counters and split-K partial
    sums of the decode kernel); what follows it is scratch of the prefill kernels with no invariant."""
    return workspace[:qqq_gemm_workspace_zero_bytes(M, N, K)]


def new_workspace(M: int, N: int, K: int, device="cuda") -> torch.Tensor:
    """Zero-filled workspace (zeroed once here; every GEMM call leaves it zero)."""
    return torch.zeros((max(qqq_gemm_workspace_bytes(M, N, K), 16),), dtype=torch.uint8, device=device)


def qqq_gemm_w4a8_perchannel(a_q, s_a, w_packed, s_w, workspace, y=None, acc_out=None, N=None):
    M, K = a_q.shape
    N = s_w.shape[0] if N is None else N
    if y is None:
        y = torch.empty((M, N), dtype=torch.float16, device=a_q.device)
    _check(lib().qqq_gemm_w4a8_perchannel(
        _ptr(a_q, torch.int8), _ptr(s_a, torch.float32), _ptr(w_packed, torch.uint8),
        _ptr(s_w, torch.float16), _ptr(y, torch.float16), _ptr(acc_out, torch.int32), M, N, K,
        _ptr(workspace, torch.uint8), workspace.numel(), _stream()))
    return y


def qqq_gemm_w4a8_pergroup(a_q, s_a, w_packed, s_g, s_w, workspace, sg_max=0, y=None, acc_out=None,
                           group=GROUP):
    M, K = a_q.shape
    N = s_w.shape[0]
    if y is None:
        y = torch.empty((M, N), dtype=torch.float16, device=a_q.device)
    _check(lib().qqq_gemm_w4a8_pergroup(
        _ptr(a_q, torch.int8), _ptr(s_a, torch.float32), _ptr(w_packed, torch.uint8),
        _ptr(s_g, torch.int8), _ptr(s_w, torch.float16), group, sg_max, _ptr(y, torch.float16),
        _ptr(acc_out, torch.int32), M, N, K, _ptr(workspace, torch.uint8), workspace.numel(),
        _stream()))
    return y


def qqq_gemm_w4a8_pergroup_f16scale(a_q, s_a, w_packed, s_g_fp16, s_w, workspace, y=None,
                                    acc_out=None, group=GROUP):
    """Per-group GEMM with the real-valued fp16 fused scale s*_Wg [K/128, N] (no saturation)."""
    M, K = a_q.shape
    N = s_w.shape[0]
    if y is None:
        y = torch.empty((M, N), dtype=torch.float16, device=a_q.device)
    _check(lib().qqq_gemm_w4a8_pergroup_f16scale(
        _ptr(a_q, torch.int8), _ptr(s_a, torch.float32), _ptr(w_packed, torch.uint8),
        _ptr(s_g_fp16, torch.float16), _ptr(s_w, torch.float16), group, _ptr(y, torch.float16),
        _ptr(acc_out, torch.int32), M, N, K, _ptr(workspace, torch.uint8), workspace.numel(),
        _stream()))
    return y


def qqq_linear_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().qqq_linear_workspace_bytes(M, N, K))


def new_linear_workspace(M: int, N: int, K: int, device="cuda") -> torch.Tensor:
    """Zero-filled workspace for the qqq_linear_* calls (zeroed once here)."""
    return torch.zeros((max(qqq_linear_workspace_bytes(M, N, K), 16),), dtype=torch.uint8, device=device)


def _fp16_rows(a_fp16):
    if a_fp16.dtype != _F16 or a_fp16.dim() != 2:
        raise ValueError("a_fp16 must be a 2-D fp16 tensor with unit inner stride")
    lda, inner = a_fp16.stride()
    if inner != 1:
        raise ValueError("a_fp16 must be a 2-D fp16 tensor with unit inner stride")
    if not a_fp16.is_cuda:
        raise ValueError("libqqq takes device tensors only")
    M, K = a_fp16.shape
    return M, K, (lda if M > 1 or lda > K else K)


# A one-row call is shorter on the GPU (5 us) than its marshalling is here (6.4 us): the extension takes plain calls, what it declines goes on below
def qqq_linear_w4a8_perchannel(a_fp16, w_packed, s_w, workspace, y=None, acc_out=None):
    if a_fp16.is_cuda:
        out = _native_linear(a_fp16, w_packed, None, s_w, workspace, y, acc_out, 0, 0, _raw_stream(_device()))
        if out is not None:
            if out.__class__ is int:
                _check(out)
            return out
    M, K, lda = _fp16_rows(a_fp16)
    N = s_w.shape[0]
    if y is None:
        y = a_fp16.new_empty(M, N)
    rc = (_lib or lib()).qqq_linear_w4a8_perchannel(
        a_fp16.data_ptr(), lda, _ptr(w_packed, _U8), _ptr(s_w, _F16), _ptr(y, _F16),
        None if acc_out is None else _ptr(acc_out, _I32), M, N, K, _ptr(workspace, _U8), workspace.numel(),
        _raw_stream(_device()))
    if rc:
        _check(rc)
    return y


def qqq_linear_w4a8_perchannel_static(a_fp16, w_packed, s_w, y, acc_out=None):
    """qqq_linear_w4a8_perchannel on the library's static device scratch: no workspace, and the
    caller passes the output tensor too, so nothing is allocated on the way."""
    M, K, lda = _fp16_rows(a_fp16)
    N = s_w.shape[0]
    _check(lib().qqq_linear_w4a8_perchannel_static(
        ctypes.c_void_p(a_fp16.data_ptr()), lda, _ptr(w_packed, torch.uint8), _ptr(s_w, torch.float16),
        _ptr(y, torch.float16), _ptr(acc_out, torch.int32), M, N, K, _stream()))
    return y


def qqq_linear_w4a8_pergroup(a_fp16, w_packed, s_g, s_w, workspace, sg_max=0, y=None, acc_out=None,
                             group=GROUP):
    if s_g is not None and a_fp16.is_cuda:
        out = _native_linear(a_fp16, w_packed, s_g, s_w, workspace, y, acc_out, group, sg_max, _raw_stream(_device()))
        if out is not None:
            if out.__class__ is int:
                _check(out)
            return out
    M, K, lda = _fp16_rows(a_fp16)
    N = s_w.shape[0]
    if y is None:
        y = a_fp16.new_empty(M, N)
    rc = (_lib or lib()).qqq_linear_w4a8_pergroup(
        a_fp16.data_ptr(), lda, _ptr(w_packed, _U8), _ptr(s_g, _I8), _ptr(s_w, _F16), group, sg_max, _ptr(y, _F16),
        None if acc_out is None else _ptr(acc_out, _I32), M, N, K, _ptr(workspace, _U8), workspace.numel(),
        _raw_stream(_device()))
    if rc:
        _check(rc)
    return y


# ---- offline stage (include/qqq_calib.h): adaptive smoothing and Hessian-based compensation

def _fp16_matrix(t):
    if t.dtype != torch.float16 or t.dim() != 2 or not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous 2-D fp16 device tensor")
    return t.shape


def qqq_adaptive_smoothing(x_fp16, w_fp16, grid_points=20):
    """Sec. 3.1 on one layer: X [M,K], W [N,K] fp16 -> dict(xs, ws, s, sigmas, losses, best); best is a
    device tensor (no synchronisation here)."""
    (M, K), (N, K2) = _fp16_matrix(x_fp16), _fp16_matrix(w_fp16)
    if K != K2:
        raise ValueError("X and W disagree on K")
    dev = x_fp16.device
    xs, ws = torch.empty_like(x_fp16), torch.empty_like(w_fp16)
    s = torch.empty((K,), dtype=torch.float32, device=dev)
    sigmas = torch.empty((grid_points,), dtype=torch.float32, device=dev)
    losses = torch.empty((grid_points,), dtype=torch.float64, device=dev)
    best = torch.empty((1,), dtype=torch.int32, device=dev)
    nbytes = int(lib().qqq_smoothing_workspace_bytes(M, N, K))
    work = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=dev)
    _check(lib().qqq_adaptive_smoothing(_ptr(x_fp16), _ptr(w_fp16), M, N, K, grid_points, _ptr(xs), _ptr(ws),
                                        _ptr(s), _ptr(sigmas), _ptr(losses), _ptr(best), _ptr(work),
                                        work.numel(), _stream()))
    return {"xs": xs, "ws": ws, "s": s, "sigmas": sigmas, "losses": losses, "best": best}


def qqq_channel_absmax(x_fp16):
    M, K = _fp16_matrix(x_fp16)
    out = torch.empty((K,), dtype=torch.float32, device=x_fp16.device)
    _check(lib().qqq_channel_absmax(_ptr(x_fp16), M, K, _ptr(out), _stream()))
    return out


def qqq_smooth_apply(x_fp16, w_fp16, absmax, sigma):
    """sigma: 1-element fp32 device tensor.  -> (xs, ws, s)."""
    (M, K), (N, _) = _fp16_matrix(x_fp16), _fp16_matrix(w_fp16)
    xs, ws = torch.empty_like(x_fp16), torch.empty_like(w_fp16)
    s = torch.empty((K,), dtype=torch.float32, device=x_fp16.device)
    _check(lib().qqq_smooth_apply(_ptr(x_fp16), _ptr(w_fp16), _ptr(absmax, torch.float32), _ptr(sigma, torch.float32),
                                  M, N, K, _ptr(xs), _ptr(ws), _ptr(s), _stream()))
    return xs, ws, s


def qqq_fp16_gemm_nt(x_fp16, w_fp16):
    (M, K), (N, _) = _fp16_matrix(x_fp16), _fp16_matrix(w_fp16)
    y = torch.empty((M, N), dtype=torch.float32, device=x_fp16.device)
    _check(lib().qqq_fp16_gemm_nt(_ptr(x_fp16), _ptr(w_fp16), M, N, K, _ptr(y), _stream()))
    return y


def qqq_hessian(x_fp16):
    M, K = _fp16_matrix(x_fp16)
    H = torch.empty((K, K), dtype=torch.float64, device=x_fp16.device)
    _check(lib().qqq_hessian(_ptr(x_fp16), M, K, _ptr(H), _stream()))
    return H


def qqq_gptq_quantize_w4_perchannel(w_fp16, H, percdamp=0.01):
    """Sec. 3.2 on one layer: W [N,K] fp16, H [K,K] fp64 -> (w_nat int32 [N,K/8], s_w fp16 [N])."""
    N, K = _fp16_matrix(w_fp16)
    dev = w_fp16.device
    w_nat = torch.empty((N, K // 8), dtype=torch.int32, device=dev)
    s_w = torch.empty((N,), dtype=torch.float16, device=dev)
    nbytes = int(lib().qqq_gptq_workspace_bytes(N, K))
    work = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=dev)
    _check(lib().qqq_gptq_quantize_w4_perchannel(_ptr(w_fp16), _ptr(H, torch.float64), N, K, float(percdamp),
                                                 _ptr(w_nat, torch.int32), _ptr(s_w, torch.float16), _ptr(work),
                                                 work.numel(), _stream()))
    return w_nat, s_w


def qqq_gptq_quantize_w4_pergroup(w_fp16, H, percdamp=0.01, want_int=True):
    """Sec. 3.2 with the group-128 quantiser of Sec. 3.3.2 on one layer: W [N,K] fp16, H [K,K] fp64 ->
    (w_nat int32 [N,K/8], s_wg fp16 [K/128,N], s_star fp16 [K/128,N], s_int int8 [K/128,N] or None, s_wc fp16 [N])."""
    N, K = _fp16_matrix(w_fp16)
    dev = w_fp16.device
    G = K // GROUP
    w_nat = torch.empty((N, K // 8), dtype=torch.int32, device=dev)
    s_wg = torch.empty((G, N), dtype=torch.float16, device=dev)
    s_star = torch.empty((G, N), dtype=torch.float16, device=dev)
    s_int = torch.empty((G, N), dtype=torch.int8, device=dev) if want_int else None
    s_wc = torch.empty((N,), dtype=torch.float16, device=dev)
    nbytes = int(lib().qqq_gptq_workspace_bytes(N, K))
    work = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=dev)
    _check(lib().qqq_gptq_quantize_w4_pergroup(_ptr(w_fp16), _ptr(H, torch.float64), N, K, GROUP, float(percdamp),
                                               _ptr(w_nat, torch.int32), _ptr(s_wg, torch.float16),
                                               _ptr(s_star, torch.float16), _ptr(s_int, torch.int8),
                                               _ptr(s_wc, torch.float16), _ptr(work), work.numel(), _stream()))
    return w_nat, s_wg, s_star, s_int, s_wc


# ---- between the linear calls (include/qqq_layer.h): norm and gated activation to int8, the 8-bit cache, attention over it

def _rows(t, name):
    if t.dtype != torch.float16 or t.dim() != 2 or t.stride(1) != 1 or not t.is_cuda:
        raise ValueError("%s must be a 2-D fp16 device tensor with unit inner stride" % name)
    M, K = t.shape
    return M, K, (t.stride(0) if M > 1 else max(K, t.stride(0)))


def _checked(out):
    """What the extension gives: the outputs, or the library's error code."""
    if out.__class__ is int:
        _check(out)
    return out


def _rmsnorm_args(x, gain, residual, sum_out):
    M, K, ldx = _rows(x, "x")
    if tuple(gain.shape) != (K,):
        raise ValueError("gain must have the %d values of a row" % K)
    if residual is None:
        if sum_out is not None:
            raise ValueError("sum_out without a residual")
        return M, K, ldx, None, 0, 0, None, 0
    if residual.dtype not in (torch.float16, torch.float32) or residual.shape != x.shape or residual.stride(1) != 1 or not residual.is_cuda:
        raise ValueError("residual must be an fp16 or fp32 device tensor of x's shape with unit inner stride")
    if sum_out is None:
        sum_out = torch.empty((M, K), dtype=residual.dtype, device=x.device)
    elif sum_out.dtype != residual.dtype or sum_out.shape != x.shape or sum_out.stride(1) != 1 or not sum_out.is_cuda:
        raise ValueError("sum_out must be a device tensor of the residual's type and shape with unit inner stride")
    ldr, lds = (residual.stride(0), sum_out.stride(0)) if M > 1 else (max(K, residual.stride(0)), max(K, sum_out.stride(0)))
    return M, K, ldx, residual.data_ptr(), ldr, 1 if residual.dtype == torch.float16 else 2, sum_out, lds


def qqq_add_rmsnorm(x, gain, residual=None, eps=1e-6, y=None, sum_out=None):
    """x [M,K] fp16 (+ residual fp16 or fp32) -> (their sum in the residual's type or None, y fp16 [M,K] = norm(sum) * gain).
    sum_out may be the residual itself."""
    out = _native_rmsnorm(x, gain, residual, eps, sum_out, y, None, False, _raw_stream(_device())) if _lib and x.is_cuda else None
    if out is not None:
        return _checked(out)
    M, K, ldx, res, ldr, kind, sum_out, lds = _rmsnorm_args(x, gain, residual, sum_out)
    if y is None:
        y = torch.empty((M, K), dtype=torch.float16, device=x.device)
    elif y.shape != x.shape:
        raise ValueError("y must have x's shape")
    _check(lib().qqq_add_rmsnorm(x.data_ptr(), ldx, res, ldr, kind, _ptr(gain, _F16), eps, M, K, None if sum_out is None else sum_out.data_ptr(), lds,
                                 _ptr(y, _F16), _stream()))
    return sum_out, y


def qqq_add_rmsnorm_quant(x, gain, residual=None, eps=1e-6, a_q=None, s_a=None, sum_out=None):
    """The same straight to codes -> (sum or None, a_q int8 [M,K], s_a fp32 [M]), as qqq_quant_act gives them."""
    out = _native_rmsnorm(x, gain, residual, eps, sum_out, a_q, s_a, True, _raw_stream(_device())) if _lib and x.is_cuda else None
    if out is not None:
        return _checked(out)
    M, K, ldx, res, ldr, kind, sum_out, lds = _rmsnorm_args(x, gain, residual, sum_out)
    a_q, s_a = _codes_out(M, K, a_q, s_a, x.device)
    _check(lib().qqq_add_rmsnorm_quant(x.data_ptr(), ldx, res, ldr, kind, _ptr(gain, _F16), eps, M, K, None if sum_out is None else sum_out.data_ptr(),
                                       lds, _ptr(a_q, _I8), _ptr(s_a, torch.float32), _stream()))
    return sum_out, a_q, s_a


def _codes_out(M, K, a_q, s_a, device):
    if a_q is None:
        a_q = torch.empty((M, K), dtype=torch.int8, device=device)
    if s_a is None:
        s_a = torch.empty((M,), dtype=torch.float32, device=device)
    if tuple(a_q.shape) != (M, K) or s_a.numel() != M:
        raise ValueError("codes and scales must be of %d rows of %d" % (M, K))
    return a_q, s_a


_ACTS = {"silu": 0, "gelu_tanh": 1}


def qqq_gated_act_quant(gate, up, act="silu", a_q=None, s_a=None):
    """gate, up [M,F] fp16 (views of one projection's output allowed) -> (a_q int8 [M,F], s_a fp32 [M]) of act(gate) * up; act "silu" or "gelu_tanh"."""
    if act not in _ACTS:
        raise ValueError("act must be one of %s" % ", ".join(_ACTS))
    out = _native_gated(gate, up, _ACTS[act], a_q, s_a, _raw_stream(_device())) if _lib and gate.is_cuda else None
    if out is not None:
        return _checked(out)
    M, F, ldg = _rows(gate, "gate")
    M2, F2, ldu = _rows(up, "up")
    if (M, F) != (M2, F2):
        raise ValueError("gate and up disagree on their shape")
    a_q, s_a = _codes_out(M, F, a_q, s_a, gate.device)
    _check(lib().qqq_gated_act_quant(gate.data_ptr(), ldg, up.data_ptr(), ldu, _ACTS[act], M, F, _ptr(a_q, _I8), _ptr(s_a, torch.float32), _stream()))
    return a_q, s_a


class KV8Cache(typing.NamedTuple):
    """A layer's keys and values in 8 bits with a scale for each page and head (layout: include/qqq_layer.h)."""
    k_codes: torch.Tensor   # uint8 [pages, kv_heads, page_tokens, head_dim], offset binary
    k_scale: torch.Tensor   # fp32 [pages, kv_heads]
    v_codes: torch.Tensor   # uint8 [pages, kv_heads, head_dim, page_tokens]
    v_scale: torch.Tensor   # fp32 [pages, kv_heads]
    k_tail: torch.Tensor    # fp16 [slots, kv_heads, page_tokens, head_dim]: the pages that are not full
    v_tail: torch.Tensor    # fp16 [slots, kv_heads, head_dim, page_tokens]


class KV8Batch(typing.NamedTuple):
    """The sequences of a step: b holds kv_len[b] tokens, the last cu[b+1] - cu[b] of them new (rows cu[b] .. of the tensors beside it)."""
    page_table: torch.Tensor  # int32 [sequences, columns]
    kv_len: torch.Tensor      # int32 [sequences], the new tokens included
    cu: torch.Tensor          # int32 [sequences + 1]
    slots: typing.Optional[torch.Tensor]  # int32 [sequences]: tail slots; None: sequence b has slot b
    max_new: int              # bounds of the new tokens and of kv_len
    max_len: int


def new_kv8_cache(pages, kv_heads, head_dim, page_tokens=64, slots=1, device="cuda") -> KV8Cache:
    """An empty cache."""
    u8 = lambda *s: torch.full(s, 128, dtype=torch.uint8, device=device)  # noqa: E731
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16, device=device)  # noqa: E731
    scale = torch.zeros((2, pages, kv_heads), dtype=torch.float32, device=device)
    return KV8Cache(u8(pages, kv_heads, page_tokens, head_dim), scale[0], u8(pages, kv_heads, head_dim, page_tokens), scale[1],
                    f16(slots, kv_heads, page_tokens, head_dim), f16(slots, kv_heads, head_dim, page_tokens))


class _Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_codes", "k_scale", "v_codes", "v_scale", "k_tail", "v_tail")] + [
        ("pages", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("slots", "kv_heads", "head_dim", "page_tokens")]


class _Batch(ctypes.Structure):
    _fields_ = [("page_table", ctypes.c_void_p), ("table_stride", ctypes.c_int64)] + [(n, ctypes.c_void_p) for n in ("kv_len", "cu", "slots")] + [
        (n, ctypes.c_int32) for n in ("columns", "sequences", "max_new", "max_len")]


def _kv8_structs(cache, batch):
    kc, ks, vc, vs, kt, vt = cache
    table, kv_len, cu, slots, max_new, max_len = batch
    if kc.dim() != 4 or kt.dim() != 4 or table.dim() != 2 or table.stride(1) != 1 or not table.is_cuda or table.dtype != _I32:
        raise ValueError("codes and tails must be 4-D, page_table a 2-D int32 device tensor with unit inner stride")
    (pages, H, P, D), B = kc.shape, table.shape[0]
    nslots = kt.shape[0]
    if vc.shape != (pages, H, D, P) or ks.shape != (pages, H) or vs.shape != (pages, H) or kt.shape != (nslots, H, P, D) or vt.shape != (nslots, H, D, P):
        raise ValueError("the cache's tensors disagree on their shape")
    if kv_len.shape != (B,) or cu.shape != (B + 1,) or (slots is not None and slots.shape != (B,)):
        raise ValueError("kv_len, cu and slots must be of page_table's %d sequences" % B)
    if slots is None and nslots < B:
        raise ValueError("%d tail slots for %d sequences" % (nslots, B))
    f32 = torch.float32
    return (_Cache(_ptr(kc, _U8), _ptr(ks, f32), _ptr(vc, _U8), _ptr(vs, f32), _ptr(kt, _F16), _ptr(vt, _F16), pages, nslots, H, D, P),
            _Batch(table.data_ptr(), table.stride(0) if B > 1 else max(table.shape[1], table.stride(0)), _ptr(kv_len, _I32), _ptr(cu, _I32),
                   _ptr(slots, _I32), table.shape[1], B, max_new, max_len), H, D)


def _heads(t, heads, D, name):
    if t.dtype != torch.float16 or t.dim() != 3 or t.stride(2) != 1 or not t.is_cuda or t.shape[2] != D or (heads and t.shape[1] != heads):
        raise ValueError("%s must be an fp16 device tensor [tokens, heads, %d] with unit inner stride" % (name, D))
    return t.shape[0], t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0


def qqq_kv8_append(cache: KV8Cache, batch: KV8Batch, k, v):
    """Puts the step's new keys and values [tokens, kv_heads, head_dim] fp16 (strided views allowed) into the cache."""
    rc = _native_append(cache, batch, k, v, _raw_stream(_device())) if _lib and k.is_cuda else None
    if rc is not None:
        return _check(rc)
    c, b, H, D = _kv8_structs(cache, batch)
    (T, kt, kh), (T2, vt, vh) = _heads(k, H, D, "k"), _heads(v, H, D, "v")
    if T != T2:
        raise ValueError("k and v disagree on their tokens")
    _check(lib().qqq_kv8_append(ctypes.byref(c), ctypes.byref(b), k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, T, _stream()))


def qqq_kv8_read(cache: KV8Cache, batch: KV8Batch, k=None, v=None, tokens=None):
    """The last cu[b+1] - cu[b] tokens of each sequence as the cache holds them -> (k, v) fp16 [tokens, kv_heads, head_dim]; tokens: rows of the
    outputs where they are not given."""
    if k is not None and v is not None and _lib and k.is_cuda:
        rc = _native_read(cache, batch, k, v, _raw_stream(_device()))
        if rc is not None:
            _check(rc)
            return k, v
    c, b, H, D = _kv8_structs(cache, batch)
    if (k is None or v is None) and tokens is None:
        raise ValueError("tokens is needed where k or v is not given")
    if k is None:
        k = torch.empty((tokens, H, D), dtype=torch.float16, device=cache[0].device)
    if v is None:
        v = torch.empty((tokens, H, D), dtype=torch.float16, device=cache[0].device)
    if k.dim() != 3 or k.shape[1:] != (H, D) or v.shape != k.shape:
        raise ValueError("k and v must be [tokens, %d, %d]" % (H, D))
    _check(lib().qqq_kv8_read(ctypes.byref(c), ctypes.byref(b), _ptr(k, _F16), _ptr(v, _F16), k.shape[0], _stream()))
    return k, v


def qqq_attention_kv8_workspace_bytes(cache: KV8Cache, batch: KV8Batch, q_heads: int, tokens: int) -> int:
    c, b, _, _ = _kv8_structs(cache, batch)
    return int(lib().qqq_attention_kv8_workspace_bytes(ctypes.byref(c), ctypes.byref(b), q_heads, tokens))


def qqq_attention_kv8(cache: KV8Cache, batch: KV8Batch, q, scale=None, causal=True, window=0, out=None, lse=None, workspace=None):
    """Attention of the new tokens' queries [tokens, q_heads, head_dim] fp16 (strided views allowed) over the cache -> (out fp16 of that shape, lse
    fp32 [tokens, q_heads], or None where none is given).  scale: 1 / sqrt(head_dim).  workspace: a uint8 tensor of
    qqq_attention_kv8_workspace_bytes(); without one torch's allocator lends it."""
    given = _native_attention(cache, batch, q, scale, causal, window, out, lse, workspace, _raw_stream(_device())) if _lib and q.is_cuda else None
    if given is not None:
        return _checked(given)
    c, b, H, D = _kv8_structs(cache, batch)
    T, qt, qh = _heads(q, 0, D, "q")
    Hq = q.shape[1]
    if out is None:
        out = torch.empty((T, Hq, D), dtype=torch.float16, device=q.device)
    elif out.shape != q.shape:
        raise ValueError("out must have q's shape")
    if lse is not None and lse.shape != (T, Hq):
        raise ValueError("lse must be [tokens, q_heads]")
    L = lib()
    if workspace is None:
        nbytes = L.qqq_attention_kv8_workspace_bytes(ctypes.byref(c), ctypes.byref(b), Hq, T)
        workspace = torch.empty((nbytes,), dtype=torch.uint8, device=q.device) if nbytes else None
    _check(L.qqq_attention_kv8(ctypes.byref(c), ctypes.byref(b), q.data_ptr(), qt, qh, Hq, T, D ** -0.5 if scale is None else scale, int(causal), window,
                               _ptr(out, _F16), None if lse is None else _ptr(lse, torch.float32), _ptr(workspace, _U8),
                               0 if workspace is None else workspace.numel(), _stream()))
    return out, lse


def last_route() -> str:
    """The kernels the most recent GEMM / linear call of this thread enqueued (include/qqq_tuning.h)."""
    return lib().qqq_last_route().decode()


def count_sg_violations(s_g: torch.Tensor, sg_max: int) -> int:
    """Entries of the integer group-scale table [K/128, N] outside 0..sg_max (diagnostic; synchronises)."""
    G, N = s_g.shape
    out = torch.empty((1,), dtype=torch.int32, device=s_g.device)
    _check(lib().qqq_debug_count_sg_violations(_ptr(s_g, torch.int8), N, G * GROUP, sg_max,
                                               _ptr(out, torch.int32), _stream()))
    return int(out.item())


def probe_stream_read(buf: torch.Tensor, nbytes: int, workgroups: int, sink: torch.Tensor, offset: int = 0):
    """One launch of the streaming-read ceiling probe over buf[offset : offset + nbytes] (uint8 tensor)."""
    _check(lib().qqq_probe_stream_read(ctypes.c_void_p(buf.data_ptr() + offset), nbytes, workgroups,
                                       _ptr(sink, torch.int32), _stream()))


def probe_mfma_i8(a_pool: torch.Tensor, b_pool: torch.Tensor, iters: int, workgroups: int, sink: torch.Tensor):
    """One launch of the int8 MFMA ceiling probe (a_pool 128 KiB, b_pool 32 KiB of int8 operand values)."""
    if a_pool.numel() != 4 * 4 * 512 * 16 or b_pool.numel() != 2 * 2 * 512 * 16:
        raise ValueError("operand pools must hold 4*4*512 and 2*2*512 16-byte values")
    _check(lib().qqq_probe_mfma_i8(_ptr(a_pool, torch.int8), _ptr(b_pool, torch.int8), iters, workgroups,
                                   _ptr(sink, torch.int32), _stream()))


PROBE_A_READS, PROBE_W_READS, PROBE_CONVERT, PROBE_DMA, PROBE_FORM_32X32X32 = 1, 2, 4, 8, 16
PROBE_LOOP_STAGE = 51200


def probe_prefill_loop(src: torch.Tensor, region_bytes: int, steps: int, parts: int, workgroups: int,
                       sink: torch.Tensor):
    """One launch of the prefill k-loop probe: src is a uint8 tensor of workgroups * region_bytes bytes."""
    if src.numel() < workgroups * region_bytes:
        raise ValueError("src must hold workgroups * region_bytes bytes")
    _check(lib().qqq_probe_prefill_loop(_ptr(src, torch.uint8), region_bytes, steps, parts, workgroups,
                                        _ptr(sink, torch.int32), _stream()))


def set_fused_quant(enable: int) -> int:
    return lib().qqq_set_fused_quant(enable)


def set_kernel_override(family: int) -> int:
    return lib().qqq_set_kernel_override(family)


def set_group_mode_override(mode: int) -> int:
    return lib().qqq_set_group_mode_override(mode)


def set_skinny_tuning(channel_tiles: int, k_slices: int, waves: int = 0, depth: int = 0) -> int:
    return lib().qqq_set_skinny_tuning(channel_tiles, k_slices, waves, depth)


def set_prefill_tuning(waves: int) -> int:
    return lib().qqq_set_prefill_tuning(waves)



def set_prefill_ksplit(k_splits: int) -> int:
    """Diagnostic: K splits of the per-tile prefill kernel for 64 < M <= 512 (0 = automatic)."""
    return lib().qqq_set_prefill_ksplit(k_splits)


def set_factor_workgroups(most: int) -> int:
    """Diagnostic: the most workgroups of the compensation's factorisation (0 = automatic)."""
    return lib().qqq_set_factor_workgroups(most)
