"""Integer-only relative-positional MHSA (I-Parakeet, Sec. 3.1) on GB300.

A thin Python binding over the C ABI of ``include/ip_mhsa.h``: argument
marshalling only.  Every step of the attention runs in the CUDA kernels of
``libipmhsa.so``; there is no CPU fallback, and a missing or unloadable
library raises :class:`LibraryError`.  PyTorch serves for device memory and
streams only.
"""
from __future__ import annotations

import ctypes
import operator
import sys
import threading
import warnings
from dataclasses import dataclass

from . import build as _build

IP_DH = 128
IP_MAX_T = 2048

ERRORS = {
    0: "IP_OK", -1: "IP_ERR_NULL", -2: "IP_ERR_SHAPE", -3: "IP_ERR_ALIGN",
    -4: "IP_ERR_UNSUPPORTED", -5: "IP_ERR_CUDA", -6: "IP_ERR_TIMEOUT",
    -7: "IP_ERR_PARAM", -8: "IP_ERR_WORKSPACE",
}

EXPORTS = (
    "ip_relpos_mhsa_workspace_bytes", "ip_relpos_mhsa_i8", "ip_relpos_mhsa_status",
    "ip_relpos_mhsa_host_arena_bytes", "ip_relpos_mhsa_i8_host", "ip_strerror",
    "ip_debug_set_timeout_cycles", "ip_debug_set_stall_injection", "ip_dyadic_multiplier",
    "ip_dyadic_pair",
    "ip_isoftmax_params_from_scale", "ip_probe_int8_mma", "ip_relpos_mhsa_i8_noalloc",
    "ip_debug_set_split_mode", "ip_debug_set_wide_sums", "ip_linear_i8", "ip_linear_swish_i8", "ip_swish_params_from_scales",
    "ip_layernorm_i8", "ip_layernorm_constants", "ip_relpos_mhsa_i8_ex", "ip_residual_i8",
    "ip_residual_params", "ip_linear_glu_i8", "ip_glu_params", "ip_dwconv_swish_i8",
    "ip_swish16_params_from_scales", "ip_relpos_mhsa_i8_host_async", "ip_relpos_mhsa_host_status",
    "ip_set_workspace", "ip_probe_int8_mix", "ip_linear_residual_i8",
    "ip_relpos_layer_constants", "ip_linear_constants", "ip_relpos_mhsa_noalloc_status",
    "ip_quantize_rows_i8", "ip_linear_scaled_i8", "ip_kv4_page_bytes", "ip_kv4_append", "ip_kv4_read",
    "ip_kv4_attention_workspace_bytes", "ip_kv4_attention",
    "ip_fp4_block_bytes", "ip_quantize_fp4", "ip_rmsnorm_i8", "ip_rmsnorm_fp4", "ip_dequantize_i8",
    "ip_dequantize_fp4", "ip_token_logprobs_workspace_bytes", "ip_token_logprobs",
    "ip_linear_fp4",
)

ROWS = 0    # IP_LAYOUT_ROWS:  [B][T][C]
HEADS = 1   # IP_LAYOUT_HEADS: [G][B][C/G/128][T][128]
ACT_NONE = 0    # IP_ACT_NONE
ACT_SWISH = 1   # IP_ACT_SWISH: z / (1 + exp(-z))


class LibraryError(RuntimeError):
    """The GPU library could not be built or loaded."""


class IpError(RuntimeError):
    """A library call returned an IP_ERR_* code."""

    def __init__(self, fn: str, code: int, text: str):
        super().__init__(f"{fn}: {ERRORS.get(code, code)} ({text})")
        self.code = code


class SwishParams(ctypes.Structure):
    _fields_ = [("q_c", ctypes.c_int32), ("q_one", ctypes.c_int32), ("m", ctypes.c_int32),
                ("s", ctypes.c_int32)]


class Swish16Params(ctypes.Structure):
    _fields_ = [("q_c", ctypes.c_int32), ("q_one", ctypes.c_longlong), ("m", ctypes.c_int32),
                ("s", ctypes.c_int32)]


class SoftmaxParams(ctypes.Structure):
    _fields_ = [("q_ln2", ctypes.c_int32), ("q_b", ctypes.c_int32), ("q_c", ctypes.c_int32)]


class _Int:
    """An int argument of an entry point.  What 32 bits do not hold becomes the end of their range,
    which the entry points refuse, where c_int would wrap it to a value they may take."""

    @classmethod
    def from_param(cls, v):
        return ctypes.c_int(max(-1 << 31, min(operator.index(v), (1 << 31) - 1)))


_lock = threading.Lock()
_lib = None


def build(force: bool = False) -> str:
    """Compile libipmhsa.so for sm_103a (nvcc) and return its path."""
    return _build.build(force=force)


def load(build_if_missing: bool = True) -> ctypes.CDLL:
    """Load libipmhsa.so and declare the C signatures."""
    global _lib, _short
    with _lock:
        if _lib is not None:
            return _lib
        try:
            path = _build.build() if build_if_missing else _build.LIB
            lib = ctypes.CDLL(path)
        except Exception as exc:  # noqa: BLE001 - reported with context
            raise LibraryError(f"cannot build or load the GPU library: {exc}") from exc
        P = ctypes.c_void_p
        I = ctypes.c_int
        i32p = ctypes.POINTER(ctypes.c_int32)
        lib.ip_relpos_mhsa_workspace_bytes.argtypes = [I, I, I, I]
        lib.ip_relpos_mhsa_workspace_bytes.restype = ctypes.c_size_t
        lib.ip_relpos_mhsa_host_arena_bytes.argtypes = [I, I, I, I]
        lib.ip_relpos_mhsa_host_arena_bytes.restype = ctypes.c_size_t
        sig = [P] * 6 + [P, P, ctypes.POINTER(SoftmaxParams), P] + [I] * 4 + [P, P, ctypes.c_size_t, P]
        lib.ip_relpos_mhsa_i8.argtypes = sig
        lib.ip_relpos_mhsa_i8.restype = I
        lib.ip_relpos_mhsa_i8_host.argtypes = sig
        lib.ip_relpos_mhsa_i8_host.restype = I
        lib.ip_relpos_mhsa_i8_noalloc.argtypes = sig[:15] + [P]
        lib.ip_relpos_mhsa_i8_noalloc.restype = I
        lib.ip_relpos_mhsa_noalloc_status.argtypes = [P]
        lib.ip_relpos_mhsa_noalloc_status.restype = I
        lib.ip_relpos_mhsa_status.argtypes = [P, P]
        lib.ip_relpos_mhsa_status.restype = I
        lib.ip_set_workspace.argtypes = [P, ctypes.c_size_t]
        lib.ip_set_workspace.restype = I
        lib.ip_strerror.argtypes = [I]
        lib.ip_strerror.restype = ctypes.c_char_p
        lib.ip_debug_set_timeout_cycles.argtypes = [ctypes.c_longlong]
        lib.ip_debug_set_timeout_cycles.restype = I
        lib.ip_debug_set_stall_injection.argtypes = [I]
        lib.ip_debug_set_stall_injection.restype = I
        lib.ip_debug_set_split_mode.argtypes = [I]
        lib.ip_debug_set_split_mode.restype = I
        lib.ip_debug_set_wide_sums.argtypes = [I]
        lib.ip_debug_set_wide_sums.restype = I
        lib.ip_dyadic_multiplier.argtypes = [ctypes.c_double, i32p, i32p]
        lib.ip_dyadic_multiplier.restype = I
        lib.ip_dyadic_pair.argtypes = [ctypes.c_double, ctypes.c_double, i32p, i32p, i32p]
        lib.ip_dyadic_pair.restype = I
        lib.ip_isoftmax_params_from_scale.argtypes = [ctypes.c_double, ctypes.POINTER(SoftmaxParams)]
        lib.ip_isoftmax_params_from_scale.restype = I
        D_ = ctypes.c_double
        lib.ip_relpos_layer_constants.argtypes = [D_] * 6 + [I, P, P, ctypes.POINTER(SoftmaxParams)]
        lib.ip_relpos_layer_constants.restype = I
        lib.ip_linear_constants.argtypes = [D_, ctypes.POINTER(D_), ctypes.POINTER(D_), I,
                                            ctypes.POINTER(ctypes.c_int32),
                                            ctypes.POINTER(ctypes.c_int32)]
        lib.ip_linear_constants.restype = I
        lib.ip_relpos_mhsa_i8_ex.argtypes = [P] * 6 + [P, P, ctypes.POINTER(SoftmaxParams), P] + [
            I] * 4 + [P, I, P, ctypes.c_size_t, P]
        lib.ip_relpos_mhsa_i8_ex.restype = I
        lib.ip_relpos_mhsa_i8_host_async.argtypes = lib.ip_relpos_mhsa_i8_host.argtypes
        lib.ip_relpos_mhsa_i8_host_async.restype = I
        lib.ip_relpos_mhsa_host_status.argtypes = [P, I, I, I, I, P]
        lib.ip_relpos_mhsa_host_status.restype = I
        lib.ip_linear_i8.argtypes = [P, I, P, P, P, P, I, I, I, I, I, P, I, P, ctypes.c_size_t, P]
        lib.ip_linear_i8.restype = I
        lib.ip_linear_swish_i8.argtypes = [P, P, P, P, P, ctypes.POINTER(SwishParams), I, I, I, I,
                                           P, P, ctypes.c_size_t, P]
        lib.ip_linear_swish_i8.restype = I
        lib.ip_swish_params_from_scales.argtypes = [ctypes.c_double, ctypes.c_double,
                                                    ctypes.POINTER(SwishParams)]
        lib.ip_swish_params_from_scales.restype = I
        LL = ctypes.c_longlong
        lib.ip_layernorm_i8.argtypes = [P, LL, I, LL, P, P, P, P, P, ctypes.c_size_t, P]
        lib.ip_layernorm_i8.restype = I
        D = ctypes.c_double
        lib.ip_layernorm_constants.argtypes = [D, P, P, I, D, D, ctypes.POINTER(LL), P, P, P]
        lib.ip_layernorm_constants.restype = I
        i32p_ = ctypes.POINTER(ctypes.c_int32)
        lib.ip_residual_i8.argtypes = [P, P, ctypes.c_longlong, I, I, I, P, P]
        lib.ip_residual_i8.restype = I
        lib.ip_residual_params.argtypes = [D, D, D, D, i32p_, i32p_, i32p_]
        lib.ip_residual_params.restype = I
        lib.ip_linear_glu_i8.argtypes = [P, P, P, P, P, ctypes.POINTER(SwishParams), I, I, I, I, P,
                                         P, ctypes.c_size_t, P]
        lib.ip_linear_glu_i8.restype = I
        lib.ip_linear_residual_i8.argtypes = [P, P, P, P, P, P, I, I, I, I, I, I, I, P, P,
                                              ctypes.c_size_t, P]
        lib.ip_linear_residual_i8.restype = I
        lib.ip_glu_params.argtypes = [D, D, D, ctypes.POINTER(SwishParams)]
        lib.ip_glu_params.restype = I
        lib.ip_dwconv_swish_i8.argtypes = [P, I, I, I, P, I, P, P, P, ctypes.POINTER(Swish16Params),
                                           P, P, ctypes.c_size_t, P]
        lib.ip_dwconv_swish_i8.restype = I
        lib.ip_swish16_params_from_scales.argtypes = [D, D, ctypes.POINTER(Swish16Params)]
        lib.ip_swish16_params_from_scales.restype = I
        N, S, F = _Int, ctypes.c_size_t, ctypes.c_float
        for name, args, result in (
                ("ip_quantize_rows_i8", [P, N, LL, N, LL, P, LL, P, P], I),
                ("ip_linear_scaled_i8", [P, LL, P, P, LL, P, P, N, LL, N, N, P, LL, N, P, S, P], I),
                ("ip_kv4_page_bytes", [N, N], S),
                ("ip_kv4_append", [P, P, N, P, P, P, P, N, N, N, N, P, N, P, N, N, P, S, P], I),
                ("ip_kv4_read", [P, N, N, P, N, P, P, N, N, N, N, P, P, N, P, S, P], I),
                ("ip_kv4_attention_workspace_bytes", [N] * 5, S),
                ("ip_kv4_attention", [P, N, P, P, P, N, F, N, N, N, N, N, N, P, N, P, N, N, P, P, S, P], I),
                ("ip_fp4_block_bytes", [LL, N], S),
                ("ip_quantize_fp4", [P, N, LL, N, LL, P, LL, P, P, P], I),
                ("ip_rmsnorm_i8", [P, LL, P, LL, P, F, N, LL, N, P, LL, P, LL, P, P], I),
                ("ip_rmsnorm_fp4", [P, LL, P, LL, P, F, N, LL, N, P, LL, P, LL, P, P, P], I),
                ("ip_dequantize_i8", [P, LL, P, LL, N, P, LL, N, P], I),
                ("ip_dequantize_fp4", [P, LL, P, P, LL, N, P, LL, N, P], I),
                ("ip_linear_fp4", [P, LL, P, P, P, LL, P, P, P, N, LL, N, N, P, LL, N, P, S, P], I),
                ("ip_token_logprobs_workspace_bytes", [LL, N, N], S),
                ("ip_token_logprobs", [P, N, LL, N, LL, P, N, F, N, P, P, P, P, P, S, P], I)):
            fn = getattr(lib, name, None)      # a library built before these calls does the others
            if fn is not None:
                fn.argtypes, fn.restype = args, result
        lib.ip_probe_int8_mma.argtypes = [I, I, P, P]
        lib.ip_probe_int8_mma.restype = ctypes.c_longlong
        lib.ip_probe_int8_mix.argtypes = [I, I, I, P, P]
        lib.ip_probe_int8_mix.restype = ctypes.c_longlong
        # a process that has not imported torch has no use for them yet
        _short = _bound_short(lib) if "torch" in sys.modules else _Pending(lib)
        _lib = lib
        return lib


def strerror(code: int) -> str:
    return load().ip_strerror(code).decode()


def _check(fn: str, code: int):
    if code != 0:
        raise IpError(fn, code, strerror(code))


# ---------------------------------------------------------------- constants

@dataclass(frozen=True)
class LayerConstants:
    multipliers: tuple[int, int, int]   # m_c, m_p, m_o
    shifts: tuple[int, int]             # s_s, s_o (right shift 31 + s)
    softmax: tuple[int, int, int]       # q_ln2, q_b, q_c


def dyadic_multiplier(ratio: float) -> tuple[int, int]:
    m, s = ctypes.c_int32(), ctypes.c_int32()
    _check("ip_dyadic_multiplier", load().ip_dyadic_multiplier(ratio, ctypes.byref(m), ctypes.byref(s)))
    return m.value, s.value


def dyadic_pair(r_c: float, r_p: float) -> tuple[int, int, int]:
    a, b, s = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check("ip_dyadic_pair", load().ip_dyadic_pair(r_c, r_p, ctypes.byref(a), ctypes.byref(b), ctypes.byref(s)))
    return a.value, b.value, s.value


def isoftmax_params_from_scale(S_s: float) -> tuple[int, int, int]:
    prm = SoftmaxParams()
    _check("ip_isoftmax_params_from_scale", load().ip_isoftmax_params_from_scale(S_s, ctypes.byref(prm)))
    return prm.q_ln2, prm.q_b, prm.q_c


def layer_constants(scales: dict, dh: int = IP_DH) -> LayerConstants:
    """Integer constants of one layer from its real scales S_Q, S_K, S_P,
    S_V, S_s, S_O (offline, Eq. 7 and Eq. 11), by ip_relpos_layer_constants."""
    mult = (ctypes.c_int32 * 3)()
    sh = (ctypes.c_int32 * 2)()
    sm = SoftmaxParams()
    _check("ip_relpos_layer_constants", load().ip_relpos_layer_constants(
        float(scales["S_Q"]), float(scales["S_K"]), float(scales["S_P"]), float(scales["S_V"]),
        float(scales["S_s"]), float(scales["S_O"]), int(dh), mult, sh, ctypes.byref(sm)))
    return LayerConstants(tuple(mult), tuple(sh), (sm.q_ln2, sm.q_b, sm.q_c))


# ---------------------------------------------------------------- device path

def workspace_bytes(B: int, H: int, T: int, dh: int = IP_DH) -> int:
    n = load().ip_relpos_mhsa_workspace_bytes(B, H, T, dh)
    if n == 0:
        raise IpError("ip_relpos_mhsa_workspace_bytes", -2, "invalid shape")
    return n


def host_arena_bytes(B: int, H: int, T: int, dh: int = IP_DH) -> int:
    n = load().ip_relpos_mhsa_host_arena_bytes(B, H, T, dh)
    if n == 0:
        raise IpError("ip_relpos_mhsa_host_arena_bytes", -2, "invalid shape")
    return n


def set_timeout_cycles(cycles: int) -> None:
    """Bound of every kernel barrier wait (clock cycles; negative: default)."""
    load().ip_debug_set_timeout_cycles(int(cycles))


def set_stall_injection(on: bool) -> None:
    """Test hook: make the kernels wait on a barrier nothing arrives on."""
    load().ip_debug_set_stall_injection(1 if on else 0)


def set_split_mode(mode: int) -> None:
    """Test hook: -1 planned tail split (default), 0 never split, 1 split
    every 64-row tile into two key-split halves, 2 into four key-split
    quarters."""
    load().ip_debug_set_split_mode(int(mode))


def set_wide_sums(on: bool) -> None:
    """Test hook: always take the general softmax arithmetic (64-bit partial
    row sums, probabilities from the full 64-bit product); False: the fast
    paths where the host has shown they give the same integers."""
    load().ip_debug_set_wide_sums(1 if on else 0)


def _arr(vals, ctype):
    return (ctype * len(vals))(*vals)


def _stream_handle(stream):
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _stream(stream):
    """The same handle as an int, for the calls that have CUDA tensors in hand
    (so that CUDA is initialised): 0.2 us on a Grace core instead of the 3 us of
    making a Stream object."""
    if stream is None:
        import torch
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _dev_ptr(t, name, dtype, shape):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _ptrs(tensor, checks):
    """Device pointers of (t, name, dtype, shape) in order: the checks of _dev_ptr
    in one pass over plain tensors (0.4 us each instead of 0.7), _dev_ptr itself
    for the error of one that fails and for tensor subclasses.  A short call's
    host time is what its kernel hides behind: attention 17 -> 9 us, LayerNorm
    12 -> 6 us a call."""
    return [t.data_ptr() if t.__class__ is tensor and t.dtype is dtype and t.shape == shape
            and t.is_cuda and t.is_contiguous() else _dev_ptr(t, name, dtype, shape)
            for t, name, dtype, shape in checks]


def relpos_mhsa_i8(q, k, v, p, u, v_bias, consts: LayerConstants, lengths=None, out=None,
                   workspace=None, stream=None, out_layout: int = HEADS):
    """Whole layer on the GPU.  q, k, v: int8 [B, H, T, 128] CUDA tensors;
    p: int8 [H, 2T-1, 128]; u, v_bias: int8 [H, 128]; lengths: int32 [B]
    CUDA tensor or None.  Returns out: int8 [B, H, T, 128] (HEADS) or
    [B, T, H, 128] (ROWS, the frames' rows of the output projection).
    Asynchronous on `stream` (default: torch's current stream)."""
    import torch
    B, H, T, dh = q.shape
    shp, bshp, i8 = (B, H, T, dh), (H, dh), torch.int8
    oshp = shp if out_layout == HEADS else (B, T, H, dh)
    checks = [(q, "q", i8, shp), (k, "k", i8, shp), (v, "v", i8, shp),
              (p, "p", i8, (H, 2 * T - 1, dh)), (u, "u", i8, bshp), (v_bias, "v_bias", i8, bshp)]
    args = _ptrs(torch.Tensor, checks)
    if out is None:
        out = torch.empty(oshp, dtype=torch.int8, device=q.device)
    lens = None if lengths is None else _ptrs(torch.Tensor, [(lengths, "lengths", torch.int32, (B,))])[0]
    if workspace is None and _default_workspace is None:
        workspace = torch.zeros(workspace_bytes(B, H, T, dh), dtype=torch.uint8, device=q.device)
    # workspace None here: the library uses the registered default workspace
    ws_ptr, ws_len = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())
    rc = (_lib or load()).ip_relpos_mhsa_i8_ex(
        *args, _arr(consts.multipliers, ctypes.c_int32), _arr(consts.shifts, ctypes.c_int32),
        SoftmaxParams(*consts.softmax), lens, B, H, T, dh,
        *_ptrs(torch.Tensor, [(out, "out", i8, oshp)]), out_layout, ws_ptr, ws_len, _stream(stream))
    if rc:
        _check("ip_relpos_mhsa_i8_ex", rc)
    return out


def int8_mma_peak_tops(iters: int = 4096, repeats: int = 3) -> float:
    """Measured integer warp-MMA throughput of the current GPU in TOPS
    (best of `repeats` timed launches, CUDA events on the launching stream)."""
    import torch
    props = torch.cuda.get_device_properties(torch.cuda.current_device())
    blocks = props.multi_processor_count * 8
    sink = torch.empty(blocks * 256, dtype=torch.int32, device="cuda")
    st = torch.cuda.current_stream()
    lib = load()
    h = ctypes.c_void_p(st.cuda_stream)
    lib.ip_probe_int8_mma(blocks, iters, ctypes.c_void_p(sink.data_ptr()), h)   # warm-up
    best = 0.0
    for _ in range(repeats):
        e0 = torch.cuda.Event(enable_timing=True)
        e1 = torch.cuda.Event(enable_timing=True)
        e0.record(st)
        ops = lib.ip_probe_int8_mma(blocks, iters, ctypes.c_void_p(sink.data_ptr()), h)
        e1.record(st)
        e1.synchronize()
        if ops < 0:
            raise IpError("ip_probe_int8_mma", -5, "launch failed")
        best = max(best, ops / (e0.elapsed_time(e1) * 1e-3) / 1e12)
    return best


def int8_pipe_rates(iters: int = 2048, repeats: int = 3) -> dict:
    """Measured integer throughput (TOPS, best of `repeats` launches, CUDA
    events) of the integer MMA pipe alone, the dp4a pipe alone, and both at
    once (half the warps on each)."""
    import torch
    props = torch.cuda.get_device_properties(torch.cuda.current_device())
    blocks = props.multi_processor_count * 2
    sink = torch.empty(blocks * 256, dtype=torch.int32, device="cuda")
    st = torch.cuda.current_stream()
    lib = load()
    h = ctypes.c_void_p(st.cuda_stream)
    out = {}
    for name, mw in (("imma", 8), ("dp4a", 0), ("imma_plus_dp4a", 4)):
        lib.ip_probe_int8_mix(blocks, iters, mw, ctypes.c_void_p(sink.data_ptr()), h)   # warm-up
        best = 0.0
        for _ in range(repeats):
            e0 = torch.cuda.Event(enable_timing=True)
            e1 = torch.cuda.Event(enable_timing=True)
            e0.record(st)
            ops = lib.ip_probe_int8_mix(blocks, iters, mw, ctypes.c_void_p(sink.data_ptr()), h)
            e1.record(st)
            e1.synchronize()
            if ops < 0:
                raise IpError("ip_probe_int8_mix", -5, "launch failed")
            best = max(best, ops / (e0.elapsed_time(e1) * 1e-3) / 1e12)
        out[name] = best
    return out


def status(workspace=None, stream=None) -> int:
    """Synchronises the stream and returns the device-side status code of
    the last call that used `workspace` (0 = ok); None: the default
    workspace registered by set_workspace."""
    ptr = None if workspace is None else ctypes.c_void_p(workspace.data_ptr())
    return load().ip_relpos_mhsa_status(ptr, _stream_handle(stream))


def noalloc_status(stream=None) -> int:
    """Synchronises the stream and returns the device-side status code of
    the ip_relpos_mhsa_i8_noalloc calls on the current device since the
    last read (0 = ok), clearing it."""
    return load().ip_relpos_mhsa_noalloc_status(_stream_handle(stream))


_default_workspace = None


def set_workspace(workspace) -> None:
    """Registers `workspace` (a zero-filled uint8 CUDA tensor of at least
    workspace_bytes(...) bytes) as the default of the attention calls that
    pass none; None releases it.  The binding keeps the tensor alive while
    it is registered.  Calls that share it must run on one stream."""
    global _default_workspace
    if workspace is None:
        _check("ip_set_workspace", load().ip_set_workspace(None, 0))
        _default_workspace = None
        return
    import torch
    if not (isinstance(workspace, torch.Tensor) and workspace.is_cuda and
            workspace.dtype == torch.uint8 and workspace.is_contiguous()):
        raise TypeError("workspace: a contiguous uint8 CUDA tensor")
    _check("ip_set_workspace", load().ip_set_workspace(ctypes.c_void_p(workspace.data_ptr()),
                                                       workspace.numel()))
    _default_workspace = workspace


def linear_constants(s_x: float, s_w, s_y):
    """Per-output-channel constants of Eq. 7 (offline), by
    ip_linear_constants: int32 arrays m, s of the length of s_w (s_y: one
    grid per channel, or one for all)."""
    import numpy as np
    s_w = np.ascontiguousarray(s_w, dtype=np.float64).reshape(-1)
    s_y = np.ascontiguousarray(np.broadcast_to(np.asarray(s_y, dtype=np.float64).reshape(-1)
                                               if np.ndim(s_y) else np.float64(s_y), s_w.shape))
    m = np.empty(s_w.shape, dtype=np.int32)
    s = np.empty(s_w.shape, dtype=np.int32)
    dp = ctypes.POINTER(ctypes.c_double)
    ip32 = ctypes.POINTER(ctypes.c_int32)
    _check("ip_linear_constants", load().ip_linear_constants(
        float(s_x), s_w.ctypes.data_as(dp), s_y.ctypes.data_as(dp), int(s_w.size),
        m.ctypes.data_as(ip32), s.ctypes.data_as(ip32)))
    return m, s


def _linear_ptrs(x, xs, w, bias, m, s, out, ys):
    """Checked pointers of a linear layer's tensors (bias may be None)."""
    import torch
    i8, i32, n = torch.int8, torch.int32, (w.shape[0],)
    checks = [(x, "x", i8, xs), (w, "w", i8, (n[0], w.shape[1])), (m, "m", i32, n), (s, "s", i32, n),
              (out, "out", i8, ys)]
    if bias is not None:
        checks.append((bias, "bias", i32, n))
    px, pw, pm, ps, po, *pb = _ptrs(torch.Tensor, checks)
    return px, pw, pb[0] if pb else None, pm, ps, po


def linear_i8(x, w, bias, m, s, *, x_layout: int = ROWS, y_layout: int = ROWS, groups: int = 1,
              out=None, workspace=None, stream=None):
    """Integer linear layer (Eqs. 6-7) on the GPU.  x: int8 [B, T, K] (ROWS)
    or [B, K/128, T, 128] (HEADS); w: int8 [N, K]; bias: int32 [N] or None;
    m, s: int32 [N] (per output channel); all CUDA tensors.  Returns out:
    int8 [B, T, N] (ROWS) or [G, B, N/G/128, T, 128] (HEADS).  Asynchronous
    on `stream` (default: torch's current stream)."""
    import torch
    N, K = w.shape
    if x_layout == ROWS:
        B, T, _ = x.shape
        xs = (B, T, K)
    else:
        B, _, T, _ = x.shape
        xs = (B, K // 128, T, 128)
    ys = (B, T, N) if y_layout == ROWS else (groups, B, N // max(groups, 1) // 128, T, 128)
    if out is None:
        out = torch.empty(ys, dtype=torch.int8, device=w.device)
    if workspace is None:
        workspace = torch.zeros(256, dtype=torch.uint8, device=w.device)
    px, pw, pb, pm, ps, po = _linear_ptrs(x, xs, w, bias, m, s, out, ys)
    rc = (_lib or load()).ip_linear_i8(px, x_layout, pw, pb, pm, ps, B, T, K, N, groups, po, y_layout,
                                       workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc:
        _check("ip_linear_i8", rc)
    return out


def linear_residual_i8(x, w, bias, m, s, res, m_x: int, m_y: int, s_r: int, *, out=None,
                       workspace=None, stream=None):
    """Integer linear layer with the residual addition of its output fused:
    out = residual(res, linear(x)) with (m_x, m_y, s_r) from residual_params.
    x: int8 [B, T, K]; w: int8 [N, K]; bias, m, s as linear_i8; res: int8
    [B, T, N] (not aliasing out); all CUDA tensors, row-major."""
    import torch
    N, K = w.shape
    B, T, _ = x.shape
    if out is None:
        out = torch.empty((B, T, N), dtype=torch.int8, device=w.device)
    if workspace is None:
        workspace = torch.zeros(256, dtype=torch.uint8, device=w.device)
    ys = (B, T, N)
    px, pw, pb, pm, ps, po = _linear_ptrs(x, (B, T, K), w, bias, m, s, out, ys)
    pr, = _ptrs(torch.Tensor, [(res, "res", torch.int8, ys)])
    rc = (_lib or load()).ip_linear_residual_i8(px, pw, pb, pm, ps, pr, int(m_x), int(m_y), int(s_r), B, T, K,
                                                N, po, workspace.data_ptr(), workspace.numel(),
                                                _stream(stream))
    if rc:
        _check("ip_linear_residual_i8", rc)
    return out


def swish_params_from_scales(S_z: float, S_y: float) -> tuple[int, int, int, int]:
    """Integer constants (q_c, q_one, m, s) of the minimax Swish for an int8
    input on grid S_z and an int8 output on grid S_y (Eqs. 12-13)."""
    prm = SwishParams()
    _check("ip_swish_params_from_scales",
           load().ip_swish_params_from_scales(S_z, S_y, ctypes.byref(prm)))
    return prm.q_c, prm.q_one, prm.m, prm.s


def linear_swish_i8(x, w, bias, m, s, swish: tuple[int, int, int, int], *, out=None,
                    workspace=None, stream=None):
    """Feed-forward projection with the fused minimax Swish: x int8 [B, T, K],
    w int8 [N, K], bias int32 [N] or None, m, s int32 [N] (onto the Swish
    input grid), swish = (q_c, q_one, m, s).  Returns int8 [B, T, N]."""
    import torch
    N, K = w.shape
    B, T, _ = x.shape
    if out is None:
        out = torch.empty((B, T, N), dtype=torch.int8, device=w.device)
    if workspace is None:
        workspace = torch.zeros(256, dtype=torch.uint8, device=w.device)
    px, pw, pb, pm, ps, po = _linear_ptrs(x, (B, T, K), w, bias, m, s, out, (B, T, N))
    rc = (_lib or load()).ip_linear_swish_i8(px, pw, pb, pm, ps, SwishParams(*swish), B, T, K, N, po,
                                             workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc:
        _check("ip_linear_swish_i8", rc)
    return out


@dataclass(frozen=True)
class NormConstants:
    eps_c: int
    M: "np.ndarray"     # int32 [d]
    B: "np.ndarray"     # int64 [d]
    E: "np.ndarray"     # int32 [d]


def layernorm_constants(s_x: float, gamma, beta, s_y: float, eps: float = 1e-5) -> NormConstants:
    """Offline constants of the integer LayerNorm (host, float64)."""
    import numpy as np
    g = np.ascontiguousarray(gamma, dtype=np.float64)
    b = np.ascontiguousarray(beta, dtype=np.float64)
    d = g.size
    M = np.empty(d, np.int32)
    B = np.empty(d, np.int64)
    E = np.empty(d, np.int32)
    ec = ctypes.c_longlong()
    _check("ip_layernorm_constants", load().ip_layernorm_constants(
        s_x, g.ctypes.data, b.ctypes.data, d, s_y, eps, ctypes.byref(ec), M.ctypes.data,
        B.ctypes.data, E.ctypes.data))
    return NormConstants(ec.value, M, B, E)


def layernorm_i8(x, M, B, E, eps_c: int, *, out=None, workspace=None, stream=None):
    """Integer LayerNorm over the last axis of int8 x (CUDA, d in {512, 1024,
    1536, 2048}); M int32, B int64, E int32 [d] CUDA tensors.  Returns int8
    like x.  Asynchronous on `stream`."""
    import torch
    d = x.shape[-1]
    rows = x.numel() // d if d else 0
    if out is None:
        out = torch.empty_like(x)
    if workspace is None:
        workspace = torch.zeros(256, dtype=torch.uint8, device=x.device)
    px, pM, pB, pE, po = _ptrs(torch.Tensor, [
        (x, "x", torch.int8, x.shape), (M, "M", torch.int32, (d,)), (B, "B", torch.int64, (d,)),
        (E, "E", torch.int32, (d,)), (out, "out", torch.int8, x.shape)])
    rc = (_lib or load()).ip_layernorm_i8(px, rows, d, int(eps_c), pM, pB, pE, po, workspace.data_ptr(),
                                          workspace.numel(), _stream(stream))
    if rc:
        _check("ip_layernorm_i8", rc)
    return out


def residual_params(s_x: float, s_y: float, s_z: float, alpha: float = 1.0):
    """(m_x, m_y, s) of z = x + alpha y onto S_z (Eqs. 1-4)."""
    a, b, s = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check("ip_residual_params", load().ip_residual_params(s_x, s_y, s_z, alpha, ctypes.byref(a),
                                                          ctypes.byref(b), ctypes.byref(s)))
    return a.value, b.value, s.value


def residual_i8(x, y, m_x: int, m_y: int, s: int, *, out=None, stream=None):
    """Residual addition of two int8 CUDA tensors of one shape."""
    import torch
    if out is None:
        out = torch.empty_like(x)
    n = x.numel()
    px, py, po = _ptrs(torch.Tensor, [(x, "x", torch.int8, x.shape), (y, "y", torch.int8, x.shape),
                                      (out, "out", torch.int8, x.shape)])
    rc = (_lib or load()).ip_residual_i8(px, py, n, m_x, m_y, s, po, _stream(stream))
    if rc:
        _check("ip_residual_i8", rc)
    return out


def glu_params(s_a: float, s_b: float, s_y: float) -> tuple[int, int, int, int]:
    """(q_c, q_one, m, s) of GLU(a, b) = a sigma(b) (Eq. 5, minimax tanh)."""
    prm = SwishParams()
    _check("ip_glu_params", load().ip_glu_params(s_a, s_b, s_y, ctypes.byref(prm)))
    return prm.q_c, prm.q_one, prm.m, prm.s


def linear_glu_i8(x, w_interleaved, bias, m, s, glu: tuple[int, int, int, int], *, out=None,
                  workspace=None, stream=None):
    """Pointwise convolution with the GLU fused: x int8 [B, T, K]; w int8 [N, K]
    with rows (a_c, b_c) interleaved; bias, m, s int32 [N]; returns int8
    [B, T, N/2]."""
    import torch
    N, K = w_interleaved.shape
    B, T, _ = x.shape
    if out is None:
        out = torch.empty((B, T, N // 2), dtype=torch.int8, device=x.device)
    if workspace is None:
        workspace = torch.zeros(256, dtype=torch.uint8, device=x.device)
    px, pw, pb, pm, ps, po = _linear_ptrs(x, (B, T, K), w_interleaved, bias, m, s, out, (B, T, N // 2))
    rc = (_lib or load()).ip_linear_glu_i8(px, pw, pb, pm, ps, SwishParams(*glu), B, T, K, N, po,
                                           workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc:
        _check("ip_linear_glu_i8", rc)
    return out


def swish16_params(s_z: float, s_y: float) -> tuple[int, int, int, int]:
    """(q_c, q_one, m, s) of the Swish of an INT16 input grid."""
    prm = Swish16Params()
    _check("ip_swish16_params_from_scales",
           load().ip_swish16_params_from_scales(s_z, s_y, ctypes.byref(prm)))
    return prm.q_c, prm.q_one, prm.m, prm.s


def dwconv_swish_i8(x, w, bias, m, s, sw16: tuple[int, int, int, int], *, out=None,
                    workspace=None, stream=None):
    """Depthwise convolution over time (folded BatchNorm, INT16) + Swish:
    x int8 [B, T, C]; w int8 [C, K]; bias, m, s int32 [C]; returns int8
    [B, T, C]."""
    import torch
    B, T, C = x.shape
    K = w.shape[1]
    if out is None:
        out = torch.empty_like(x)
    if workspace is None:
        workspace = torch.zeros(256, dtype=torch.uint8, device=x.device)
    px, pw, pb, pm, ps, po = _ptrs(torch.Tensor, [
        (x, "x", torch.int8, (B, T, C)), (w, "w", torch.int8, (C, K)), (bias, "bias", torch.int32, (C,)),
        (m, "m", torch.int32, (C,)), (s, "s", torch.int32, (C,)), (out, "out", torch.int8, (B, T, C))])
    rc = (_lib or load()).ip_dwconv_swish_i8(px, B, T, C, pw, K, pb, pm, ps, Swish16Params(*sw16), po,
                                             workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc:
        _check("ip_dwconv_swish_i8", rc)
    return out


# ------------------------------------------------------- run-time scales
#
# A decoder's single-token calls are shorter on the GPU than in Python (2 us for a 1024 x 4096
# product), so a call with its usual arguments first goes to its short form in ip_torch.cpp,
# which makes the same checks natively; everything else and every error is left to the forms here.
# (On a Grace core, us a call over ctypes / natively: quantize_rows_i8 15 / 4.4, linear_scaled_i8
# 19 / 3.7, kv4_append 15 / 2.1, kv4_attention 21 / 3.5, kv4_read 21 / 4.7.)

class _Unbound:
    """Stands for the short forms until the library is loaded."""

    @staticmethod
    def quantize_rows(*args):
        return None

    linear_scaled = kv4_append = kv4_read = kv4_attention = quantize_rows
    quantize_fp4 = linear_fp4 = rmsnorm_i8 = rmsnorm_fp4 = dequantize_i8 = dequantize_fp4 = token_logprobs = quantize_rows


_short = _Unbound


def _bind_short(lib):
    """The short forms, bound to the library; none without torch (the C entry points need none).  What they
    return is what the general forms do; new outputs of up to 1 MB a call in all share one storage."""
    path = _build.torch_extension()
    if path is None:
        return _Unbound
    import importlib.util
    import torch  # noqa: F401 - its libraries have to be there
    spec = importlib.util.spec_from_file_location("ip_torch", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    mod.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.ip_quantize_rows_i8, lib.ip_linear_scaled_i8, lib.ip_kv4_append, lib.ip_kv4_read, lib.ip_kv4_attention,
        lib.ip_quantize_fp4, lib.ip_linear_fp4, lib.ip_rmsnorm_i8, lib.ip_rmsnorm_fp4, lib.ip_dequantize_i8,
        lib.ip_dequantize_fp4, lib.ip_token_logprobs)))
    return mod


def _bound_short(lib):
    try:
        return _bind_short(lib)
    except Exception as exc:  # noqa: BLE001 - reported with context
        warnings.warn(f"cannot load the native short forms: {exc}; the calls take their general forms",
                      RuntimeWarning, stacklevel=3)
        return _Unbound


class _Pending:
    """Stands for the short forms from the library's loading to the first call that may take them:
    they need torch, which the calls without tensors do not."""

    def __init__(self, lib):
        self._lib, self._forms = lib, None

    def __getattr__(self, name):
        global _short
        if self._forms is None:
            self._forms = _bound_short(self._lib)
            if _short is self:
                _short = self._forms
        return getattr(self._forms, name)


def _dtype_code(dtype, name="dtype"):
    import torch
    code = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}.get(dtype)
    if code is None:
        raise TypeError(f"{name} must be torch.float32, float16 or bfloat16, got {dtype}")
    return code


def _need(t, name, dtype=None, shape=None, device=None):
    """Checks a CUDA tensor's type, shape and device; its strides are the caller's."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    return t


def _dense(t, name, dtype, shape, device):
    if not _need(t, name, dtype, shape, device).is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _as_rows(t, name):
    """(rows, columns, row stride) of the last axis's rows; the leading axes must be
    walked with one stride (a matrix, a contiguous tensor, column slices of either)."""
    d = t.shape[-1] if t.dim() else 0
    if t.dim() < 1 or d < 1:
        raise ValueError(f"{name} needs a last axis of at least one element")
    if t.stride(-1) != 1 and d > 1:
        raise ValueError(f"{name}'s last axis must be contiguous")
    rows, stride = 1, None
    for size, st in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size != 1 and rows:
            if stride is None:
                stride = st
            elif st != stride * rows:
                raise ValueError(f"{name}'s rows must follow one another with one stride")
        rows *= size
    if rows < 2:
        stride = -(-d // 16) * 16      # one row (or none): any stride does
    if stride < d:
        raise ValueError(f"{name}'s rows must not overlap")
    return rows, d, stride


class _On:
    """Makes `device` and `stream` (None: the device's current one) current, so that what
    a call allocates belongs to the stream that uses it, and gives the raw handle."""

    def __init__(self, device, stream):
        import torch
        if stream is not None and stream.device != device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
        self.ctx = torch.cuda.stream(stream) if stream is not None else (
            torch.cuda.device(device) if device.index != torch._C._cuda_getDevice() else None)

    def __enter__(self):
        import torch
        if self.ctx is not None:
            self.ctx.__enter__()
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)


def _status_space(workspace, device, size=256):
    """Pointer and bytes of the caller's workspace, or of a fresh zeroed one."""
    import torch
    if workspace is None:
        workspace = torch.zeros(size, dtype=torch.uint8, device=device)
    else:
        _dense(workspace, "workspace", torch.uint8, (workspace.numel(),), device)
    return workspace, workspace.data_ptr(), workspace.numel()


def quantize_rows_i8(x, *, q=None, scale=None, stream=None):
    """Rows (the last axis) of a float32, float16 or bfloat16 CUDA tensor to int8 with a
    scale each: scale = amax / 127 (float32), q = 127 x / amax to the nearest integer,
    ties to even.  A row of zeros gives scale 0; one with a NaN or an infinity the scale
    NaN and q 0.  Returns (q, scale): int8 of x's shape and float32 of x.shape[:-1].  A
    new q has rows of a multiple of 16 bytes, as linear_scaled_i8 reads them, so it
    is a view of them where 16 does not divide the last axis.  Asynchronous on
    `stream` (default: torch's current stream)."""
    if stream is None:
        r = _short.quantize_rows(x, q, scale)
        if r is not None:
            return r if r.__class__ is tuple else _check("ip_quantize_rows_i8", r)
    import torch
    code = _dtype_code(_need(x, "x").dtype, "x")
    rows, d, ldx = _as_rows(x, "x")
    lib = _lib or load()
    with _On(x.device, stream) as handle:
        if q is None:
            ldq = -(-d // 16) * 16
            q = torch.empty((*x.shape[:-1], ldq), dtype=torch.int8, device=x.device)
            q = q if ldq == d else q[..., :d]
        else:
            ldq = _as_rows(_need(q, "q", torch.int8, x.shape, x.device), "q")[2]
        if scale is None:
            scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
        rc = lib.ip_quantize_rows_i8(
            x.data_ptr(), code, rows, d, ldx, q.data_ptr(), ldq,
            _dense(scale, "scale", torch.float32, x.shape[:-1], x.device), handle)
    if rc:
        _check("ip_quantize_rows_i8", rc)
    return q, scale


def linear_scaled_i8(x, sx, w, sw, bias=None, *, act: int = ACT_NONE, dtype=None, out=None,
                     workspace=None, stream=None):
    """Int8 matrix product with a scale per token and per channel:
    out[..., n] = act(sx sw[n] sum_k x[..., k] w[n, k] + bias[n]), the sum exact, the rest
    in float32.  x: int8 [..., K], sx: float32 [...] (quantize_rows_i8); w: int8 [N, K], sw:
    float32 [N]; bias: float32 [N] or None; act: ACT_NONE or ACT_SWISH; all CUDA tensors.
    K and N may be any size; the rows of x and w start on multiples of 16 bytes.
    Returns out: [..., N] of `dtype` (bfloat16 unless out gives it).  Asynchronous on
    `stream` (default: torch's current stream)."""
    if stream is None:
        r = _short.linear_scaled(x, sx, w, sw, bias, act, dtype, out, workspace)
        if r is not None:
            return r if r.__class__ is not int else _check("ip_linear_scaled_i8", r)
    import torch
    rows, K, ldx = _as_rows(_need(x, "x", torch.int8), "x")
    if _need(w, "w", torch.int8, None, x.device).dim() != 2 or w.shape[1] != K:
        raise ValueError(f"w must have shape (N, {K}), got {tuple(w.shape)}")
    N, _, ldw = _as_rows(w, "w")
    shape = (*x.shape[:-1], N)
    if out is not None:
        dtype = out.dtype if dtype is None else dtype
        ldy = _as_rows(_need(out, "out", dtype, shape, x.device), "out")[2]
    else:
        dtype, ldy = dtype or torch.bfloat16, N
    code = _dtype_code(dtype)
    psx = _dense(sx, "sx", torch.float32, x.shape[:-1], x.device)
    psw = _dense(sw, "sw", torch.float32, (N,), x.device)
    pb = None if bias is None else _dense(bias, "bias", torch.float32, (N,), x.device)
    lib = _lib or load()
    with _On(x.device, stream) as handle:
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=x.device)
        workspace, ws, wsb = _status_space(workspace, x.device)
        rc = lib.ip_linear_scaled_i8(
            x.data_ptr(), ldx, psx, w.data_ptr(), ldw, psw, pb, int(act), rows, K, N, out.data_ptr(),
            ldy, code, ws, wsb, handle)
    if rc:
        _check("ip_linear_scaled_i8", rc)
    return out


# ------------------------------------------------------- 4-bit rows, norm

def fp4_block_shape(rows: int, d: int) -> tuple[int, int, int]:
    """Shape of the block scales of `rows` 4-bit rows of d elements: uint8 [ceil(rows / 128),
    ceil(d / 64), 512], the scale of row m and block b (16 elements) at [m // 128, b // 4,
    16 (m % 32) + 4 (m % 128 // 32) + b % 4]."""
    return -(-rows // 128), -(-d // 64), 512


def _fp4_out(q, blocks, scale, lead, rows, d, dev):
    """New or checked (q, its row stride, blocks, scale) of 4-bit rows."""
    import torch
    n = -(-d // 2)
    if q is None:
        ldq = -(-n // 16) * 16
        q = torch.empty((*lead, ldq), dtype=torch.uint8, device=dev)
        q = q if ldq == n else q[..., :n]
    else:
        ldq = _as_rows(_need(q, "q", torch.uint8, (*lead, n), dev), "q")[2]
    if blocks is None:
        blocks = torch.empty(fp4_block_shape(rows, d), dtype=torch.uint8, device=dev)
    _dense(blocks, "blocks", torch.uint8, fp4_block_shape(rows, d), dev)
    if scale is None:
        scale = torch.empty(lead, dtype=torch.float32, device=dev)
    _dense(scale, "scale", torch.float32, lead, dev)
    return q, ldq, blocks, scale


def quantize_fp4(x, *, q=None, blocks=None, scale=None, stream=None):
    """Rows (the last axis, d elements) of a float32, float16 or bfloat16 CUDA tensor to 4-bit
    floating point: e2m1 codes, an e4m3 scale s for each 16 of them, a float32 scale r a row, an
    element being code s r.  r is the least power of two with amax <= 2688 r, s and the codes
    are rounded to nearest, ties to even, exactly.  A row of zeros gives scale 0; one with a
    NaN or an infinity the scale NaN and codes 0.  Returns (q, blocks, scale): uint8
    [..., ceil(d / 2)] (the first code in the low nibble; a new q has rows of a multiple of 16
    bytes, as linear_fp4 reads them, so it may be a view of them), uint8
    fp4_block_shape(rows, d) and float32 of x.shape[:-1].  New outputs of up to 1 MB in all may share one
    storage: clone one that is to be kept, saved or resized by itself.
    Asynchronous on `stream` (default: torch's current stream)."""
    if stream is None:
        r = _short.quantize_fp4(x, q, blocks, scale)
        if r is not None:
            return r if r.__class__ is not int else _check("ip_quantize_fp4", r)
    code = _dtype_code(_need(x, "x").dtype, "x")
    rows, d, ldx = _as_rows(x, "x")
    lib = _lib or load()
    with _On(x.device, stream) as handle:
        q, ldq, blocks, scale = _fp4_out(q, blocks, scale, x.shape[:-1], rows, d, x.device)
        rc = lib.ip_quantize_fp4(x.data_ptr(), code, rows, d, ldx, q.data_ptr(), ldq, blocks.data_ptr(),
                                 scale.data_ptr(), handle)
    if rc:
        _check("ip_quantize_fp4", rc)
    return q, blocks, scale


def _norm_in(x, weight, residual, out):
    """What the two norms check of their inputs: the type's code, rows, d, the row strides of x,
    residual and the sum's tensor (None: to be made)."""
    code = _dtype_code(_need(x, "x").dtype, "x")
    rows, d, ldx = _as_rows(x, "x")
    _dense(weight, "weight", x.dtype, (d,), x.device)
    ldr = lds = 0
    if residual is not None:
        ldr = _as_rows(_need(residual, "residual", x.dtype, x.shape, x.device), "residual")[2]
        lds = d if out is None else _as_rows(_need(out, "out", x.dtype, x.shape, x.device), "out")[2]
    elif out is not None:
        raise ValueError("out is the sum with a residual, and there is none")
    return code, rows, d, ldx, ldr, lds


def rmsnorm_i8(x, weight, residual=None, *, eps: float = 1e-5, out=None, q=None, scale=None, stream=None):
    """Root-mean-square norm over the last axis (d elements) with the residual's addition,
    its rows in int8: h = x + residual (rounded to x's type), then h weight / sqrt(mean(h^2) + eps)
    as quantize_rows_i8 rounds rows (the row's factor leaves the codes as they are: they are
    exactly those of h weight).  x, residual: float32, float16 or bfloat16 [..., d] CUDA
    tensors; weight: x's type [d].  Returns (q, scale, h): int8 of x's shape (a new q has rows of
    a multiple of 16 bytes), float32 of x.shape[:-1], and h of x's type, None without a residual; new ones may share one
    storage (quantize_fp4).  out: where h goes, which may be x or residual itself.
    Asynchronous on `stream`."""
    if stream is None:
        r = _short.rmsnorm_i8(x, weight, residual, eps, out, q, scale)
        if r is not None:
            return r if r.__class__ is not int else _check("ip_rmsnorm_i8", r)
    import torch
    code, rows, d, ldx, ldr, lds = _norm_in(x, weight, residual, out)
    dev, lib = x.device, _lib or load()
    with _On(dev, stream) as handle:
        if q is None:
            ldq = -(-d // 16) * 16
            q = torch.empty((*x.shape[:-1], ldq), dtype=torch.int8, device=dev)
            q = q if ldq == d else q[..., :d]
        else:
            ldq = _as_rows(_need(q, "q", torch.int8, x.shape, dev), "q")[2]
        if scale is None:
            scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=dev)
        _dense(scale, "scale", torch.float32, x.shape[:-1], dev)
        if residual is not None and out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=dev)
        rc = lib.ip_rmsnorm_i8(x.data_ptr(), ldx, None if residual is None else residual.data_ptr(), ldr,
                               weight.data_ptr(), eps, code, rows, d, None if out is None else out.data_ptr(), lds,
                               q.data_ptr(), ldq, scale.data_ptr(), handle)
    if rc:
        _check("ip_rmsnorm_i8", rc)
    return q, scale, out


def rmsnorm_fp4(x, weight, residual=None, *, eps: float = 1e-5, out=None, q=None, blocks=None, scale=None,
                stream=None):
    """rmsnorm_i8 with 4-bit rows (quantize_fp4): returns (q, blocks, scale, h)."""
    if stream is None:
        r = _short.rmsnorm_fp4(x, weight, residual, eps, out, q, blocks, scale)
        if r is not None:
            return r if r.__class__ is not int else _check("ip_rmsnorm_fp4", r)
    import torch
    code, rows, d, ldx, ldr, lds = _norm_in(x, weight, residual, out)
    dev, lib = x.device, _lib or load()
    with _On(dev, stream) as handle:
        q, ldq, blocks, scale = _fp4_out(q, blocks, scale, x.shape[:-1], rows, d, dev)
        if residual is not None and out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=dev)
        rc = lib.ip_rmsnorm_fp4(x.data_ptr(), ldx, None if residual is None else residual.data_ptr(), ldr,
                                weight.data_ptr(), eps, code, rows, d, None if out is None else out.data_ptr(), lds,
                                q.data_ptr(), ldq, blocks.data_ptr(), scale.data_ptr(), handle)
    if rc:
        _check("ip_rmsnorm_fp4", rc)
    return q, blocks, scale, out


def _values_out(out, dtype, shape, dev):
    """(out or None, its type, its row stride) of a call that writes values of rows."""
    import torch
    if out is None:
        return dtype or torch.bfloat16, shape[-1]
    dtype = out.dtype if dtype is None else dtype
    return dtype, _as_rows(_need(out, "out", dtype, shape, dev), "out")[2]


def dequantize_i8(q, scale, *, dtype=None, out=None, stream=None):
    """The values of int8 rows (quantize_rows_i8, rmsnorm_i8): q scale, rounded once to `dtype`
    (bfloat16 unless out gives it).  q: int8 [..., d], scale: float32 [...], CUDA tensors.
    Asynchronous on `stream`."""
    if stream is None:
        r = _short.dequantize_i8(q, scale, dtype, out)
        if r is not None:
            return r if r.__class__ is not int else _check("ip_dequantize_i8", r)
    import torch
    rows, d, ldq = _as_rows(_need(q, "q", torch.int8), "q")
    ps = _dense(scale, "scale", torch.float32, q.shape[:-1], q.device)
    dtype, ldy = _values_out(out, dtype, q.shape, q.device)
    code, lib = _dtype_code(dtype), _lib or load()
    with _On(q.device, stream) as handle:
        if out is None:
            out = torch.empty(q.shape, dtype=dtype, device=q.device)
        rc = lib.ip_dequantize_i8(q.data_ptr(), ldq, ps, rows, d, out.data_ptr(), ldy, code, handle)
    if rc:
        _check("ip_dequantize_i8", rc)
    return out


def _fp4_in(q, blocks, scale, names, d=None):
    """Checked (rows, d, row stride) of 4-bit rows; d: elements a row (default: two a byte)."""
    import torch
    rows, n, ldq = _as_rows(_need(q, names[0], torch.uint8), names[0])
    d = 2 * n if d is None else d
    if -(-d // 2) != n:
        raise ValueError(f"{names[0]}'s rows of {n} bytes do not hold {d} elements")
    _dense(blocks, names[1], torch.uint8, fp4_block_shape(rows, d), q.device)
    _dense(scale, names[2], torch.float32, q.shape[:-1], q.device)
    return rows, d, ldq


def dequantize_fp4(q, blocks, scale, d=None, *, dtype=None, out=None, stream=None):
    """The values of 4-bit rows (quantize_fp4, rmsnorm_fp4), code s r in float32, rounded once to
    `dtype` (bfloat16 unless out gives it): [..., d], d twice q's bytes unless given.
    Asynchronous on `stream`."""
    if stream is None:
        r = _short.dequantize_fp4(q, blocks, scale, d, dtype, out)
        if r is not None:
            return r if r.__class__ is not int else _check("ip_dequantize_fp4", r)
    import torch
    rows, d, ldq = _fp4_in(q, blocks, scale, ("q", "blocks", "scale"), d)
    shape = (*q.shape[:-1], d)
    dtype, ldy = _values_out(out, dtype, shape, q.device)
    code, lib = _dtype_code(dtype), _lib or load()
    with _On(q.device, stream) as handle:
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=q.device)
        rc = lib.ip_dequantize_fp4(q.data_ptr(), ldq, blocks.data_ptr(), scale.data_ptr(), rows, d, out.data_ptr(),
                                   ldy, code, handle)
    if rc:
        _check("ip_dequantize_fp4", rc)
    return out


def linear_fp4(x, x_blocks, sx, w, w_blocks, sw, bias=None, *, act: int = ACT_NONE, dtype=None, out=None,
               workspace=None, stream=None):
    """Product of 4-bit rows (quantize_fp4, rmsnorm_fp4) on the block-scaled tensor cores (a few rows go by
    ordinary lanes):
    out[..., n] = act(sum of the products of the values of x's and w's rows + bias[n]), codes and
    scales exact, sums in float32.  Block scales are from 0 on (bytes 0 to 0x7e: the tensor cores'
    have no sign), as the writing calls give them.  x: uint8 [..., ceil(K / 2)] with its block scales and sx:
    float32 [...]; w: uint8 [N, ceil(K / 2)], w_blocks, sw: float32 [N] (quantize_fp4 of the weights); bias: float32 [N]
    or None; act: ACT_NONE or ACT_SWISH; all CUDA tensors.  K and N may be any size; the rows of x
    and w start on multiples of 16 bytes.  Returns out: [..., N] of `dtype` (bfloat16 unless out
    gives it).  Asynchronous on `stream` (default: torch's current stream)."""
    if stream is None:
        r = _short.linear_fp4(x, x_blocks, sx, w, w_blocks, sw, bias, act, dtype, out, workspace)
        if r is not None:
            return r if r.__class__ is not int else _check("ip_linear_fp4", r)
    import torch
    rows, K, ldx = _fp4_in(x, x_blocks, sx, ("x", "x_blocks", "sx"))
    if _need(w, "w", torch.uint8, None, x.device).dim() != 2 or w.shape[1] != x.shape[-1]:
        raise ValueError(f"w must have shape (N, {x.shape[-1]}), got {tuple(w.shape)}")
    N, _, ldw = _fp4_in(w, w_blocks, sw, ("w", "w_blocks", "sw"))
    shape = (*x.shape[:-1], N)
    dtype, ldy = _values_out(out, dtype, shape, x.device)
    code = _dtype_code(dtype)
    pb = None if bias is None else _dense(bias, "bias", torch.float32, (N,), x.device)
    lib = _lib or load()
    with _On(x.device, stream) as handle:
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=x.device)
        workspace, ws, wsb = _status_space(workspace, x.device)
        rc = lib.ip_linear_fp4(x.data_ptr(), ldx, x_blocks.data_ptr(), sx.data_ptr(), w.data_ptr(), ldw,
                               w_blocks.data_ptr(), sw.data_ptr(), pb, int(act), rows, K, N, out.data_ptr(), ldy, code,
                               ws, wsb, handle)
    if rc:
        _check("ip_linear_fp4", rc)
    return out


def kv4_page_bytes(page: int, dh: int = IP_DH) -> int:
    """Bytes of one page of one head of a 4-bit cache (144 a token)."""
    n = load().ip_kv4_page_bytes(page, dh)
    if n == 0:
        raise IpError("ip_kv4_page_bytes", -4, "pages of 16, 32 or 64 tokens, heads of 128")
    return n


def kv4_cache(n_pages: int, heads: int, page: int = 64, device="cuda"):
    """A cache of n_pages pages of `page` tokens: uint8 [n_pages, heads, 144 page]."""
    import torch
    return torch.zeros((n_pages, heads, kv4_page_bytes(page)), dtype=torch.uint8, device=device)


def _strides(t, name):
    st = t.stride()
    if st[3] != 1:
        raise ValueError(f"{name}'s channels must be contiguous")
    return _Stride3(*st[:3])


_Stride3 = ctypes.c_longlong * 3


def _kv4_args(x, cache, table, workspace, lens, names):
    """Checks what the calls on a cache share: x [B, T, H, 128] (or B, for a call without
    one), the cache, its table and the int32 [B] tensors lens; returns B, the cache's
    (pages, heads, page size, table width) and the pointers of lens."""
    import torch
    B = x if x.__class__ is int else x.shape[0]
    dev = _need(cache, "cache", torch.uint8).device
    if x is not B:
        _need(x, names[0], None, None, dev)
    if cache.dim() != 3 or cache.shape[2] % 144 or not cache.is_contiguous():
        raise ValueError("cache must be a contiguous uint8 tensor [pages, heads, 144 page]")
    if _need(table, "page_table", torch.int32, None, dev).dim() != 2 or table.shape[0] != B:
        raise ValueError(f"page_table must have shape ({B}, pages), got {tuple(table.shape)}")
    if not table.is_contiguous():
        raise ValueError("page_table must be contiguous")
    ptrs = [None if i is None else _dense(i, n, torch.int32, (B,), dev) for i, n in zip(lens, names[1:])]
    if workspace is not None:
        _dense(workspace, "workspace", torch.uint8, (workspace.numel(),), dev)
    load()
    return B, (cache.shape[0], cache.shape[1], cache.shape[2] // 144, table.shape[1]), ptrs


def kv4_append(k, v, start, page_table, cache, *, count=None, workspace=None, stream=None):
    """Quantises k, v (float32, float16 or bfloat16 [B, T, H, 128], any strides with
    contiguous channels) to 4 bits into the cache: rows t < count[b] (int32 [B]; None:
    T) go to the positions start[b] + t (int32 [B]) of sequence b, whose pages are
    page_table[b] (int32 [B, pages]).  No two rows may meet in one place.  All CUDA
    tensors; asynchronous on `stream`.  Pages or positions that do not exist are
    skipped and reported by status(workspace)."""
    if stream is None:
        rc = _short.kv4_append(k, v, start, page_table, cache, count, workspace)
        if rc is not None:
            return _check("ip_kv4_append", rc) if rc else cache
    code = _dtype_code(_need(k, "k").dtype, "k")
    if k.dim() != 4 or k.shape[3] != IP_DH:
        raise ValueError(f"k must have shape (B, T, H, 128), got {tuple(k.shape)}")
    _, T, H, dh = k.shape
    _need(v, "v", k.dtype, k.shape, k.device)
    if start is None:
        raise TypeError("start must be a CUDA tensor")
    B, (n_pages, heads, page, width), (pst, pct) = _kv4_args(k, cache, page_table, workspace, (start, count),
                                                             ("k", "start", "count"))
    if heads != H:
        raise ValueError(f"cache holds {heads} heads, not {H}")
    kst, vst = _strides(k, "k"), _strides(v, "v")
    with _On(k.device, stream) as handle:
        workspace, ws, wsb = _status_space(workspace, k.device)
        rc = _lib.ip_kv4_append(k.data_ptr(), v.data_ptr(), code, kst, vst, pst, pct, B, T, H, dh,
                                page_table.data_ptr(), width, cache.data_ptr(), n_pages, page, ws, wsb, handle)
    if rc:
        _check("ip_kv4_append", rc)
    return cache


def kv4_read(cache, start, page_table, T: int, *, count=None, dtype=None, out=None, workspace=None,
             stream=None):
    """Positions start[b] .. start[b] + T - 1 of every sequence back as real values:
    (k, v), each [B, T, H, 128] of `dtype` (bfloat16 unless out gives it), zeros in rows
    t >= count[b].  out: such a pair, contiguous.  Arguments as kv4_append."""
    if out is None and stream is None:
        r = _short.kv4_read(cache, start, page_table, T, count, dtype, workspace)
        if r is not None:
            return r if r.__class__ is tuple else _check("ip_kv4_read", r)
    import torch
    B, (n_pages, H, page, width), (pst, pct) = _kv4_args(
        _need(start, "start").numel(), cache, page_table, workspace, (start, count), ("", "start", "count"))
    if T < 0:
        raise ValueError(f"T must not be negative, got {T}")
    dev, shape = cache.device, (B, T, H, IP_DH)
    dtype = dtype or (torch.bfloat16 if out is None else out[0].dtype)
    code = _dtype_code(dtype)
    with _On(dev, stream) as handle:
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=dev), torch.empty(shape, dtype=dtype, device=dev)
        pk, pv = _dense(out[0], "out[0]", dtype, shape, dev), _dense(out[1], "out[1]", dtype, shape, dev)
        workspace, ws, wsb = _status_space(workspace, dev)
        rc = _lib.ip_kv4_read(cache.data_ptr(), n_pages, page, page_table.data_ptr(), width, pst, pct, B, T, H,
                              IP_DH, pk, pv, code, ws, wsb, handle)
    if rc:
        _check("ip_kv4_read", rc)
    return out


def kv4_attention_workspace_bytes(B: int, T: int, heads: int, cache_heads: int, max_len: int) -> int:
    """Bytes of workspace of kv4_attention for these sizes."""
    n = load().ip_kv4_attention_workspace_bytes(B, T, heads, cache_heads, max_len)
    if n == 0:
        raise IpError("ip_kv4_attention_workspace_bytes", -2, "invalid shape")
    return n


def kv4_attention(q, lengths, page_table, cache, *, count=None, causal: bool = True, scale=None,
                  max_len=None, out=None, workspace=None, stream=None):
    """Attention of q (float16 or bfloat16 [B, T, H, 128], any strides with contiguous
    channels) over a 4-bit cache of Hkv heads, H a multiple of Hkv: softmax(scale q K^T) V
    with scale 1/sqrt(128) unless given.  lengths (int32 [B]): cached tokens, with this
    call's own; count (int32 [B], None: T): query tokens, which causal makes the last
    ones of the sequence; causal=False lets every query see all cached tokens.  A query that
    sees none, and rows past count, give 0.  In float32, but for the weights of the output
    product, which are rounded to float16.  max_len: a host bound of lengths (default: what
    the table can hold); a close one splits the work better.  Returns [B, T, H, 128] of
    q's type.  workspace: a zero-filled uint8 tensor of kv4_attention_workspace_bytes(B, T,
    H, Hkv, max_len).  Asynchronous on `stream`."""
    if stream is None:
        r = _short.kv4_attention(q, lengths, page_table, cache, count, causal, scale, max_len, out, workspace)
        if r is not None:
            return r if r.__class__ is not int else _check("ip_kv4_attention", r)
    import torch
    code = _dtype_code(_need(q, "q").dtype, "q")
    if code == 0:
        raise TypeError(f"q must be float16 or bfloat16, got {q.dtype}")
    if q.dim() != 4 or q.shape[3] != IP_DH:
        raise ValueError(f"q must have shape (B, T, H, 128), got {tuple(q.shape)}")
    _, T, H, dh = q.shape
    if lengths is None:
        raise TypeError("lengths must be a CUDA tensor")
    B, (n_pages, Hkv, page, width), (pln, pct) = _kv4_args(q, cache, page_table, workspace, (lengths, count),
                                                           ("q", "lengths", "count"))
    if max_len is None:
        max_len = width * page
    qst, dev = _strides(q, "q"), q.device
    size = 0 if workspace is not None else kv4_attention_workspace_bytes(B, T, H, Hkv, max_len)
    with _On(dev, stream) as handle:
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=dev)
        po = _dense(out, "out", q.dtype, q.shape, dev)
        workspace, ws, wsb = _status_space(workspace, dev, size)
        rc = _lib.ip_kv4_attention(q.data_ptr(), code, qst, pln, pct, 1 if causal else 0,
                                   dh ** -0.5 if scale is None else scale, B, T, H, Hkv, dh, max_len,
                                   page_table.data_ptr(), width, cache.data_ptr(), n_pages, page, po, ws, wsb, handle)
    if rc:
        _check("ip_kv4_attention", rc)
    return out


# ------------------------------------------------------- log probabilities

def token_logprobs_workspace_bytes(rows: int, V: int, top: int = 0) -> int:
    """Bytes of workspace of token_logprobs for these sizes."""
    n = load().ip_token_logprobs_workspace_bytes(rows, V, top)
    if n == 0:
        raise IpError("ip_token_logprobs_workspace_bytes", -2, "invalid shape")
    return n


def token_logprobs(logits, tokens=None, *, top: int = 0, scale: float = 1.0, out=None, workspace=None, stream=None):
    """Log probabilities of given tokens, entropy and the best tokens of each row of logits
    (float32, float16 or bfloat16 [..., V] CUDA tensor), of the distribution softmax(scale logits), in
    float32.  tokens: int32 or int64 [...], or None; one below 0 (padding) gives 0, one past
    V - 1 NaN.  top: how many of the best tokens to give, up to 32, the largest logit first, the
    lowest index first of equal ones.  scale: 1 / temperature.  Returns (logprob, entropy,
    top_logprob, top_token): float32 [...] (None without tokens), float32 [...], float32 and int32
    [..., top] (None for top = 0).  A row with a NaN or +inf, or of nothing but -inf, gives NaN and
    tokens -1.  New outputs may share one storage (quantize_fp4).  out: such a tuple, contiguous.  workspace: a uint8 tensor of
    token_logprobs_workspace_bytes(rows, V, top).  Asynchronous on `stream` (default: torch's
    current stream)."""
    if stream is None and out is None:
        r = _short.token_logprobs(logits, tokens, top, scale, workspace)
        if r is not None:
            return r if r.__class__ is tuple else _check("ip_token_logprobs", r)
    import torch
    code = _dtype_code(_need(logits, "logits").dtype, "logits")
    rows, V, ld = _as_rows(logits, "logits")
    dev, lead, wide = logits.device, logits.shape[:-1], 0
    if tokens is not None:
        wide = 1 if _need(tokens, "tokens").dtype == torch.int64 else 0
        _dense(tokens, "tokens", torch.int64 if wide else torch.int32, lead, dev)
    size = 0 if workspace is not None else token_logprobs_workspace_bytes(rows, V, top)
    f32, best = torch.float32, (*lead, top)
    with _On(dev, stream) as handle:
        if out is None:
            new = lambda shape, dtype, on: torch.empty(shape, dtype=dtype, device=dev) if on else None
            out = (new(lead, f32, tokens is not None), new(lead, f32, True), new(best, f32, top > 0),
                   new(best, torch.int32, top > 0))
        lp, ent, tlp, ttok = out
        ptrs = [_dense(t, f"out[{i}]", dtype, shape, dev) if on else None for i, (t, dtype, shape, on) in enumerate((
            (lp, f32, lead, tokens is not None), (ent, f32, lead, True), (tlp, f32, best, top > 0),
            (ttok, torch.int32, best, top > 0)))]
        workspace, ws, wsb = _status_space(workspace, dev, size)
        rc = (_lib or load()).ip_token_logprobs(
            logits.data_ptr(), code, rows, V, ld, None if tokens is None else tokens.data_ptr(), wide, scale, top,
            *ptrs, ws, wsb, handle)
    if rc:
        _check("ip_token_logprobs", rc)
    return out


def relpos_mhsa_i8_host(q, k, v, p, u, v_bias, consts: LayerConstants, lengths, out, arena,
                        stream=None, wait: bool = True):
    """Whole layer from host buffers (torch CPU tensors, ideally pinned):
    copies in, runs, copies the result into `out` and synchronises.  With
    wait=False the call only enqueues (ip_relpos_mhsa_i8_host_async): `out`
    is valid after the stream synchronises, and host_status() reports
    errors."""
    import torch
    B, H, T, dh = q.shape
    for name, t in (("q", q), ("k", k), ("v", v), ("p", p), ("u", u), ("v_bias", v_bias), ("out", out)):
        if t.is_cuda or t.dtype != torch.int8 or not t.is_contiguous():
            raise TypeError(f"{name} must be a contiguous int8 CPU tensor")
    lens = None
    if lengths is not None:
        if lengths.is_cuda or lengths.dtype != torch.int32 or tuple(lengths.shape) != (B,):
            raise TypeError("lengths must be an int32 [B] CPU tensor")
        lens = ctypes.c_void_p(lengths.data_ptr())
    sm = SoftmaxParams(*consts.softmax)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    fn = load().ip_relpos_mhsa_i8_host if wait else load().ip_relpos_mhsa_i8_host_async
    rc = fn(ptr(q), ptr(k), ptr(v), ptr(p), ptr(u), ptr(v_bias),
            _arr(consts.multipliers, ctypes.c_int32), _arr(consts.shifts, ctypes.c_int32),
            ctypes.byref(sm), lens, B, H, T, dh, ptr(out), ctypes.c_void_p(arena.data_ptr()),
            arena.numel(), _stream_handle(stream))
    _check("ip_relpos_mhsa_i8_host" if wait else "ip_relpos_mhsa_i8_host_async", rc)
    return out


def host_status(arena, B: int, H: int, T: int, dh: int = IP_DH, stream=None) -> int:
    """Synchronises `stream` and returns the status of the last asynchronous
    host-buffer call that used `arena` (0 = ok)."""
    return load().ip_relpos_mhsa_host_status(ctypes.c_void_p(arena.data_ptr()), B, H, T, dh,
                                             _stream_handle(stream))


__all__ = ["build", "load", "relpos_mhsa_i8", "relpos_mhsa_i8_host", "status", "workspace_bytes",
           "host_arena_bytes", "layer_constants", "LayerConstants", "dyadic_multiplier",
           "dyadic_pair", "isoftmax_params_from_scale", "set_timeout_cycles", "strerror",
           "int8_mma_peak_tops", "set_stall_injection", "set_split_mode", "linear_i8",
           "linear_constants", "ROWS", "HEADS", "linear_swish_i8", "swish_params_from_scales",
           "layernorm_i8", "layernorm_constants", "NormConstants", "residual_i8",
           "residual_params", "linear_glu_i8", "glu_params", "dwconv_swish_i8", "swish16_params",
           "host_status", "set_workspace", "int8_pipe_rates", "linear_residual_i8",
           "quantize_rows_i8", "linear_scaled_i8", "ACT_NONE", "ACT_SWISH",
           "kv4_page_bytes", "kv4_cache", "kv4_append", "kv4_read", "kv4_attention",
           "kv4_attention_workspace_bytes",
           "fp4_block_shape", "quantize_fp4", "linear_fp4", "dequantize_fp4", "dequantize_i8", "rmsnorm_i8", "rmsnorm_fp4",
           "token_logprobs", "token_logprobs_workspace_bytes",
           "IpError", "LibraryError", "EXPORTS"]
