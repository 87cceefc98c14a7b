"""ctypes binding over libgoom's C ABI (``include/goom.h``), same names as the C calls.

Marshalling only: every step of the computation runs in the HIP kernels.  PyTorch is
used for device memory and streams.  Tensors must be contiguous CUDA (ROCm) tensors on
the context's device; complex64 / complex128 tensors carry GOOMs (real = log-magnitude,
imag = 0 or pi).
"""
from __future__ import annotations

import ctypes as C
import math
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libgoom.so")
_lib = None

C64, C128 = 0, 1
ZERO_NEG_INF, ZERO_FLOOR = 0, 1
LMME_FAST, LMME_EXACT = 0, 1
RESET_ALWAYS, RESET_COLINEAR, RESET_NEVER = 1, 0, -1
AFFINE_TIME_INVARIANT = 1
REAL_F32, REAL_BF16, REAL_F16 = 16, 17, 18
ACTIVATIONS = {"none": 0, "silu": 1, "gelu": 2}
ROTARY_INTERLEAVED, ROTARY_BACK = 1, 2
NORM_KINDS = {"rms": 0, "layer": 1}

EXPORTS = [
    "goom_version", "goom_create", "goom_destroy", "goom_set_stream", "goom_last_error",
    "goom_status_name", "goom_probe_bandwidth", "goom_probe_matrix_unit", "goom_profile_enable", "goom_profile_count", "goom_profile_get", "goom_to_goom", "goom_from_goom", "goom_lmme", "goom_lmme_workspace_bytes",
    "goom_scan", "goom_scan_workspace_bytes", "goom_scan_static", "goom_reduce", "goom_reduce_workspace_bytes",
    "goom_scan_real", "goom_scan_real_workspace_bytes", "goom_reduce_real", "goom_reduce_real_workspace_bytes",
    "goom_scan_reset", "goom_scan_reset_workspace_bytes", "goom_scan_reset_tree", "goom_scan_reset_tree_workspace_bytes", "goom_lyapunov_spectrum",
    "goom_lyapunov_spectrum_per_step", "goom_lyapunov_spectrum_per_step_workspace_bytes",
    "goom_largest_lyapunov", "goom_largest_lyapunov_workspace_bytes",
    "goom_affine_scan", "goom_affine_scan_workspace_bytes", "goom_affine_scan_scaled",
    "goom_affine_scan_scaled_workspace_bytes", "goom_scaled_exp", "goom_log_add_exp",
    "goom_count_nonfinite", "goom_to_goom_backward", "goom_from_goom_backward", "goom_affine_scan_backward", "goom_affine_scan_backward_workspace_bytes",
    "goom_lmme_backward", "goom_lmme_backward_workspace_bytes", "goom_scan_backward", "goom_scan_backward_workspace_bytes", "goom_scaled_exp_backward",
    "goom_linear_attention", "goom_linear_attention_workspace_bytes", "goom_linear_attention_step",
    "goom_linear_attention_backward", "goom_linear_attention_backward_workspace_bytes",
    "goom_gated_delta", "goom_gated_delta_workspace_bytes", "goom_gated_delta_step", "goom_gated_delta_backward", "goom_gated_delta_backward_workspace_bytes",
    "goom_group_norm", "goom_group_norm_workspace_bytes", "goom_group_norm_backward", "goom_group_norm_backward_workspace_bytes",
    "goom_rotary", "goom_norm_after", "goom_norm_before", "goom_norm_after_backward", "goom_norm_before_backward", "goom_block_norm_backward_workspace_bytes",
    "goom_embedding", "goom_embedding_backward", "goom_embedding_backward_workspace_bytes",
]


class GoomError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{status_name(status)}: {message}")
        self.status = status


class ScanOpts(C.Structure):
    _fields_ = [("chunk_len", C.c_int64), ("flags", C.c_uint32)]


class ResetOpts(C.Structure):
    _fields_ = [("chunk_len", C.c_int64), ("policy", C.c_int32), ("cos_threshold", C.c_float)]


class AttentionShape(C.Structure):
    _fields_ = [("seqs", C.c_int64), ("tokens", C.c_int64), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("dk", C.c_int32), ("dv", C.c_int32),
                ("type", C.c_int32), ("flags", C.c_int32), ("scale", C.c_double), ("q_token", C.c_int64), ("q_head", C.c_int64),
                ("k_token", C.c_int64), ("k_head", C.c_int64), ("v_token", C.c_int64), ("v_head", C.c_int64)]


class DeltaShape(C.Structure):
    _fields_ = [("seqs", C.c_int64), ("tokens", C.c_int64), ("heads", C.c_int32), ("qk_heads", C.c_int32), ("dk", C.c_int32), ("dv", C.c_int32),
                ("type", C.c_int32), ("flags", C.c_int32), ("scale", C.c_double), ("q_token", C.c_int64), ("q_head", C.c_int64),
                ("k_token", C.c_int64), ("k_head", C.c_int64), ("v_token", C.c_int64), ("v_head", C.c_int64)]


class NormShape(C.Structure):
    _fields_ = [("items", C.c_int64), ("length", C.c_int64), ("channels", C.c_int32), ("groups", C.c_int32), ("type", C.c_int32),
                ("param_type", C.c_int32), ("activation", C.c_int32), ("flags", C.c_int32), ("eps", C.c_double)]


class RotaryShape(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("dim", C.c_int32), ("pairs", C.c_int32), ("type", C.c_int32), ("flags", C.c_int32),
                ("scale", C.c_double), ("q_token", C.c_int64), ("q_head", C.c_int64), ("k_token", C.c_int64), ("k_head", C.c_int64)]


class BlockNormShape(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("channels", C.c_int32), ("groups", C.c_int32), ("type", C.c_int32), ("param_type", C.c_int32), ("activation", C.c_int32),
                ("flags", C.c_int32), ("eps", C.c_double)]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libgoom.so.  It must have been built (``python -m paper_2510_03426_amd.build`` or
    ``__graft_entry__.build()``); there is no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise GoomErrorNoLib()
    lib = C.CDLL(_LIB_PATH)
    vp, i32, i64, u32, sz = C.c_void_p, C.c_int, C.c_int64, C.c_uint32, C.c_size_t
    lib.goom_version.restype = i32
    lib.goom_create.argtypes = [C.POINTER(vp), i32, vp]
    lib.goom_destroy.argtypes = [vp]
    lib.goom_set_stream.argtypes = [vp, vp]
    lib.goom_last_error.argtypes = [vp]
    lib.goom_last_error.restype = C.c_char_p
    lib.goom_status_name.argtypes = [i32]
    lib.goom_status_name.restype = C.c_char_p
    lib.goom_profile_enable.argtypes = [vp, i32]
    lib.goom_profile_count.argtypes = [vp]
    lib.goom_profile_get.argtypes = [vp, i32, C.POINTER(C.c_char_p), C.POINTER(C.c_float)]
    lib.goom_to_goom.argtypes = [vp, vp, vp, sz, i32, u32]
    lib.goom_from_goom.argtypes = [vp, vp, vp, sz, i32]
    lib.goom_lmme.argtypes = [vp, vp, vp, vp, i64, i32, i32, i32, i32, u32, vp, sz]
    lib.goom_lmme_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, u32]
    lib.goom_lmme_workspace_bytes.restype = sz
    po = C.POINTER(ScanOpts)
    lib.goom_scan.argtypes = [vp, vp, vp, vp, i64, i32, i32, i64, i32, po, vp, sz]
    lib.goom_scan_workspace_bytes.argtypes = [i64, i32, i32, i64, i32, po]
    lib.goom_scan_workspace_bytes.restype = sz
    lib.goom_scan_static.argtypes = [vp, vp, vp, vp, i64, i32, i32, i64, i32, po]
    lib.goom_reduce.argtypes = [vp, vp, vp, vp, i64, i32, i32, i64, i32, po, vp, sz]
    lib.goom_reduce_workspace_bytes.argtypes = [i64, i32, i32, i64, i32, po]
    lib.goom_reduce_workspace_bytes.restype = sz
    lib.goom_scan_real.argtypes = [vp, vp, vp, vp, i64, i32, i32, i64, i32, po, vp, sz]
    lib.goom_scan_real_workspace_bytes.argtypes = [i64, i32, i32, i64, i32, po]
    lib.goom_scan_real_workspace_bytes.restype = sz
    lib.goom_reduce_real.argtypes = [vp, vp, vp, vp, i64, i32, i32, i64, i32, po, vp, sz]
    lib.goom_reduce_real_workspace_bytes.argtypes = [i64, i32, i32, i64, i32, po]
    lib.goom_reduce_real_workspace_bytes.restype = sz
    pr = C.POINTER(ResetOpts)
    lib.goom_scan_reset.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, i64, i32, pr, vp, sz]
    lib.goom_scan_reset_workspace_bytes.argtypes = [i64, i32, i64, i32, pr]
    lib.goom_scan_reset_workspace_bytes.restype = sz
    lib.goom_scan_reset_tree.argtypes = [vp, vp, vp, vp, vp, i64, i32, i64, i32, pr, vp, sz]
    lib.goom_scan_reset_tree_workspace_bytes.argtypes = [i64, i32, i64, i32]
    lib.goom_scan_reset_tree_workspace_bytes.restype = sz
    lib.goom_lyapunov_spectrum.argtypes = [vp, vp, vp, vp, vp, i64, i32, C.c_double, i64, i32, pr, vp, sz]
    lib.goom_lyapunov_spectrum_per_step.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, C.c_double, i64, i32, pr, vp, sz]
    lib.goom_lyapunov_spectrum_per_step_workspace_bytes.argtypes = [i64, i32, i64, i32, pr, i32, i32]
    lib.goom_lyapunov_spectrum_per_step_workspace_bytes.restype = sz
    lib.goom_largest_lyapunov.argtypes = [vp, vp, vp, vp, i64, i32, C.c_double, i64, i32, po, vp, sz]
    lib.goom_largest_lyapunov_workspace_bytes.argtypes = [i64, i32, i64, i32, po]
    lib.goom_largest_lyapunov_workspace_bytes.restype = sz
    lib.goom_scaled_exp.argtypes = [vp, vp, vp, vp, sz, i32, i32]
    lib.goom_log_add_exp.argtypes = [vp, vp, vp, vp, sz, i32]
    lib.goom_affine_scan.argtypes = [vp, vp, vp, vp, vp, i64, i32, i64, i32, po, vp, sz]
    lib.goom_affine_scan_workspace_bytes.argtypes = [i64, i32, i64, i32, po]
    lib.goom_affine_scan_workspace_bytes.restype = sz
    lib.goom_probe_bandwidth.argtypes = [vp, vp, vp, sz, i32]
    lib.goom_probe_matrix_unit.argtypes = [vp, vp, i64, i32]
    lib.goom_affine_scan_scaled.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, i64, i32, po, vp, sz]
    lib.goom_affine_scan_scaled_workspace_bytes.argtypes = [i64, i32, i64, i32, po]
    lib.goom_affine_scan_scaled_workspace_bytes.restype = sz
    lib.goom_count_nonfinite.argtypes = [vp, vp, sz, i32, vp]
    lib.goom_to_goom_backward.argtypes = [vp, vp, vp, vp, sz, i32, C.c_double]
    lib.goom_from_goom_backward.argtypes = [vp, vp, vp, vp, sz, i32, C.c_double]
    lib.goom_affine_scan_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, i32, i64, i32, po, vp, sz]
    lib.goom_affine_scan_backward_workspace_bytes.argtypes = [i64, i32, i64, i32, po]
    lib.goom_affine_scan_backward_workspace_bytes.restype = sz
    lib.goom_lmme_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i32, i32, i32, i32, u32, vp, sz]
    lib.goom_lmme_backward_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, u32]
    lib.goom_lmme_backward_workspace_bytes.restype = sz
    lib.goom_scaled_exp_backward.argtypes = [vp, vp, vp, vp, sz, i32]
    lib.goom_scan_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i32, i32, i64, i32, po, vp, sz]
    lib.goom_scan_backward_workspace_bytes.argtypes = [i64, i32, i32, i64, i32, po, i32]
    lib.goom_scan_backward_workspace_bytes.restype = sz
    pa = C.POINTER(AttentionShape)
    lib.goom_linear_attention.argtypes = [vp, pa, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz]
    lib.goom_linear_attention_workspace_bytes.argtypes = [pa, i32]
    lib.goom_linear_attention_workspace_bytes.restype = sz
    lib.goom_linear_attention_step.argtypes = [vp, pa, vp, vp, vp, vp, vp, vp, vp]
    lib.goom_linear_attention_backward.argtypes = [vp, pa, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz]
    lib.goom_linear_attention_backward_workspace_bytes.argtypes = [pa, i32]
    lib.goom_linear_attention_backward_workspace_bytes.restype = sz
    lib.goom_rotary.argtypes = [vp, C.POINTER(RotaryShape)] + [vp] * 6
    pb = C.POINTER(BlockNormShape)
    lib.goom_norm_after.argtypes = [vp, pb] + [vp] * 9
    lib.goom_norm_before.argtypes = [vp, pb] + [vp] * 10
    lib.goom_norm_after_backward.argtypes = [vp, pb] + [vp] * 14 + [sz]
    lib.goom_norm_before_backward.argtypes = [vp, pb] + [vp] * 16 + [sz]
    lib.goom_block_norm_backward_workspace_bytes.argtypes = [pb]
    lib.goom_block_norm_backward_workspace_bytes.restype = sz
    pd = C.POINTER(DeltaShape)
    lib.goom_gated_delta.argtypes = [vp, pd, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz]
    lib.goom_gated_delta_step.argtypes = [vp, pd, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.goom_gated_delta_backward.argtypes = [vp, pd] + [vp] * 16 + [sz]
    for f in (lib.goom_gated_delta_workspace_bytes, lib.goom_gated_delta_backward_workspace_bytes):
        f.argtypes = [pd, i32]
        f.restype = sz
    pn = C.POINTER(NormShape)
    lib.goom_group_norm.argtypes = [vp, pn, vp, vp, vp, vp, vp, vp, vp, sz]
    lib.goom_group_norm_backward.argtypes = [vp, pn, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz]
    for f in (lib.goom_group_norm_workspace_bytes, lib.goom_group_norm_backward_workspace_bytes):
        f.argtypes, f.restype = [pn], sz
    lib.goom_embedding.argtypes = [vp, vp, vp, vp, i64, i64, i32, i32, C.c_double]
    lib.goom_embedding_backward.argtypes = [vp, vp, vp, vp, i64, i64, i32, i32, i32, C.c_double, vp, sz]
    lib.goom_embedding_backward_workspace_bytes.argtypes = [i64, i64, i32]
    lib.goom_embedding_backward_workspace_bytes.restype = sz
    _lib = lib
    return lib


class GoomErrorNoLib(RuntimeError):
    def __init__(self):
        super().__init__(f"{_LIB_PATH} is not built; run __graft_entry__.build() (hipcc, gfx950). "
                         "There is no CPU fallback.")


def status_name(status: int) -> str:
    return load_library().goom_status_name(status).decode()


def _dtype_code(t):
    import torch
    if t.dtype in (torch.complex64, torch.float32):
        return C64
    if t.dtype in (torch.complex128, torch.float64):
        return C128
    raise TypeError(f"unsupported tensor dtype {t.dtype}")


_real_codes = {}  # torch dtype -> GOOM_REAL_*


def _real_code(t):
    code = _real_codes.get(t.dtype)
    if code is None:
        import torch
        _real_codes.update({torch.float32: REAL_F32, torch.bfloat16: REAL_BF16, torch.float16: REAL_F16})
        code = _real_codes.get(t.dtype)
        if code is None:
            raise TypeError(f"unsupported tensor dtype {t.dtype}")
    return code


def _at(t):
    """Address of a contiguous device tensor, None for None."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("libgoom takes contiguous device tensors")
    return t.data_ptr()


def _rows(t, name):
    """Address and strides (token, head; 0, 0: contiguous) of [..., heads, d] whose last axis is contiguous and whose leading axes
    follow one another in memory, as in a slice of a fused projection.  Axes that were expanded are refused."""
    if not t.is_cuda:
        raise ValueError("libgoom takes device tensors")
    if t.is_contiguous():
        return t.data_ptr(), 0, 0
    st, sh = t.stride(), t.shape
    if sh[-1] != 1 and st[-1] != 1:
        raise ValueError(f"{name}: the last axis must be contiguous")
    head = sh[-1] if sh[-2] == 1 else st[-2]
    token = None  # the innermost axis of tokens that is longer than one
    for i in range(t.dim() - 3, -1, -1):
        if sh[i] == 1:
            continue
        if token is None:
            token, run = st[i], sh[i]
        elif st[i] != run * token:
            raise ValueError(f"{name}: the tokens do not follow one another in memory")
        else:
            run *= sh[i]
    if head < sh[-1] or (token is not None and token < sh[-1]):  # (0, 0 would be taken for contiguous)
        raise ValueError(f"{name}: rows share memory, as those of an expanded tensor do")
    return t.data_ptr(), sh[-2] * head if token is None else token, head


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("libgoom takes contiguous device tensors")
    return C.c_void_p(t.data_ptr())


def rotary_frequencies(pairs: int, base: float = 10000.0, factor: float = 1.0, method: str = "none", trained: int = 0, low: float = 1.0, high: float = 32.0,
                       device="cpu"):
    """Frequencies for Goom.rotary, float32 [pairs], base^(-i / pairs) radians a position, and the scale that goes with them.  For contexts
    `factor` times as long as the `trained` one a method other than "none" (which leaves them and 1.0):
        "linear": all of them divided by the factor;
        "base":   base times factor^(pairs / (pairs - 1)), so that the first stays and the last is divided by the factor;
        "parts":  waves that turn at least `high` times within the trained context stay, those that turn at most `low` times are divided by the factor, the ones
                  between in proportion; the scale is 0.1 log(factor) + 1, on q and on k."""
    import torch
    if pairs < 1 or not base > 1 or not factor >= 1 or method not in ("none", "linear", "base", "parts"):
        raise ValueError('pairs >= 1, base > 1, factor >= 1, method "none", "linear", "base" or "parts"')
    if method == "base":
        base *= factor ** (pairs / max(1, pairs - 1))
    f = torch.pow(torch.tensor(base, dtype=torch.float64), -torch.arange(pairs, dtype=torch.float64) / pairs)
    scale = 1.0
    if method == "linear":
        f = f / factor
    elif method == "parts":
        if trained < 1 or not high > low:
            raise ValueError("parts: the trained context's length, and low < high")
        stay = ((trained * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f * stay + f / factor * (1 - stay)
        scale = 0.1 * math.log(factor) + 1.0
    return f.to(torch.float32).to(device), scale


class Goom:
    """A libgoom context on one device, bound to torch's current stream at creation (or
    to ``stream``).  Methods mirror the C entry points and allocate outputs/workspaces
    with torch."""

    def __init__(self, device: int = 0, stream=None):
        import torch
        self.torch = torch
        self.lib = load_library()
        self.device = torch.device("cuda", device)
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        self._stream = stream
        self._ctx = C.c_void_p()
        st = self.lib.goom_create(C.byref(self._ctx), device, C.c_void_p(stream.cuda_stream))
        if st != 0:
            raise GoomError(st, self.lib.goom_last_error(None).decode())
        self._ws = None

    def close(self):
        if self._ctx:
            self.lib.goom_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st):
        if st != 0:
            raise GoomError(st, self.lib.goom_last_error(self._ctx).decode())

    def set_stream(self, stream):
        self._stream = stream
        self._check(self.lib.goom_set_stream(self._ctx, C.c_void_p(stream.cuda_stream)))

    def probe_bandwidth(self, a, b, mode: int):
        """One streaming pass (0 read a, 1 fill b, 2 copy a to b) on the context's stream; the caller times it."""
        nbytes = b.numel() * b.element_size()
        self._check(self.lib.goom_probe_bandwidth(self._ctx, _ptr(a), _ptr(b), nbytes, mode))

    PROBE_MATRIX_FLOP_PER_ITER = 134217728

    def probe_matrix_unit(self, sink, iters: int, double: bool = False):
        """A kernel of nothing but matrix instructions (PROBE_MATRIX_FLOP_PER_ITER * iters flop) on the context's
        stream; sink: a device tensor of at least 4 bytes; the caller times it."""
        self._check(self.lib.goom_probe_matrix_unit(self._ctx, _ptr(sink), iters, 1 if double else 0))

    def profile_enable(self, on: bool = True):
        self._check(self.lib.goom_profile_enable(self._ctx, int(on)))

    def profile_records(self):
        """[(label, milliseconds)] for the kernels of the last compute call (waits for them)."""
        out = []
        for i in range(self.lib.goom_profile_count(self._ctx)):
            label, ms = C.c_char_p(), C.c_float()
            self._check(self.lib.goom_profile_get(self._ctx, i, C.byref(label), C.byref(ms)))
            out.append((label.value.decode(), float(ms.value)))
        return out

    def workspace(self, nbytes: int):
        """A cached 256-byte aligned scratch tensor of at least nbytes (None for 0), of the context's stream: what comes after it in memory that was let go
        waits for that stream's work, whatever torch's current one is.  A call that is captured (torch.cuda.graph, torch.cuda.CUDAGraph) has one of its own, from
        the graph's memory: the cached one is let go when a later call needs more, and replays may go side by side.  Captures that torch does not know of have no
        such memory: they take the C entry points, with a workspace that their program keeps."""
        if nbytes == 0:
            return None, 0
        captured = self.torch.cuda.is_current_stream_capturing()
        if captured or self._ws is None or self._ws.numel() < nbytes:
            with self.torch.cuda.stream(self._stream):
                ws = self.torch.empty(nbytes, dtype=self.torch.uint8, device=self.device)
            if captured:
                return ws, nbytes
            self._ws = ws
        return self._ws, self._ws.numel()

    # ---- codecs
    def to_goom(self, x, flags: int = ZERO_NEG_INF, out=None):
        torch = self.torch
        code = _dtype_code(x)
        if out is None:
            out = torch.empty(x.shape, dtype=torch.complex64 if code == C64 else torch.complex128, device=x.device)
        self._check(self.lib.goom_to_goom(self._ctx, _ptr(x), _ptr(out), x.numel(), code, flags))
        return out

    def from_goom(self, y, out=None):
        torch = self.torch
        code = _dtype_code(y)
        if out is None:
            out = torch.empty(y.shape, dtype=torch.float32 if code == C64 else torch.float64, device=y.device)
        self._check(self.lib.goom_from_goom(self._ctx, _ptr(y), _ptr(out), y.numel(), code))
        return out

    # ---- LMME
    def lmme(self, a, b, flags: int = LMME_FAST, out=None):
        torch = self.torch
        code = _dtype_code(a)
        n, d = a.shape[-2:]
        d2, m = b.shape[-2:]
        assert d == d2 and a.shape[:-2] == b.shape[:-2] and a.dtype == b.dtype
        batch = 1
        for s in a.shape[:-2]:
            batch *= s
        if out is None:
            out = torch.empty(a.shape[:-2] + (n, m), dtype=a.dtype, device=a.device)
        ws, wsn = self.workspace(self.lib.goom_lmme_workspace_bytes(batch, n, d, m, code, flags))
        self._check(self.lib.goom_lmme(self._ctx, _ptr(a), _ptr(b), _ptr(out), batch, n, d, m, code, flags,
                                       _ptr(ws), wsn))
        return out

    # ---- scans
    def _scan_shapes(self, mats, init):
        T, d, d2 = mats.shape[-3:]
        assert d == d2
        lead = mats.shape[:-3]
        batch = 1
        for s in lead:
            batch *= s
        if init is not None:
            assert init.shape[:-2] == lead and init.shape[-2] == d and init.dtype == mats.dtype
            m = init.shape[-1]
        else:
            m = d
        return lead, batch, T, d, m

    def scan(self, mats, init=None, chunk_len: int = 0, out=None):
        torch = self.torch
        code = _dtype_code(mats)
        lead, batch, T, d, m = self._scan_shapes(mats, init)
        opts = ScanOpts(chunk_len, 0)
        if out is None:
            out = torch.empty(lead + (T, d, m), dtype=mats.dtype, device=mats.device)
        ws, wsn = self.workspace(self.lib.goom_scan_workspace_bytes(T, d, m, batch, code, C.byref(opts)))
        self._check(self.lib.goom_scan(self._ctx, _ptr(mats), _ptr(init), _ptr(out), T, d, m, batch, code,
                                       C.byref(opts), _ptr(ws), wsn))
        return out

    STATIC_SCRATCH_BYTES = 40 << 20

    def scan_static(self, mats, out, init=None, chunk_len: int = 0):
        """goom_scan_static: the scan with the library's static scratch array as its workspace.  `out` is the
        caller's; nothing is allocated here or in the library."""
        code = _dtype_code(mats)
        lead, batch, T, d, m = self._scan_shapes(mats, init)
        assert tuple(out.shape) == tuple(lead + (T, d, m)) and out.dtype == mats.dtype
        opts = ScanOpts(chunk_len, 0)
        self._check(self.lib.goom_scan_static(self._ctx, _ptr(mats), _ptr(init), _ptr(out), T, d, m, batch, code,
                                              C.byref(opts)))
        return out

    def reduce(self, mats, init=None, chunk_len: int = 0, out=None):
        torch = self.torch
        code = _dtype_code(mats)
        lead, batch, T, d, m = self._scan_shapes(mats, init)
        opts = ScanOpts(chunk_len, 0)
        if out is None:
            out = torch.empty(lead + (d, m), dtype=mats.dtype, device=mats.device)
        ws, wsn = self.workspace(self.lib.goom_reduce_workspace_bytes(T, d, m, batch, code, C.byref(opts)))
        self._check(self.lib.goom_reduce(self._ctx, _ptr(mats), _ptr(init), _ptr(out), T, d, m, batch, code,
                                         C.byref(opts), _ptr(ws), wsn))
        return out

    def scan_real(self, x, init=None, chunk_len: int = 0, out=None, final_only: bool = False):
        """Prefix products (or, with final_only, the last one) of real matrices x: [..., T, d, d], as GOOMs."""
        torch = self.torch
        ctype = torch.complex64 if x.dtype == torch.float32 else torch.complex128
        code = C64 if x.dtype == torch.float32 else C128
        T, d = x.shape[-3], x.shape[-1]
        lead = x.shape[:-3]
        m = d if init is None else init.shape[-1]
        batch = 1
        for s in lead:
            batch *= s
        opts = ScanOpts(chunk_len, 0)
        if out is None:
            out = torch.empty(lead + ((d, m) if final_only else (T, d, m)), dtype=ctype, device=x.device)
        if final_only:
            ws, wsn = self.workspace(self.lib.goom_reduce_real_workspace_bytes(T, d, m, batch, code, C.byref(opts)))
            self._check(self.lib.goom_reduce_real(self._ctx, _ptr(x), _ptr(init), _ptr(out), T, d, m, batch, code,
                                                  C.byref(opts), _ptr(ws), wsn))
        else:
            ws, wsn = self.workspace(self.lib.goom_scan_real_workspace_bytes(T, d, m, batch, code, C.byref(opts)))
            self._check(self.lib.goom_scan_real(self._ctx, _ptr(x), _ptr(init), _ptr(out), T, d, m, batch, code,
                                                C.byref(opts), _ptr(ws), wsn))
        return out

    def affine_scan(self, a, bias, h0=None, chunk_len: int = 0, out=None, time_invariant: bool = False):
        """h_t = A_t h_{t-1} + bias_t.  a: [..., T, d, d], or [..., d, d] with time_invariant=True."""
        torch = self.torch
        code = _dtype_code(a)
        T, d = bias.shape[-2:]
        lead = bias.shape[:-2]
        assert a.shape == (lead + (d, d) if time_invariant else lead + (T, d, d)) and a.dtype == bias.dtype
        batch = 1
        for s in lead:
            batch *= s
        opts = ScanOpts(chunk_len, AFFINE_TIME_INVARIANT if time_invariant else 0)
        if out is None:
            out = torch.empty(lead + (T, d), dtype=a.dtype, device=a.device)
        ws, wsn = self.workspace(self.lib.goom_affine_scan_workspace_bytes(T, d, batch, code, C.byref(opts)))
        self._check(self.lib.goom_affine_scan(self._ctx, _ptr(a), _ptr(bias), _ptr(h0), _ptr(out), T, d, batch,
                                              code, C.byref(opts), _ptr(ws), wsn))
        return out

    def affine_scan_scaled(self, a, bias, h0=None, chunk_len: int = 0, time_invariant: bool = False,
                           want_logscale: bool = False):
        """The recurrence's states as exp(h - max Re h + 2), real, and optionally the log scales."""
        torch = self.torch
        code = _dtype_code(a)
        T, d = bias.shape[-2:]
        lead = bias.shape[:-2]
        assert a.shape == (lead + (d, d) if time_invariant else lead + (T, d, d)) and a.dtype == bias.dtype
        batch = 1
        for s in lead:
            batch *= s
        opts = ScanOpts(chunk_len, AFFINE_TIME_INVARIANT if time_invariant else 0)
        comp = torch.float32 if a.dtype == torch.complex64 else torch.float64
        out = torch.empty(lead + (T, d), dtype=comp, device=a.device)
        c = torch.empty(lead + (T,), dtype=comp, device=a.device) if want_logscale else None
        ws, wsn = self.workspace(self.lib.goom_affine_scan_scaled_workspace_bytes(T, d, batch, code, C.byref(opts)))
        self._check(self.lib.goom_affine_scan_scaled(self._ctx, _ptr(a), _ptr(bias), _ptr(h0), _ptr(out), _ptr(c), T, d,
                                                     batch, code, C.byref(opts), _ptr(ws), wsn))
        return (out, c) if want_logscale else out

    def scan_reset(self, jac, s0=None, chunk_len: int = 0, policy: int = RESET_ALWAYS,
                   cos_threshold: float = 0.99, want_states: bool = True):
        torch = self.torch
        code = _dtype_code(jac)
        T, d, _ = jac.shape[-3:]
        lead = jac.shape[:-3]
        batch = 1
        for s in lead:
            batch *= s
        opts = ResetOpts(chunk_len, policy, cos_threshold)
        states = torch.empty(lead + (T, d, d), dtype=jac.dtype, device=jac.device)
        flags = torch.zeros(lead + (T,), dtype=torch.uint8, device=jac.device)
        growth = torch.zeros(lead + (d,), dtype=torch.float64, device=jac.device)
        ws, wsn = self.workspace(self.lib.goom_scan_reset_workspace_bytes(T, d, batch, code, C.byref(opts)))
        self._check(self.lib.goom_scan_reset(self._ctx, _ptr(jac), _ptr(s0), _ptr(states), _ptr(flags), _ptr(growth),
                                             T, d, batch, code, C.byref(opts), _ptr(ws), wsn))
        return states, flags, growth

    def scan_reset_tree(self, jac, s0=None, policy: int = RESET_COLINEAR, cos_threshold: float = 0.99):
        """The selective-resetting scan in the order of the paper's parallel prefix scan; returns (states, flags)."""
        torch = self.torch
        code = _dtype_code(jac)
        T, d, _ = jac.shape[-3:]
        lead = jac.shape[:-3]
        batch = 1
        for s in lead:
            batch *= s
        opts = ResetOpts(0, policy, cos_threshold)
        states = torch.empty(lead + (T, d, d), dtype=jac.dtype, device=jac.device)
        flags = torch.zeros(lead + (T,), dtype=torch.uint8, device=jac.device)
        ws, wsn = self.workspace(self.lib.goom_scan_reset_tree_workspace_bytes(T, d, batch, code))
        self._check(self.lib.goom_scan_reset_tree(self._ctx, _ptr(jac), _ptr(s0), _ptr(states), _ptr(flags), T, d, batch, code,
                                                  C.byref(opts), _ptr(ws), wsn))
        return states, flags

    def lyapunov_spectrum(self, jac, dt: float, s0=None, chunk_len: int = 0, policy: int = RESET_ALWAYS,
                          cos_threshold: float = 0.99):
        torch = self.torch
        code = _dtype_code(jac)
        T, d, _ = jac.shape[-3:]
        lead = jac.shape[:-3]
        batch = 1
        for s in lead:
            batch *= s
        opts = ResetOpts(chunk_len, policy, cos_threshold)
        lam = torch.zeros(lead + (d,), dtype=torch.float64, device=jac.device)
        ws, wsn = self.workspace(self.lib.goom_scan_reset_workspace_bytes(T, d, batch, code, C.byref(opts)))
        self._check(self.lib.goom_lyapunov_spectrum(self._ctx, _ptr(jac), _ptr(s0), None, _ptr(lam), T, d, dt, batch,
                                                    code, C.byref(opts), _ptr(ws), wsn))
        return lam

    def lyapunov_spectrum_per_step(self, jac, dt: float, s0=None, chunk_len: int = 0, policy: int = RESET_ALWAYS,
                                   cos_threshold: float = 0.99, want_step_logs: bool = False):
        """Spectrum by the four groups of parallel computations (two QRs per step)."""
        torch = self.torch
        code = _dtype_code(jac)
        T, d, _ = jac.shape[-3:]
        lead = jac.shape[:-3]
        batch = 1
        for s in lead:
            batch *= s
        opts = ResetOpts(chunk_len, policy, cos_threshold)
        lam = torch.zeros(lead + (d,), dtype=torch.float64, device=jac.device)
        logs = torch.zeros(lead + (T, d), dtype=torch.float64, device=jac.device) if want_step_logs else None
        ws, wsn = self.workspace(self.lib.goom_lyapunov_spectrum_per_step_workspace_bytes(
            T, d, batch, code, C.byref(opts), 0, 1 if want_step_logs else 0))
        self._check(self.lib.goom_lyapunov_spectrum_per_step(self._ctx, _ptr(jac), _ptr(s0), None, _ptr(logs), _ptr(lam),
                                                             T, d, dt, batch, code, C.byref(opts), _ptr(ws), wsn))
        return (lam, logs) if want_step_logs else lam

    def largest_lyapunov(self, jac, dt: float, u0=None, chunk_len: int = 0):
        """Largest exponent as LSE(2 v') / (2 dt T), v' = J_T ... J_1 u_0 over GOOMs."""
        torch = self.torch
        code = _dtype_code(jac)
        T, d, _ = jac.shape[-3:]
        lead = jac.shape[:-3]
        batch = 1
        for s in lead:
            batch *= s
        opts = ScanOpts(chunk_len, 0)
        lle = torch.zeros(lead, dtype=torch.float64, device=jac.device)
        ws, wsn = self.workspace(self.lib.goom_largest_lyapunov_workspace_bytes(T, d, batch, code, C.byref(opts)))
        self._check(self.lib.goom_largest_lyapunov(self._ctx, _ptr(jac), _ptr(u0), _ptr(lle), T, d, dt, batch, code,
                                                   C.byref(opts), _ptr(ws), wsn))
        return lle

    def count_nonfinite(self, z) -> int:
        """Entries of a GOOM tensor whose log-magnitude is +inf or NaN (synchronises to return the number)."""
        cnt = self.torch.zeros(1, dtype=self.torch.int64, device=z.device)
        self._check(self.lib.goom_count_nonfinite(self._ctx, _ptr(z), z.numel(), _dtype_code(z), _ptr(cnt)))
        return int(cnt.item())

    def to_goom_backward(self, x, grad_re, eps: float):
        """grad_re * s(x) / (|x| + eps): backward of to_goom with the paper's redefined derivatives."""
        out = self.torch.empty_like(x)
        self._check(self.lib.goom_to_goom_backward(self._ctx, _ptr(x), _ptr(grad_re), _ptr(out), x.numel(), _dtype_code(x), eps))
        return out

    def from_goom_backward(self, y, grad_x, eps: float):
        """grad_x * (x + s(x) eps): backward of from_goom with the paper's redefined derivative."""
        out = self.torch.empty_like(grad_x)
        self._check(self.lib.goom_from_goom_backward(self._ctx, _ptr(y), _ptr(grad_x), _ptr(out), y.numel(), _dtype_code(y), eps))
        return out

    def affine_scan_backward(self, a, bias, h, grad_h, h0=None, chunk_len: int = 0, time_invariant: bool = False):
        """Gradients of a loss with respect to the log-magnitudes of a, bias (and h0), given grad_h = dL / d Re h.
        time_invariant: a is [..., d, d], one matrix for all steps, and so is its gradient."""
        torch = self.torch
        code = _dtype_code(a)
        T, d = bias.shape[-2:]
        lead = bias.shape[:-2]
        batch = 1
        for s in lead:
            batch *= s
        comp = torch.float32 if a.dtype == torch.complex64 else torch.float64
        ashape = lead + ((d, d) if time_invariant else (T, d, d))
        assert a.shape == ashape and h.shape == bias.shape and grad_h.shape == bias.shape and grad_h.dtype == comp
        opts = ScanOpts(chunk_len, AFFINE_TIME_INVARIANT if time_invariant else 0)
        ga = torch.empty(ashape, dtype=comp, device=a.device)
        gb = torch.empty(lead + (T, d), dtype=comp, device=a.device)
        gh0 = torch.empty(lead + (d,), dtype=comp, device=a.device) if h0 is not None else None
        ws, wsn = self.workspace(self.lib.goom_affine_scan_backward_workspace_bytes(T, d, batch, code, C.byref(opts)))
        self._check(self.lib.goom_affine_scan_backward(self._ctx, _ptr(a), _ptr(bias), _ptr(h0), _ptr(h), _ptr(grad_h), _ptr(ga), _ptr(gb),
                                                       _ptr(gh0), T, d, batch, code, C.byref(opts), _ptr(ws), wsn))
        return ga, gb, gh0

    def lmme_backward(self, a, b, c, grad_c, flags: int = LMME_FAST):
        """Gradients of a loss with respect to the log-magnitudes of a and b, given c = lmme(a, b) and grad_c = dL / d Re c."""
        torch = self.torch
        code = _dtype_code(a)
        n, d = a.shape[-2:]
        m = b.shape[-1]
        lead = a.shape[:-2]
        batch = 1
        for s in lead:
            batch *= s
        comp = torch.float32 if a.dtype == torch.complex64 else torch.float64
        assert b.shape == lead + (d, m) and c.shape == lead + (n, m) and grad_c.shape == c.shape
        assert b.dtype == a.dtype and c.dtype == a.dtype and grad_c.dtype == comp
        ga = torch.empty(lead + (n, d), dtype=comp, device=a.device)
        gb = torch.empty(lead + (d, m), dtype=comp, device=a.device)
        ws, wsn = self.workspace(self.lib.goom_lmme_backward_workspace_bytes(batch, n, d, m, code, flags))
        self._check(self.lib.goom_lmme_backward(self._ctx, _ptr(a), _ptr(b), _ptr(c), _ptr(grad_c), _ptr(ga), _ptr(gb), batch, n, d, m, code,
                                                flags, _ptr(ws), wsn))
        return ga, gb

    def scan_backward(self, mats, p, grad_p, init=None, chunk_len: int = 0):
        """Gradients of a loss with respect to the log-magnitudes of the factors (and of init), given the scan's states p and
        grad_p = dL / d Re p."""
        torch = self.torch
        code = _dtype_code(mats)
        lead, batch, T, d, m = self._scan_shapes(mats, init)
        comp = torch.float32 if mats.dtype == torch.complex64 else torch.float64
        assert p.shape == lead + (T, d, m) and grad_p.shape == p.shape and p.dtype == mats.dtype and grad_p.dtype == comp
        opts = ScanOpts(chunk_len, 0)
        gm = torch.empty(lead + (T, d, d), dtype=comp, device=mats.device)
        gi = torch.empty(lead + (d, m), dtype=comp, device=mats.device) if init is not None else None
        ws, wsn = self.workspace(self.lib.goom_scan_backward_workspace_bytes(T, d, m, batch, code, C.byref(opts), int(init is not None)))
        self._check(self.lib.goom_scan_backward(self._ctx, _ptr(mats), _ptr(init), _ptr(p), _ptr(grad_p), _ptr(gm), _ptr(gi), T, d, m, batch, code,
                                                C.byref(opts), _ptr(ws), wsn))
        return gm, gi

    def scaled_exp(self, z, want_logscale: bool = False):
        """Scaled exponentiation over the last axis: exp(z - max Re z + 2), real."""
        torch = self.torch
        code = _dtype_code(z)
        d = z.shape[-1]
        nvec = z.numel() // d
        comp = torch.float32 if z.dtype == torch.complex64 else torch.float64
        out = torch.empty(z.shape, dtype=comp, device=z.device)
        c = torch.empty(z.shape[:-1], dtype=comp, device=z.device) if want_logscale else None
        self._check(self.lib.goom_scaled_exp(self._ctx, _ptr(z), _ptr(out), _ptr(c), nvec, d, code))
        return (out, c) if want_logscale else out

    def scaled_exp_backward(self, scaled, grad_scaled):
        """Gradient with respect to Re z of scaled = scaled_exp(z), the log-scaling constant detached."""
        assert scaled.shape == grad_scaled.shape and scaled.dtype == grad_scaled.dtype
        out = self.torch.empty_like(scaled)
        self._check(self.lib.goom_scaled_exp_backward(self._ctx, _ptr(scaled), _ptr(grad_scaled), _ptr(out), scaled.numel(), _dtype_code(scaled)))
        return out

    def log_add_exp(self, x, y, out=None):
        """Elementwise GOOM of exp(x) + exp(y)."""
        assert x.shape == y.shape and x.dtype == y.dtype
        if out is None:
            out = self.torch.empty_like(x)
        self._check(self.lib.goom_log_add_exp(self._ctx, _ptr(x), _ptr(y), _ptr(out), x.numel(), _dtype_code(x)))
        return out

    # ---- linear attention with a decay for each head
    def _attention(self, q, k, v, log_decay, offsets, scale, step=False):
        """The shape structure and the addresses of q, k, v."""
        code = _real_code(q)
        if k.dtype != q.dtype or v.dtype != q.dtype or log_decay.dtype != self.torch.float32:
            raise TypeError("q, k, v have one type, log_decay is float32")
        sq, sk, sv = tuple(q.shape), tuple(k.shape), tuple(v.shape)
        lead, (heads, dk), (kv_heads, dv) = sq[:-2], sq[-2:], sv[-2:]
        if len(sq) < 3 or sk != lead + (kv_heads, dk) or sv[:-2] != lead or tuple(log_decay.shape) != (heads,):
            raise ValueError("shapes of q, k, v, log_decay do not fit")
        tokens = math.prod(lead)
        if offsets is not None:
            if offsets.dtype != self.torch.int64 or offsets.dim() != 1 or offsets.numel() < 1 or len(lead) != 1:
                raise ValueError("offsets: int64 [sequences + 1], with q, k, v [tokens, heads, d]")
            seqs = offsets.numel() - 1
        elif step:
            seqs = tokens
        else:
            seqs = math.prod(lead[:-1])
        pq, q_token, q_head = _rows(q, "q")
        pk, k_token, k_head = _rows(k, "k")
        pv, v_token, v_head = _rows(v, "v")
        return AttentionShape(seqs, tokens, heads, kv_heads, dk, dv, code, 0, scale, q_token, q_head, k_token, k_head, v_token, v_head), pq, pk, pv

    def _state(self, t, shape, name):
        if t is None:
            return None
        if tuple(t.shape) != (shape.seqs, shape.heads, shape.dk, shape.dv) or t.dtype != self.torch.float32:
            raise ValueError(f"{name}: float32 {[shape.seqs, shape.heads, shape.dk, shape.dv]}")
        return _at(t)

    def linear_attention(self, q, k, v, log_decay, state=None, offsets=None, scale: float = 1.0, want_state: bool = False):
        """o_t = scale q_t^T S_t, S_t = exp(log_decay) S_{t-1} + k_t v_t^T for every head.  q: [batch, T, heads, dk], k: [batch, T,
        kv_heads, dk], v: [batch, T, kv_heads, dv], or without the batch axis and with offsets (int64 [sequences + 1]) where
        sequences of different lengths lie behind one another (what is returned for tokens that no sequence has is not set); state, and the final one that want_state adds: float32 [sequences,
        heads, dk, dv].  q, k, v may be slices of one projection's output."""
        torch = self.torch
        shape, pq, pk, pv = self._attention(q, k, v, log_decay, offsets, scale)
        ps = self._state(state, shape, "state")
        o = torch.empty(q.shape[:-1] + (shape.dv,), dtype=q.dtype, device=q.device)
        last = torch.empty((shape.seqs, shape.heads, shape.dk, shape.dv), dtype=torch.float32, device=q.device) if want_state else None
        ws, wsn = self.workspace(self.lib.goom_linear_attention_workspace_bytes(C.byref(shape), int(offsets is not None)))
        self._check(self.lib.goom_linear_attention(self._ctx, C.byref(shape), pq, pk, pv, _at(log_decay), _at(offsets), ps, o.data_ptr(), _at(last),
                                                   _at(ws), wsn))
        return (o, last) if want_state else o

    def linear_attention_step(self, q, k, v, log_decay, state, scale: float = 1.0, out_state=None):
        """One token of each sequence: q: [batch, heads, dk], k: [batch, kv_heads, dk], v: [batch, kv_heads, dv]; state: float32 [batch,
        heads, dk, dv], replaced by the next one, or left as it is if out_state receives that."""
        if q.dim() != 3:
            raise ValueError("q: [batch, heads, dk]")
        shape, pq, pk, pv = self._attention(q, k, v, log_decay, None, scale, step=True)
        ps = self._state(state, shape, "state")
        pn = ps if out_state is None else self._state(out_state, shape, "out_state")
        o = self.torch.empty((shape.seqs, shape.heads, shape.dv), dtype=q.dtype, device=q.device)
        self._check(self.lib.goom_linear_attention_step(self._ctx, C.byref(shape), pq, pk, pv, _at(log_decay), ps, o.data_ptr(), pn))
        return o

    def linear_attention_backward(self, q, k, v, log_decay, grad_o, state=None, grad_state=None, offsets=None, scale: float = 1.0):
        """Gradients with respect to q, k, v and (None without one) the initial state, given those with respect to the outputs and
        (None: none) the final state.  Tokens that no sequence has: as above."""
        empty = self.torch.empty
        shape, pq, pk, pv = self._attention(q, k, v, log_decay, offsets, scale)
        if grad_o.shape != q.shape[:-1] + (shape.dv,) or grad_o.dtype != q.dtype:
            raise ValueError("grad_o: of o's shape and type")
        gq, gk, gv = (empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        ps, pg = self._state(state, shape, "state"), self._state(grad_state, shape, "grad_state")
        gs = empty(state.shape, dtype=state.dtype, device=state.device) if state is not None else None
        ws, wsn = self.workspace(self.lib.goom_linear_attention_backward_workspace_bytes(C.byref(shape), int(offsets is not None)))
        self._check(self.lib.goom_linear_attention_backward(self._ctx, C.byref(shape), pq, pk, pv, _at(log_decay), _at(offsets), ps, _at(grad_o), pg,
                                                            gq.data_ptr(), gk.data_ptr(), gv.data_ptr(), _at(gs), _at(ws), wsn))
        return gq, gk, gv, gs

    # ---- the gated delta rule
    def _delta(self, q, k, v, log_decay, beta, offsets, scale, step=False):
        """The shape structure and the addresses of q, k, v."""
        code = _real_code(q)
        if k.dtype != q.dtype or v.dtype != q.dtype or log_decay.dtype != self.torch.float32 or beta.dtype != self.torch.float32:
            raise TypeError("q, k, v have one type, log_decay and beta are float32")
        sq, sv = tuple(q.shape), tuple(v.shape)
        lead, (qk_heads, dk), (heads, dv) = sq[:-2], sq[-2:], sv[-2:]
        if len(sq) < 3 or tuple(k.shape) != sq or sv[:-2] != lead or tuple(log_decay.shape) != lead + (heads,) or tuple(beta.shape) != lead + (heads,):
            raise ValueError("shapes of q, k, v, log_decay, beta do not fit")
        tokens = math.prod(lead)
        if offsets is not None:
            if offsets.dtype != self.torch.int64 or offsets.dim() != 1 or offsets.numel() < 1 or len(lead) != 1:
                raise ValueError("offsets: int64 [sequences + 1], with q, k, v [tokens, heads, d]")
            seqs = offsets.numel() - 1
        elif step:
            seqs = tokens
        else:
            seqs = math.prod(lead[:-1])
        pq, q_token, q_head = _rows(q, "q")
        pk, k_token, k_head = _rows(k, "k")
        pv, v_token, v_head = _rows(v, "v")
        return DeltaShape(seqs, tokens, heads, qk_heads, dk, dv, code, 0, scale, q_token, q_head, k_token, k_head, v_token, v_head), pq, pk, pv

    def gated_delta(self, q, k, v, log_decay, beta, state=None, offsets=None, scale: float = 1.0, want_state: bool = False):
        """o_t = scale q_t^T S_t, S_t = a_t (S_{t-1} - beta_t k_t k_t^T S_{t-1}) + beta_t k_t v_t^T for every head, a_t = exp(log_decay_t).
        q, k: [batch, T, qk_heads, dk], v: [batch, T, heads, dv], log_decay, beta: float32 [batch, T, heads], or without the batch axis and with
        offsets (int64 [sequences + 1]) where sequences of different lengths lie behind one another (what is returned for tokens that no
        sequence has is not set); state, and the final one that want_state adds: float32 [sequences, heads, dk, dv].  q, k, v may be slices
        of one projection's output."""
        torch = self.torch
        shape, pq, pk, pv = self._delta(q, k, v, log_decay, beta, offsets, scale)
        ps = self._state(state, shape, "state")
        o = torch.empty(v.shape, dtype=v.dtype, device=v.device)
        last = torch.empty((shape.seqs, shape.heads, shape.dk, shape.dv), dtype=torch.float32, device=q.device) if want_state else None
        ws, wsn = self.workspace(self.lib.goom_gated_delta_workspace_bytes(C.byref(shape), int(offsets is not None)))
        self._check(self.lib.goom_gated_delta(self._ctx, C.byref(shape), pq, pk, pv, _at(log_decay), _at(beta), _at(offsets), ps, o.data_ptr(), _at(last), _at(ws), wsn))
        return (o, last) if want_state else o

    def gated_delta_step(self, q, k, v, log_decay, beta, state, scale: float = 1.0, out_state=None):
        """One token of each sequence: q, k: [batch, qk_heads, dk], v: [batch, heads, dv], log_decay, beta: [batch, heads]; state: float32
        [batch, heads, dk, dv], replaced by the next one, or left as it is if out_state receives that."""
        if q.dim() != 3:
            raise ValueError("q: [batch, qk_heads, dk]")
        shape, pq, pk, pv = self._delta(q, k, v, log_decay, beta, None, scale, step=True)
        ps = self._state(state, shape, "state")
        pn = ps if out_state is None else self._state(out_state, shape, "out_state")
        o = self.torch.empty_like(v, memory_format=self.torch.contiguous_format)
        self._check(self.lib.goom_gated_delta_step(self._ctx, C.byref(shape), pq, pk, pv, _at(log_decay), _at(beta), ps, o.data_ptr(), pn))
        return o

    def gated_delta_backward(self, q, k, v, log_decay, beta, grad_o, state=None, grad_state=None, offsets=None, scale: float = 1.0):
        """Gradients with respect to q, k, v, log_decay, beta and (None without one) the initial state, given those with respect to the outputs
        and (None: none) the final state.  Tokens that no sequence has: as above."""
        empty = self.torch.empty
        shape, pq, pk, pv = self._delta(q, k, v, log_decay, beta, offsets, scale)
        if grad_o.shape != v.shape or grad_o.dtype != v.dtype:
            raise ValueError("grad_o: of o's shape and type")
        gq, gk, gv, ga, gb = (empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v, log_decay, beta))
        ps, pg = self._state(state, shape, "state"), self._state(grad_state, shape, "grad_state")
        gs = empty(state.shape, dtype=state.dtype, device=state.device) if state is not None else None
        ws, wsn = self.workspace(self.lib.goom_gated_delta_backward_workspace_bytes(C.byref(shape), int(offsets is not None)))
        self._check(self.lib.goom_gated_delta_backward(self._ctx, C.byref(shape), pq, pk, pv, _at(log_decay), _at(beta), _at(offsets), ps, _at(grad_o), pg, gq.data_ptr(),
                                                       gk.data_ptr(), gv.data_ptr(), ga.data_ptr(), gb.data_ptr(), _at(gs), _at(ws), wsn))
        return gq, gk, gv, ga, gb, gs

    # ---- group norm with an activation, channels last
    def _norm(self, x, groups, weight, bias, eps, activation):
        sh = tuple(x.shape)
        act = ACTIVATIONS.get(activation)
        if len(sh) < 2 or act is None:
            raise ValueError("x: [items, ..., channels]; activation: one of " + ", ".join(ACTIVATIONS))
        code = REAL_F32
        for p in (weight, bias):
            if p is not None and tuple(p.shape) != sh[-1:]:
                raise ValueError("weight and bias: [channels]")
        if weight is not None:
            code = _real_code(weight)
            if bias is not None and bias.dtype != weight.dtype:
                raise TypeError("weight and bias have one type")
        elif bias is not None:
            code = _real_code(bias)
        return NormShape(sh[0], math.prod(sh[1:-1]), sh[-1], groups, _real_code(x), code, act, 0, eps)

    def group_norm(self, x, groups: int, weight=None, bias=None, eps: float = 1e-5, activation: str = "none", want_stats: bool = False):
        """act(normalised x * weight + bias); x: [items, ..., channels], statistics over the axes between and channels / groups
        neighbouring channels ([tokens, channels]: every token by itself).  want_stats: also mean and rstd, float32 [items, groups]."""
        torch = self.torch
        shape = self._norm(x, groups, weight, bias, eps, activation)
        px = _at(x)
        y = torch.empty_like(x)
        mean = rstd = pm = pr = None
        if want_stats:
            mean = torch.empty((shape.items, groups), dtype=torch.float32, device=x.device)
            rstd = torch.empty_like(mean)
            pm, pr = mean.data_ptr(), rstd.data_ptr()
        ws, wsn = self.workspace(self.lib.goom_group_norm_workspace_bytes(C.byref(shape)))
        self._check(self.lib.goom_group_norm(self._ctx, C.byref(shape), px, _at(weight), _at(bias), y.data_ptr(), pm, pr, _at(ws), wsn))
        return (y, mean, rstd) if want_stats else y

    def group_norm_backward(self, x, grad_y, mean, rstd, groups: int, weight=None, bias=None, activation: str = "none"):
        """Gradients with respect to x, weight and bias (of their type; float32 where there is none)."""
        torch = self.torch
        shape = self._norm(x, groups, weight, bias, 0.0, activation)
        if grad_y.shape != x.shape or grad_y.dtype != x.dtype or tuple(mean.shape) != (shape.items, groups) or mean.shape != rstd.shape \
                or mean.dtype != torch.float32 or rstd.dtype != torch.float32:
            raise ValueError("grad_y: of x's shape and type; mean, rstd: float32 [items, groups]")
        px = _at(x)
        gx = torch.empty_like(x)
        gw = torch.empty(shape.channels, dtype=weight.dtype if weight is not None else bias.dtype if bias is not None else torch.float32, device=x.device)
        gb = torch.empty_like(gw)
        ws, wsn = self.workspace(self.lib.goom_group_norm_backward_workspace_bytes(C.byref(shape)))
        self._check(self.lib.goom_group_norm_backward(self._ctx, C.byref(shape), px, _at(grad_y), _at(mean), _at(rstd), _at(weight), _at(bias), gx.data_ptr(),
                                                      gw.data_ptr(), gb.data_ptr(), _at(ws), wsn))
        return gx, gw, gb

    # ---- rotary positions
    def _rotary(self, q, k, positions, frequencies, interleaved, scale, flags):
        torch = self.torch
        code = _real_code(q)
        lead, (heads, dim) = tuple(q.shape[:-2]), tuple(q.shape[-2:])
        if q.dim() < 3 or positions.dtype != torch.int64 or tuple(positions.shape) != lead or frequencies.dtype != torch.float32 or frequencies.dim() != 1:
            raise ValueError("q: [..., heads, dim]; positions: int64 of q's leading shape; frequencies: float32 [pairs]")
        pq, q_token, q_head = _rows(q, "q")
        kv_heads, pk, k_token, k_head, out_k = 0, None, 0, 0, None
        if k is not None:
            if k.dtype != q.dtype or k.dim() != q.dim() or tuple(k.shape[:-2]) != lead or k.shape[-1] != dim or k.shape[-2] < 1:
                raise ValueError("k: [..., kv_heads, dim] of q's leading shape and type")
            kv_heads = k.shape[-2]
            pk, k_token, k_head = _rows(k, "k")
            out_k = torch.empty_like(k, memory_format=torch.contiguous_format)
        out_q = torch.empty_like(q, memory_format=torch.contiguous_format)
        shape = RotaryShape(math.prod(lead), heads, kv_heads, dim, frequencies.numel(), code, flags | (ROTARY_INTERLEAVED if interleaved else 0), scale, q_token, q_head, k_token, k_head)
        self._check(self.lib.goom_rotary(self._ctx, C.byref(shape), pq, pk, _at(positions), _at(frequencies), out_q.data_ptr(), _at(out_k)))
        return out_q, out_k

    def rotary(self, q, k, positions, frequencies, interleaved: bool = False, scale: float = 1.0):
        """q [..., heads, dim] and (unless None) k [..., kv_heads, dim] with their first 2 pairs entries turned by position times frequency, times
        scale; positions: int64 [...]; frequencies: float32 [pairs] (rotary_frequencies).  Pairs are (i, pairs + i), or (2 i, 2 i + 1) if interleaved;
        entries behind them are copied.  q and k may be slices of one projection's output."""
        return self._rotary(q, k, positions, frequencies, interleaved, scale, 0)

    def rotary_backward(self, grad_q, grad_k, positions, frequencies, interleaved: bool = False, scale: float = 1.0):
        """Gradients with respect to rotary's q and k."""
        return self._rotary(grad_q, grad_k, positions, frequencies, interleaved, scale, ROTARY_BACK)

    # ---- norms before and after a block
    def _block_norm(self, x, groups, weight, bias, scale, gate, residual, kind, activation, eps):
        act = ACTIVATIONS.get(activation)
        if x.dim() < 1 or act is None or kind not in NORM_KINDS:
            raise ValueError("x: [..., channels]; kind: one of " + ", ".join(NORM_KINDS) + "; activation: one of " + ", ".join(ACTIVATIONS))
        sh, dtype = x.shape, x.dtype
        channels, code = sh[-1], REAL_F32
        given = [p for p in (weight, bias, scale) if p is not None]
        if given:
            first, code = given[0].dtype, _real_code(given[0])
            for p in given:
                if p.dim() != 1 or p.shape[0] != channels:
                    raise ValueError("weight, bias and scale: [channels]")
                if p.dtype != first:
                    raise TypeError("weight, bias and scale have one type")
        for t in (gate, residual):
            if t is not None and (t.shape != sh or t.dtype != dtype):
                raise ValueError("gate and residual: of x's shape and type")
        return BlockNormShape(x.numel() // channels if channels else 0, channels, groups, _real_code(x), code, act, NORM_KINDS[kind], eps)

    def _stats(self, x, groups, kind, want):
        if not want:
            return None, None
        rstd = x.new_empty(x.shape[:-1] + (groups,), dtype=self.torch.float32)
        return self.torch.empty_like(rstd) if kind == "layer" else None, rstd

    def norm_after(self, x, groups: int = 1, weight=None, bias=None, scale=None, gate=None, residual=None, kind: str = "rms", activation: str = "silu", eps: float = 1e-5,
                   want_stats: bool = False):
        """residual + scale * (norm(x) * weight + bias) * act(gate): what closes a block whose output is x, [..., channels].  Every group of channels /
        groups neighbouring channels is normalised by itself, by its root mean square ("rms") or, less its mean, by its deviation ("layer").
        weight, bias, scale: [channels]; gate, residual: of x's shape.  want_stats: also mean (None for "rms") and rstd, float32 [..., groups]."""
        shape = self._block_norm(x, groups, weight, bias, scale, gate, residual, kind, activation, eps)
        px = _at(x)
        y = self.torch.empty_like(x)
        mean, rstd = self._stats(x, groups, kind, want_stats)
        self._check(self.lib.goom_norm_after(self._ctx, C.byref(shape), px, _at(gate), _at(residual), _at(weight), _at(bias), _at(scale), y.data_ptr(), _at(mean), _at(rstd)))
        return (y, mean, rstd) if want_stats else y

    def norm_before(self, x, groups: int = 1, weight=None, bias=None, scale=None, gate=None, residual=None, kind: str = "rms", activation: str = "silu", eps: float = 1e-5,
                    want_stats: bool = False):
        """h = residual + scale * x * act(gate), y = norm(h) * weight + bias: what opens the next block, x being the last one's output.  Returns y and
        h (x itself where there is nothing to add), with want_stats also mean (None for "rms") and rstd.  Arguments as for norm_after."""
        shape = self._block_norm(x, groups, weight, bias, scale, gate, residual, kind, activation, eps)
        px = _at(x)
        y = self.torch.empty_like(x)
        h = x if scale is None and gate is None and residual is None else self.torch.empty_like(x)
        mean, rstd = self._stats(x, groups, kind, want_stats)
        self._check(self.lib.goom_norm_before(self._ctx, C.byref(shape), px, _at(gate), _at(residual), _at(weight), _at(bias), _at(scale), None if h is x else h.data_ptr(),
                                              y.data_ptr(), _at(mean), _at(rstd)))
        return (y, h, mean, rstd) if want_stats else (y, h)

    def _norm_grads(self, x, grads, mean, rstd, groups, kind, params, gate):
        for t in grads:
            if t is not None and (t.shape != x.shape or t.dtype != x.dtype):
                raise ValueError("gradients and h: of x's shape and type")
        for t in (mean, rstd) if kind == "layer" else (rstd,):
            if t is None or tuple(t.shape) != tuple(x.shape[:-1]) + (groups,) or t.dtype != self.torch.float32:
                raise ValueError("mean (for layer), rstd: float32 [..., groups]")
        new = [None if p is None else self.torch.empty_like(p) for p in params]
        return self.torch.empty_like(x), None if gate is None else self.torch.empty_like(x), new

    def norm_after_backward(self, x, grad_y, mean, rstd, groups: int = 1, weight=None, bias=None, scale=None, gate=None, kind: str = "rms", activation: str = "silu"):
        """Gradients with respect to x, gate, weight, bias and scale (None for those that there are not); the residual's is grad_y."""
        shape = self._block_norm(x, groups, weight, bias, scale, gate, None, kind, activation, 0.0)
        gx, ggate, (gw, gb, gs) = self._norm_grads(x, (grad_y,), mean, rstd, groups, kind, (weight, bias, scale), gate)
        ws, wsn = self.workspace(self.lib.goom_block_norm_backward_workspace_bytes(C.byref(shape)))
        self._check(self.lib.goom_norm_after_backward(self._ctx, C.byref(shape), _at(x), _at(gate), _at(grad_y), _at(mean), _at(rstd), _at(weight), _at(bias), _at(scale),
                                                      gx.data_ptr(), _at(ggate), _at(gw), _at(gb), _at(gs), _at(ws), wsn))
        return gx, ggate, gw, gb, gs

    def norm_before_backward(self, x, h, grad_y, mean, rstd, grad_h=None, groups: int = 1, weight=None, bias=None, scale=None, gate=None, kind: str = "rms",
                             activation: str = "silu"):
        """Gradients with respect to residual, x, gate, weight, bias and scale (None for those that there are not; without gate and scale residual's and
        x's are one tensor), given those with respect to y and (None: none) to h."""
        shape = self._block_norm(x, groups, weight, bias, scale, gate, None, kind, activation, 0.0)
        gres, ggate, (gw, gb, gs) = self._norm_grads(x, (h, grad_y, grad_h), mean, rstd, groups, kind, (weight, bias, scale), gate)
        gx = gres if gate is None and scale is None else self.torch.empty_like(x)
        ws, wsn = self.workspace(self.lib.goom_block_norm_backward_workspace_bytes(C.byref(shape)))
        self._check(self.lib.goom_norm_before_backward(self._ctx, C.byref(shape), _at(x), _at(gate), _at(h), _at(grad_y), _at(grad_h), _at(mean), _at(rstd), _at(weight), _at(scale),
                                                       gres.data_ptr(), None if gx is gres else gx.data_ptr(), _at(ggate), _at(gw), _at(gb), _at(gs), _at(ws), wsn))
        return gres, gx, ggate, gw, gb, gs

    # ---- token embeddings
    def embedding(self, table, tokens, scale: float = 1.0, out=None):
        """scale * table[tokens], zeros for tokens outside the table (padding); table: [vocab, width], tokens: int64."""
        torch = self.torch
        if table.dim() != 2 or tokens.dtype != torch.int64:
            raise ValueError("table: [vocab, width]; tokens: int64")
        vocab, width = table.shape
        if out is None:
            out = torch.empty(tokens.shape + (width,), dtype=table.dtype, device=table.device)
        elif out.shape != tokens.shape + (width,) or out.dtype != table.dtype:
            raise ValueError("out: the tokens' shape with the table's width, of its type")
        self._check(self.lib.goom_embedding(self._ctx, _at(table), _at(tokens), _at(out), tokens.numel(), vocab, width, _real_code(table), scale))
        return out

    def embedding_backward(self, tokens, grad, vocab: int, scale: float = 1.0, dtype=None):
        """Gradient with respect to the table, [vocab, width], of type `dtype` (grad's if None), given grad: the tokens' shape with
        the width."""
        torch = self.torch
        if tokens.dtype != torch.int64 or grad.shape[:-1] != tokens.shape:
            raise ValueError("tokens: int64; grad: the tokens' shape with the width")
        n, width = tokens.numel(), grad.shape[-1]
        out = torch.empty((vocab, width), dtype=dtype or grad.dtype, device=grad.device)
        ws, wsn = self.workspace(self.lib.goom_embedding_backward_workspace_bytes(n, vocab, width))
        self._check(self.lib.goom_embedding_backward(self._ctx, _at(tokens), _at(grad), out.data_ptr(), n, vocab, width, _real_code(grad), _real_code(out), scale,
                                                     _at(ws), wsn))
        return out
