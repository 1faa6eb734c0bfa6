"""ctypes binding of libsparsecomm.so: same names as the C ABI, argument marshalling only.

torch is used for device memory and streams; every step of the path runs in the
library's CUDA kernels.  There is no CPU fallback: if the shared library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

SC_TOPK, SC_RANDK, SC_RANDBLOCK, SC_RANDBLOCK_WRAP = 0, 1, 2, 3
SCHEMES = {"topk": SC_TOPK, "randk": SC_RANDK, "randblock": SC_RANDBLOCK, "randblock_wrap": SC_RANDBLOCK_WRAP}

SC_BF16, SC_F16, SC_F32 = 0, 1, 2
SC_ACT_NONE, SC_ACT_RELU, SC_ACT_GELU, SC_ACT_GELU_TANH, SC_ACT_SILU = 0, 1, 2, 3, 4
ACTIVATIONS = {"none": SC_ACT_NONE, "relu": SC_ACT_RELU, "gelu": SC_ACT_GELU, "gelu_tanh": SC_ACT_GELU_TANH, "silu": SC_ACT_SILU}
CHECKPOINT_GROUP = 32
_TYPES = {torch.bfloat16: SC_BF16, torch.float16: SC_F16, torch.float32: SC_F32}

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsparsecomm.so")

EXPORTS = ["sc_create", "sc_destroy", "sc_strerror", "sc_sync_status", "sc_set_gamma", "sc_scratch_bytes", "sc_launch_count",
           "sc_topk_path_counts", "sc_topk_path_detail", "sc_debug_set_poll_limits", "sc_debug_wait_probe", "sc_profile", "sc_profile_kinds", "sc_profile_name", "sc_profile_read",
           "sc_compress", "sc_compress_batch", "sc_aggregate", "sc_aggregate_shared", "sc_aggregate_static", "sc_aggregate_apply",
           "sc_aggregate_apply_shared", "sc_step", "sc_step_apply", "sc_step_host",
           "sc_layer_reserve", "sc_debug_layer_tiles", "sc_checkpoint_pack", "sc_checkpoint_unpack", "sc_activation_grad", "sc_linear", "sc_linear_grad_input",
           "sc_linear_grad_weight", "sc_quantize", "sc_dequantize", "sc_linear_quantized", "sc_dropout", "sc_rms_norm", "sc_rms_norm_grad"]


_LAYER_CALLS = ("sc_checkpoint_pack", "sc_checkpoint_unpack", "sc_activation_grad", "sc_linear", "sc_linear_grad_input", "sc_linear_grad_weight",
                "sc_quantize", "sc_dequantize", "sc_linear_quantized", "sc_dropout", "sc_rms_norm", "sc_rms_norm_grad")


class ScSegment(ctypes.Structure):
    _fields_ = [("offset", ctypes.c_uint64), ("n", ctypes.c_uint64), ("k", ctypes.c_uint64)]


class SparseCommError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {strerror(code)} ({code})")
        self.code = code


_lib: Optional[ctypes.CDLL] = None


def load_library() -> ctypes.CDLL:
    """Loads the CUDA library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2009_09271_b200.build` "
                           "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, u64, sz, ci = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_int
    lib.sc_create.argtypes = [ctypes.POINTER(vp), sz, ci, ci]
    lib.sc_create.restype = ci
    lib.sc_destroy.argtypes = [vp]
    lib.sc_destroy.restype = None
    lib.sc_strerror.argtypes = [ci]
    lib.sc_strerror.restype = ctypes.c_char_p
    lib.sc_set_gamma.argtypes = [vp, ctypes.c_float]
    lib.sc_set_gamma.restype = ci
    lib.sc_sync_status.argtypes = [vp, vp]
    lib.sc_sync_status.restype = ci
    lib.sc_scratch_bytes.argtypes = [vp]
    lib.sc_scratch_bytes.restype = sz
    lib.sc_launch_count.argtypes = [vp]
    lib.sc_launch_count.restype = u64
    lib.sc_topk_path_counts.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_uint32)]
    lib.sc_topk_path_counts.restype = ci
    lib.sc_topk_path_detail.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_uint32)]
    lib.sc_topk_path_detail.restype = ci
    lib.sc_debug_set_poll_limits.argtypes = [vp, ctypes.c_uint32, ctypes.c_uint32]
    lib.sc_debug_set_poll_limits.restype = ci
    lib.sc_debug_wait_probe.argtypes = [vp, ci, vp]
    lib.sc_debug_wait_probe.restype = ci
    lib.sc_profile.argtypes = [vp, ci]
    lib.sc_profile.restype = ci
    lib.sc_profile_kinds.argtypes = []
    lib.sc_profile_kinds.restype = ci
    lib.sc_profile_name.argtypes = [ci]
    lib.sc_profile_name.restype = ctypes.c_char_p
    lib.sc_profile_read.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(u64)]
    lib.sc_profile_read.restype = ci
    lib.sc_compress.argtypes = [vp, ci, vp, vp, sz, sz, u64, vp, vp, vp]
    lib.sc_compress.restype = ci
    lib.sc_compress_batch.argtypes = [vp, ci, ci, vp, vp, sz, ctypes.POINTER(ScSegment), ci,
                                      ctypes.POINTER(u64), vp, vp, vp]
    lib.sc_compress_batch.restype = ci
    lib.sc_aggregate.argtypes = [vp, ci, vp, vp, sz, sz, vp, vp]
    lib.sc_aggregate.restype = ci
    lib.sc_aggregate_shared.argtypes = [vp, ci, vp, vp, sz, sz, vp, vp]
    lib.sc_aggregate_shared.restype = ci
    for name in ("sc_aggregate_apply", "sc_aggregate_apply_shared"):
        getattr(lib, name).argtypes = [vp, ci, vp, vp, sz, sz, vp, vp]
        getattr(lib, name).restype = ci
    lib.sc_aggregate_static.argtypes = [ci, vp, vp, sz, sz, vp, vp]
    lib.sc_aggregate_static.restype = ci
    lib.sc_step.argtypes = [vp, ci, ci, vp, vp, sz, ctypes.POINTER(ScSegment), ci, ctypes.POINTER(u64),
                            vp, vp, vp, vp]
    lib.sc_step.restype = ci
    lib.sc_step_apply.argtypes = lib.sc_step.argtypes
    lib.sc_step_apply.restype = ci
    lib.sc_step_host.argtypes = [vp, ci, ci, vp, vp, sz, ctypes.POINTER(ScSegment), ci, ctypes.POINTER(u64),
                                 vp, vp]
    lib.sc_step_host.restype = ci
    lib.sc_layer_reserve.argtypes = [vp, sz, sz, sz]
    lib.sc_debug_layer_tiles.argtypes = [vp, ci, ci, ci]
    lib.sc_checkpoint_pack.argtypes = [vp, ci, vp, sz, sz, sz, vp, vp, vp]
    lib.sc_checkpoint_unpack.argtypes = [vp, ci, vp, vp, sz, sz, vp, sz, vp]
    lib.sc_activation_grad.argtypes = [vp, ci, ci, vp, sz, vp, vp, sz, sz, vp, sz, vp, ci, vp]
    lib.sc_linear.argtypes = [vp, ci, ci, vp, sz, vp, sz, vp, vp, sz, sz, sz, sz, vp, sz, vp, vp, vp]
    lib.sc_linear_grad_input.argtypes = [vp, ci, ci, vp, sz, vp, sz, vp, sz, vp, vp, sz, sz, sz, vp, sz, vp]
    lib.sc_linear_grad_weight.argtypes = [vp, ci, vp, sz, vp, sz, vp, vp, sz, sz, sz, vp, sz, ci, vp]
    lib.sc_quantize.argtypes = [vp, ci, vp, sz, sz, sz, vp, sz, vp, vp]
    lib.sc_dequantize.argtypes = [vp, ci, vp, sz, vp, sz, sz, vp, sz, vp]
    lib.sc_linear_quantized.argtypes = [vp, ci, ci, vp, sz, vp, vp, sz, vp, vp, vp, sz, sz, sz, sz, vp, sz, vp, vp, vp]
    lib.sc_dropout.argtypes = [vp, ci, vp, sz, vp, sz, ctypes.c_double, u64, sz, sz, vp, sz, vp]
    lib.sc_rms_norm.argtypes = [vp, ci, vp, sz, vp, sz, vp, ctypes.c_float, ctypes.c_double, u64, sz, sz, vp, sz, vp, sz, vp, sz, vp, vp]
    lib.sc_rms_norm_grad.argtypes = [vp, ci, vp, sz, vp, sz, vp, ctypes.c_float, vp, sz, ctypes.c_double, u64, sz, sz, vp, sz, vp, sz, vp, ci, vp]
    for name in ("sc_layer_reserve", "sc_debug_layer_tiles") + _LAYER_CALLS:
        getattr(lib, name).restype = ci
    _lib = lib
    return lib


def strerror(code: int) -> str:
    return load_library().sc_strerror(code).decode()


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# the current stream's handle, without the Stream object that torch.cuda.current_stream() makes around it (3 us)
_raw_stream, _current_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(_current_device()) or None
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


def _segments(segs: Sequence) -> "ctypes.Array[ScSegment]":
    arr = (ScSegment * max(len(segs), 1))()
    for i, s in enumerate(segs):
        off, n, k = (s.offset, s.n, s.k) if hasattr(s, "offset") else s
        arr[i] = ScSegment(int(off), int(n), int(k))
    return arr


def _seeds(seeds: Sequence[int]):
    return (ctypes.c_uint64 * max(len(seeds), 1))(*[int(s) & 0xFFFFFFFFFFFFFFFF for s in seeds])


def _check(code: int, what: str) -> None:
    if code != 0:
        raise SparseCommError(code, what)


def _want(t: torch.Tensor, dtype, name: str, cuda: bool = True) -> None:
    if t.dtype != dtype or not t.is_contiguous() or (cuda and not t.is_cuda):
        raise TypeError(f"{name}: expected a contiguous {'CUDA ' if cuda else ''}{dtype} tensor")


def _matrix(t: torch.Tensor, rows: int, cols: int, dtype, name: str) -> int:
    """Checks a CUDA matrix [rows, cols] whose rows are contiguous; returns the distance between rows in elements."""
    if t.dtype is dtype and t.is_cuda and t.shape == (rows, cols):
        ld, step = t.stride()
        if ld >= cols and step == 1:
            return ld
        if (step == 1 or cols <= 1) and (ld >= cols or rows <= 1):
            return max(ld, cols)
        raise TypeError(f"{name}: the last dimension must be contiguous and rows must not overlap")
    if t.dtype != dtype or not t.is_cuda or t.dim() != 2:
        raise TypeError(f"{name}: expected a 2-D CUDA {dtype} tensor")
    raise ValueError(f"{name}: expected shape {(rows, cols)}, got {tuple(t.shape)}")


def _vector(t: torch.Tensor, n: int, dtype, name: str) -> None:
    if t.dtype is dtype and t.is_cuda and t.numel() == n and t.is_contiguous():
        return
    _want(t, dtype, name)
    if t.numel() != n:
        raise ValueError(f"{name}: expected {n} elements, got {t.numel()}")


def _kept(q, scales, rows: int, cols: int) -> None:
    """Checks a checkpoint of a [rows, cols] matrix; matrices have its shape, views of other dimensions its number of elements."""
    groups = -(-cols // CHECKPOINT_GROUP)
    if (q is not None and scales is not None and q.dtype is torch.int8 and scales.dtype is torch.uint8 and q.is_cuda and scales.is_cuda
            and q.shape == (rows, cols) and scales.shape == (rows, groups) and q.is_contiguous() and scales.is_contiguous()):
        return
    if q is None or scales is None:
        raise ValueError("q and scales: a checkpoint is both or neither")
    _vector(q, rows * cols, torch.int8, "q")
    _vector(scales, rows * groups, torch.uint8, "scales")
    for t, want, name in ((q, (rows, cols), "q"), (scales, (rows, groups), "scales")):
        if t.dim() == 2 and t.shape != want:
            raise ValueError(f"{name}: expected shape {want}, got {tuple(t.shape)}")


def _layer_type(t: torch.Tensor, name: str, f32: bool = False) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None or (kind == SC_F32 and not f32):
        raise TypeError(f"{name}: expected bfloat16 or float16{' or float32' if f32 else ''}, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{name}: expected a matrix, got shape {tuple(t.shape)}")
    return kind


def checkpoint_buffers(rows: int, cols: int, device="cuda"):
    """(q, scales) for the 8-bit checkpoint of a [rows, cols] matrix."""
    return (torch.empty(rows, cols, dtype=torch.int8, device=device),
            torch.empty(rows, -(-cols // CHECKPOINT_GROUP), dtype=torch.uint8, device=device))


def quantized_buffers(rows: int, cols: int, device="cuda"):
    """(q, scales) for the 8-bit rows of a [rows, cols] matrix: int8, and one float32 a row."""
    return torch.empty(rows, cols, dtype=torch.int8, device=device), torch.empty(rows, dtype=torch.float32, device=device)


def _eight_bit_rows(q, scales, rows: int, cols: int, name: str = "q", scales_name: str = "scales") -> int:
    """Checks 8-bit rows [rows, cols] and their scales; returns the distance between rows."""
    if q is None or scales is None:
        raise ValueError(f"{name} and {scales_name}: 8-bit rows are both or neither")
    _vector(scales, rows, torch.float32, scales_name)
    return _matrix(q, rows, cols, torch.int8, name)


def _probability(p: float) -> float:
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"p: expected a probability, got {p}")
    return p


STATIC_MAX_N, STATIC_MAX_W = 1 << 24, 64


def sc_aggregate_static(W: int, vals, idx, k: int, n: int, out, stream=None) -> None:
    """sc_aggregate without a Context, for callers that may not allocate device memory (the
    library's own scratch for it is a fixed device array).  Limits: W <= 64, n <= 2**24.
    All calls on one GPU share that scratch, so calls that may overlap on the GPU race."""
    lib = load_library()
    _want(vals, torch.float32, "vals"), _want(idx, torch.int32, "idx"), _want(out, torch.float32, "out")
    if vals.numel() < W * k or idx.numel() < W * k or out.numel() < n:
        raise ValueError("buffer sizes do not match W, k and n")
    code = lib.sc_aggregate_static(W, _ptr(vals), _ptr(idx), k, n, _ptr(out), _stream(stream))
    if code != 0:
        raise SparseCommError(code, f"sc_aggregate_static (limits: W <= {STATIC_MAX_W}, n <= {STATIC_MAX_N})")


_calls = None


def _layer_calls(lib):
    """The layer operators' entry points: from the compiled caller where it was built, else through ctypes (same arguments)."""
    global _calls
    if _calls is None:
        try:
            from . import _sc_calls
            _sc_calls.bind(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _LAYER_CALLS))
            _calls = _sc_calls
        except ImportError:
            _calls = lib
    return _calls


def _tensor_calls(calls):
    """The compiled caller's functions that take tensors, where it was built for this torch; without them (None) the binding's own checks do."""
    built_for = getattr(calls, "torch_version", None)
    return calls if built_for is not None and torch.__version__.split("+")[0] == built_for.split("+")[0] else None


class Context:
    """Owns an sc_ctx (scratch memory on the current CUDA device)."""

    def __init__(self, max_n: int, max_W: int = 1, max_segments: int = 1):
        lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("sparsecomm needs a CUDA device (there is no CPU fallback)")
        torch.cuda.init()
        torch.zeros(1, device="cuda")          # make sure the primary context exists
        self._lib = lib
        self._h = ctypes.c_void_p()
        _check(lib.sc_create(ctypes.byref(self._h), max_n, max_W, max_segments), "sc_create")
        self._layer, self._handle = _layer_calls(lib), self._h.value
        self._device = torch.cuda.current_device()
        self._direct = _tensor_calls(self._layer)

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h:
            self._lib.sc_destroy(self._h)
            self._h = self._handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def scratch_bytes(self) -> int:
        return self._lib.sc_scratch_bytes(self._h)

    @property
    def launch_count(self) -> int:
        return self._lib.sc_launch_count(self._h)

    def sc_topk_path_counts(self, stream=None) -> tuple:
        """(small-segment radix select, one-pass path, radix select after a missed bracket)."""
        out = (ctypes.c_uint32 * 3)()
        _check(self._lib.sc_topk_path_counts(self._h, _stream(stream), out), "sc_topk_path_counts")
        return tuple(out)

    PATH_DETAIL = ("short", "one_pass", "radix_after_failure", "tie_key_seen", "ties_admitted",
                   "failed_list_overflow", "failed_bracket", "failed_short_list")

    def sc_topk_path_detail(self, stream=None) -> dict:
        out = (ctypes.c_uint32 * 8)()
        _check(self._lib.sc_topk_path_detail(self._h, _stream(stream), out), "sc_topk_path_detail")
        return dict(zip(self.PATH_DETAIL, out))

    def sc_debug_set_poll_limits(self, lookback_polls: int = 0, barrier_polls: int = 0) -> None:
        _check(self._lib.sc_debug_set_poll_limits(self._h, lookback_polls, barrier_polls), "sc_debug_set_poll_limits")

    def sc_debug_wait_probe(self, which: int, stream=None) -> None:
        _check(self._lib.sc_debug_wait_probe(self._h, which, _stream(stream)), "sc_debug_wait_probe")

    def sc_profile(self, enable: bool) -> None:
        _check(self._lib.sc_profile(self._h, 1 if enable else 0), "sc_profile")

    def sc_profile_read(self) -> dict:
        """{kernel kind: (milliseconds, launches)} since sc_profile(True)."""
        kinds = self._lib.sc_profile_kinds()
        ms = (ctypes.c_double * kinds)()
        cnt = (ctypes.c_uint64 * kinds)()
        _check(self._lib.sc_profile_read(self._h, ms, cnt), "sc_profile_read")
        return {self._lib.sc_profile_name(i).decode(): (ms[i], cnt[i]) for i in range(kinds)}

    # -- the C ABI, one method per entry point ---------------------------------
    def sc_set_gamma(self, gamma: float) -> None:
        _check(self._lib.sc_set_gamma(self._h, float(gamma)), "sc_set_gamma")

    def sc_sync_status(self, stream=None) -> int:
        return self._lib.sc_sync_status(self._h, _stream(stream))

    def sc_compress(self, scheme: int, grad, residual, k: int, seed: int, out_vals, out_idx, stream=None) -> None:
        _want(grad, torch.float32, "grad"), _want(residual, torch.float32, "residual")
        _want(out_vals, torch.float32, "out_vals"), _want(out_idx, torch.int32, "out_idx")
        if residual.numel() != grad.numel() or out_vals.numel() < k or out_idx.numel() < k:
            raise ValueError("buffer sizes do not match n and k")
        _check(self._lib.sc_compress(self._h, scheme, _ptr(grad), _ptr(residual), grad.numel(), k,
                                     int(seed) & 0xFFFFFFFFFFFFFFFF, _ptr(out_vals), _ptr(out_idx),
                                     _stream(stream)), "sc_compress")

    def sc_compress_batch(self, scheme: int, grads, residuals, segs, seeds, out_vals, out_idx, stream=None) -> None:
        W, n = grads.shape
        _want(grads, torch.float32, "grads"), _want(residuals, torch.float32, "residuals")
        _want(out_vals, torch.float32, "out_vals"), _want(out_idx, torch.int32, "out_idx")
        K = sum((s.k if hasattr(s, "k") else s[2]) for s in segs)
        if residuals.shape != grads.shape or len(seeds) != W or out_vals.numel() < W * K or out_idx.numel() < W * K:
            raise ValueError("buffer sizes do not match W, n and the segment table")
        _check(self._lib.sc_compress_batch(self._h, scheme, W, _ptr(grads), _ptr(residuals), n, _segments(segs),
                                           len(segs), _seeds(seeds), _ptr(out_vals), _ptr(out_idx),
                                           _stream(stream)), "sc_compress_batch")

    def sc_aggregate(self, W: int, vals, idx, k: int, n: int, out, stream=None) -> None:
        _want(vals, torch.float32, "vals"), _want(idx, torch.int32, "idx"), _want(out, torch.float32, "out")
        if vals.numel() < W * k or idx.numel() < W * k or out.numel() < n:
            raise ValueError("buffer sizes do not match W, k and n")
        _check(self._lib.sc_aggregate(self._h, W, _ptr(vals), _ptr(idx), k, n, _ptr(out), _stream(stream)),
               "sc_aggregate")

    def sc_aggregate_shared(self, W: int, vals, idx, k: int, n: int, out, stream=None) -> None:
        _want(vals, torch.float32, "vals"), _want(idx, torch.int32, "idx"), _want(out, torch.float32, "out")
        if vals.numel() < W * k or idx.numel() < k or out.numel() < n:
            raise ValueError("buffer sizes do not match W, k and n")
        _check(self._lib.sc_aggregate_shared(self._h, W, _ptr(vals), _ptr(idx), k, n, _ptr(out), _stream(stream)),
               "sc_aggregate_shared")

    def sc_aggregate_apply(self, W: int, vals, idx, k: int, n: int, x, stream=None, shared: bool = False) -> None:
        """x <- x - average of the W messages, touching only the coordinates that were sent."""
        _want(vals, torch.float32, "vals"), _want(idx, torch.int32, "idx"), _want(x, torch.float32, "x")
        if vals.numel() < W * k or idx.numel() < (k if shared else W * k) or x.numel() < n:
            raise ValueError("buffer sizes do not match W, k and n")
        fn = self._lib.sc_aggregate_apply_shared if shared else self._lib.sc_aggregate_apply
        _check(fn(self._h, W, _ptr(vals), _ptr(idx), k, n, _ptr(x), _stream(stream)), "sc_aggregate_apply")

    def sc_step(self, scheme: int, grads, residuals, segs, seeds, out_vals, out_idx, out, stream=None) -> None:
        W, n = grads.shape
        _want(grads, torch.float32, "grads"), _want(residuals, torch.float32, "residuals")
        _want(out_vals, torch.float32, "out_vals"), _want(out_idx, torch.int32, "out_idx")
        _want(out, torch.float32, "out")
        K = sum((s.k if hasattr(s, "k") else s[2]) for s in segs)
        if (residuals.shape != grads.shape or len(seeds) != W or out_vals.numel() < W * K
                or out_idx.numel() < W * K or out.numel() < n):
            raise ValueError("buffer sizes do not match W, n and the segment table")
        _check(self._lib.sc_step(self._h, scheme, W, _ptr(grads), _ptr(residuals), n, _segments(segs), len(segs),
                                 _seeds(seeds), _ptr(out_vals), _ptr(out_idx), _ptr(out), _stream(stream)),
               "sc_step")

    def sc_step_apply(self, scheme: int, grads, residuals, segs, seeds, out_vals, out_idx, x, stream=None) -> None:
        """Compress W workers, then x <- x - average of their messages at the sent coordinates only."""
        W, n = grads.shape
        _want(grads, torch.float32, "grads"), _want(residuals, torch.float32, "residuals")
        _want(out_vals, torch.float32, "out_vals"), _want(out_idx, torch.int32, "out_idx")
        _want(x, torch.float32, "x")
        K = sum((s.k if hasattr(s, "k") else s[2]) for s in segs)
        if (residuals.shape != grads.shape or len(seeds) != W or out_vals.numel() < W * K
                or out_idx.numel() < W * K or x.numel() < n):
            raise ValueError("buffer sizes do not match W, n and the segment table")
        _check(self._lib.sc_step_apply(self._h, scheme, W, _ptr(grads), _ptr(residuals), n, _segments(segs), len(segs),
                                       _seeds(seeds), _ptr(out_vals), _ptr(out_idx), _ptr(x), _stream(stream)),
               "sc_step_apply")

    def sc_step_host(self, scheme: int, h_grads, residuals, segs, seeds, h_out, stream=None) -> None:
        W, n = h_grads.shape
        _want(h_grads, torch.float32, "h_grads", cuda=False), _want(h_out, torch.float32, "h_out", cuda=False)
        _want(residuals, torch.float32, "residuals")
        if h_grads.is_cuda or h_out.is_cuda:
            raise TypeError("h_grads and h_out must be host tensors")
        if residuals.shape != h_grads.shape or len(seeds) != W or h_out.numel() < n:
            raise ValueError("buffer sizes do not match W and n")
        _check(self._lib.sc_step_host(self._h, scheme, W, _ptr(h_grads), _ptr(residuals), n, _segments(segs),
                                      len(segs), _seeds(seeds), _ptr(h_out), _stream(stream)), "sc_step_host")

    # -- layer operators ---------------------------------------------------------
    def sc_layer_reserve(self, M: int, N: int, K: int) -> None:
        """Allocates ahead the workspace of layer calls of at most these sizes (before a stream capture, for instance)."""
        _check(self._lib.sc_layer_reserve(self._h, M, N, K), "sc_layer_reserve")

    def sc_debug_layer_tiles(self, rows: int = 0, cols: int = 0, parts: int = 0) -> None:
        _check(self._lib.sc_debug_layer_tiles(self._h, rows, cols, parts), "sc_debug_layer_tiles")

    def sc_checkpoint_pack(self, x, q, scales, stream=None) -> None:
        """q, scales <- the 8-bit checkpoint of x [rows, cols] (bfloat16, float16 or float32)."""
        kind = _layer_type(x, "x", f32=True)
        rows, cols = x.shape
        ldx = _matrix(x, rows, cols, x.dtype, "x")
        _kept(q, scales, rows, cols)
        _check(self._layer.sc_checkpoint_pack(self._handle, kind, _ptr(x), ldx, rows, cols, _ptr(q), _ptr(scales), _stream(stream)),
               "sc_checkpoint_pack")

    def sc_checkpoint_unpack(self, q, scales, out, stream=None) -> None:
        """out [rows, cols] <- the values that a checkpoint holds."""
        kind = _layer_type(out, "out", f32=True)
        rows, cols = out.shape
        ldo = _matrix(out, rows, cols, out.dtype, "out")
        _kept(q, scales, rows, cols)
        _check(self._layer.sc_checkpoint_unpack(self._handle, kind, _ptr(q), _ptr(scales), rows, cols, _ptr(out), ldo, _stream(stream)),
               "sc_checkpoint_unpack")

    def sc_activation_grad(self, act: int, dy, q, scales, dz, db=None, accumulate: bool = False, stream=None) -> None:
        """dz <- dy * act'(z^), db <- (db +) column sums of dz; z^ is the checkpoint (q, scales), unused for SC_ACT_NONE.
        dz or db may be None; dz may be dy."""
        kind = _layer_type(dy, "dy")
        rows, cols = dy.shape
        lddy = _matrix(dy, rows, cols, dy.dtype, "dy")
        if act != SC_ACT_NONE:
            _kept(q, scales, rows, cols)
        lddz = cols if dz is None else _matrix(dz, rows, cols, dy.dtype, "dz")
        if db is not None:
            _vector(db, cols, torch.float32, "db")
        _check(self._layer.sc_activation_grad(self._handle, kind, act, _ptr(dy), lddy, _ptr(q), _ptr(scales), rows, cols, _ptr(dz), lddz,
                                            _ptr(db), 1 if accumulate else 0, _stream(stream)), "sc_activation_grad")

    def sc_linear(self, act: int, x, w, y, bias=None, residual=None, q=None, scales=None, stream=None) -> None:
        """y [M, N] <- act(x W^T + bias) + residual, x [M, K], w [N, K]; q, scales <- the checkpoint of x W^T + bias."""
        kind = _layer_type(x, "x")
        M, K = x.shape
        ldx = _matrix(x, M, K, x.dtype, "x")
        if w.dim() != 2:
            raise ValueError("w: expected a matrix")
        N = w.shape[0]
        ldw = _matrix(w, N, K, x.dtype, "w")
        ldy = _matrix(y, M, N, x.dtype, "y")
        if bias is not None:
            _vector(bias, N, x.dtype, "bias")
        ldr = N if residual is None else _matrix(residual, M, N, x.dtype, "residual")
        if q is not None or scales is not None:
            _kept(q, scales, M, N)
        _check(self._layer.sc_linear(self._handle, kind, act, _ptr(x), ldx, _ptr(w), ldw, _ptr(bias), _ptr(residual), ldr, M, N, K,
                                   _ptr(y), ldy, _ptr(q), _ptr(scales), _stream(stream)), "sc_linear")

    def sc_linear_grad_input(self, dz, w, dx, residual=None, act: int = SC_ACT_NONE, q=None, scales=None, stream=None) -> None:
        """dx [M, K] <- (dz W + residual) * act'(z^), dz [M, N], w [N, K], z^ [M, K] the checkpoint below the layer."""
        kind = _layer_type(dz, "dz")
        M, N = dz.shape
        lddz = _matrix(dz, M, N, dz.dtype, "dz")
        if w.dim() != 2:
            raise ValueError("w: expected a matrix")
        K = w.shape[1]
        ldw = _matrix(w, N, K, dz.dtype, "w")
        lddx = _matrix(dx, M, K, dz.dtype, "dx")
        ldr = K if residual is None else _matrix(residual, M, K, dz.dtype, "residual")
        if act != SC_ACT_NONE:
            _kept(q, scales, M, K)
        _check(self._layer.sc_linear_grad_input(self._handle, kind, act, _ptr(dz), lddz, _ptr(w), ldw, _ptr(residual), ldr, _ptr(q), _ptr(scales),
                                              M, N, K, _ptr(dx), lddx, _stream(stream)), "sc_linear_grad_input")

    def sc_linear_grad_weight(self, dz, dw, x=None, q=None, scales=None, accumulate: bool = False, stream=None) -> None:
        """dw [N, K] fp32 <- (dw +) dz^T x, dz [M, N]; the layer's input is given as x [M, K] or as its checkpoint (q, scales)."""
        kind = _layer_type(dz, "dz")
        M, N = dz.shape
        lddz = _matrix(dz, M, N, dz.dtype, "dz")
        if dw.dim() != 2:
            raise ValueError("dw: expected a matrix")
        K = dw.shape[1]
        lddw = _matrix(dw, N, K, torch.float32, "dw")
        if (x is None) == (q is None):
            raise ValueError("the layer's input is given once: as x, or as a checkpoint")
        ldx = K
        if x is not None:
            ldx = _matrix(x, M, K, dz.dtype, "x")
        else:
            _kept(q, scales, M, K)
        _check(self._layer.sc_linear_grad_weight(self._handle, kind, _ptr(dz), lddz, _ptr(x), ldx, _ptr(q), _ptr(scales), M, N, K,
                                               _ptr(dw), lddw, 1 if accumulate else 0, _stream(stream)), "sc_linear_grad_weight")

    # -- 8-bit rows, norm, dropout -----------------------------------------------
    def _here(self, *tensors) -> None:
        """The tensors (None: not given) are on the context's device."""
        for t in tensors:
            if t is not None and t.get_device() != self._device:
                raise ValueError(f"tensors must be on the context's device, cuda:{self._device}; got one on {t.device}")

    def _queue(self, stream) -> Optional[int]:
        """The given stream, or the current one of the context's device, whichever device is current."""
        if stream is None and _raw_stream is not None:
            return _raw_stream(self._device) or None
        return _stream(torch.cuda.current_stream(self._device) if stream is None else stream)

    def sc_quantize(self, x, q, scales, stream=None) -> None:
        """q, scales <- the 8-bit rows of x [rows, cols] (bfloat16, float16 or float32)."""
        if self._direct is not None:
            code = self._direct.quantize(self._handle, self._device, x, q, scales, self._queue(stream))
            if code is not None:
                return _check(code, "sc_quantize") if code else None
        kind = _layer_type(x, "x", f32=True)
        rows, cols = x.shape
        ldx = _matrix(x, rows, cols, x.dtype, "x")
        ldq = _eight_bit_rows(q, scales, rows, cols)
        self._here(x, q, scales)
        _check(self._layer.sc_quantize(self._handle, kind, _ptr(x), ldx, rows, cols, _ptr(q), ldq, _ptr(scales), self._queue(stream)), "sc_quantize")

    def sc_dequantize(self, q, scales, out, stream=None) -> None:
        """out [rows, cols] <- the values of 8-bit rows."""
        if self._direct is not None:
            code = self._direct.dequantize(self._handle, self._device, q, scales, out, self._queue(stream))
            if code is not None:
                return _check(code, "sc_dequantize") if code else None
        kind = _layer_type(out, "out", f32=True)
        rows, cols = out.shape
        ldo = _matrix(out, rows, cols, out.dtype, "out")
        ldq = _eight_bit_rows(q, scales, rows, cols)
        self._here(q, scales, out)
        _check(self._layer.sc_dequantize(self._handle, kind, _ptr(q), ldq, _ptr(scales), rows, cols, _ptr(out), ldo, self._queue(stream)), "sc_dequantize")

    def sc_linear_quantized(self, act: int, x, x_scales, w, w_scales, y, bias=None, residual=None, q=None, scales=None, stream=None) -> None:
        """y [M, N] <- act(z) + residual, z = (x W^T) x_scales w_scales + bias with 8-bit rows x [M, K] and w [N, K]; q, scales <- the
        checkpoint of z."""
        if self._direct is not None:
            code = self._direct.linear_quantized(self._handle, self._device, act, x, x_scales, w, w_scales, y, bias, residual, q, scales, self._queue(stream))
            if code is not None:
                return _check(code, "sc_linear_quantized") if code else None
        kind = _layer_type(y, "y")
        M, N = y.shape
        ldy = _matrix(y, M, N, y.dtype, "y")
        if x is None or x.dim() != 2:
            raise ValueError("x: expected a matrix")
        K = x.shape[1]
        ldx = _eight_bit_rows(x, x_scales, M, K, "x", "x_scales")
        ldw = _eight_bit_rows(w, w_scales, N, K, "w", "w_scales")
        if bias is not None:
            _vector(bias, N, y.dtype, "bias")
        ldr = N if residual is None else _matrix(residual, M, N, y.dtype, "residual")
        if q is not None or scales is not None:
            _kept(q, scales, M, N)
        self._here(x, x_scales, w, w_scales, y, bias, residual, q, scales)
        _check(self._layer.sc_linear_quantized(self._handle, kind, act, _ptr(x), ldx, _ptr(x_scales), _ptr(w), ldw, _ptr(w_scales), _ptr(bias),
                                               _ptr(residual), ldr, M, N, K, _ptr(y), ldy, _ptr(q), _ptr(scales), self._queue(stream)),
               "sc_linear_quantized")

    def sc_dropout(self, x, y, p: float, seed: int, residual=None, stream=None) -> None:
        """y <- residual + dropout(x): each element kept with probability 1 - p and scaled by its reciprocal, by the mask that (seed, row,
        column) give.  The gradient is the same call on dy, without a residual.  y may be x or residual.  A captured call keeps its seed."""
        if self._direct is not None:
            code = self._direct.dropout(self._handle, self._device, x, y, p, seed, residual, self._queue(stream))
            if code is not None:
                return _check(code, "sc_dropout") if code else None
        kind = _layer_type(x, "x")
        rows, cols = x.shape
        ldx = _matrix(x, rows, cols, x.dtype, "x")
        ldy = _matrix(y, rows, cols, x.dtype, "y")
        ldr = cols if residual is None else _matrix(residual, rows, cols, x.dtype, "residual")
        self._here(x, y, residual)
        _check(self._layer.sc_dropout(self._handle, kind, _ptr(x), ldx, _ptr(residual), ldr, _probability(p), int(seed) & 0xFFFFFFFFFFFFFFFF, rows, cols,
                                      _ptr(y), ldy, self._queue(stream)), "sc_dropout")

    def sc_rms_norm(self, x, gamma, eps: float, y=None, q=None, scales=None, residual=None, h=None, p: float = 0.0, seed: int = 0, stream=None) -> None:
        """h <- residual + dropout(x; p, seed); y, or its 8-bit rows q and scales, or both <- h / sqrt(mean(h^2) + eps) * gamma."""
        if self._direct is not None:
            code = self._direct.rms_norm(self._handle, self._device, x, gamma, eps, y, q, scales, residual, h, p, seed, self._queue(stream))
            if code is not None:
                return _check(code, "sc_rms_norm") if code else None
        kind = _layer_type(x, "x")
        rows, cols = x.shape
        dtype = x.dtype
        ldx = _matrix(x, rows, cols, dtype, "x")
        _vector(gamma, cols, dtype, "gamma")
        if y is None and q is None:
            raise ValueError("y, or q and scales, must be given")
        ldy = cols if y is None else _matrix(y, rows, cols, dtype, "y")
        ldq = cols if q is None and scales is None else _eight_bit_rows(q, scales, rows, cols)
        ldr = cols if residual is None else _matrix(residual, rows, cols, dtype, "residual")
        ldh = cols if h is None else _matrix(h, rows, cols, dtype, "h")
        self._here(x, gamma, y, q, scales, residual, h)
        _check(self._layer.sc_rms_norm(self._handle, kind, _ptr(x), ldx, _ptr(residual), ldr, _ptr(gamma), eps, _probability(p),
                                       int(seed) & 0xFFFFFFFFFFFFFFFF, rows, cols, _ptr(h), ldh, _ptr(y), ldy, _ptr(q), ldq, _ptr(scales),
                                       self._queue(stream)), "sc_rms_norm")

    def sc_rms_norm_grad(self, dy, h, gamma, eps: float, dh=None, dgamma=None, residual=None, dx=None, p: float = 0.0, seed: int = 0,
                         accumulate: bool = False, stream=None) -> None:
        """dh <- residual + the norm's gradient at h; dx <- dropout(dh; p, seed); dgamma <- (dgamma +) column sums of dy h / rms(h), float32."""
        if self._direct is not None:
            code = self._direct.rms_norm_grad(self._handle, self._device, dy, h, gamma, eps, dh, dgamma, residual, dx, p, seed, accumulate, self._queue(stream))
            if code is not None:
                return _check(code, "sc_rms_norm_grad") if code else None
        kind = _layer_type(dy, "dy")
        rows, cols = dy.shape
        dtype = dy.dtype
        lddy = _matrix(dy, rows, cols, dtype, "dy")
        ldh = _matrix(h, rows, cols, dtype, "h")
        _vector(gamma, cols, dtype, "gamma")
        if dh is None and dx is None and dgamma is None:
            raise ValueError("dh, dx or dgamma must be given")
        lddh = cols if dh is None else _matrix(dh, rows, cols, dtype, "dh")
        lddx = cols if dx is None else _matrix(dx, rows, cols, dtype, "dx")
        ldr = cols if residual is None else _matrix(residual, rows, cols, dtype, "residual")
        if dgamma is not None:
            _vector(dgamma, cols, torch.float32, "dgamma")
        self._here(dy, h, gamma, dh, dgamma, residual, dx)
        _check(self._layer.sc_rms_norm_grad(self._handle, kind, _ptr(dy), lddy, _ptr(h), ldh, _ptr(gamma), eps, _ptr(residual), ldr, _probability(p),
                                            int(seed) & 0xFFFFFFFFFFFFFFFF, rows, cols, _ptr(dh), lddh, _ptr(dx), lddx, _ptr(dgamma),
                                            1 if accumulate else 0, self._queue(stream)), "sc_rms_norm_grad")
