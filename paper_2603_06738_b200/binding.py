"""Thin Python binding of the C ABI in ``include/rib_window_attn.h``.

Argument marshalling only: torch supplies device memory and the current stream, every step of
the computation runs in the CUDA kernels of ``librib_window_attn.so``.  There is no CPU or
PyTorch fallback: if the shared library has not been built, importing this module's functions
raises ``RibLibraryMissing``.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import warnings
from pathlib import Path

import torch

from .build import marshal_identity


def _load_marshal():
    """The checks, allocations and the C call of the hot entry points in native code (csrc/rib_marshal.cpp), or None.  It answers None
    for arguments that are not plain tensors of the right kind, and the Python form below takes over."""
    try:
        from . import _rib_marshal as module
    except ImportError:         # not built, or symbols that this torch does not have
        return None
    return module if _fits(module) else None


def _fits(module) -> bool:
    """Was the marshaller compiled for this torch and this Python?  It would import for many others, and read their tensors wrongly."""
    built_for = getattr(module, "built_for", None)
    if built_for == marshal_identity():
        return True
    warnings.warn(f"{module.__name__} was built for {built_for}, this is {marshal_identity()}: calls are marshalled in Python "
                  "until `python -m paper_2603_06738_b200.build` has been run", RuntimeWarning, stacklevel=2)
    return False


_marshal = _load_marshal()

_LIB_PATH = Path(__file__).resolve().parent / "librib_window_attn.so"
_lib = None

RIB_OK = 0
RIB_ERR_DEVICE_WAIT = -7
RIB_PATH_NONE, RIB_PATH_GENERIC, RIB_PATH_SM100, RIB_PATH_SM100_EXACT = 0, 1, 2, 3

EXPORTS = (
    "rib_window_attn_fwd", "rib_window_attn_bwd", "rib_window_attn_bwd_workspace",
    "rib_query_status", "rib_status_string", "rib_set_path", "rib_last_path", "rib_kernel_launches",
    "rib_window_attn_bwd_noalloc", "rib_profile_begin", "rib_profile_end",
    "rib_generate_features", "rib_generate_features_bwd",
    "rib_window_attn_fwd_headwise", "rib_window_attn_bwd_headwise", "rib_window_attn_bwd_headwise_workspace",
    "rib_window_attn_fwd_padded", "rib_cla_gate", "rib_window_attn_fwd_gated",
    "rib_window_attn_bwd_padded", "rib_window_attn_bwd_padded_workspace",
    "rib_window_attn_fwd_masked", "rib_window_attn_bwd_masked", "rib_window_cycle_bwd", "rib_window_cycle_bwd_workspace",
    "rib_cla_product", "rib_cla_product_bwd", "rib_cla_gate_bwd", "rib_cla_gate_bwd_workspace",
    "rib_wait_probe", "rib_exp_probe", "rib_tensor_map_cache_counts", "rib_window_cycle_fwd",
    "rib_window_attn_fwd_bucketed", "rib_window_attn_bwd_bucketed", "rib_window_attn_bwd_bucketed_workspace",
    "rib_checkpoint_store", "rib_checkpoint_restore",
    "rib_window_attn_bwd_checkpointed", "rib_window_attn_bwd_checkpointed_workspace",
    "rib_window_attn_bwd_bucketed_checkpointed", "rib_window_attn_bwd_bucketed_checkpointed_workspace",
    "rib_rope_table", "rib_qk_norm_rope_fwd", "rib_qk_norm_rope_bwd", "rib_qk_norm_rope_bwd_workspace",
    "rib_cross_attn_fwd", "rib_cross_attn_fwd_workspace", "rib_cross_attn_bwd", "rib_cross_attn_bwd_workspace",
)
KERNEL_NAMES = {1: "rib_fwd_sm100_kernel", 2: "rib_bwd_prepare_kernel", 3: "rib_bwd_sm100_kernel",
                4: "rib_bwd_finish_kernel", 6: "generic_fwd_kernel",
                7: "rowdot_kernel", 8: "generic_bwd_dq_kernel", 9: "generic_bwd_dkv_kernel",
                10: "rib_generator_fwd_kernel", 11: "rib_generator_bwd_kernel", 12: "rib_cla_gate_kernel",
                13: "rib_cla_bwd_pw_kernel", 14: "rib_cla_bwd_dw_kernel", 15: "rib_cla_product_kernel", 16: "rib_cla_bwd_tc_kernel",
                17: "rib_fwd_frame_sm100_kernel", 18: "rib_window8_fwd_kernel", 19: "rib_window8_clear_kernel", 20: "rib_window8_bwd_kernel",
                21: "rib_window16_fwd_kernel", 22: "rib_window16_clear_kernel", 23: "rib_window16_bwd_kernel", 24: "rib_generator_clear_kernel",
                25: "rib_bias_scatter_kernel, rib_bias_convert_kernel", 26: "rib_checkpoint_store_kernel", 27: "rib_checkpoint_restore_kernel", 28: "rib_bias_fwd_kernel",
                29: "rib_bias_bwd_prepare_kernel", 30: "rib_bias_bwd_kernel", 31: "rib_bias_bwd_finish_kernel",
                32: "rib_bias_small_fwd_kernel", 33: "rib_bias_small_bwd_kernel",
                34: "rib_rope_table_kernel", 35: "rib_qk_norm_rope_kernel", 36: "rib_qk_norm_rope_kernel (backward)", 37: "rib_qk_norm_rope_sum_kernel",
                38: "rib_cross_fwd_kernel", 39: "rib_cross_join_kernel", 40: "rib_cross_bwd_prepare_kernel", 41: "rib_cross_bwd_dq_kernel", 42: "rib_cross_bwd_dkv_kernel",
                43: "rib_cross_bwd_sum_kernel"}
RIB_DTYPE_F32, RIB_DTYPE_BF16 = 0, 1
RIB_NOALLOC_SCRATCH_BYTES = 32 << 20


class RibLibraryMissing(RuntimeError):
    pass


class RibError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(f"rib call failed with {code}: {rib_status_string(code)}")


def library() -> ctypes.CDLL:
    """Load (once) the in-tree shared library and declare the C signatures."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RibLibraryMissing(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2603_06738_b200.build`")
        lib = ctypes.CDLL(str(_LIB_PATH))
        vp, ci, fp = ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p
        lib.rib_window_attn_fwd.restype = ci
        lib.rib_window_attn_fwd.argtypes = [vp] * 5 + [ci] * 8 + [vp, fp, vp]
        lib.rib_window_attn_bwd.restype = ci
        lib.rib_window_attn_bwd.argtypes = [vp] * 8 + [ci] * 8 + [vp] * 5 + [vp, ctypes.c_size_t, vp]
        ll = ctypes.c_longlong
        lib.rib_window_attn_fwd_headwise.restype = ci
        lib.rib_window_attn_fwd_headwise.argtypes = [vp] * 5 + [ll] + [ci] * 8 + [vp, fp, vp]
        lib.rib_window_attn_fwd_padded.restype = ci
        lib.rib_window_attn_fwd_padded.argtypes = [vp] * 5 + [ll] + [ci] * 8 + [vp, fp, vp]
        lib.rib_window_attn_bwd_padded.restype = ci
        lib.rib_window_attn_bwd_padded.argtypes = [vp] * 5 + [ll] + [vp] * 3 + [ci] * 8 + [vp] * 5 + [vp, ctypes.c_size_t, vp]
        lib.rib_window_cycle_bwd.restype = ci
        lib.rib_window_cycle_bwd.argtypes = [vp] * 8 + [vp, vp, ci] + [ci] * 6 + [vp] * 5 + [vp, ctypes.c_size_t, vp]
        lib.rib_window_cycle_bwd_workspace.restype = ctypes.c_size_t
        lib.rib_window_cycle_bwd_workspace.argtypes = [vp, ci] + [ci] * 6
        lib.rib_window_attn_fwd_masked.restype = ci
        lib.rib_window_attn_fwd_masked.argtypes = [vp] * 5 + [ll] + [ci] * 8 + [vp, fp, vp]
        lib.rib_window_attn_bwd_masked.restype = ci
        lib.rib_window_attn_bwd_masked.argtypes = [vp] * 5 + [ll] + [vp] * 3 + [ci] * 8 + [vp] * 5 + [vp, ctypes.c_size_t, vp]
        lib.rib_window_attn_bwd_padded_workspace.restype = ctypes.c_size_t
        lib.rib_window_attn_bwd_padded_workspace.argtypes = [ll] + [ci] * 7
        lib.rib_cla_gate.restype = ci
        lib.rib_cla_gate.argtypes = [vp] * 5 + [ci] * 4 + [vp, vp]
        lib.rib_cla_product.restype = ci
        lib.rib_cla_product.argtypes = [vp, vp, ll, vp, vp]
        lib.rib_cla_product_bwd.restype = ci
        lib.rib_cla_product_bwd.argtypes = [vp, vp, vp, ll, vp, vp, vp]
        lib.rib_cla_gate_bwd.restype = ci
        lib.rib_cla_gate_bwd.argtypes = [vp] * 6 + [ci] * 4 + [vp] * 5 + [vp, ctypes.c_size_t, vp]
        lib.rib_cla_gate_bwd_workspace.restype = ctypes.c_size_t
        lib.rib_cla_gate_bwd_workspace.argtypes = [ci] * 4
        lib.rib_window_attn_fwd_gated.restype = ci
        lib.rib_window_attn_fwd_gated.argtypes = [vp] * 5 + [ll, vp] + [ci] * 8 + [vp, fp, vp]
        lib.rib_window_attn_bwd_headwise.restype = ci
        lib.rib_window_attn_bwd_headwise.argtypes = [vp] * 5 + [ll] + [vp] * 3 + [ci] * 8 + [vp] * 5 + [vp, ctypes.c_size_t, vp]
        lib.rib_window_attn_bwd_headwise_workspace.restype = ctypes.c_size_t
        lib.rib_window_attn_bwd_headwise_workspace.argtypes = [ll] + [ci] * 7
        lib.rib_window_attn_bwd_noalloc.restype = ci
        lib.rib_window_attn_bwd_noalloc.argtypes = [vp] * 8 + [ci] * 8 + [vp] * 5 + [vp]
        lib.rib_generate_features.restype = ci
        lib.rib_generate_features.argtypes = [vp] * 4 + [ci] * 4 + [vp] * 3
        lib.rib_generate_features_bwd.restype = ci
        lib.rib_generate_features_bwd.argtypes = [vp] * 6 + [ci] * 4 + [vp] * 5
        lib.rib_profile_begin.restype = ci
        lib.rib_profile_begin.argtypes = [ci]
        lib.rib_profile_end.restype = ci
        lib.rib_profile_end.argtypes = [ctypes.POINTER(ci), ctypes.POINTER(ctypes.c_float), ci]
        lib.rib_window_attn_bwd_workspace.restype = ctypes.c_size_t
        lib.rib_window_attn_bwd_workspace.argtypes = [ci] * 7
        lib.rib_query_status.restype = ci
        lib.rib_query_status.argtypes = [vp]
        lib.rib_status_string.restype = ctypes.c_char_p
        lib.rib_status_string.argtypes = [ci]
        lib.rib_set_path.restype = ci
        lib.rib_set_path.argtypes = [ci]
        lib.rib_last_path.restype = ci
        lib.rib_last_path.argtypes = []
        lib.rib_kernel_launches.restype = ctypes.c_longlong
        lib.rib_kernel_launches.argtypes = []
        lib.rib_window_cycle_fwd.restype = ci
        lib.rib_window_cycle_fwd.argtypes = [ctypes.POINTER(vp)] * 5 + [ctypes.POINTER(ci)] * 2 + [ci] * 7 + [ctypes.POINTER(vp)] * 2 + [vp]
        lib.rib_tensor_map_cache_counts.restype = None
        lib.rib_tensor_map_cache_counts.argtypes = [ctypes.POINTER(ctypes.c_longlong)] * 2
        lib.rib_wait_probe.restype = ci
        lib.rib_wait_probe.argtypes = [ctypes.c_ulonglong, vp]
        lib.rib_exp_probe.restype = ctypes.c_longlong
        lib.rib_exp_probe.argtypes = [vp, ci, ci, vp]
        size = ctypes.c_size_t
        lib.rib_window_attn_fwd_bucketed.restype = ci
        lib.rib_window_attn_fwd_bucketed.argtypes = [vp] * 4 + [ci, ll, vp, ci] + [ci] * 8 + [vp, fp, vp]
        lib.rib_window_attn_bwd_bucketed.restype = ci
        lib.rib_window_attn_bwd_bucketed.argtypes = [vp] * 4 + [ci, ll, vp, ci] + [vp] * 3 + [ci] * 8 + [vp] * 5 + [size, vp]
        lib.rib_window_attn_bwd_bucketed_workspace.restype = size
        lib.rib_window_attn_bwd_bucketed_workspace.argtypes = [ll] + [ci] * 7
        lib.rib_checkpoint_store.restype = ci
        lib.rib_checkpoint_store.argtypes = [vp, ll, ci, vp, vp, vp]
        lib.rib_checkpoint_restore.restype = ci
        lib.rib_checkpoint_restore.argtypes = [vp, vp, ll, ci, vp, vp]
        lib.rib_window_attn_bwd_checkpointed.restype = ci
        lib.rib_window_attn_bwd_checkpointed.argtypes = [vp] * 3 + [ll, vp, vp] + [ci] * 9 + [vp] * 6 + [size, vp]
        lib.rib_window_attn_bwd_checkpointed_workspace.restype = size
        lib.rib_window_attn_bwd_checkpointed_workspace.argtypes = [ll] + [ci] * 7
        lib.rib_window_attn_bwd_bucketed_checkpointed.restype = ci
        lib.rib_window_attn_bwd_bucketed_checkpointed.argtypes = [vp, vp, ci, ll, vp, ci, vp, vp] + [ci] * 8 + [vp] * 5 + [size, vp]
        lib.rib_window_attn_bwd_bucketed_checkpointed_workspace.restype = size
        lib.rib_window_attn_bwd_bucketed_checkpointed_workspace.argtypes = [ll] + [ci] * 7
        f32 = ctypes.c_float
        lib.rib_rope_table.restype = ci
        lib.rib_rope_table.argtypes = [vp, ci, ci, ci, ll, ll, f32, vp, vp]
        lib.rib_qk_norm_rope_fwd.restype = ci
        lib.rib_qk_norm_rope_fwd.argtypes = [vp, ll, vp, ll, vp, vp, ci, vp] + [ci] * 8 + [f32, vp, vp, vp]
        lib.rib_qk_norm_rope_bwd_workspace.restype = size
        lib.rib_qk_norm_rope_bwd_workspace.argtypes = [ci] * 7
        lib.rib_qk_norm_rope_bwd.restype = ci
        lib.rib_qk_norm_rope_bwd.argtypes = [vp, ll, vp, ll, vp, vp, ci, vp, vp, vp] + [ci] * 8 + [f32, vp, ll, vp, ll, vp, vp, vp, size, vp]
        for name in ("rib_cross_attn_fwd_workspace", "rib_cross_attn_bwd_workspace"):
            getattr(lib, name).restype = size
            getattr(lib, name).argtypes = [ci] * 8
        lib.rib_cross_attn_fwd.restype = ci
        lib.rib_cross_attn_fwd.argtypes = [vp] * 4 + [ci] * 8 + [vp, vp, vp, size, vp]
        lib.rib_cross_attn_bwd.restype = ci
        lib.rib_cross_attn_bwd.argtypes = [vp] * 7 + [ci] * 8 + [vp] * 4 + [size, vp]
        lib.rib_addresses = {name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in EXPORTS}
        _lib = lib
    return _lib


def _native(call, entry, *args):
    """The results of a call through the native marshaller, or None: the caller then goes on in Python."""
    got = call((_lib or library()).rib_addresses[entry], *args)
    if type(got) is int:
        raise RibError(got)
    return got


def _stream_ptr(stream) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return int(s.cuda_stream)


def _elsewhere(stream) -> bool:
    """Is the stream that a call is given another one than the current one?"""
    return int(stream.cuda_stream) != int(torch.cuda.current_stream(getattr(stream, "device", None)).cuda_stream)


def _tensors(x):
    if isinstance(x, torch.Tensor):
        yield x
    elif isinstance(x, (tuple, list)):
        for y in x:
            yield from _tensors(y)


def _beside(stream, call, *args):
    """A call on a stream that is not the current one: made with that stream current, so that its results and its scratch are memory of that stream, which
    nothing on the current one still uses; and no tensor of the call is handed out again before the call (its arguments) or what the current stream does
    with them (its results) is through."""
    given = [t for t in _tensors(args) if t.is_cuda]
    device = given[0].device if given else None
    current = torch.cuda.current_stream(device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream.cuda_stream), device=device)
    if device is not None and stream.device != device:
        raise ValueError(f"stream is one of {stream.device}, the tensors are on {device}")
    try:
        with torch.cuda.stream(stream):
            results = call(*args)
    finally:
        for t in given:
            t.record_stream(stream)
    for t in _tensors(results):
        t.record_stream(current)
    return results


def _ptr(t) -> int | None:
    return None if t is None else int(t.data_ptr())


def _check_image(name, t, shape=None):
    if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 5:
        raise ValueError(f"{name} must be a contiguous CUDA bfloat16 tensor [B,H,W,heads,d]")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _check_pos(name, t, n):
    if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 2 or t.shape[0] != n:
        raise ValueError(f"{name} must be a contiguous CUDA bfloat16 tensor [n={n}, r]")


def _check_pos_headwise(name, t, heads, n):
    if (t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 3
            or t.shape[0] != heads or t.shape[1] != n):
        raise ValueError(f"{name} must be a contiguous CUDA bfloat16 tensor [heads={heads}, n={n}, r]")


def rib_status_string(code: int) -> str:
    return library().rib_status_string(int(code)).decode()


def rib_set_path(path: int) -> int:
    return int(library().rib_set_path(int(path)))


def rib_last_path() -> int:
    return int(library().rib_last_path())


def rib_kernel_launches() -> int:
    return int(library().rib_kernel_launches())


def rib_profile_begin(max_launches: int) -> None:
    rc = int(library().rib_profile_begin(int(max_launches)))
    if rc != RIB_OK:
        raise RibError(rc)


def rib_profile_end(capacity: int) -> list[tuple[int, float]]:
    """Ends the per-kernel timing session; returns [(kernel id, device milliseconds), ...] in launch order."""
    ids = (ctypes.c_int * capacity)()
    ms = (ctypes.c_float * capacity)()
    n = int(library().rib_profile_end(ids, ms, capacity))
    if n < 0:
        raise RibError(n)
    return [(int(ids[i]), float(ms[i])) for i in range(n)]


def rib_query_status(stream=None) -> int:
    return int(library().rib_query_status(_stream_ptr(stream)))


def rib_tensor_map_cache_counts() -> tuple[int, int]:
    """(hits, misses) of the library's tensor-map cache in this process."""
    h, m = ctypes.c_longlong(0), ctypes.c_longlong(0)
    library().rib_tensor_map_cache_counts(ctypes.byref(h), ctypes.byref(m))
    return int(h.value), int(m.value)


def rib_wait_probe(limit_ns: int, stream=None) -> None:
    """Enqueue the self-test kernel whose bounded wait runs out after `limit_ns` nanoseconds."""
    rc = int(library().rib_wait_probe(int(limit_ns), _stream_ptr(stream)))
    if rc != RIB_OK:
        raise RibError(rc)


def rib_exp_probe(sink, blocks: int, iters: int, stream=None) -> int:
    """Enqueue the exp-throughput kernel; returns the number of exponentials it evaluates."""
    n = int(library().rib_exp_probe(_ptr(sink), int(blocks), int(iters), _stream_ptr(stream)))
    if n < 0:
        raise RibError(n)
    return n


def rib_window_attn_bwd_workspace(B, H, W, heads, d, r, window) -> int:
    return int(library().rib_window_attn_bwd_workspace(B, H, W, heads, d, r, window))


def rib_window_attn_fwd(q, k, v, pq, pk, window, shift=0, out=None, lse=None, stream=None, want_lse=True):
    """Enqueue the forward pass; returns (out bf16 [B,H,W,heads,d], lse fp32 [B,heads,H,W] or None)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_fwd, q, k, v, pq, pk, window, shift, out, lse, None, want_lse)
    if _marshal is not None and out is None and lse is None:
        got = _native(_marshal.fwd, "rib_window_attn_fwd_headwise", q, k, v, pq, pk, 1, window, shift, want_lse, stream)
        if got is not None:
            return got
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    _check_image("k", k, q.shape)
    _check_image("v", v, q.shape)
    n = window * window
    _check_pos("pq", pq, n)
    _check_pos("pk", pk, n)
    r = pq.shape[1]
    if out is None:
        out = torch.empty_like(q)
    if lse is None and want_lse:
        lse = torch.empty((B, heads, H, W), dtype=torch.float32, device=q.device)
    rc = library().rib_window_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(pq), _ptr(pk), B, H, W, heads, d, r,
                                       window, shift, _ptr(out), _ptr(lse), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return out, lse


def rib_window_attn_bwd(q, k, v, pq, pk, out, lse, dout, window, shift=0, workspace=None, stream=None):
    """Enqueue the backward pass; returns (dq, dk, dv bf16, dpq, dpk fp32 [n,r])."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_bwd, q, k, v, pq, pk, out, lse, dout, window, shift, workspace)
    if _marshal is not None and workspace is not None:
        got = _native(_marshal.bwd, "rib_window_attn_bwd_headwise", q, k, v, pq, pk, out, lse, dout, 1, window, shift, workspace, stream)
        if got is not None:
            return got
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    for name, t in (("k", k), ("v", v), ("out", out), ("dout", dout)):
        _check_image(name, t, q.shape)
    n = window * window
    _check_pos("pq", pq, n)
    _check_pos("pk", pk, n)
    r = pq.shape[1]
    if lse.dtype != torch.float32 or tuple(lse.shape) != (B, heads, H, W) or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous fp32 tensor [B,heads,H,W]")
    need = rib_window_attn_bwd_workspace(B, H, W, heads, d, r, window)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    dpq = torch.empty((n, r), dtype=torch.float32, device=q.device)
    dpk = torch.empty((n, r), dtype=torch.float32, device=q.device)
    rc = library().rib_window_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(pq), _ptr(pk), _ptr(out), _ptr(lse),
                                       _ptr(dout), B, H, W, heads, d, r, window, shift, _ptr(dq), _ptr(dk),
                                       _ptr(dv), _ptr(dpq), _ptr(dpk), _ptr(workspace), workspace.numel(),
                                       _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dq, dk, dv, dpq, dpk


def rib_window_attn_bwd_headwise_workspace(pos_head_stride, B, H, W, heads, d, r, window) -> int:
    return int(library().rib_window_attn_bwd_headwise_workspace(pos_head_stride, B, H, W, heads, d, r, window))


def rib_window_attn_fwd_headwise(q, k, v, pq, pk, window, shift=0, stream=None, want_lse=True):
    """Forward pass with one Pq/Pk table per head: pq, pk bf16 [heads, n, r]; returns (out, lse)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_fwd_headwise, q, k, v, pq, pk, window, shift, None, want_lse)
    if _marshal is not None:
        got = _native(_marshal.fwd, "rib_window_attn_fwd_headwise", q, k, v, pq, pk, 2, window, shift, want_lse, stream)
        if got is not None:
            return got
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    _check_image("k", k, q.shape)
    _check_image("v", v, q.shape)
    n = window * window
    _check_pos_headwise("pq", pq, heads, n)
    _check_pos_headwise("pk", pk, heads, n)
    r = pq.shape[2]
    out = torch.empty_like(q)
    lse = torch.empty((B, heads, H, W), dtype=torch.float32, device=q.device) if want_lse else None
    rc = library().rib_window_attn_fwd_headwise(_ptr(q), _ptr(k), _ptr(v), _ptr(pq), _ptr(pk), n * r, B, H, W, heads,
                                                d, r, window, shift, _ptr(out), _ptr(lse), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return out, lse


def rib_window_attn_fwd_padded(q, k, v, pq, pk, window, shift=0, stream=None, want_lse=True):
    """Forward pass on a map whose sides need not be multiples of the window (positions of the extended map
    beyond H x W are not tokens); pq, pk are [n, r] or [heads, n, r].  Returns (out, lse)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_fwd_padded, q, k, v, pq, pk, window, shift, None, want_lse)
    if _marshal is not None:
        got = _native(_marshal.fwd, "rib_window_attn_fwd_padded", q, k, v, pq, pk, 3, window, shift, want_lse, stream)
        if got is not None:
            return got
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    _check_image("k", k, q.shape)
    _check_image("v", v, q.shape)
    n = window * window
    headwise = pq.dim() == 3
    if headwise:
        _check_pos_headwise("pq", pq, heads, n)
        _check_pos_headwise("pk", pk, heads, n)
    else:
        _check_pos("pq", pq, n)
        _check_pos("pk", pk, n)
    r = pq.shape[-1]
    out = torch.empty_like(q)
    lse = torch.empty((B, heads, H, W), dtype=torch.float32, device=q.device) if want_lse else None
    rc = library().rib_window_attn_fwd_padded(_ptr(q), _ptr(k), _ptr(v), _ptr(pq), _ptr(pk), n * r if headwise else 0,
                                              B, H, W, heads, d, r, window, shift, _ptr(out), _ptr(lse), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return out, lse


def rib_window_cycle_fwd(qs, ks, vs, pqs, pks, windows, shifts=None, stream=None, want_lse=True):
    """The cyclic window strategy in one call: layer l attends qs[l], ks[l], vs[l] in windows of side windows[l] with the tables
    pqs[l], pks[l] ([windows[l]^2, r]).  Returns (outs, lses), one tensor per layer."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_cycle_fwd, qs, ks, vs, pqs, pks, windows, shifts, None, want_lse)
    layers = len(windows)
    if not (len(qs) == len(ks) == len(vs) == len(pqs) == len(pks) == layers) or (shifts is not None and len(shifts) != layers):
        raise ValueError("one q, k, v, pq, pk (and shift) per layer")
    _check_image("q", qs[0])
    B, H, W, heads, d = qs[0].shape
    r = pqs[0].shape[1]
    for l in range(layers):
        for name, t in (("q", qs[l]), ("k", ks[l]), ("v", vs[l])):
            _check_image(name, t, qs[0].shape)
        _check_pos("pq", pqs[l], windows[l] * windows[l])
        _check_pos("pk", pks[l], windows[l] * windows[l])
        if pqs[l].shape[1] != r or pks[l].shape[1] != r:
            raise ValueError("every layer uses the same rank")
    outs = [torch.empty_like(qs[0]) for _ in range(layers)]
    lses = [torch.empty((B, heads, H, W), dtype=torch.float32, device=qs[0].device) if want_lse else None for _ in range(layers)]
    arr = lambda ts: (ctypes.c_void_p * layers)(*[_ptr(t) for t in ts])
    ints = lambda xs: (ctypes.c_int * layers)(*[int(x) for x in xs])
    rc = library().rib_window_cycle_fwd(arr(qs), arr(ks), arr(vs), arr(pqs), arr(pks), ints(windows),
                                        ints(shifts) if shifts is not None else None, layers, B, H, W, heads, d, r,
                                        arr(outs), arr(lses) if want_lse else None, _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return outs, lses


def rib_window_cycle_bwd(qs, ks, vs, pqs, pks, outs, lses, douts, windows, shifts=None, workspace=None, stream=None):
    """Backward passes of the layers of rib_window_cycle_fwd.  Returns (dqs, dks, dvs, dpqs, dpks), one tensor per layer."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_cycle_bwd, qs, ks, vs, pqs, pks, outs, lses, douts, windows, shifts, workspace)
    layers = len(windows)
    lists = (qs, ks, vs, pqs, pks, outs, lses, douts)
    if any(len(x) != layers for x in lists) or (shifts is not None and len(shifts) != layers):
        raise ValueError("one q, k, v, pq, pk, out, lse, dout (and shift) per layer")
    _check_image("q", qs[0])
    B, H, W, heads, d = qs[0].shape
    r = pqs[0].shape[1]
    for l in range(layers):
        for name, t in (("q", qs[l]), ("k", ks[l]), ("v", vs[l]), ("out", outs[l]), ("dout", douts[l])):
            _check_image(name, t, qs[0].shape)
        _check_pos("pq", pqs[l], windows[l] * windows[l])
        _check_pos("pk", pks[l], windows[l] * windows[l])
        if lses[l].dtype != torch.float32 or tuple(lses[l].shape) != (B, heads, H, W) or not lses[l].is_contiguous():
            raise ValueError("lse must be a contiguous fp32 tensor [B,heads,H,W]")
    ints = lambda xs: (ctypes.c_int * layers)(*[int(x) for x in xs])
    arr = lambda ts: (ctypes.c_void_p * layers)(*[_ptr(t) for t in ts])
    need = int(library().rib_window_cycle_bwd_workspace(ints(windows), layers, B, H, W, heads, d, r))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=qs[0].device)
    dqs, dks, dvs = ([torch.empty_like(qs[0]) for _ in range(layers)] for _ in range(3))
    dpqs = [torch.empty(tuple(t.shape), dtype=torch.float32, device=t.device) for t in pqs]
    dpks = [torch.empty(tuple(t.shape), dtype=torch.float32, device=t.device) for t in pks]
    rc = library().rib_window_cycle_bwd(arr(qs), arr(ks), arr(vs), arr(pqs), arr(pks), arr(outs), arr(lses), arr(douts), ints(windows),
                                        ints(shifts) if shifts is not None else None, layers, B, H, W, heads, d, r,
                                        arr(dqs), arr(dks), arr(dvs), arr(dpqs), arr(dpks), _ptr(workspace), workspace.numel(),
                                        _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dqs, dks, dvs, dpqs, dpks


def rib_window_attn_bwd_padded(q, k, v, pq, pk, out, lse, dout, window, shift=0, workspace=None, stream=None):
    """Backward pass on a map whose sides need not be multiples of the window; pq, pk [n, r] or [heads, n, r].
    Returns (dq, dk, dv bf16, dpq, dpk fp32 of the shape of pq)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_bwd_padded, q, k, v, pq, pk, out, lse, dout, window, shift, workspace)
    if _marshal is not None and workspace is not None:
        got = _native(_marshal.bwd, "rib_window_attn_bwd_padded", q, k, v, pq, pk, out, lse, dout, 3, window, shift, workspace, stream)
        if got is not None:
            return got
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    for name, t in (("k", k), ("v", v), ("out", out), ("dout", dout)):
        _check_image(name, t, q.shape)
    n = window * window
    headwise = pq.dim() == 3
    if headwise:
        _check_pos_headwise("pq", pq, heads, n)
        _check_pos_headwise("pk", pk, heads, n)
    else:
        _check_pos("pq", pq, n)
        _check_pos("pk", pk, n)
    r = pq.shape[-1]
    stride = n * r if headwise else 0
    if lse.dtype != torch.float32 or tuple(lse.shape) != (B, heads, H, W) or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous fp32 tensor [B,heads,H,W]")
    need = int(library().rib_window_attn_bwd_padded_workspace(stride, B, H, W, heads, d, r, window))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    dpq = torch.empty(tuple(pq.shape), dtype=torch.float32, device=q.device)
    dpk = torch.empty(tuple(pk.shape), dtype=torch.float32, device=q.device)
    rc = library().rib_window_attn_bwd_padded(_ptr(q), _ptr(k), _ptr(v), _ptr(pq), _ptr(pk), stride, _ptr(out), _ptr(lse),
                                              _ptr(dout), B, H, W, heads, d, r, window, shift, _ptr(dq), _ptr(dk), _ptr(dv),
                                              _ptr(dpq), _ptr(dpk), _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dq, dk, dv, dpq, dpk


def rib_window_attn_fwd_masked(q, k, v, pq, pk, window, shift=0, stream=None, want_lse=True):
    """Forward pass with shifted windows whose wrapped parts do not attend to each other (H, W multiples of the
    window); pq, pk are [n, r] or [heads, n, r].  Returns (out, lse)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_fwd_masked, q, k, v, pq, pk, window, shift, None, want_lse)
    if _marshal is not None:
        got = _native(_marshal.fwd, "rib_window_attn_fwd_masked", q, k, v, pq, pk, 3, window, shift, want_lse, stream)
        if got is not None:
            return got
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    _check_image("k", k, q.shape)
    _check_image("v", v, q.shape)
    n = window * window
    headwise = pq.dim() == 3
    if headwise:
        _check_pos_headwise("pq", pq, heads, n)
        _check_pos_headwise("pk", pk, heads, n)
    else:
        _check_pos("pq", pq, n)
        _check_pos("pk", pk, n)
    r = pq.shape[-1]
    out = torch.empty_like(q)
    lse = torch.empty((B, heads, H, W), dtype=torch.float32, device=q.device) if want_lse else None
    rc = library().rib_window_attn_fwd_masked(_ptr(q), _ptr(k), _ptr(v), _ptr(pq), _ptr(pk), n * r if headwise else 0,
                                              B, H, W, heads, d, r, window, shift, _ptr(out), _ptr(lse), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return out, lse


def rib_window_attn_bwd_masked(q, k, v, pq, pk, out, lse, dout, window, shift=0, workspace=None, stream=None):
    """Backward pass of rib_window_attn_fwd_masked; pq, pk [n, r] or [heads, n, r].
    Returns (dq, dk, dv bf16, dpq, dpk fp32 of the shape of pq)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_bwd_masked, q, k, v, pq, pk, out, lse, dout, window, shift, workspace)
    if _marshal is not None and workspace is not None:
        got = _native(_marshal.bwd, "rib_window_attn_bwd_masked", q, k, v, pq, pk, out, lse, dout, 3, window, shift, workspace, stream)
        if got is not None:
            return got
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    for name, t in (("k", k), ("v", v), ("out", out), ("dout", dout)):
        _check_image(name, t, q.shape)
    n = window * window
    headwise = pq.dim() == 3
    if headwise:
        _check_pos_headwise("pq", pq, heads, n)
        _check_pos_headwise("pk", pk, heads, n)
    else:
        _check_pos("pq", pq, n)
        _check_pos("pk", pk, n)
    r = pq.shape[-1]
    stride = n * r if headwise else 0
    if lse.dtype != torch.float32 or tuple(lse.shape) != (B, heads, H, W) or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous fp32 tensor [B,heads,H,W]")
    need = int(library().rib_window_attn_bwd_padded_workspace(stride, B, H, W, heads, d, r, window))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    dpq = torch.empty(tuple(pq.shape), dtype=torch.float32, device=q.device)
    dpk = torch.empty(tuple(pk.shape), dtype=torch.float32, device=q.device)
    rc = library().rib_window_attn_bwd_masked(_ptr(q), _ptr(k), _ptr(v), _ptr(pq), _ptr(pk), stride, _ptr(out), _ptr(lse),
                                              _ptr(dout), B, H, W, heads, d, r, window, shift, _ptr(dq), _ptr(dk), _ptr(dv),
                                              _ptr(dpq), _ptr(dpk), _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dq, dk, dv, dpq, dpk


def rib_cla_gate(x, w_dw, b_dw, w_pw, b_pw, stream=None):
    """CLA gate (Eq. 8): x bf16 [B,H,W,D]; w_dw fp32 [D,3,3]; b_dw fp32 [D]; w_pw fp32 [D,D] (out, in); b_pw fp32 [D].
    Returns the gate, bf16 [B,H,W,D]."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_cla_gate, x, w_dw, b_dw, w_pw, b_pw)
    if x.dtype != torch.bfloat16 or not x.is_cuda or not x.is_contiguous() or x.dim() != 4:
        raise ValueError("x must be a contiguous CUDA bfloat16 tensor [B,H,W,D]")
    B, H, W, D = x.shape
    for name, t, shape in (("w_dw", w_dw, (D, 3, 3)), ("b_dw", b_dw, (D,)), ("w_pw", w_pw, (D, D)), ("b_pw", b_pw, (D,))):
        if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != shape:
            raise ValueError(f"{name} must be a contiguous CUDA fp32 tensor of shape {shape}")
    gate = torch.empty_like(x)
    rc = library().rib_cla_gate(_ptr(x), _ptr(w_dw), _ptr(b_dw), _ptr(w_pw), _ptr(b_pw), B, H, W, D, _ptr(gate), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return gate


def _check_bf16_like(name, t, like=None):
    if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA bfloat16 tensor")
    if like is not None and t.numel() != like.numel():
        raise ValueError(f"{name} must have as many elements as out")


def rib_cla_product(out, gate, stream=None):
    """Eq. 9 on its own: out [B,H,W,heads,d] (or [B,H,W,D]) times gate [B,H,W,D], both bf16; returns out's shape."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_cla_product, out, gate)
    _check_bf16_like("out", out)
    _check_bf16_like("gate", gate, out)
    res = torch.empty_like(out)
    rc = library().rib_cla_product(_ptr(out), _ptr(gate), out.numel(), _ptr(res), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return res


def rib_cla_product_bwd(out, gate, dout_gated, stream=None):
    """Chain rule of Eq. 9: returns (dout in out's shape, dgate in gate's shape), bf16."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_cla_product_bwd, out, gate, dout_gated)
    _check_bf16_like("out", out)
    _check_bf16_like("gate", gate, out)
    _check_bf16_like("dout_gated", dout_gated, out)
    dout = torch.empty_like(out)
    dgate = torch.empty_like(gate)
    rc = library().rib_cla_product_bwd(_ptr(out), _ptr(gate), _ptr(dout_gated), out.numel(), _ptr(dout), _ptr(dgate),
                                       _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dout, dgate


def rib_cla_gate_bwd(x, w_dw, b_dw, w_pw, b_pw, dgate, workspace=None, stream=None):
    """Chain rule of Eq. 8: x, dgate bf16 [B,H,W,D]; weights as for rib_cla_gate.
    Returns (dx bf16 [B,H,W,D], dw_dw [D,3,3], db_dw [D], dw_pw [D,D], db_pw [D] fp32)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_cla_gate_bwd, x, w_dw, b_dw, w_pw, b_pw, dgate, workspace)
    if x.dtype != torch.bfloat16 or not x.is_cuda or not x.is_contiguous() or x.dim() != 4:
        raise ValueError("x must be a contiguous CUDA bfloat16 tensor [B,H,W,D]")
    B, H, W, D = x.shape
    if dgate.dtype != torch.bfloat16 or not dgate.is_cuda or not dgate.is_contiguous() or dgate.shape != x.shape:
        raise ValueError("dgate must be a contiguous CUDA bfloat16 tensor of x's shape")
    for name, t, shape in (("w_dw", w_dw, (D, 3, 3)), ("b_dw", b_dw, (D,)), ("w_pw", w_pw, (D, D)), ("b_pw", b_pw, (D,))):
        if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != shape:
            raise ValueError(f"{name} must be a contiguous CUDA fp32 tensor of shape {shape}")
    need = library().rib_cla_gate_bwd_workspace(B, H, W, D)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
    dx = torch.empty_like(x)
    grads = [torch.empty_like(t) for t in (w_dw, b_dw, w_pw, b_pw)]
    rc = library().rib_cla_gate_bwd(_ptr(x), _ptr(w_dw), _ptr(b_dw), _ptr(w_pw), _ptr(b_pw), _ptr(dgate), B, H, W, D, _ptr(dx),
                                    *[_ptr(g) for g in grads], _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return (dx, *grads)


def rib_window_attn_fwd_gated(q, k, v, pq, pk, gate, window, shift=0, stream=None, want_lse=True):
    """Forward pass whose output is multiplied by the CLA gate (Eq. 9); gate bf16 [B,H,W,heads*d]; pq, pk [n,r] or
    [heads,n,r].  Returns (out, lse)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_fwd_gated, q, k, v, pq, pk, gate, window, shift, None, want_lse)
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    _check_image("k", k, q.shape)
    _check_image("v", v, q.shape)
    if gate.dtype != torch.bfloat16 or not gate.is_cuda or not gate.is_contiguous() or tuple(gate.shape) != (B, H, W, heads * d):
        raise ValueError("gate must be a contiguous CUDA bfloat16 tensor [B,H,W,heads*d]")
    n = window * window
    headwise = pq.dim() == 3
    if headwise:
        _check_pos_headwise("pq", pq, heads, n)
        _check_pos_headwise("pk", pk, heads, n)
    else:
        _check_pos("pq", pq, n)
        _check_pos("pk", pk, n)
    r = pq.shape[-1]
    out = torch.empty_like(q)
    lse = torch.empty((B, heads, H, W), dtype=torch.float32, device=q.device) if want_lse else None
    rc = library().rib_window_attn_fwd_gated(_ptr(q), _ptr(k), _ptr(v), _ptr(pq), _ptr(pk), n * r if headwise else 0, _ptr(gate),
                                             B, H, W, heads, d, r, window, shift, _ptr(out), _ptr(lse), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return out, lse


def rib_window_attn_bwd_headwise(q, k, v, pq, pk, out, lse, dout, window, shift=0, workspace=None, stream=None):
    """Backward pass with one Pq/Pk table per head; returns (dq, dk, dv bf16, dpq, dpk fp32 [heads, n, r])."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_bwd_headwise, q, k, v, pq, pk, out, lse, dout, window, shift, workspace)
    if _marshal is not None and workspace is not None:
        got = _native(_marshal.bwd, "rib_window_attn_bwd_headwise", q, k, v, pq, pk, out, lse, dout, 2, window, shift, workspace, stream)
        if got is not None:
            return got
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    for name, t in (("k", k), ("v", v), ("out", out), ("dout", dout)):
        _check_image(name, t, q.shape)
    n = window * window
    _check_pos_headwise("pq", pq, heads, n)
    _check_pos_headwise("pk", pk, heads, n)
    r = pq.shape[2]
    if lse.dtype != torch.float32 or tuple(lse.shape) != (B, heads, H, W) or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous fp32 tensor [B,heads,H,W]")
    need = rib_window_attn_bwd_headwise_workspace(n * r, B, H, W, heads, d, r, window)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    dpq = torch.empty((heads, n, r), dtype=torch.float32, device=q.device)
    dpk = torch.empty((heads, n, r), dtype=torch.float32, device=q.device)
    rc = library().rib_window_attn_bwd_headwise(_ptr(q), _ptr(k), _ptr(v), _ptr(pq), _ptr(pk), n * r, _ptr(out),
                                                _ptr(lse), _ptr(dout), B, H, W, heads, d, r, window, shift, _ptr(dq),
                                                _ptr(dk), _ptr(dv), _ptr(dpq), _ptr(dpk), _ptr(workspace),
                                                workspace.numel(), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dq, dk, dv, dpq, dpk


def rib_window_attn_bwd_noalloc(q, k, v, pq, pk, out, lse, dout, dq, dk, dv, dpq, dpk, window, shift=0, stream=None):
    """Backward pass into caller-provided result tensors, using the library's built-in scratch.

    For callers that must not allocate on the device: nothing is allocated here either, so every
    result tensor is passed in.  Shapes that need more than ``RIB_NOALLOC_SCRATCH_BYTES`` of
    scratch raise ``RibError`` (RIB_ERR_TOO_LARGE).  Calls on one device share the scratch: keep
    them on one stream.
    """
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_bwd_noalloc, q, k, v, pq, pk, out, lse, dout, dq, dk, dv, dpq, dpk, window, shift)
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    for name, t in (("k", k), ("v", v), ("out", out), ("dout", dout), ("dq", dq), ("dk", dk), ("dv", dv)):
        _check_image(name, t, q.shape)
    n = window * window
    _check_pos("pq", pq, n)
    _check_pos("pk", pk, n)
    r = pq.shape[1]
    for name, t in (("dpq", dpq), ("dpk", dpk)):
        if t.dtype != torch.float32 or tuple(t.shape) != (n, r) or not t.is_contiguous() or not t.is_cuda:
            raise ValueError(f"{name} must be a contiguous CUDA fp32 tensor [n, r]")
    if lse.dtype != torch.float32 or tuple(lse.shape) != (B, heads, H, W) or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous fp32 tensor [B,heads,H,W]")
    rc = library().rib_window_attn_bwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(pq), _ptr(pk), _ptr(out), _ptr(lse),
                                               _ptr(dout), B, H, W, heads, d, r, window, shift, _ptr(dq), _ptr(dk),
                                               _ptr(dv), _ptr(dpq), _ptr(dpk), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)


_SAME_DEVICE = contextlib.nullcontext()


def _on(device, *tensors):
    """The calls below launch on the device of their tensors, whichever is current (a stream that is given has to be one of its)."""
    for t in tensors:
        if t.device != device:
            raise ValueError(f"all tensors of a call have to be on one device: got {t.device} beside {device}")
    return _SAME_DEVICE if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _check_bias(bias, buckets, heads, window, device):
    """(dtype, elements between the heads' tables, number of buckets) of a bias [heads, buckets] or [buckets] (shared by the heads)."""
    if bias.dtype not in (torch.float32, torch.bfloat16) or not bias.is_contiguous() or bias.device != device:
        raise ValueError("bias must be a contiguous float32 or bfloat16 tensor [heads, num_buckets] or [num_buckets] on q's device")
    if bias.dim() not in (1, 2) or bias.shape[-1] < 1 or (bias.dim() == 2 and bias.shape[0] != heads):
        raise ValueError(f"bias has shape {tuple(bias.shape)}, expected [{heads}, num_buckets] or [num_buckets]")
    side = 2 * window - 1
    if buckets.dtype != torch.int32 or not buckets.is_contiguous() or buckets.device != device or tuple(buckets.shape) != (side, side):
        raise ValueError(f"buckets must be a contiguous int32 tensor [{side}, {side}] on q's device")
    count = bias.shape[-1]
    return RIB_DTYPE_BF16 if bias.dtype == torch.bfloat16 else RIB_DTYPE_F32, count if bias.dim() == 2 else 0, count


def rib_window_attn_fwd_bucketed(q, k, v, bias, buckets, window, shift=0, masked=False, stream=None, want_lse=True):
    """Forward pass with a learned bias for relative positions: bias fp32 or bf16 [heads, num_buckets] (or [num_buckets], shared by
    the heads), buckets int32 [2 window - 1, 2 window - 1], the bucket of every offset key - query (outside [0, num_buckets): not
    attended to).  Any H and W; `masked` keeps the wrapped parts of shifted windows apart (H, W multiples of the window).
    Returns (out, lse)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_fwd_bucketed, q, k, v, bias, buckets, window, shift, masked, None, want_lse)
    if _marshal is not None:
        got = _native(_marshal.fwd_bucketed, "rib_window_attn_fwd_bucketed", q, k, v, bias, buckets, window, shift, masked, want_lse, stream)
        if got is not None:
            return got
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    _check_image("k", k, q.shape)
    _check_image("v", v, q.shape)
    dtype, stride, count = _check_bias(bias, buckets, heads, window, q.device)
    with _on(q.device, k, v):
        out = torch.empty_like(q)
        lse = torch.empty((B, heads, H, W), dtype=torch.float32, device=q.device) if want_lse else None
        rc = library().rib_window_attn_fwd_bucketed(_ptr(q), _ptr(k), _ptr(v), _ptr(bias), dtype, stride, _ptr(buckets), count, B, H, W, heads, d,
                                                    window, shift, int(masked), _ptr(out), _ptr(lse), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return out, lse


def _check_lse(lse, B, heads, H, W, device):
    if lse.dtype != torch.float32 or tuple(lse.shape) != (B, heads, H, W) or not lse.is_contiguous() or lse.device != device:
        raise ValueError("lse must be a contiguous fp32 tensor [B,heads,H,W] on q's device")


def rib_window_attn_bwd_bucketed_workspace(bias_head_stride, num_buckets, B, H, W, heads, d, window) -> int:
    return int(library().rib_window_attn_bwd_bucketed_workspace(bias_head_stride, num_buckets, B, H, W, heads, d, window))


def rib_window_attn_bwd_bucketed(q, k, v, bias, buckets, out, lse, dout, window, shift=0, masked=False, workspace=None, stream=None):
    """Backward pass of rib_window_attn_fwd_bucketed.  Returns (dq, dk, dv bf16, dbias of bias's shape and type)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_bwd_bucketed, q, k, v, bias, buckets, out, lse, dout, window, shift, masked, workspace)
    if _marshal is not None:
        call = lambda address, *args: _marshal.bwd_bucketed(address, _lib.rib_addresses["rib_window_attn_bwd_bucketed_workspace"], *args)  # noqa: E731
        got = _native(call, "rib_window_attn_bwd_bucketed", q, k, v, bias, buckets, out, lse, dout, window, shift, masked, workspace, stream)
        if got is not None:
            return got
    _check_image("q", q)
    B, H, W, heads, d = q.shape
    for name, t in (("k", k), ("v", v), ("out", out), ("dout", dout)):
        _check_image(name, t, q.shape)
    dtype, stride, count = _check_bias(bias, buckets, heads, window, q.device)
    _check_lse(lse, B, heads, H, W, q.device)
    if workspace is None:
        need = rib_window_attn_bwd_bucketed_workspace(stride, count, B, H, W, heads, d, window)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    with _on(q.device, k, v, out, dout, workspace):
        dq, dk, dv, dbias = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q), torch.empty_like(bias)
        rc = library().rib_window_attn_bwd_bucketed(_ptr(q), _ptr(k), _ptr(v), _ptr(bias), dtype, stride, _ptr(buckets), count, _ptr(out), _ptr(lse),
                                                    _ptr(dout), B, H, W, heads, d, window, shift, int(masked), _ptr(dq), _ptr(dk), _ptr(dv),
                                                    _ptr(dbias), _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dq, dk, dv, dbias


def rib_checkpoint_store(x, stream=None):
    """x bf16 [..., d], d <= 64, as (codes int8 of x's shape, scales fp32 of x's shape without its last dimension)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_checkpoint_store, x)
    if _marshal is not None:
        got = _native(_marshal.store, "rib_checkpoint_store", x, stream)
        if got is not None:
            return got
    if x.dtype != torch.bfloat16 or not x.is_cuda or not x.is_contiguous() or x.dim() < 1:
        raise ValueError("x must be a contiguous CUDA bfloat16 tensor [..., d]")
    d = x.shape[-1]
    codes = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    scales = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    if x.numel() == 0 and 0 < d <= 64:
        return codes, scales
    with _on(x.device):
        rc = library().rib_checkpoint_store(_ptr(x), scales.numel(), d, _ptr(codes), _ptr(scales), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return codes, scales


def _check_checkpoint(name, codes, scales, shape=None):
    if codes.dtype != torch.int8 or not codes.is_cuda or not codes.is_contiguous() or codes.dim() < 1 or (shape is not None and tuple(codes.shape) != tuple(shape)):
        raise ValueError(f"the codes of {name} must be a contiguous CUDA int8 tensor " + (f"of shape {tuple(shape)}" if shape is not None else "[..., d]"))
    if scales.dtype != torch.float32 or not scales.is_contiguous() or scales.device != codes.device or scales.shape != codes.shape[:-1]:
        raise ValueError(f"the scales of {name} must be a contiguous fp32 tensor of shape {tuple(codes.shape[:-1])} on the codes' device")


def rib_checkpoint_restore(codes, scales, stream=None):
    """What rib_checkpoint_store kept, as bf16."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_checkpoint_restore, codes, scales)
    if _marshal is not None:
        got = _native(_marshal.restore, "rib_checkpoint_restore", codes, scales, stream)
        if got is not None:
            return got[0]
    _check_checkpoint("x", codes, scales)
    x = torch.empty(codes.shape, dtype=torch.bfloat16, device=codes.device)
    if x.numel() == 0 and 0 < codes.shape[-1] <= 64:
        return x
    with _on(x.device):
        rc = library().rib_checkpoint_restore(_ptr(codes), _ptr(scales), scales.numel(), codes.shape[-1], _ptr(x), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return x


def _saved(q, k, v, out, dout):
    """The C call's array of the checkpoints (codes, scales) of q, k, v and out."""
    _check_image("dout", dout)
    for name, pair in (("q", q), ("k", k), ("v", v), ("out", out)):
        _check_checkpoint(name, *pair, shape=dout.shape)
    return (ctypes.c_void_p * 8)(*[_ptr(t) for pair in (q, k, v, out) for t in pair])


def rib_window_attn_bwd_checkpointed(q, k, v, out, pq, pk, lse, dout, window, shift=0, masked=False, workspace=None, stream=None):
    """Backward pass of a layer that kept q, k, v and out as checkpoints (codes, scales); pq, pk [n, r] or [heads, n, r].  On a map whose
    sides are not multiples of the window as rib_window_attn_bwd_padded, with `masked` as rib_window_attn_bwd_masked.
    Returns (dq, dk, dv bf16, dpq, dpk fp32 of the shape of pq)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_bwd_checkpointed, q, k, v, out, pq, pk, lse, dout, window, shift, masked, workspace)
    if _marshal is not None:
        call = lambda address, *args: _marshal.bwd_checkpointed(address, _lib.rib_addresses["rib_window_attn_bwd_checkpointed_workspace"], *args)  # noqa: E731
        got = _native(call, "rib_window_attn_bwd_checkpointed", q, k, v, out, pq, pk, lse, dout, window, shift, masked, workspace, stream)
        if got is not None:
            return got
    saved = _saved(q, k, v, out, dout)
    B, H, W, heads, d = dout.shape
    n = window * window
    headwise = pq.dim() == 3
    for name, t in (("pq", pq), ("pk", pk)):
        if headwise:
            _check_pos_headwise(name, t, heads, n)
        else:
            _check_pos(name, t, n)
    r = pq.shape[-1]
    stride = n * r if headwise else 0
    _check_lse(lse, B, heads, H, W, dout.device)
    if workspace is None:
        need = int(library().rib_window_attn_bwd_checkpointed_workspace(stride, B, H, W, heads, d, r, window))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dout.device)
    with _on(dout.device, q[0], k[0], v[0], out[0], pq, pk, workspace):
        dq, dk, dv = torch.empty_like(dout), torch.empty_like(dout), torch.empty_like(dout)
        dpq = torch.empty(tuple(pq.shape), dtype=torch.float32, device=dout.device)
        dpk = torch.empty(tuple(pk.shape), dtype=torch.float32, device=dout.device)
        rc = library().rib_window_attn_bwd_checkpointed(saved, _ptr(pq), _ptr(pk), stride, _ptr(lse), _ptr(dout), B, H, W, heads, d, r, window, shift,
                                                        int(masked), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dpq), _ptr(dpk), _ptr(workspace),
                                                        workspace.numel(), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dq, dk, dv, dpq, dpk


def rib_window_attn_bwd_bucketed_checkpointed(q, k, v, out, bias, buckets, lse, dout, window, shift=0, masked=False, workspace=None, stream=None):
    """Backward pass of rib_window_attn_fwd_bucketed for a layer that kept q, k, v and out as checkpoints (codes, scales).
    Returns (dq, dk, dv bf16, dbias of bias's shape and type)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_window_attn_bwd_bucketed_checkpointed, q, k, v, out, bias, buckets, lse, dout, window, shift, masked, workspace)
    if _marshal is not None:
        call = lambda address, *args: _marshal.bwd_bucketed_checkpointed(address, _lib.rib_addresses["rib_window_attn_bwd_bucketed_checkpointed_workspace"], *args)  # noqa: E731
        got = _native(call, "rib_window_attn_bwd_bucketed_checkpointed", q, k, v, out, bias, buckets, lse, dout, window, shift, masked, workspace, stream)
        if got is not None:
            return got
    saved = _saved(q, k, v, out, dout)
    B, H, W, heads, d = dout.shape
    dtype, stride, count = _check_bias(bias, buckets, heads, window, dout.device)
    _check_lse(lse, B, heads, H, W, dout.device)
    if workspace is None:
        need = int(library().rib_window_attn_bwd_bucketed_checkpointed_workspace(stride, count, B, H, W, heads, d, window))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dout.device)
    with _on(dout.device, q[0], k[0], v[0], out[0], workspace):
        dq, dk, dv, dbias = torch.empty_like(dout), torch.empty_like(dout), torch.empty_like(dout), torch.empty_like(bias)
        rc = library().rib_window_attn_bwd_bucketed_checkpointed(saved, _ptr(bias), dtype, stride, _ptr(buckets), count, _ptr(lse), _ptr(dout), B, H, W,
                                                                 heads, d, window, shift, int(masked), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dbias),
                                                                 _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dq, dk, dv, dbias


def _check_f32(name, t, shape):
    if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be a contiguous CUDA float32 tensor of shape {tuple(shape)}")


def rib_generate_features(w_h, b_h, w_pq, w_pk, window, stream=None):
    """Pq, Pk (bf16 [window^2, r]) from the generator weights (Eq. 1-3); L is read off w_h's height 2 + 4 L."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_generate_features, w_h, b_h, w_pq, w_pk, window)
    if _marshal is not None:
        got = _native(_marshal.generate, "rib_generate_features", w_h, b_h, w_pq, w_pk, window, stream)
        if got is not None:
            return got
    rows, dh = w_h.shape
    L, r = (rows - 2) // 4, w_pq.shape[1]
    _check_f32("w_h", w_h, (2 + 4 * L, dh)); _check_f32("b_h", b_h, (dh,))
    _check_f32("w_pq", w_pq, (dh, r)); _check_f32("w_pk", w_pk, (dh, r))
    pq = torch.empty((window * window, r), dtype=torch.bfloat16, device=w_h.device)
    pk = torch.empty_like(pq)
    rc = library().rib_generate_features(_ptr(w_h), _ptr(b_h), _ptr(w_pq), _ptr(w_pk), window, L, dh, r, _ptr(pq), _ptr(pk),
                                         _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return pq, pk


def rib_generate_features_bwd(w_h, b_h, w_pq, w_pk, dpq, dpk, window, stream=None):
    """Gradients (dw_h, db_h, dw_pq, dw_pk) of the generator weights given dpq, dpk fp32 [window^2, r]."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_generate_features_bwd, w_h, b_h, w_pq, w_pk, dpq, dpk, window)
    if _marshal is not None:
        got = _native(_marshal.generate_bwd, "rib_generate_features_bwd", w_h, b_h, w_pq, w_pk, dpq, dpk, window, stream)
        if got is not None:
            return got
    rows, dh = w_h.shape
    L, r = (rows - 2) // 4, w_pq.shape[1]
    _check_f32("w_h", w_h, (2 + 4 * L, dh)); _check_f32("b_h", b_h, (dh,))
    _check_f32("w_pq", w_pq, (dh, r)); _check_f32("w_pk", w_pk, (dh, r))
    _check_f32("dpq", dpq, (window * window, r)); _check_f32("dpk", dpk, (window * window, r))
    outs = tuple(torch.empty_like(t) for t in (w_h, b_h, w_pq, w_pk))
    rc = library().rib_generate_features_bwd(_ptr(w_h), _ptr(b_h), _ptr(w_pq), _ptr(w_pk), _ptr(dpq), _ptr(dpk), window, L, dh, r,
                                             *[_ptr(t) for t in outs], _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return outs


def rib_rope_frequencies(rot, base=100.0, sequence=False, scaling=None, scale=1.0, trained=None, device="cuda"):
    """Frequencies fp32 [2, rot / 2] for rib_rope_table: the i-th of the n pairs of an axis turns by base^(-i / n), from 1 down to a little above 1 / base; the
    first half of the pairs (the larger, when their number is odd) turns along the rows and the second along the columns; with `sequence` all along the rows.  For maps larger than those a model was trained on, by a factor `scale`:
    `scaling` "linear" divides every frequency by it, "base" raises the base such that the lowest frequency is divided by it and the highest is kept, and
    "by_parts" divides those that turn less than once over `trained` positions, keeps those that turn more than 32 times, and goes over linearly in between."""
    if rot < 2 or rot % 2 or not base > 0 or not scale > 0:
        raise ValueError(f"rot has to be even and positive, base and scale positive: got {rot}, {base}, {scale}")
    if scaling not in (None, "linear", "base", "by_parts") or (scaling == "by_parts") != (trained is not None):
        raise ValueError('scaling is None, "linear", "base" or "by_parts", and `trained` (positions) goes with the last')
    pairs = rot // 2
    counts = (pairs, 0) if sequence else ((pairs + 1) // 2, pairs // 2)
    frequencies = torch.zeros(2, pairs, dtype=torch.float64)
    for axis, (first, count) in enumerate(zip((0, counts[0]), counts)):
        along = torch.arange(count, dtype=torch.float64) / max(1, count)
        raised = base * scale ** (count / (count - 1)) if scaling == "base" and count > 1 else base
        f = raised ** -along
        if scaling == "linear":
            f = f / scale
        elif scaling == "by_parts":
            kept = ((trained * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
            f = f * kept + f / scale * (1 - kept)
        frequencies[axis, first:first + count] = f
    return frequencies.float().to(device)


def rib_rope_table(frequencies, H, W, y0=0, x0=0, magnitude=1.0, stream=None):
    """Cosines and sines of a map's rows and columns, fp32 [H + W, rot / 2, 2], from frequencies fp32 [2, rot / 2] (per row, per column); (y0, x0) is the place of the
    map's first token, `magnitude` a factor of the rotated channels.  A sequence of L tokens is a map of L rows and one column.  The first H entries are the rows, and nothing in a table's
    shape says how many they are: it serves maps of these H and W, not of W and H."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_rope_table, frequencies, H, W, y0, x0, magnitude)
    if _marshal is not None:
        got = _native(_marshal.rope_table, "rib_rope_table", frequencies, H, W, y0, x0, magnitude, stream)
        if got is not None:
            return got[0]
    if frequencies.dtype != torch.float32 or not frequencies.is_cuda or not frequencies.is_contiguous() or frequencies.dim() != 2 or frequencies.shape[0] != 2:
        raise ValueError("frequencies must be a contiguous CUDA float32 tensor [2, rot / 2]")
    pairs = frequencies.shape[1]
    if H < 1 or W < 1 or pairs < 1:
        raise ValueError(f"a table needs rows, columns and pairs: got H={H}, W={W}, {pairs} pairs")
    with _on(frequencies.device):
        table = torch.empty((H + W, pairs, 2), dtype=torch.float32, device=frequencies.device)
        rc = library().rib_rope_table(_ptr(frequencies), H, W, pairs, y0, x0, magnitude, _ptr(table), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return table


def _token_rows(name, t, like=None):
    """Elements between the tokens of a bf16 tensor [B, H, W, heads, d] whose heads lie behind one another: contiguous, or a slice of heads of a contiguous one."""
    if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 5:
        raise ValueError(f"{name} must be a CUDA bfloat16 tensor [B,H,W,heads,d]")
    if like is not None and tuple(t.shape) != tuple(like):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(like)}")
    B, H, W, heads, d = t.shape
    strides = t.stride()
    for size, stride, want in ((d, strides[4], 1), (heads, strides[3], d)):
        if size > 1 and stride != want:
            raise ValueError(f"the heads of a token of {name} have to lie behind one another, got strides {strides}")
    token, tokens = None, 1                         # strides of axes of size 1 say nothing
    for size, stride in ((W, strides[2]), (H, strides[1]), (B, strides[0])):
        if size > 1:
            if token is None:
                token = stride // tokens
            if stride != token * tokens:
                raise ValueError(f"the tokens of {name} have to be evenly spaced, got strides {strides}")
        tokens *= size
    return heads * d if token is None else token


def _check_rope(q, k, q_weight, k_weight, table):
    """(q_stride, k_stride, kv_heads, weights per head, rot)"""
    q_stride = _token_rows("q", q)
    B, H, W, heads, d = q.shape
    k_stride, kv_heads = 0, 0
    if k is not None:
        k_stride = _token_rows("k", k)
        kv_heads = k.shape[3]
        if tuple(k.shape) != (B, H, W, kv_heads, d):
            raise ValueError(f"k has shape {tuple(k.shape)}, expected [{B},{H},{W},kv_heads,{d}]")
    elif k_weight is not None:
        raise ValueError("k_weight is given without k")
    per_head = None
    for name, w, count in (("q_weight", q_weight, heads), ("k_weight", k_weight, kv_heads)):
        if w is None:
            continue
        if w.dtype != torch.float32 or not w.is_contiguous() or w.device != q.device or tuple(w.shape) not in ((d,), (count, d)):
            raise ValueError(f"{name} must be a contiguous float32 tensor [{d}] or [{count}, {d}] on q's device")
        if per_head is not None and per_head != (w.dim() == 2):
            raise ValueError("q_weight and k_weight are both per head or both shared by the heads")
        per_head = w.dim() == 2
    rot = 0
    if table is not None:
        if table.dtype != torch.float32 or not table.is_contiguous() or table.device != q.device or table.dim() != 3 or table.shape[0] != H + W or table.shape[2] != 2:
            raise ValueError(f"table must be a contiguous float32 tensor [{H + W}, rot / 2, 2] on q's device")
        rot = 2 * table.shape[1]
        if rot > d:
            raise ValueError(f"the table rotates {rot} channels of a head of {d}")
    return q_stride, k_stride, kv_heads, int(bool(per_head)), rot


def rib_qk_norm_rope_fwd(q, k, q_weight=None, k_weight=None, table=None, interleaved=False, eps=1e-6, stream=None):
    """Norm of each head and rotation by position, in one pass: q bf16 [B,H,W,heads,d], k bf16 [B,H,W,kv_heads,d] or None, contiguous or slices of heads of one
    projection's output; weights fp32 [d] or [heads, d] ([kv_heads, d]), None: not normalised; table from rib_rope_table, None: not rotated.
    Returns (q, k), contiguous (k None if there is none)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_qk_norm_rope_fwd, q, k, q_weight, k_weight, table, interleaved, eps)
    if _marshal is not None:
        got = _native(_marshal.rope_fwd, "rib_qk_norm_rope_fwd", q, k, q_weight, k_weight, table, interleaved, eps, stream)
        if got is not None:
            return got
    q_stride, k_stride, kv_heads, per_head, rot = _check_rope(q, k, q_weight, k_weight, table)
    B, H, W, heads, d = q.shape
    with _on(q.device, *([] if k is None else [k])):
        q_out = torch.empty((B, H, W, heads, d), dtype=q.dtype, device=q.device)
        k_out = None if k is None else torch.empty((B, H, W, kv_heads, d), dtype=q.dtype, device=q.device)
        rc = library().rib_qk_norm_rope_fwd(_ptr(q), q_stride, _ptr(k), k_stride, _ptr(q_weight), _ptr(k_weight), per_head, _ptr(table), B, H, W, heads, kv_heads, d, rot,
                                            int(interleaved), eps, _ptr(q_out), _ptr(k_out), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return q_out, k_out


def rib_qk_norm_rope_bwd_workspace(B, H, W, heads, kv_heads, d, weight_per_head) -> int:
    return int(library().rib_qk_norm_rope_bwd_workspace(B, H, W, heads, kv_heads, d, int(weight_per_head)))


def rib_qk_norm_rope_bwd(q, k, q_weight, k_weight, table, dq_out, dk_out, interleaved=False, eps=1e-6, dq=None, dk=None, workspace=None, stream=None):
    """Backward pass of rib_qk_norm_rope_fwd, given the gradients dq_out, dk_out of its results.  Returns (dq, dk, dq_weight, dk_weight), the weights' fp32 in their
    shape (None where there is none).  dq and dk may be given: tensors, or slices of heads of the gradient of one projection's output, that are written."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_qk_norm_rope_bwd, q, k, q_weight, k_weight, table, dq_out, dk_out, interleaved, eps, dq, dk, workspace)
    if _marshal is not None and dq is None and dk is None:
        call = lambda address, *args: _marshal.rope_bwd(address, _lib.rib_addresses["rib_qk_norm_rope_bwd_workspace"], *args)  # noqa: E731
        got = _native(call, "rib_qk_norm_rope_bwd", q, k, q_weight, k_weight, table, dq_out, dk_out, interleaved, eps, workspace, stream)
        if got is not None:
            return got
    q_stride, k_stride, kv_heads, per_head, rot = _check_rope(q, k, q_weight, k_weight, table)
    B, H, W, heads, d = q.shape
    _check_image("dq_out", dq_out, q.shape)
    if (k is None) != (dk_out is None) or (k is None and dk is not None):
        raise ValueError("dk_out (and dk) go with k")
    if k is not None:
        _check_image("dk_out", dk_out, k.shape)
    if workspace is None:
        workspace = torch.empty(max(rib_qk_norm_rope_bwd_workspace(B, H, W, heads, kv_heads, d, per_head), 256), dtype=torch.uint8, device=q.device)
    given = [t for t in (k, dq_out, dk_out, dq, dk, workspace) if t is not None]
    with _on(q.device, *given):
        if dq is None:
            dq = torch.empty((B, H, W, heads, d), dtype=q.dtype, device=q.device)
        if dk is None and k is not None:
            dk = torch.empty((B, H, W, kv_heads, d), dtype=q.dtype, device=q.device)
        dq_stride, dk_stride = _token_rows("dq", dq, q.shape), 0 if k is None else _token_rows("dk", dk, k.shape)
        dq_weight, dk_weight = (None if w is None else torch.empty_like(w) for w in (q_weight, k_weight))
        rc = library().rib_qk_norm_rope_bwd(_ptr(q), q_stride, _ptr(k), k_stride, _ptr(q_weight), _ptr(k_weight), per_head, _ptr(table), _ptr(dq_out), _ptr(dk_out),
                                            B, H, W, heads, kv_heads, d, rot, int(interleaved), eps, _ptr(dq), dq_stride, _ptr(dk), dk_stride, _ptr(dq_weight),
                                            _ptr(dk_weight), _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dq, dk, dq_weight, dk_weight


def _check_states(q, k, v, lengths):
    """(kv_heads, L, contexts)"""
    _check_image("q", q)
    B, _, _, heads, d = q.shape
    for name, t in (("k", k), ("v", v)):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{name} must be a contiguous CUDA bfloat16 tensor [contexts,L,kv_heads,d]")
        if t.shape[0] not in (1, B) or t.shape[3] != d or t.shape != k.shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected [{B} or 1,L,kv_heads,{d}], k and v alike")
    contexts, L, kv_heads, _ = k.shape
    if kv_heads < 1 or heads % kv_heads:
        raise ValueError(f"{heads} query heads do not divide among {kv_heads} heads of states")
    if lengths is not None and (lengths.dtype != torch.int32 or not lengths.is_contiguous() or lengths.device != q.device or tuple(lengths.shape) != (contexts,)):
        raise ValueError(f"lengths must be a contiguous int32 tensor [{contexts}] on q's device")
    return kv_heads, L, contexts


def rib_cross_attn_fwd_workspace(B, H, W, heads, kv_heads, d, L, contexts) -> int:
    return int(library().rib_cross_attn_fwd_workspace(B, H, W, heads, kv_heads, d, L, contexts))


def rib_cross_attn_fwd(q, k, v, lengths=None, workspace=None, stream=None, want_lse=True):
    """Attention of a map's tokens q bf16 [B,H,W,heads,d] to states k, v bf16 [B,L,kv_heads,d] ([1,L,kv_heads,d]: the same for all maps); lengths int32 [B] (or [1]):
    the states of each context that are attended to.  Returns (out, lse)."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_cross_attn_fwd, q, k, v, lengths, workspace, None, want_lse)
    if _marshal is not None:
        call = lambda address, *args: _marshal.cross_fwd(address, _lib.rib_addresses["rib_cross_attn_fwd_workspace"], *args)  # noqa: E731
        got = _native(call, "rib_cross_attn_fwd", q, k, v, lengths, workspace, want_lse, stream)
        if got is not None:
            return got
    kv_heads, L, contexts = _check_states(q, k, v, lengths)
    B, H, W, heads, d = q.shape
    need = rib_cross_attn_fwd_workspace(B, H, W, heads, kv_heads, d, L, contexts)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    with _on(q.device, k, v, *([] if workspace is None else [workspace])):
        out = torch.empty_like(q)
        lse = torch.empty((B, heads, H, W), dtype=torch.float32, device=q.device) if want_lse else None
        rc = library().rib_cross_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(lengths), B, H, W, heads, kv_heads, d, L, contexts, _ptr(out), _ptr(lse),
                                          _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return out, lse


def rib_cross_attn_bwd_workspace(B, H, W, heads, kv_heads, d, L, contexts) -> int:
    return int(library().rib_cross_attn_bwd_workspace(B, H, W, heads, kv_heads, d, L, contexts))


def rib_cross_attn_bwd(q, k, v, out, lse, dout, lengths=None, workspace=None, stream=None):
    """Backward pass of rib_cross_attn_fwd.  Returns (dq, dk, dv), bf16 in the shapes of q, k, v."""
    if stream is not None and _elsewhere(stream):
        return _beside(stream, rib_cross_attn_bwd, q, k, v, out, lse, dout, lengths, workspace)
    if _marshal is not None:
        call = lambda address, *args: _marshal.cross_bwd(address, _lib.rib_addresses["rib_cross_attn_bwd_workspace"], *args)  # noqa: E731
        got = _native(call, "rib_cross_attn_bwd", q, k, v, out, lse, dout, lengths, workspace, stream)
        if got is not None:
            return got
    kv_heads, L, contexts = _check_states(q, k, v, lengths)
    B, H, W, heads, d = q.shape
    for name, t in (("out", out), ("dout", dout)):
        _check_image(name, t, q.shape)
    _check_lse(lse, B, heads, H, W, q.device)
    if workspace is None:
        workspace = torch.empty(max(rib_cross_attn_bwd_workspace(B, H, W, heads, kv_heads, d, L, contexts), 256), dtype=torch.uint8, device=q.device)
    with _on(q.device, k, v, out, dout, workspace):
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        rc = library().rib_cross_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(lengths), _ptr(out), _ptr(lse), _ptr(dout), B, H, W, heads, kv_heads, d, L, contexts,
                                          _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != RIB_OK:
        raise RibError(rc)
    return dq, dk, dv
