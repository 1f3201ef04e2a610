"""Python binding of libhsa, the GB300 hot path of Heterogeneous Step Allocation.

Argument marshalling only: each function below has the name of a C entry
point of include/hsa.h, turns torch tensors into raw pointers and sizes, calls
the C function through ctypes on the current torch CUDA stream (or the stream
given), and raises HsaError on a negative status.  Every step runs in the
library's CUDA kernels; there is no Python or CPU fallback, and importing this
package fails loudly when libhsa.so has not been built.

Device tensors must be contiguous and live on the current CUDA device.
"""
from __future__ import annotations

import ctypes
import math
import os

import torch

__all__ = [
    "HsaError", "lib", "library_path", "HSA_BF16", "HSA_F32",
    "hsa_status_string", "hsa_version", "hsa_check_budgets", "hsa_window_margin",
    "hsa_active_count", "hsa_sigma_schedule", "hsa_partition_workspace_bytes",
    "hsa_partition", "hsa_partition_static", "hsa_uniform_stat", "hsa_reserve_first_frame",
    "hsa_reorder_tokens", "hsa_partition_active", "hsa_gather_active",
    "hsa_kv_sync_scatter", "hsa_check_indices", "hsa_check_indices_workspace_bytes",
    "hsa_rope_table", "hsa_rope_rows", "hsa_kv_sync_scatter_rope",
    "hsa_active_attention", "hsa_active_attention_prefix",
    "hsa_active_attention_workspace_bytes",
    "hsa_cached_euler", "hsa_cached_euler_l1rel",
    "HSA_E4M3", "hsa_kv_quant_scatter", "hsa_kv_dequant_gather",
    "hsa_paged_attention", "hsa_paged_attention_workspace_bytes",
    "hsa_packed_attention", "hsa_packed_attention_workspace_bytes",
    "hsa_get_device_error", "hsa_launch_count", "hsa_test_inject_attention_stall",
    "hsa_test_f32_cluster",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
library_path = os.path.join(_HERE, "libhsa.so")

HSA_BF16, HSA_F32, HSA_E4M3 = 0, 1, 2
HSA_PARTITION_STATIC_MAX_TOKENS = 524288
STATUS = {0: "HSA_OK", -1: "HSA_ERR_INVALID_ARG", -2: "HSA_ERR_NOT_DIVISOR",
          -3: "HSA_ERR_BAD_COUNTS", -4: "HSA_ERR_UNSUPPORTED", -5: "HSA_ERR_NONFINITE",
          -6: "HSA_ERR_INDEX", -7: "HSA_ERR_TIMEOUT", -8: "HSA_ERR_CUDA",
          -9: "HSA_ERR_WORKSPACE"}


class HsaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)} ({status})")


_c_int, _c_p, _c_sz, _c_f, _c_d = (ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t,
                                   ctypes.c_float, ctypes.c_double)
_c_ll = ctypes.c_longlong
_SIGS = {
    "hsa_status_string": ([_c_int], ctypes.c_char_p),
    "hsa_version": ([], _c_int),
    "hsa_check_budgets": ([_c_int, _c_p, _c_p, _c_int, _c_int], _c_int),
    "hsa_window_margin": ([_c_int, _c_int], _c_int),
    "hsa_active_count": ([_c_p, _c_p, _c_int, _c_int, _c_int, _c_int], _c_int),
    "hsa_sigma_schedule": ([_c_int, _c_d, _c_p], _c_int),
    "hsa_partition_workspace_bytes": ([_c_int], _c_sz),
    "hsa_partition": ([_c_p, _c_int, _c_int, _c_p, _c_p, _c_int, _c_p, _c_p, _c_sz, _c_p],
                      _c_int),
    "hsa_partition_static": ([_c_p, _c_int, _c_int, _c_p, _c_p, _c_int, _c_p, _c_p], _c_int),
    "hsa_uniform_stat": ([_c_p, _c_int, _c_p], _c_int),
    "hsa_reserve_first_frame": ([_c_p, _c_int, _c_int, _c_p], _c_int),
    "hsa_partition_active": ([_c_p, _c_int, _c_int, _c_p, _c_int, _c_int, _c_int, _c_p, _c_p,
                              _c_p], _c_int),
    "hsa_gather_active": ([_c_p, _c_sz, _c_int, _c_p, _c_int, _c_p, _c_p], _c_int),
    "hsa_kv_sync_scatter": ([_c_p, _c_p, _c_p, _c_p, _c_p, _c_int, _c_int, _c_int, _c_int,
                             _c_int, _c_p], _c_int),
    "hsa_active_attention": ([_c_p, _c_p, _c_int, _c_p, _c_p, _c_int, _c_int, _c_int, _c_f,
                              _c_p, _c_int, _c_p, _c_sz, _c_p], _c_int),
    "hsa_active_attention_prefix": ([_c_p, _c_p, _c_int, _c_p, _c_p, _c_int, _c_p, _c_p, _c_int,
                                     _c_int, _c_int, _c_f, _c_p, _c_int, _c_p, _c_sz, _c_p],
                                    _c_int),
    "hsa_check_indices_workspace_bytes": ([_c_int], _c_sz),
    "hsa_check_indices": ([_c_p, _c_int, _c_int, _c_p, _c_sz, _c_p], _c_int),
    "hsa_rope_table": ([_c_int, _c_int, _c_int, _c_int, _c_d, _c_p], _c_int),
    "hsa_rope_rows": ([_c_p, _c_p, _c_int, _c_int, _c_int, _c_p, _c_int, _c_p], _c_int),
    "hsa_kv_sync_scatter_rope": ([_c_p, _c_p, _c_p, _c_p, _c_p, _c_int, _c_int, _c_int, _c_int,
                                  _c_p, _c_p], _c_int),
    "hsa_reorder_tokens": ([_c_p, _c_int, _c_int, _c_p, _c_p, _c_p, _c_p], _c_int),
    "hsa_active_attention_workspace_bytes": ([_c_int, _c_int, _c_int, _c_int, _c_int], _c_sz),
    "hsa_cached_euler": ([_c_p, _c_p, _c_p, _c_p, _c_int, _c_int, _c_int, _c_f, _c_p], _c_int),
    "hsa_cached_euler_l1rel": ([_c_p, _c_p, _c_p, _c_p, _c_int, _c_int, _c_int, _c_f, _c_p,
                                _c_f, _c_p], _c_int),
    "hsa_kv_quant_scatter": ([_c_p] * 7 + [_c_int] * 5 + [_c_p, _c_p, _c_int, _c_p], _c_int),
    "hsa_kv_dequant_gather": ([_c_p] * 5 + [_c_int] * 4 + [_c_p, _c_p, _c_int, _c_p], _c_int),
    "hsa_paged_attention": ([_c_p, _c_int, _c_int, _c_int] + [_c_p] * 4 + [_c_int] * 5 +
                            [_c_p, _c_int, _c_p, _c_f, _c_p, _c_p, _c_sz, _c_p], _c_int),
    "hsa_paged_attention_workspace_bytes": ([_c_int] * 5, _c_sz),
    "hsa_packed_attention": ([_c_p, _c_ll, _c_p, _c_ll, _c_p, _c_ll, _c_p, _c_p] + [_c_int] * 7 +
                             [_c_f, _c_p, _c_int, _c_p, _c_sz, _c_p], _c_int),
    "hsa_packed_attention_workspace_bytes": ([_c_int] * 3, _c_sz),
    "hsa_get_device_error": ([_c_p], _c_int),
    "hsa_launch_count": ([], ctypes.c_ulonglong),
    "hsa_test_inject_attention_stall": ([_c_int], _c_int),
    "hsa_test_f32_cluster": ([_c_int] * 7, _c_int),
}

_lib = None
# torch's own, not part of its public interface: None where a torch lacks them
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def lib() -> ctypes.CDLL:
    """The loaded libhsa.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(library_path):
            raise ImportError(
                f"libhsa.so not found at {library_path}; build it with "
                "`python -m paper_2605_06892_gb300.build` (or __graft_entry__.build())")
        handle = ctypes.CDLL(library_path)
        for name, (args, res) in _SIGS.items():
            f = getattr(handle, name)
            f.argtypes = args
            f.restype = res
        _lib = handle
    return _lib


# ------------------------------------------------------------- marshalling

def _p(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensors passed to libhsa must be contiguous"
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        # The current stream's handle as torch keeps it: 0.2 us, against 2.9 us
        # for building the torch.cuda.Stream object (a third of a small call's
        # host time on the Grace host).  Before CUDA is initialised, and on a torch
        # without these two functions, the object's constructor serves.
        if _raw_stream and _current_device and torch.cuda.is_initialized():
            return _raw_stream(_current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# int arrays of the usual group counts; looking the type up costs more than
# filling it
_INT_ARRAYS = tuple(ctypes.c_int * max(1, n) for n in range(33))


def _host_ints(xs) -> ctypes.Array:
    n = len(xs := tuple(xs))
    return (_INT_ARRAYS[n] if n < len(_INT_ARRAYS) else ctypes.c_int * n)(*xs)


def _check(st: int, where: str) -> int:
    if st < 0:
        raise HsaError(st, where)
    return st


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return HSA_BF16
    if t.dtype == torch.float32:
        return HSA_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _place(name, t, dtype, device):
    """The address of a contiguous tensor of this dtype on this device; any other is
    refused.  What C cannot see of a tensor is checked here; sizes are compared apart."""
    if t.dtype is dtype and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    if t.dtype is not dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, not {dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, not on the current CUDA device")
    raise ValueError(f"{name} is not contiguous")


def _sized(name, t, shape):
    """Refuses a tensor of another shape."""
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")


def _device() -> int:
    """The current CUDA device; -2 where there is none, since a CPU tensor says -1."""
    if _current_device and torch.cuda.is_initialized():
        return _current_device()
    return torch.cuda.current_device() if torch.cuda.is_available() else -2


def _scratch(t, device):
    """Address and bytes of a workspace (None: none)."""
    if t is None:
        return None, 0
    return _place("workspace", t, t.dtype, device), t.numel() * t.element_size()


# ---------------------------------------------------------- host helpers

def hsa_status_string(status: int) -> str:
    return lib().hsa_status_string(status).decode()


def hsa_version() -> int:
    return lib().hsa_version()


def hsa_check_budgets(T: int, budgets, counts, N: int) -> int:
    c = None if counts is None else _host_ints(counts)
    return lib().hsa_check_budgets(T, _host_ints(budgets), c, len(budgets), N)


def hsa_window_margin(T: int, window_pct: int) -> int:
    return _check(lib().hsa_window_margin(T, window_pct), "hsa_window_margin")


def hsa_active_count(budgets, counts, T: int, iter_: int, window_pct: int = 100) -> int:
    return _check(lib().hsa_active_count(_host_ints(budgets), _host_ints(counts), len(budgets),
                                         T, iter_, window_pct), "hsa_active_count")


def hsa_sigma_schedule(T: int, shift: float = 1.0) -> list:
    buf = (ctypes.c_double * (T + 1))()
    _check(lib().hsa_sigma_schedule(T, float(shift), buf), "hsa_sigma_schedule")
    return list(buf)


# ----------------------------------------------------------- device calls

def hsa_partition_workspace_bytes(N: int) -> int:
    return lib().hsa_partition_workspace_bytes(N)


def hsa_partition(stat, T: int, budgets, counts, group_of, workspace, stream=None) -> None:
    """group_of[N] (int32, device) <- group of each token; workspace: uint8 device
    tensor of at least hsa_partition_workspace_bytes(N) bytes."""
    N = stat.numel()
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().hsa_partition(_p(stat), N, T, _host_ints(budgets), _host_ints(counts),
                               len(budgets), _p(group_of), _p(workspace), ws_bytes,
                               _stream(stream)), "hsa_partition")


def hsa_partition_static(stat, T: int, budgets, counts, group_of, stream=None) -> None:
    """hsa_partition with the library's own fixed scratch instead of a caller
    workspace (N <= HSA_PARTITION_STATIC_MAX_TOKENS); calls must not overlap
    on the GPU."""
    _check(lib().hsa_partition_static(_p(stat), stat.numel(), T, _host_ints(budgets),
                                      _host_ints(counts), len(budgets), _p(group_of),
                                      _stream(stream)), "hsa_partition_static")


def hsa_uniform_stat(stat, stream=None) -> None:
    """stat[n] <- uniform-allocation statistic (App. B, U)."""
    _check(lib().hsa_uniform_stat(_p(stat), stat.numel(), _stream(stream)), "hsa_uniform_stat")


def hsa_reserve_first_frame(stat, frame_tokens: int, stream=None) -> None:
    """stat[:frame_tokens] <- FLT_MAX (App. B, F)."""
    _check(lib().hsa_reserve_first_frame(_p(stat), stat.numel(), frame_tokens,
                                         _stream(stream)), "hsa_reserve_first_frame")


def hsa_partition_active(group_of, T: int, budgets, iter_: int, idx, pos=None,
                         window_pct: int = 100, stream=None) -> None:
    _check(lib().hsa_partition_active(_p(group_of), group_of.numel(), T, _host_ints(budgets),
                                      len(budgets), iter_, window_pct, _p(idx), _p(pos),
                                      _stream(stream)), "hsa_partition_active")


def hsa_gather_active(src, idx, n_active: int, dst, stream=None) -> None:
    """dst[:n_active] = src[idx[:n_active]] (rows = first dimension)."""
    N = src.shape[0]
    row_bytes = (src.numel() // max(N, 1)) * src.element_size()
    _check(lib().hsa_gather_active(_p(src), row_bytes, N, _p(idx), n_active, _p(dst),
                                   _stream(stream)), "hsa_gather_active")


def hsa_kv_sync_scatter(k_cache, v_cache, k_fresh, v_fresh, idx, n_active: int,
                        stream=None) -> None:
    N, H, D = k_cache.shape
    _check(lib().hsa_kv_sync_scatter(_p(k_cache), _p(v_cache), _p(k_fresh), _p(v_fresh),
                                     _p(idx), n_active, N, H, D, _dtype_code(k_cache),
                                     _stream(stream)), "hsa_kv_sync_scatter")


def hsa_check_indices_workspace_bytes(N: int) -> int:
    return lib().hsa_check_indices_workspace_bytes(N)


def hsa_check_indices(idx, n: int, N: int, workspace, stream=None) -> None:
    """Opt-in check of idx[:n]: HSA_ERR_INDEX (via hsa_get_device_error) when an
    entry is outside [0, N) or repeated; workspace: uint8 device tensor of at
    least hsa_check_indices_workspace_bytes(N) bytes."""
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().hsa_check_indices(_p(idx), n, N, _p(workspace), ws_bytes, _stream(stream)),
           "hsa_check_indices")


def hsa_rope_table(grid, D: int, theta: float = 10000.0) -> torch.Tensor:
    """Host fp32 [N, D/2, 2] (cos, sin) table of a (F, Hh, Ww) token grid."""
    F, Hh, Ww = grid
    out = torch.empty((F * Hh * Ww, D // 2, 2), dtype=torch.float32)
    _check(lib().hsa_rope_table(F, Hh, Ww, D, float(theta), out.data_ptr()), "hsa_rope_table")
    return out


def hsa_rope_rows(x, idx, n: int, table, stream=None) -> None:
    _, H, D = x.shape
    _check(lib().hsa_rope_rows(_p(x), _p(idx), n, H, D, _p(table), table.shape[0],
                               _stream(stream)), "hsa_rope_rows")


def hsa_kv_sync_scatter_rope(k_cache, v_cache, k_fresh, v_fresh, idx, n_active: int, table,
                             stream=None) -> None:
    N, H, D = k_cache.shape
    _check(lib().hsa_kv_sync_scatter_rope(_p(k_cache), _p(v_cache), _p(k_fresh), _p(v_fresh),
                                          _p(idx), n_active, N, H, D, _p(table),
                                          _stream(stream)), "hsa_kv_sync_scatter_rope")


def hsa_active_attention_prefix(q, q_idx, n_active: int, k_cache, v_cache, k_base, v_base, out,
                                scale: float = 0.0, workspace=None, stream=None) -> None:
    """Attention against the M cached rows followed by the B baseline rows."""
    M, H, D = k_cache.shape
    B = k_base.shape[0]
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().hsa_active_attention_prefix(
        _p(q), _p(q_idx), n_active, _p(k_cache) if M else None, _p(v_cache) if M else None, M,
        _p(k_base) if B else None, _p(v_base) if B else None, B, H, D, float(scale), _p(out),
        _dtype_code(k_cache if M else k_base), _p(workspace), ws_bytes, _stream(stream)),
        "hsa_active_attention_prefix")


def hsa_reorder_tokens(group_of, n_baseline: int, order, where=None, group_new=None,
                       stream=None) -> None:
    _check(lib().hsa_reorder_tokens(_p(group_of), group_of.numel(), n_baseline, _p(order),
                                    _p(where), _p(group_new), _stream(stream)),
           "hsa_reorder_tokens")


def hsa_active_attention_workspace_bytes(n_active: int, N: int, H: int, D: int,
                                         dtype: int = HSA_BF16) -> int:
    return lib().hsa_active_attention_workspace_bytes(n_active, N, H, D, dtype)


def hsa_active_attention(q, q_idx, n_active: int, k_cache, v_cache, out, scale: float = 0.0,
                         workspace=None, stream=None) -> None:
    """out[j] = attention of query row q_idx[j] (q: [N,H,D]) or j (q_idx None,
    q: [n_active,H,D]) against the full cache; `workspace` (optional uint8
    device tensor) lets the last wave of CTAs be split along the keys."""
    N, H, D = k_cache.shape
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().hsa_active_attention(_p(q), _p(q_idx), n_active, _p(k_cache), _p(v_cache), N,
                                      H, D, float(scale), _p(out), _dtype_code(k_cache),
                                      _p(workspace), ws_bytes, _stream(stream)),
           "hsa_active_attention")


def hsa_cached_euler(x, v_cache, v_fresh, pos, dsigma: float, n_fresh: int | None = None,
                     stream=None) -> None:
    N, C = x.shape
    if n_fresh is None:
        n_fresh = 0 if v_fresh is None else v_fresh.shape[0]
    _check(lib().hsa_cached_euler(_p(x), _p(v_cache), _p(v_fresh), _p(pos), n_fresh, N, C,
                                  float(dsigma), _stream(stream)), "hsa_cached_euler")


def hsa_cached_euler_l1rel(x, v_cache, v_fresh, pos, dsigma: float, stat, weight: float,
                           n_fresh: int | None = None, stream=None) -> None:
    N, C = x.shape
    if n_fresh is None:
        n_fresh = v_fresh.shape[0]
    _check(lib().hsa_cached_euler_l1rel(_p(x), _p(v_cache), _p(v_fresh), _p(pos), n_fresh, N, C,
                                        float(dsigma), _p(stat), float(weight),
                                        _stream(stream)), "hsa_cached_euler_l1rel")


# ------------------------------------------------ 8-bit cache, paged attention

_MOST = 2 ** 31 - 1   # C's int: ctypes would pass on a larger number's low 32 bits


def _rows_of(name, t, size, n):
    """Refuses fewer than n rows, or rows of other sizes than a cache of this shape has."""
    shape = t.shape
    if n > _MOST:
        raise ValueError(f"{name}: {n} rows are more than a call takes")
    if len(shape) != 3 or shape[1] != size[-2] or shape[2] != size[-1] or not 0 <= n <= shape[0]:
        raise ValueError(f"{name} has shape {tuple(shape)}, not {n} or more rows of {size[-2]} "
                         f"heads x {size[-1]}")
    return shape


def _ids(name, t, n, device):
    """Address of at least n indices."""
    if t.numel() < n:
        raise ValueError(f"{name} holds fewer than {n} indices")
    return _place(name, t, torch.int32, device)


def _cache8(k_cache, v_cache, k_scale, v_scale, size, device):
    """Addresses of an 8-bit cache's four tensors, its rows, heads and dimensions."""
    code = k_cache.dtype
    if code is not torch.float8_e4m3fn and code is not torch.uint8:
        raise TypeError(f"the cache's codes have dtype {code}, not float8_e4m3fn or uint8")
    *lead, H, D = size
    N = math.prod(lead)
    if N > _MOST:
        raise ValueError(f"k_cache holds {N} rows, more than a call takes")
    scales = (*lead, H)
    _sized("v_cache", v_cache, size)
    _sized("k_scale", k_scale, scales)
    _sized("v_scale", v_scale, scales)
    return (_place("k_cache", k_cache, code, device), _place("v_cache", v_cache, code, device),
            _place("k_scale", k_scale, torch.uint8, device),
            _place("v_scale", v_scale, torch.uint8, device), N, H, D)


def hsa_kv_quant_scatter(k_cache, v_cache, k_scale, v_scale, k_fresh, v_fresh, idx, n_active: int,
                         table=None, table_idx=None, stream=None) -> None:
    """Fresh rows [>= n_active, H, D] (bf16 or fp32) into rows idx of an 8-bit cache: codes
    [N, H, D] (float8_e4m3fn or uint8) and scale bytes [N, H] (uint8); a cache in pages [P,
    page, H, D] with scales [P, page, H] counts as P * page rows.  table: K is rotated first
    (bf16), by the table's rows table_idx (idx where that is None)."""
    dev, size, dt = _device(), k_cache.shape, k_fresh.dtype
    _sized("v_fresh", v_fresh, _rows_of("k_fresh", k_fresh, size, n_active))
    if table is not None:
        _sized("table", table, (table.shape[0], size[-1] // 2, 2))
    kc, vc, ks, vs, N, H, D = _cache8(k_cache, v_cache, k_scale, v_scale, size, dev)
    tp = ip = None
    rows = 0
    if table is not None:
        rows, tp = table.shape[0], _place("table", table, torch.float32, dev)
    if table_idx is not None:
        ip = _ids("table_idx", table_idx, n_active, dev)
    _check(lib().hsa_kv_quant_scatter(
        kc, vc, ks, vs, _place("k_fresh", k_fresh, dt, dev), _place("v_fresh", v_fresh, dt, dev),
        _ids("idx", idx, n_active, dev), n_active, N, H, D, _dtype_code(k_fresh), tp, ip, rows,
        _stream(stream)), "hsa_kv_quant_scatter")


def hsa_kv_dequant_gather(k_cache, v_cache, k_scale, v_scale, idx, n: int, k_out, v_out,
                          stream=None) -> None:
    """k_out[:n], v_out[:n] ([>= n, H, D], bf16 or fp32) <- rows idx[:n] of an 8-bit cache
    (idx None: rows 0 .. n-1); the cache as for hsa_kv_quant_scatter."""
    dev, size, dt = _device(), k_cache.shape, k_out.dtype
    _sized("v_out", v_out, _rows_of("k_out", k_out, size, n))
    kc, vc, ks, vs, N, H, D = _cache8(k_cache, v_cache, k_scale, v_scale, size, dev)
    _check(lib().hsa_kv_dequant_gather(
        kc, vc, ks, vs, None if idx is None else _ids("idx", idx, n, dev), n, N, H, D,
        _place("k_out", k_out, dt, dev), _place("v_out", v_out, dt, dev), _dtype_code(k_out),
        _stream(stream)), "hsa_kv_dequant_gather")


def hsa_paged_attention_workspace_bytes(batch: int, n_new: int, Hq: int, Hkv: int, D: int) -> int:
    return lib().hsa_paged_attention_workspace_bytes(batch, n_new, Hq, Hkv, D)


def hsa_paged_attention(q, k_pages, v_pages, page_table, seq_lens, out, k_scale=None, v_scale=None,
                        scale: float = 0.0, workspace=None, stream=None) -> None:
    """out = attention of the newest tokens q [batch, n_new, Hq, D] over each sequence's
    seq_lens[b] keys, held in pages [n_pages, page, Hkv, D] named by page_table [batch,
    max_pages]; bf16 pages, or 8-bit ones (float8_e4m3fn or uint8) with their scale bytes
    [n_pages, page, Hkv].  workspace: uint8 device tensor of at least
    hsa_paged_attention_workspace_bytes(...) bytes."""
    dev, size, pool = _device(), q.shape, k_pages.shape
    B, n_new, Hq, D = size
    n_pages, page, Hkv, Dk = pool
    batch, cols = page_table.shape
    if Dk != D or batch != B or seq_lens.shape != (B,):
        raise ValueError("q, k_pages, page_table and seq_lens disagree on the batch or the head "
                         "dimension")
    _sized("out", out, size)
    qp = _place("q", q, torch.bfloat16, dev)
    if k_scale is None and v_scale is None:
        _sized("v_pages", v_pages, pool)
        kp = _place("k_pages", k_pages, torch.bfloat16, dev)
        vp = _place("v_pages", v_pages, torch.bfloat16, dev)
        ks, vs, code = None, None, HSA_BF16
    elif k_scale is None or v_scale is None:
        raise TypeError("an 8-bit cache has both k_scale and v_scale")
    else:
        kp, vp, ks, vs, *_ = _cache8(k_pages, v_pages, k_scale, v_scale, pool, dev)
        code = HSA_E4M3
    where, room = _scratch(workspace, dev)
    _check(lib().hsa_paged_attention(
        qp, B, n_new, Hq, kp, vp, ks, vs, n_pages, page, Hkv, D,
        code, _place("page_table", page_table, torch.int32, dev), cols,
        _place("seq_lens", seq_lens, torch.int32, dev), float(scale),
        _place("out", out, torch.bfloat16, dev), where, room, _stream(stream)),
        "hsa_paged_attention")


def hsa_packed_attention_workspace_bytes(Hq: int, Hkv: int, D: int) -> int:
    return lib().hsa_packed_attention_workspace_bytes(Hq, Hkv, D)


def _token_rows(name, t, device):
    """Address of bf16 token rows [tokens, H, D] on the device whose heads lie together, and
    the elements from a row to the next: the rows may lie apart, as in a fused projection's
    output."""
    tokens, H, D = t.shape
    if t.is_contiguous():
        return _place(name, t, torch.bfloat16, device), H * D
    row, head, one = t.stride()
    if one != 1 or (head != D and H > 1):
        raise ValueError(f"{name} is not rows of {H} heads x {D} that lie together")
    _place(name, t[0], torch.bfloat16, device)
    return t.data_ptr(), row


def hsa_packed_attention(q, k, v, cu_q, cu_k, out, mask: int = 0, scale: float = 0.0,
                         workspace=None, stream=None) -> None:
    """out [total_q, Hq, D] = attention of packed sequences: queries q[cu_q[b]:cu_q[b+1]] of
    [total_q, Hq, D] over k, v[cu_k[b]:cu_k[b+1]] of [total_k, Hkv, D], bf16; mask 0: none,
    F: causal by frames of F tokens (1: causal).  The rows of q, k and v may be slices of a
    wider tensor.  workspace (optional): uint8 device tensor of
    hsa_packed_attention_workspace_bytes(Hq, Hkv, D) bytes."""
    dev, size, keys, ends = _device(), q.shape, k.shape, cu_q.shape
    total_q, Hq, D = size
    total_k, Hkv, Dk = keys
    if Dk != D or len(ends) != 1:
        raise ValueError("q and k disagree on the head dimension, or cu_q is not a vector")
    if not -_MOST <= mask <= _MOST:
        raise ValueError(f"mask is {mask}, not 0 or a frame's tokens")
    _sized("v", v, keys)
    _sized("cu_k", cu_k, ends)
    _sized("out", out, size)
    qp, q_row = _token_rows("q", q, dev)
    kp, k_row = _token_rows("k", k, dev)
    vp, v_row = _token_rows("v", v, dev)
    where, room = _scratch(workspace, dev)
    _check(lib().hsa_packed_attention(
        qp, q_row, kp, k_row, vp, v_row, _place("cu_q", cu_q, torch.int32, dev),
        _place("cu_k", cu_k, torch.int32, dev), ends[0] - 1, total_q, total_k, Hq, Hkv, D, mask,
        float(scale), _place("out", out, torch.bfloat16, dev), HSA_BF16, where, room,
        _stream(stream)), "hsa_packed_attention")


def hsa_get_device_error(stream=None) -> int:
    """Status of the device-side checks since the last call (synchronises)."""
    return lib().hsa_get_device_error(_stream(stream))


def hsa_launch_count() -> int:
    """Kernels this library has launched in this process (host counter)."""
    return int(lib().hsa_launch_count())


def hsa_test_inject_attention_stall(mode: int) -> int:
    """Test hook (include/hsa_test.h): mode 1 makes following bf16 attention
    launches never load their first value tile, so the bounded wait for it runs
    out and HSA_ERR_TIMEOUT is reported; mode 0 restores normal operation."""
    return _check(lib().hsa_test_inject_attention_stall(mode), "hsa_test_inject_attention_stall")


def hsa_test_f32_cluster(n_active: int, N: int, H: int, D: int, sms: int, wide_most: int,
                         deep_most: int) -> int:
    """Test hook (include/hsa_test.h): CTAs per cluster of the fp32 attention's launch
    plan where clusters of at most wide_most / deep_most CTAs can be resident, plus
    256 for its deep kernel.  Needs no GPU."""
    return _check(lib().hsa_test_f32_cluster(n_active, N, H, D, sms, wide_most, deep_most),
                  "hsa_test_f32_cluster")
