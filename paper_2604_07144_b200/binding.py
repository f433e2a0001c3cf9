"""ctypes binding of the C ABI in ``include/ap_serving.h``.

Argument marshalling only: every function here has the name of the C entry
point without the ``ap_`` prefix and forwards to it.  Device buffers may be
``torch`` CUDA tensors (their ``data_ptr()`` is passed), raw integer
addresses, or ``None``; host arrays are numpy.  Errors from the library raise
:class:`ApError` carrying the status code.

There is no fallback: if ``libap_serving.so`` cannot be loaded or built, the
import of the library fails with an error.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct
from typing import Optional, Sequence, Tuple

import numpy as np

AP_OK = 0
AP_ERR_INVALID_ARG = -1
AP_ERR_OUT_OF_PAGES = -2
AP_ERR_BAD_BLOCK_TABLE = -3
AP_ERR_WORKSPACE_TOO_SMALL = -4
AP_ERR_CUDA = -5
AP_ERR_TIMEOUT = -6
AP_ERR_UNSUPPORTED = -7

_HERE = os.path.dirname(os.path.abspath(__file__))
#: the shared library; ``AP_SERVING_LIB`` selects another build of the same ABI
LIB_PATH = os.environ.get("AP_SERVING_LIB") or os.path.join(_HERE, "libap_serving.so")

#: every symbol ``include/ap_serving.h`` declares
EXPORTED_SYMBOLS = (
    "ap_status_string", "ap_kv_pool_bytes", "ap_kv_pool_create", "ap_kv_pool_destroy",
    "ap_kv_pool_k_base", "ap_kv_pool_v_base", "ap_kv_pool_alloc_pages", "ap_kv_pool_free_pages",
    "ap_kv_pool_seed_free_list", "ap_kv_pool_num_free", "ap_kv_pool_set_side_by_side", "ap_plan_create", "ap_plan_destroy",
    "ap_plan_workspace_bytes", "ap_plan_get_info", "ap_plan_predict", "ap_plan_export", "ap_kv_append", "ap_kv_copy_pages",
    "ap_attention_iteration", "ap_serving_iteration_host", "ap_last_device_status",
    "ap_profile_enable", "ap_profile_collect",
    "ap_static_workspace_bytes", "ap_attention_iteration_static",
    "ap_kv_pool_set_wait_limit", "ap_selftest_wait_timeout", "ap_kv_pool_set_single_launch",
    "ap_plan_create_windowed", "ap_kv_pool_bytes_4bit", "ap_kv_pool_create_4bit", "ap_kv_append_rope", "ap_kv_read_new",
)


class ApError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__(f"{where}: {status_string(status)} ({status})")


class PoolDesc(ctypes.Structure):
    _fields_ = [("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("k_base", ctypes.c_void_p), ("v_base", ctypes.c_void_p), ("device", ctypes.c_int32)]


class BatchDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("q_lens", ctypes.c_void_p), ("ctx_lens", ctypes.c_void_p),
                ("block_tables", ctypes.c_void_p), ("table_stride", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float)]


class WindowDesc(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("sinks", ctypes.c_int32)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("base", ctypes.c_double),
                ("inv_freq", ctypes.c_void_p), ("amplitude", ctypes.c_float), ("q_row_stride", ctypes.c_int64),
                ("k_row_stride", ctypes.c_int64), ("v_row_stride", ctypes.c_int64)]


#: RopeDesc in one piece: a ctypes structure takes three times as long to fill, a twentieth of a rotated append's call
_ROPE_DESC = struct.Struct("@iidPf4xqqq")
_FP32_MAX = 3.4028234663852886e38


class PlanInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "n_new", "kv_tokens", "decode_rows", "prefill_seqs", "prefill_pairs", "decode_items",
        "decode_ctas", "merge_entries", "prefill_tiles", "launches_append", "launches_attention",
        "side_by_side", "decode_head_block")]

    def as_dict(self):
        return {n: int(getattr(self, n)) for n, _ in self._fields_}


class PlanPrediction(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in (
        "decode_bytes", "decode_flops", "prefill_bytes", "prefill_flops", "append_bytes",
        "roofline_decode_us", "roofline_prefill_us", "roofline_append_us",
        "model_decode_us", "model_prefill_us", "model_step_us")]

    def as_dict(self):
        return {n: float(getattr(self, n)) for n, _ in self._fields_}


class PlanLayout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "total_ints", "append_dst", "bt_flat", "decode_items", "cta_begin", "merge_entries",
        "prefill_tiles", "n_bt", "n_cta_begin")]


class KernelTimes(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * 4), ("launches", ctypes.c_int64 * 4)]


KERNEL_NAMES = ("kv_append", "decode_splitk", "prefill", "mixed_iteration")

_lib: Optional[ctypes.CDLL] = None


def load(build_if_missing: bool = True) -> ctypes.CDLL:
    """Loads (building first if the file is absent) ``libap_serving.so``."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        if not build_if_missing:
            raise ImportError(f"{LIB_PATH} is missing; run python -m paper_2604_07144_b200.build")
        from . import build as _build
        _build.build()
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, u64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64, ctypes.c_size_t
    sigs = {
        "ap_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "ap_kv_pool_bytes": (sz, [ctypes.POINTER(PoolDesc)]),
        "ap_kv_pool_create": (ctypes.c_int, [ctypes.POINTER(vp), ctypes.POINTER(PoolDesc)]),
        "ap_kv_pool_destroy": (ctypes.c_int, [vp]),
        "ap_kv_pool_k_base": (vp, [vp]),
        "ap_kv_pool_v_base": (vp, [vp]),
        "ap_kv_pool_alloc_pages": (ctypes.c_int, [vp, i32, vp]),
        "ap_kv_pool_free_pages": (ctypes.c_int, [vp, i32, vp]),
        "ap_kv_pool_seed_free_list": (ctypes.c_int, [vp, u64]),
        "ap_kv_pool_num_free": (i32, [vp]),
        "ap_kv_pool_set_side_by_side": (ctypes.c_int, [vp, i32]),
        "ap_plan_create": (ctypes.c_int, [ctypes.POINTER(vp), vp, ctypes.POINTER(BatchDesc), vp]),
        "ap_kv_pool_bytes_4bit": (sz, [ctypes.POINTER(PoolDesc)]),
        "ap_kv_pool_create_4bit": (ctypes.c_int, [ctypes.POINTER(vp), ctypes.POINTER(PoolDesc)]),
        "ap_kv_append_rope": (ctypes.c_int, [vp, vp, vp, vp, vp, vp, vp, vp]),      # (the description: bytes or a RopeDesc by reference)
        "ap_kv_read_new": (ctypes.c_int, [vp, vp, vp, vp, vp]),
        "ap_plan_create_windowed": (ctypes.c_int, [ctypes.POINTER(vp), vp, ctypes.POINTER(BatchDesc),
                                                   ctypes.POINTER(WindowDesc), vp]),
        "ap_plan_destroy": (ctypes.c_int, [vp]),
        "ap_plan_workspace_bytes": (sz, [vp]),
        "ap_plan_predict": (ctypes.c_int, [vp, ctypes.c_double, ctypes.c_double, ctypes.POINTER(PlanPrediction)]),
        "ap_plan_get_info": (ctypes.c_int, [vp, ctypes.POINTER(PlanInfo)]),
        "ap_plan_export": (ctypes.c_int, [vp, vp, sz, ctypes.POINTER(PlanLayout)]),
        "ap_kv_append": (ctypes.c_int, [vp, vp, vp, vp, vp]),
        "ap_kv_copy_pages": (ctypes.c_int, [vp, vp, i32, vp, vp, vp]),
        "ap_attention_iteration": (ctypes.c_int, [vp, vp, vp, vp, vp, vp, sz, vp]),
        "ap_serving_iteration_host": (ctypes.c_int, [vp, ctypes.POINTER(BatchDesc), vp, vp, vp, vp, vp, vp]),
        "ap_last_device_status": (ctypes.c_int, [vp, vp]),
        "ap_profile_enable": (ctypes.c_int, [vp, ctypes.c_int]),
        "ap_profile_collect": (ctypes.c_int, [vp, vp, ctypes.POINTER(KernelTimes)]),
        "ap_static_workspace_bytes": (sz, []),
        "ap_attention_iteration_static": (ctypes.c_int, [vp, vp, vp, vp, vp, vp]),
        "ap_kv_pool_set_single_launch": (ctypes.c_int, [vp, i32]),
        "ap_kv_pool_set_wait_limit": (ctypes.c_int, [vp, u64]),
        "ap_selftest_wait_timeout": (ctypes.c_int, [vp, u64, ctypes.c_int, vp]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _lib = lib
    return lib


def _ptr(x) -> Optional[int]:
    """Address of a device tensor / host array / raw integer (None -> NULL)."""
    if x is None:
        return None
    try:
        return x.data_ptr()
    except AttributeError:
        pass
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        return int(x.ctypes.data)
    raise TypeError(f"cannot take the address of {type(x)}")


_bf16 = _fp32 = None      # torch's dtypes, once a tensor has been seen


def _pair(x, y, nbytes: int, device: int) -> Tuple[Optional[int], Optional[int]]:
    """Addresses of two contiguous bf16 tensors on `device` (-1: a host-only pool's, any) that hold at least `nbytes`
    each; the library gets addresses only, so what it would read or write elsewhere is refused here."""
    try:
        if (x.dtype is y.dtype is _bf16 and x.nbytes >= nbytes <= y.nbytes and x.get_device() == device == y.get_device()
                and x.is_contiguous() and y.is_contiguous()):
            return x.data_ptr(), y.data_ptr()
    except AttributeError:                   # None, an address, a host array
        pass
    return _checked(x, nbytes, device, 2), _checked(y, nbytes, device, 2)


def _one(x, nbytes: int, device: int) -> Optional[int]:
    """_pair for one tensor, or None."""
    try:
        if x.dtype is _bf16 and x.nbytes >= nbytes and x.get_device() == device and x.is_contiguous():
            return x.data_ptr()
    except AttributeError:
        pass
    return _checked(x, nbytes, device, 2)


def _checked(x, nbytes: int, device: int, itemsize: Optional[int], dense: bool = True) -> Optional[int]:
    """The same at length.  `itemsize`: 2 for bf16, 4 for fp32 (or integers of that size, or bytes), None for any type."""
    if nbytes <= 0 and dense and itemsize is not None:
        return _ptr(x)                       # a plan without new tokens: nothing is read or written
    if hasattr(x, "data_ptr"):
        global _bf16, _fp32
        import torch
        _bf16, _fp32 = torch.bfloat16, torch.float32
        want = _bf16 if itemsize == 2 else _fp32
        plain = not (x.dtype.is_floating_point or x.dtype.is_complex) and x.element_size() in (1, itemsize)
        if itemsize is not None and x.dtype is not want and not plain:
            raise ValueError(f"expected {want}, not {x.dtype}")
        if device >= 0 and x.get_device() != device and not (x.get_device() < 0 and x.is_pinned()):
            raise ValueError(f"expected a tensor on cuda:{device}, not on {x.device}")
        if dense and not x.is_contiguous():
            raise ValueError("expected a contiguous tensor")
        if dense and x.nbytes < nbytes:
            raise ValueError(f"a tensor of {x.nbytes} bytes where the call takes {nbytes}")
    elif isinstance(x, np.ndarray):
        if device >= 0:
            raise ValueError("expected a device tensor, not a host array")
        if not x.flags.c_contiguous:
            raise ValueError("expected a contiguous array")
        plain = x.dtype.kind in "biu" and x.dtype.itemsize in (1, itemsize)
        like = x.dtype == np.float32 if itemsize == 4 else x.dtype.kind == "V" and x.dtype.itemsize == 2    # (numpy's own has no bf16)
        if itemsize is not None and not plain and not like:
            raise ValueError(f"expected {'bf16 bits' if itemsize == 2 else 'float32'}, not {x.dtype}")
        if x.nbytes < nbytes:
            raise ValueError(f"an array of {x.nbytes} bytes where the call takes {nbytes}")
    return _ptr(x)


def _lse_rows(x, nbytes: int, device: int) -> Optional[int]:
    """_pair for lse: one tensor of fp32, or None."""
    if x is None:
        return None
    try:
        if x.dtype is _fp32 and x.nbytes >= nbytes and x.get_device() == device and x.is_contiguous():
            return x.data_ptr()
    except AttributeError:
        pass
    return _checked(x, nbytes, device, 4)


_raw_stream = None        # torch's accessor of the current stream's handle, once torch has initialised CUDA


def _stream(stream, device: Optional[int] = None) -> Optional[int]:
    """CUDA stream handle: a torch stream, an integer, or None for torch's current stream on ``device`` (a pool's
    device; the current device where it is not given)."""
    global _raw_stream
    if stream is None:
        if _raw_stream is None:
            try:
                import torch
            except ImportError:
                return None
            if not torch.cuda.is_initialized():
                return None                  # nobody can have chosen a stream yet
            # torch.cuda.current_stream(device).cuda_stream takes 3 us, as long as a launch
            _raw_stream = torch._C._cuda_getCurrentRawStream
        if device is None or device < 0:
            import torch
            device = torch.cuda.current_device()
        return _raw_stream(device) or None
    if hasattr(stream, "cuda_stream"):
        return int(stream.cuda_stream) or None
    return int(stream) or None


def _check(status: int, where: str) -> int:
    if status != AP_OK:
        raise ApError(status, where)
    return status


def status_string(status: int) -> str:
    return load().ap_status_string(int(status)).decode()


# ------------------------------------------------------------------- pool --

class KVPool:
    """Handle returned by :func:`kv_pool_create`."""

    def __init__(self, handle: int, desc: PoolDesc, keepalive=()):
        self.handle = handle
        self.desc = desc
        self._keepalive = keepalive
        self.num_pages, self.num_kv_heads = int(desc.num_pages), int(desc.num_kv_heads)
        self.head_dim, self.device = int(desc.head_dim), int(desc.device)


def kv_pool_bytes(num_pages: int, num_kv_heads: int, head_dim: int, page_size: int = 16) -> int:
    d = PoolDesc(num_pages, page_size, num_kv_heads, head_dim, None, None, 0)
    return int(load().ap_kv_pool_bytes(ctypes.byref(d)))


def _plane(x, nbytes: int, device: int) -> Optional[int]:
    """Address of a pool plane: at least `nbytes` on `device` (any view of memory that lies together)."""
    if hasattr(x, "nbytes") and x.nbytes < nbytes:
        raise ValueError(f"a plane of {x.nbytes} bytes where the pool takes {nbytes}")
    return _checked(x, 0, device, None, dense=False)


def kv_pool_create(num_pages: int, num_kv_heads: int, head_dim: int, k_base=None, v_base=None,
                   device: int = 0, page_size: int = 16) -> KVPool:
    k_at, v_at = (_plane(x, kv_pool_bytes(num_pages, num_kv_heads, head_dim, page_size), device) for x in (k_base, v_base))
    d = PoolDesc(num_pages, page_size, num_kv_heads, head_dim, k_at, v_at, device)
    h = ctypes.c_void_p()
    _check(load().ap_kv_pool_create(ctypes.byref(h), ctypes.byref(d)), "ap_kv_pool_create")
    return KVPool(h.value, d, (k_base, v_base))


def kv_pool_bytes_4bit(num_pages: int, num_kv_heads: int, head_dim: int, page_size: int = 16) -> int:
    d = PoolDesc(num_pages, page_size, num_kv_heads, head_dim, None, None, 0)
    return int(load().ap_kv_pool_bytes_4bit(ctypes.byref(d)))


def kv_pool_create_4bit(num_pages: int, num_kv_heads: int, head_dim: int, k_base=None, v_base=None,
                        device: int = 0, page_size: int = 16) -> KVPool:
    """Pool that holds K and V in 4 bits (see ap_kv_pool_create_4bit for the planes' layout)."""
    k_at, v_at = (_plane(x, kv_pool_bytes_4bit(num_pages, num_kv_heads, head_dim, page_size), device) for x in (k_base, v_base))
    d = PoolDesc(num_pages, page_size, num_kv_heads, head_dim, k_at, v_at, device)
    h = ctypes.c_void_p()
    _check(load().ap_kv_pool_create_4bit(ctypes.byref(h), ctypes.byref(d)), "ap_kv_pool_create_4bit")
    return KVPool(h.value, d, (k_base, v_base))


def kv_pool_destroy(pool: KVPool) -> None:
    if pool.handle:
        _check(load().ap_kv_pool_destroy(pool.handle), "ap_kv_pool_destroy")
        pool.handle = None


def kv_pool_k_base(pool: KVPool) -> int:
    return int(load().ap_kv_pool_k_base(pool.handle) or 0)


def kv_pool_v_base(pool: KVPool) -> int:
    return int(load().ap_kv_pool_v_base(pool.handle) or 0)


def kv_pool_alloc_pages(pool: KVPool, n: int) -> np.ndarray:
    ids = np.empty(max(n, 1), dtype=np.int32)
    _check(load().ap_kv_pool_alloc_pages(pool.handle, n, _ptr(ids)), "ap_kv_pool_alloc_pages")
    return ids[:n]


def kv_pool_free_pages(pool: KVPool, ids: Sequence[int]) -> None:
    a = np.ascontiguousarray(ids, dtype=np.int32)
    _check(load().ap_kv_pool_free_pages(pool.handle, len(a), _ptr(a) if len(a) else None),
           "ap_kv_pool_free_pages")


def kv_pool_seed_free_list(pool: KVPool, seed: int) -> None:
    _check(load().ap_kv_pool_seed_free_list(pool.handle, seed), "ap_kv_pool_seed_free_list")


def kv_pool_set_side_by_side(pool: KVPool, mode: int) -> None:
    """0: never run decode and prefill concurrently; 1: per-plan decision (default); k >= 2: always, k decode CTAs."""
    _check(load().ap_kv_pool_set_side_by_side(pool.handle, int(mode)), "ap_kv_pool_set_side_by_side")


def kv_pool_set_single_launch(pool: KVPool, on: bool) -> None:
    """Side-by-side plans: one launch for both parts (default) or the decode and prefill kernels on two streams."""
    _check(load().ap_kv_pool_set_single_launch(pool.handle, int(bool(on))), "ap_kv_pool_set_single_launch")


def kv_pool_num_free(pool: KVPool) -> int:
    return int(load().ap_kv_pool_num_free(pool.handle))


# ------------------------------------------------------------------- plan --

class Plan:
    """Handle returned by :func:`plan_create`.  `q_bytes`, `kv_bytes`, `lse_bytes`: what the new tokens' rows take."""

    def __init__(self, handle: int, pool: KVPool, rows: int, num_q_heads: int):
        self.handle = handle
        self.pool = pool
        self.rows = rows
        self.num_q_heads = num_q_heads
        self.q_bytes = rows * num_q_heads * pool.head_dim * 2
        self.kv_bytes = rows * pool.num_kv_heads * pool.head_dim * 2
        self.lse_bytes = rows * num_q_heads * 4


def _batch_desc(q_lens, ctx_lens, block_tables, num_q_heads: int, softmax_scale: float):
    q_lens = np.ascontiguousarray(q_lens, dtype=np.int32)
    ctx_lens = np.ascontiguousarray(ctx_lens, dtype=np.int32)
    bt = np.ascontiguousarray(block_tables, dtype=np.int32)
    if bt.ndim != 2:
        bt = bt.reshape(len(q_lens), -1) if len(q_lens) else bt.reshape(0, 1)
    desc = BatchDesc(len(q_lens), num_q_heads, _ptr(q_lens), _ptr(ctx_lens), _ptr(bt),
                     bt.shape[1] if bt.ndim == 2 else 0, softmax_scale)
    return desc, (q_lens, ctx_lens, bt)


def plan_create(pool: KVPool, q_lens, ctx_lens, block_tables, num_q_heads: int,
                softmax_scale: float = 0.0, stream=None) -> Plan:
    desc, keep = _batch_desc(q_lens, ctx_lens, block_tables, num_q_heads, softmax_scale)
    h = ctypes.c_void_p()
    _check(load().ap_plan_create(ctypes.byref(h), pool.handle, ctypes.byref(desc), _stream(stream, pool.device)),
           "ap_plan_create")
    return Plan(h.value, pool, int(keep[0].sum(dtype=np.int64)), num_q_heads)


def plan_create_windowed(pool: KVPool, q_lens, ctx_lens, block_tables, num_q_heads: int, window: int, sinks: int = 0,
                         softmax_scale: float = 0.0, stream=None) -> Plan:
    """Plan of a sliding-window layer: a new token sees its last ``window`` keys (itself among them) and the
    first ``sinks`` keys of its context.  Used like a plan of :func:`plan_create`."""
    desc, keep = _batch_desc(q_lens, ctx_lens, block_tables, num_q_heads, softmax_scale)
    # (a number past 32 bits would wrap; so long a window is the whole context, and one below 1 is refused)
    win = WindowDesc(*(max(-1, min(int(x), 2 ** 31 - 1)) for x in (window, sinks)))
    h = ctypes.c_void_p()
    _check(load().ap_plan_create_windowed(ctypes.byref(h), pool.handle, ctypes.byref(desc), ctypes.byref(win),
                                          _stream(stream, pool.device)), "ap_plan_create_windowed")
    return Plan(h.value, pool, int(keep[0].sum(dtype=np.int64)), num_q_heads)


def plan_destroy(plan: Plan) -> None:
    if plan.handle:
        _check(load().ap_plan_destroy(plan.handle), "ap_plan_destroy")
        plan.handle = None


def plan_workspace_bytes(plan: Plan) -> int:
    return int(load().ap_plan_workspace_bytes(plan.handle))


def plan_get_info(plan: Plan) -> dict:
    info = PlanInfo()
    _check(load().ap_plan_get_info(plan.handle, ctypes.byref(info)), "ap_plan_get_info")
    return info.as_dict()


def plan_predict(plan: Plan, hbm_gbs: float = 0.0, tensor_tflops: float = 0.0) -> dict:
    """Algorithmic work and predicted kernel times of a plan (paper's roofline model and the planner's own)."""
    est = PlanPrediction()
    _check(load().ap_plan_predict(plan.handle, float(hbm_gbs), float(tensor_tflops), ctypes.byref(est)),
           "ap_plan_predict")
    return est.as_dict()


def plan_export(plan: Plan) -> dict:
    """Host copy of the plan's work lists as numpy arrays (see ap_plan_export)."""
    lay = PlanLayout()
    _check(load().ap_plan_export(plan.handle, None, 0, ctypes.byref(lay)), "ap_plan_export")
    blob = np.zeros(int(lay.total_ints), dtype=np.int32)
    _check(load().ap_plan_export(plan.handle, _ptr(blob), blob.size, ctypes.byref(lay)), "ap_plan_export")
    info = plan_get_info(plan)

    def sec(off, n, width=None):
        a = blob[int(off):int(off) + int(n) * (width or 1)]
        return a.reshape(-1, width) if width else a
    return {
        "append_dst": sec(lay.append_dst, info["n_new"]),
        "bt_flat": sec(lay.bt_flat, lay.n_bt),
        "decode_items": sec(lay.decode_items, info["decode_items"], 8),
        "cta_begin": sec(lay.cta_begin, lay.n_cta_begin),
        "merge_entries": sec(lay.merge_entries, info["merge_entries"], 4),
        "prefill_tiles": sec(lay.prefill_tiles, info["prefill_tiles"], 8),
        "info": info,
    }


# ---------------------------------------------------------------- kernels --

def kv_append(pool: KVPool, plan: Plan, k_new, v_new, stream=None) -> None:
    dev = pool.device
    k_at, v_at = _pair(k_new, v_new, plan.kv_bytes, dev)
    status = (_lib or load()).ap_kv_append(pool.handle, plan.handle, k_at, v_at, _stream(stream, dev))
    if status:
        _check(status, "ap_kv_append")


def _strided_rows(x, rows: int, heads: int, dim: int, nbytes: int, device: int) -> Tuple[Optional[int], int]:
    """(address, elements from one row to the next or 0 for contiguous) of an input of the rotated append."""
    try:
        if x.is_contiguous():
            return _one(x, nbytes, device), 0
        row, head, one = x.stride()
        n, h, d = x.shape
    except AttributeError:                   # an address, or not given
        return _checked(x, nbytes, device, 2), 0
    except ValueError:
        n = h = d = row = head = one = 0
    if rows <= 0:
        return _ptr(x), 0
    if one != 1 or (head != d and h > 1):
        raise ValueError("expected [rows, heads, head_dim] with a token's heads contiguous")
    if n < rows or h != heads or d != dim:
        raise ValueError(f"expected [{rows}, {heads}, {dim}], not {list(x.shape)}")
    if n < 2:
        row = 0
    elif row < heads * dim:
        raise ValueError("rows overlap (an expanded tensor?)")
    if x.dtype is _bf16 and x.get_device() == device:
        return x.data_ptr(), row
    return _checked(x, 0, device, 2, dense=False), row


def kv_append_rope(pool: KVPool, plan: Plan, k_new, v_new, q=None, q_rot=None, rotary_dim: Optional[int] = None,
                   base: float = 10000.0, interleaved: bool = False, inv_freq=None, amplitude: float = 1.0,
                   stream=None) -> None:
    """Append with the rotary embedding: K rotated by its position, V as it is, ``q`` rotated into ``q_rot``.
    Tensors [rows, heads, head_dim] may be strided by row (slices of one projection)."""
    freq = None if inv_freq is None else np.ascontiguousarray(inv_freq, dtype=np.float64)
    rotary = pool.head_dim if rotary_dim is None else max(-1, min(int(rotary_dim), 2 ** 31 - 1))
    if freq is not None and freq.shape != (rotary // 2,):
        raise ValueError("inv_freq must have rotary_dim / 2 entries")
    dev = pool.device
    n, hkv, d, kv_bytes = plan.rows, pool.num_kv_heads, pool.head_dim, plan.kv_bytes
    q_at, q_stride = (None, 0) if q is None else _strided_rows(q, n, plan.num_q_heads, d, plan.q_bytes, dev)
    k_at, k_stride = _strided_rows(k_new, n, hkv, d, kv_bytes, dev)
    v_at, v_stride = _strided_rows(v_new, n, hkv, d, kv_bytes, dev)
    if not abs(amplitude) <= _FP32_MAX:      # (NaN and what fp32 does not hold: refused by the library)
        amplitude = math.nan
    desc = _ROPE_DESC.pack(rotary, 1 if interleaved else 0, base, 0 if freq is None else freq.ctypes.data, amplitude, q_stride,
                           k_stride, v_stride)
    status = (_lib or load()).ap_kv_append_rope(pool.handle, plan.handle, desc, q_at, k_at, v_at,
                                                _one(q_rot, plan.q_bytes, dev), _stream(stream, dev))
    if status:
        _check(status, "ap_kv_append_rope")


def kv_read_new(pool: KVPool, plan: Plan, k, v, stream=None) -> None:
    """The rows of the plan's new tokens, read back as the bf16 numbers the pool holds (or, in 4 bits, stands for)."""
    dev = pool.device
    k_at, v_at = _pair(k, v, plan.kv_bytes, dev)
    status = (_lib or load()).ap_kv_read_new(pool.handle, plan.handle, k_at, v_at, _stream(stream, dev))
    if status:
        _check(status, "ap_kv_read_new")


def kv_copy_pages(dst_pool: KVPool, src_pool: KVPool, dst_ids: Sequence[int], src_ids: Sequence[int], stream=None) -> None:
    """Page ``src_ids[i]`` of ``src_pool`` -> page ``dst_ids[i]`` of ``dst_pool`` (all kv heads, K and V)."""
    dst = np.ascontiguousarray(dst_ids, dtype=np.int32)
    src = np.ascontiguousarray(src_ids, dtype=np.int32)
    if dst.shape != src.shape or dst.ndim != 1:
        raise ValueError("dst_ids and src_ids must be 1-D and of the same length")
    _check(load().ap_kv_copy_pages(dst_pool.handle, src_pool.handle, int(dst.size), dst.ctypes.data, src.ctypes.data,
                                   _stream(stream, dst_pool.device) if dst_pool.desc.device >= 0 else None), "ap_kv_copy_pages")


def attention_iteration(pool: KVPool, plan: Plan, q, out, lse=None, workspace=None,
                        workspace_bytes: Optional[int] = None, stream=None) -> None:
    dev = pool.device
    try:
        room = workspace.nbytes
        if workspace_bytes is None:
            workspace_bytes = room
        elif workspace_bytes > room:
            raise ValueError(f"a workspace of {room} bytes where the call is told {workspace_bytes}")
        workspace = workspace.data_ptr() if workspace.get_device() == dev and workspace.is_contiguous() else (
            _checked(workspace, 0, dev, None))
    except AttributeError:                   # none, or an address
        workspace, workspace_bytes = _checked(workspace, 0, dev, None), workspace_bytes or 0
    q_at, out_at = _pair(q, out, plan.q_bytes, dev)
    lse_at = None if lse is None else _lse_rows(lse, plan.lse_bytes, dev)
    status = (_lib or load()).ap_attention_iteration(pool.handle, plan.handle, q_at, out_at, lse_at, workspace, workspace_bytes,
                                                     _stream(stream, dev))
    if status:
        _check(status, "ap_attention_iteration")


def static_workspace_bytes() -> int:
    """Size of the library's built-in split-K scratch array (the largest plan
    workspace :func:`attention_iteration_static` accepts)."""
    return int(load().ap_static_workspace_bytes())


def attention_iteration_static(pool: KVPool, plan: Plan, q, out, lse=None, stream=None) -> None:
    """Same result as :func:`attention_iteration`, for callers that cannot
    allocate device memory and therefore have no workspace to pass: the split-K
    partials go to a fixed 8 MiB array inside the library.  Plans that need
    more raise ``ApError`` (``AP_ERR_WORKSPACE_TOO_SMALL``).  Calls share that
    array, so two of them must not overlap on the GPU."""
    dev = pool.device
    _check(load().ap_attention_iteration_static(pool.handle, plan.handle, *_pair(q, out, plan.q_bytes, dev),
                                                _lse_rows(lse, plan.lse_bytes, dev), _stream(stream, dev)),
           "ap_attention_iteration_static")


def serving_iteration_host(pool: KVPool, q_lens, ctx_lens, block_tables, num_q_heads: int, q_host,
                           k_new_host, v_new_host, out_host, lse_host=None, softmax_scale: float = 0.0,
                           stream=None) -> None:
    desc, keep = _batch_desc(q_lens, ctx_lens, block_tables, num_q_heads, softmax_scale)
    rows = int(keep[0].sum(dtype=np.int64))
    sizes = [rows * h * pool.head_dim * 2 for h in (num_q_heads, pool.num_kv_heads, pool.num_kv_heads, num_q_heads)]
    at = [_checked(x, size, -1, 2) for x, size in zip((q_host, k_new_host, v_new_host, out_host), sizes)]
    _check(load().ap_serving_iteration_host(pool.handle, ctypes.byref(desc), *at, _checked(lse_host, rows * num_q_heads * 4, -1, 4),
                                            _stream(stream, pool.device)), "ap_serving_iteration_host")
    del keep


def last_device_status(pool: KVPool, stream=None) -> int:
    return int(load().ap_last_device_status(pool.handle, _stream(stream, pool.device)))


def kv_pool_set_wait_limit(pool: KVPool, limit_ns: int) -> None:
    """Bound (ns) of every wait inside the kernels launched for this pool from now on; 0 = default (2 s)."""
    _check(load().ap_kv_pool_set_wait_limit(pool.handle, int(limit_ns)), "ap_kv_pool_set_wait_limit")


def selftest_wait_timeout(pool: KVPool, limit_ns: int, leave_counter: bool = False, stream=None) -> None:
    """Queues the one-warp kernel whose bounded wait always runs out (see ap_selftest_wait_timeout)."""
    _check(load().ap_selftest_wait_timeout(pool.handle, int(limit_ns), int(bool(leave_counter)), _stream(stream, pool.device)),
           "ap_selftest_wait_timeout")


# ------------------------------------------------------------ diagnostics --

def profile_enable(pool: KVPool, on: bool = True) -> None:
    _check(load().ap_profile_enable(pool.handle, int(bool(on))), "ap_profile_enable")


def profile_collect(pool: KVPool, stream=None) -> dict:
    """{kernel name: (total ms, launches)} since the last enable/collect."""
    kt = KernelTimes()
    _check(load().ap_profile_collect(pool.handle, _stream(stream, pool.device), ctypes.byref(kt)), "ap_profile_collect")
    return {name: (float(kt.ms[i]), int(kt.launches[i])) for i, name in enumerate(KERNEL_NAMES)}
