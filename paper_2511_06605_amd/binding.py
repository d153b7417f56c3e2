"""ctypes binding of the C boundary in ``include/dmalatte.h``.

Argument marshalling only: every byte is moved by the HIP kernels behind the
``dl_*`` entry points.  There is no CPU fallback: if the built library is
missing, loading fails with an error.

Device buffers may be given as integer addresses or as objects with a
``data_ptr()`` method (torch tensors); streams as ``None`` (default stream),
integer handles, or objects with a ``cuda_stream`` attribute.
"""

from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
# DL_LIBRARY names another build of the same library (the host-sanitizer build of the tests); there is still no
# fallback: whatever it names must exist.
LIB_PATH = os.environ.get("DL_LIBRARY") or os.path.join(_HERE, "libdmalatte.so")

DL_OK = 0
DL_ERR_INVALID = -1
DL_ERR_OVERLAP = -2
DL_ERR_HIP = -3
DL_ERR_TIMEOUT = -4
DL_ERR_STATE = -5
DL_ERR_EXPIRED = -6
DL_ERR_LOST = -7
DL_ERR_CAPACITY = -8
DL_STATIC_MAX_COPIES = 16384
DL_DISPATCH_DEVICE_MAX_TOKENS = 10240
DL_MAX_FANOUT = 64
DL_PLAN_FANOUT = 8
DL_MODE_ONESHOT = 0
DL_MODE_PRELAUNCH = 1
DL_MODE_SIGNAL = 2
DL_MODE_STANDBY = 3
DL_MODE_AUTO = 4
DL_OP_BATCH, DL_OP_BROADCAST, DL_OP_ALLGATHER, DL_OP_ALLTOALL, DL_OP_SWAP, DL_OP_TOKEN_DISPATCH = range(6)
DL_TYPE_F32, DL_TYPE_BF16, DL_TYPE_F16 = range(3)
DL_KV_FP8, DL_KV_INT8 = range(2)
DL_MAX_DRAFTS = 63
DL_MAX_ROWS = 1 << 27
DL_AUTO_STANDBY_TILES = 64
DL_AUTO_SIGNAL_MAX_BYTES = 288 << 20
DL_AUTO_PRELAUNCH_MAX_BYTES = 288 << 20

# every symbol include/dmalatte.h declares
EXPORTS = [
    "dl_init", "dl_shutdown", "dl_set_mode", "dl_get_mode", "dl_set_validate", "dl_strerror",
    "dl_last_hip_error", "dl_batch_copy", "dl_broadcast", "dl_allgather", "dl_alltoall",
    "dl_prelaunch_start", "dl_prelaunch_stop", "dl_last_ticket", "dl_trigger", "dl_wait", "dl_wait_armed",
    "dl_get_config",
    "dl_set_config", "dl_plan_allgather", "dl_plan_alltoall", "dl_plan_broadcast", "dl_plan_batch",
    "dl_plan_first_hazard", "dl_plan_tiles", "dl_batch_swap", "dl_alltoall_inplace", "dl_plan_alltoall_inplace",
    "dl_plan_swap_first_hazard", "dl_batch_fanout", "dl_token_dispatch", "dl_plan_token_dispatch",
    "dl_plan_batch_inferred", "dl_set_trace", "dl_get_trace", "dl_trace_clock",
    "dl_last_device_error", "dl_debug_lose_next_table", "dl_batch_copy_static",
    "dl_plan_mode", "dl_last_mode", "dl_complete", "dl_parse_config", "dl_token_dispatch_device",
    "dl_kv_write", "dl_kv_read", "dl_prefix_attention", "dl_prefix_attention_workspace", "dl_verify_draft",
    "dl_verify_draft_workspace",
]


class DlError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {strerror(status)} (status {status}, hip error {last_hip_error()})")


class CopyDesc(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("bytes", ctypes.c_size_t)]


class SwapDesc(ctypes.Structure):
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("bytes", ctypes.c_size_t)]


class Trace(ctypes.Structure):
    _fields_ = [("doorbell_seen", ctypes.c_uint64), ("copy_begin", ctypes.c_uint64), ("copy_end", ctypes.c_uint64),
                ("completion_issued", ctypes.c_uint64)]


class Config(ctypes.Structure):
    _fields_ = [
        ("tile_bytes", ctypes.c_uint32),
        ("block_threads", ctypes.c_uint32),
        ("nontemporal_min_bytes", ctypes.c_uint64),
        ("armed_blocks", ctypes.c_uint32),
        ("arm_timeout_us", ctypes.c_uint32),
        ("fuse_broadcast", ctypes.c_uint32),
        ("max_blocks", ctypes.c_uint32),
        ("fan_split", ctypes.c_uint32),
        ("infer_broadcast", ctypes.c_uint32),
        ("device_lowering", ctypes.c_uint32),
        ("table_push", ctypes.c_uint32),
        ("write_through_max_bytes", ctypes.c_uint64),
        ("stream_plain_min_bytes", ctypes.c_uint64),
        ("armed_chain_min_bytes", ctypes.c_uint64),
    ]


class PlanItem(ctypes.Structure):
    _fields_ = [
        ("src", ctypes.c_void_p),
        ("bytes", ctypes.c_size_t),
        ("k", ctypes.c_uint32),
        ("reserved", ctypes.c_uint32),
        ("dst", ctypes.c_void_p * DL_PLAN_FANOUT),
    ]


class KvCacheDesc(ctypes.Structure):
    """dl_kv_cache"""
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
        ("format", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
        ("pages", ctypes.c_int64),
        ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
        ("scale_page_stride", ctypes.c_int64), ("scale_token_stride", ctypes.c_int64), ("scale_head_stride", ctypes.c_int64),
    ]


class KvRowsDesc(ctypes.Structure):
    """dl_kv_rows"""
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("tokens", ctypes.c_int64),
        ("type", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("k_token_stride", ctypes.c_int64), ("k_head_stride", ctypes.c_int64),
        ("v_token_stride", ctypes.c_int64), ("v_head_stride", ctypes.c_int64),
    ]


class PrefixAttentionDesc(ctypes.Structure):
    """dl_prefix_attention_args"""
    _fields_ = [
        ("q", ctypes.c_void_p), ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("prefix_pages", ctypes.c_void_p),
        ("pages", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("q_lens", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("prefix_tokens", ctypes.c_int64), ("max_pages", ctypes.c_int64), ("pages_stride", ctypes.c_int64),
        ("q_seq_stride", ctypes.c_int64), ("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
        ("out_seq_stride", ctypes.c_int64), ("out_token_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64),
        ("type", ctypes.c_int32), ("batch", ctypes.c_int32), ("q_tokens", ctypes.c_int32), ("q_heads", ctypes.c_int32),
        ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
    ]


class VerifyDraftDesc(ctypes.Structure):
    """dl_verify_draft_args"""
    _fields_ = [
        ("target", ctypes.c_void_p), ("draft", ctypes.c_void_p), ("draft_tokens", ctypes.c_void_p), ("uniform", ctypes.c_void_p),
        ("race", ctypes.c_void_p), ("draft_lens", ctypes.c_void_p), ("tokens", ctypes.c_void_p), ("accepted", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("target_seq_stride", ctypes.c_int64), ("target_row_stride", ctypes.c_int64),
        ("draft_seq_stride", ctypes.c_int64), ("draft_row_stride", ctypes.c_int64), ("race_stride", ctypes.c_int64),
        ("type", ctypes.c_int32), ("batch", ctypes.c_int32), ("drafts", ctypes.c_int32), ("vocab", ctypes.c_int32),
    ]


_lib = None
_marshal = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib, _marshal
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2511_06605_amd.build` "
            "(there is no fallback path)")
    try:
        # One HIP runtime per process: PyTorch ships its own, and device memory and streams come
        # from it, so it has to be loaded first for the library to bind to that same runtime.
        import torch  # noqa: F401
    except ImportError:
        pass
    L = ctypes.CDLL(LIB_PATH)
    vp, vpp = ctypes.c_void_p, ctypes.POINTER(ctypes.c_void_p)
    szp = ctypes.POINTER(ctypes.c_size_t)
    sig = {
        "dl_init": (ctypes.c_int, [ctypes.c_int]),
        "dl_shutdown": (ctypes.c_int, []),
        "dl_set_mode": (ctypes.c_int, [ctypes.c_int]),
        "dl_get_mode": (ctypes.c_int, []),
        "dl_last_mode": (ctypes.c_int, []),
        "dl_complete": (ctypes.c_int, [vp, ctypes.c_uint64]),
        "dl_plan_mode": (ctypes.c_int, [ctypes.c_int, ctypes.c_size_t, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_uint64,
                                        ctypes.c_int]),
        "dl_set_validate": (ctypes.c_int, [ctypes.c_int]),
        "dl_strerror": (ctypes.c_char_p, [ctypes.c_int]),
        "dl_last_hip_error": (ctypes.c_int, []),
        "dl_last_device_error": (ctypes.c_int, []),
        "dl_debug_lose_next_table": (ctypes.c_int, [ctypes.c_uint32]),
        "dl_batch_copy": (ctypes.c_int, [ctypes.POINTER(CopyDesc), ctypes.c_size_t, vp]),
        "dl_batch_copy_static": (ctypes.c_int, [ctypes.POINTER(CopyDesc), ctypes.c_size_t, vp]),
        "dl_broadcast": (ctypes.c_int, [vp, vpp, ctypes.c_int, ctypes.c_size_t, vp]),
        "dl_allgather": (ctypes.c_int, [vpp, vpp, ctypes.c_int, ctypes.c_size_t, vp]),
        "dl_alltoall": (ctypes.c_int, [vpp, vpp, ctypes.c_int, szp, vp]),
        "dl_prelaunch_start": (ctypes.c_int, []),
        "dl_prelaunch_stop": (ctypes.c_int, []),
        "dl_last_ticket": (ctypes.c_uint64, []),
        "dl_trigger": (ctypes.c_int, [ctypes.c_uint64]),
        "dl_wait": (ctypes.c_int, [ctypes.c_uint64, ctypes.c_uint64]),
        "dl_wait_armed": (ctypes.c_int, [ctypes.c_uint64, ctypes.c_uint64]),
        "dl_get_config": (ctypes.c_int, [ctypes.POINTER(Config)]),
        "dl_set_config": (ctypes.c_int, [ctypes.POINTER(Config)]),
        "dl_parse_config": (ctypes.c_int, [ctypes.c_char_p, ctypes.POINTER(Config)]),
        "dl_plan_allgather": (ctypes.c_long, [vpp, vpp, ctypes.c_int, ctypes.c_size_t, ctypes.c_int,
                                              ctypes.POINTER(PlanItem), ctypes.c_size_t]),
        "dl_plan_alltoall": (ctypes.c_long, [vpp, vpp, ctypes.c_int, szp, ctypes.POINTER(PlanItem), ctypes.c_size_t]),
        "dl_plan_broadcast": (ctypes.c_long, [vp, vpp, ctypes.c_int, ctypes.c_size_t, ctypes.POINTER(PlanItem),
                                              ctypes.c_size_t]),
        "dl_plan_batch": (ctypes.c_long, [ctypes.POINTER(CopyDesc), ctypes.c_size_t, ctypes.POINTER(PlanItem),
                                          ctypes.c_size_t]),
        "dl_plan_first_hazard": (ctypes.c_long, [ctypes.POINTER(PlanItem), ctypes.c_size_t]),
        "dl_plan_tiles": (ctypes.c_uint64, [ctypes.POINTER(PlanItem), ctypes.c_size_t, ctypes.c_uint32]),
        "dl_batch_swap": (ctypes.c_int, [ctypes.POINTER(SwapDesc), ctypes.c_size_t, vp]),
        "dl_alltoall_inplace": (ctypes.c_int, [vpp, ctypes.c_int, ctypes.c_size_t, vp]),
        "dl_plan_alltoall_inplace": (ctypes.c_long, [vpp, ctypes.c_int, ctypes.c_size_t, ctypes.POINTER(SwapDesc),
                                                     ctypes.c_size_t]),
        "dl_plan_swap_first_hazard": (ctypes.c_long, [ctypes.POINTER(SwapDesc), ctypes.c_size_t]),
        "dl_set_trace": (ctypes.c_int, [ctypes.c_int]),
        "dl_get_trace": (ctypes.c_int, [ctypes.c_uint64, ctypes.POINTER(Trace)]),
        "dl_trace_clock": (ctypes.c_int, [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]),
        "dl_batch_fanout": (ctypes.c_int, [ctypes.POINTER(PlanItem), ctypes.c_size_t, vp]),
        "dl_token_dispatch": (ctypes.c_int, [vpp, vpp, ctypes.c_int, ctypes.POINTER(ctypes.c_uint32), ctypes.c_size_t,
                                             ctypes.POINTER(ctypes.c_uint8), vp]),
        "dl_token_dispatch_device": (ctypes.c_int, [vpp, vpp, ctypes.c_int, ctypes.POINTER(ctypes.c_uint32), ctypes.c_size_t,
                                                    vp, vp]),
        "dl_plan_token_dispatch": (ctypes.c_long, [vpp, vpp, ctypes.c_int, ctypes.POINTER(ctypes.c_uint32),
                                                   ctypes.c_size_t, ctypes.POINTER(ctypes.c_uint8),
                                                   ctypes.POINTER(PlanItem), ctypes.c_size_t]),
        "dl_plan_batch_inferred": (ctypes.c_long, [ctypes.POINTER(CopyDesc), ctypes.c_size_t, ctypes.POINTER(PlanItem),
                                                   ctypes.c_size_t]),
        "dl_kv_write": (ctypes.c_int, [vp, vp, vp]),
        "dl_kv_read": (ctypes.c_int, [vp, vp, vp]),
        "dl_prefix_attention": (ctypes.c_int, [vp, vp, vp]),
        "dl_prefix_attention_workspace": (ctypes.c_int64, [vp, vp]),
        "dl_verify_draft": (ctypes.c_int, [vp, vp]),
        "dl_verify_draft_workspace": (ctypes.c_int64, [vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    try:
        from . import _marshal as m  # built next to the library (build.py)
    except ImportError:
        from . import marshal_ctypes as m  # not for this Python: the same calls with ctypes objects
    m.bind(ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in m.NAMES)
    _marshal = m  # first: another thread that finds _lib set goes on to use it
    _lib = L
    return L


def _native():
    """The marshalling module, bound to the loaded library."""
    if _marshal is None:
        lib()
    return _marshal


# ------------------------------------------------------------------ marshalling

def _addr(x) -> int | None:
    if x is None:
        return None
    if hasattr(x, "data_ptr"):
        return int(x.data_ptr()) or None
    return int(x) or None


def _stream(s) -> int | None:
    if s is None:
        return None
    if hasattr(s, "cuda_stream"):
        return int(s.cuda_stream) or None
    return int(s) or None


def _ptr_array(xs):
    return (ctypes.c_void_p * max(len(xs), 1))(*[_addr(x) for x in xs])


def _chunk_array(chunk_bytes, W):
    flat = [int(v) for row in chunk_bytes for v in (row if hasattr(row, "__len__") else [row])]
    if len(flat) != W * W:
        raise ValueError("chunk_bytes must have W*W entries")
    return (ctypes.c_size_t * (W * W))(*flat)


def _desc_array(descs):
    arr = (CopyDesc * max(len(descs), 1))()
    for i, (s, d, n) in enumerate(descs):
        arr[i].src, arr[i].dst, arr[i].bytes = _addr(s), _addr(d), int(n)
    return arr


def _swap_array(descs):
    arr = (SwapDesc * max(len(descs), 1))()
    for i, (a, b, n) in enumerate(descs):
        arr[i].a, arr[i].b, arr[i].bytes = _addr(a), _addr(b), int(n)
    return arr


def _check(status: int, what: str) -> None:
    if status != DL_OK:
        raise DlError(status, what)


# ------------------------------------------------------------------- lifecycle

def strerror(status: int) -> str:
    return lib().dl_strerror(status).decode()


def last_hip_error() -> int:
    return lib().dl_last_hip_error()


def dl_last_device_error() -> int:
    """DL_ERR_LOST if a kernel has given up on its copy table since the last call (clears the report), else DL_OK."""
    return int(lib().dl_last_device_error())


def dl_debug_lose_next_table(tries: int = 4) -> None:
    _check(lib().dl_debug_lose_next_table(int(tries)), "dl_debug_lose_next_table")


def dl_init(device: int = 0) -> None:
    _check(lib().dl_init(device), "dl_init")


def dl_shutdown() -> None:
    _check(lib().dl_shutdown(), "dl_shutdown")


def dl_set_mode(mode: int) -> None:
    status = _native().set_mode(mode)
    _check(lib().dl_set_mode(mode) if status is NotImplemented else status, "dl_set_mode")


def dl_get_mode() -> int:
    return lib().dl_get_mode()


def dl_last_mode() -> int:
    return lib().dl_last_mode()


def dl_complete(stream=None, timeout_ns: int = 5_000_000_000) -> None:
    _check(lib().dl_complete(_stream(stream), timeout_ns), "dl_complete")


def dl_plan_mode(op: int, items: int, max_fanout: int, moved_bytes: int, tiles: int, known_ahead: bool) -> int:
    """The size -> mode table: the dl_mode that suits a lowered list of these dimensions."""
    m = lib().dl_plan_mode(int(op), int(items), int(max_fanout), int(moved_bytes), int(tiles), 1 if known_ahead else 0)
    if m < 0:
        raise DlError(int(m), "dl_plan_mode")
    return int(m)


def dl_set_validate(on: bool) -> None:
    _check(lib().dl_set_validate(1 if on else 0), "dl_set_validate")


def dl_get_config() -> Config:
    c = Config()
    _check(lib().dl_get_config(ctypes.byref(c)), "dl_get_config")
    return c


def dl_parse_config(text: str, cfg: Config | None = None) -> Config:
    """``text`` ("name=value,...") applied to ``cfg`` (or to an all-zero one with arm_timeout_us = 1); host-only."""
    c = cfg or Config(arm_timeout_us=1)
    _check(lib().dl_parse_config(text.encode(), ctypes.byref(c)), "dl_parse_config")
    return c


def dl_set_config(cfg: Config | None = None, **fields) -> None:
    c = cfg or dl_get_config()
    for k, v in fields.items():
        if not hasattr(c, k):
            raise AttributeError(k)
        setattr(c, k, v)
    _check(lib().dl_set_config(ctypes.byref(c)), "dl_set_config")


# ------------------------------------------------------------------ operations

def dl_batch_copy(descs, stream=None) -> None:
    """descs: sequence of (src, dst, bytes)."""
    _check(_native().batch_copy(descs, stream), "dl_batch_copy")


def dl_batch_copy_static(descs, stream=None) -> None:
    """descs: sequence of (src, dst, bytes); the variant that allocates nothing."""
    _check(_native().batch_copy_static(descs, stream), "dl_batch_copy_static")


def dl_broadcast(src, dsts, nbytes: int, stream=None) -> None:
    _check(_native().broadcast(src, dsts, nbytes, stream), "dl_broadcast")


def dl_allgather(ins, outs, bytes_per_rank: int, stream=None) -> None:
    _check(_native().allgather(ins, outs, bytes_per_rank, stream), "dl_allgather")


def dl_alltoall(ins, outs, chunk_bytes, stream=None) -> None:
    _check(_native().alltoall(ins, outs, chunk_bytes, stream), "dl_alltoall")


def dl_batch_swap(descs, stream=None) -> None:
    """descs: sequence of (a, b, bytes)."""
    _check(_native().batch_swap(descs, stream), "dl_batch_swap")


def dl_alltoall_inplace(bufs, chunk_bytes: int, stream=None) -> None:
    _check(_native().alltoall_inplace(bufs, chunk_bytes, stream), "dl_alltoall_inplace")


def _mask_bytes(dest) -> bytes:
    """A routing mask of any form, one byte per (token, rank)."""
    if hasattr(dest, "tobytes"):
        return (dest != 0).astype("uint8").tobytes()
    return bytes(bytearray(int(v) != 0 for row in dest for v in row))


def _dispatch_args(ins, outs, tokens, dest):
    ins, outs = list(ins), list(outs)
    W = len(ins)
    if len(outs) != W or len(tokens) != W:
        raise ValueError("need W send buffers, W receive buffers and W token counts")
    tok = (ctypes.c_uint32 * W)(*[int(t) for t in tokens])
    total = sum(int(t) for t in tokens)
    flat = _mask_bytes(dest)
    if len(flat) != total * W:
        raise ValueError("dest must have one entry per (token, rank)")
    d = (ctypes.c_uint8 * max(len(flat), 1)).from_buffer_copy(flat or b"\0")
    return _ptr_array(ins), _ptr_array(outs), W, tok, d


def dl_batch_fanout(items, stream=None) -> None:
    """items: sequence of dicts {src, bytes, dst: [..]} (as the dl_plan_* functions return)."""
    items = list(items)
    _check(lib().dl_batch_fanout(_items_in(items), len(items), _stream(stream)), "dl_batch_fanout")


def dl_token_dispatch(ins, outs, tokens, row_bytes: int, dest, stream=None) -> None:
    status = _native().token_dispatch(ins, outs, tokens, row_bytes, dest, stream)
    if status is NotImplemented:  # dest is no contiguous buffer of bytes (and nothing else has been looked at): make one
        status = _native().token_dispatch(ins, outs, tokens, row_bytes, _mask_bytes(dest), stream)
    _check(status, "dl_token_dispatch")


def dl_token_dispatch_device(ins, outs, tokens, row_bytes: int, dest_device, stream=None) -> None:
    """dest_device: device buffer of (total tokens) x W bytes, non-zero where a token goes to a rank."""
    _check(_native().token_dispatch_device(ins, outs, tokens, row_bytes, dest_device, stream), "dl_token_dispatch_device")


# ------------------------------------------- a paged cache in 8 bits, and decoding with drafts
#
# The descriptors below take tensors (anything with data_ptr(), shape, stride() and dtype, as torch's) and hold on to them.
# They name buffers, not contents: a program makes them once for the buffers it keeps and calls with them step after step.

_TYPES = {"float32": DL_TYPE_F32, "bfloat16": DL_TYPE_BF16, "float16": DL_TYPE_F16}
_FORMATS = {"float8_e4m3fn": DL_KV_FP8, "int8": DL_KV_INT8}


def _dtype(t) -> str:
    return str(t.dtype).rpartition(".")[2]


def _expect(t, what, dtype, shape, packed=False):
    """A tensor's address, once it is what it has to be; None in the shape: any size."""
    if _dtype(t) not in (dtype if isinstance(dtype, (tuple, list, dict)) else (dtype,)):
        raise ValueError(f"{what}: type {t.dtype}, expected {dtype if isinstance(dtype, str) else ' or '.join(dtype)}")
    if len(t.shape) != len(shape) or any(w is not None and int(w) != int(n) for n, w in zip(t.shape, shape)):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {tuple('any' if w is None else int(w) for w in shape)}")
    if t.numel() and (getattr(t, "is_cuda", True) is False):
        raise ValueError(f"{what}: not in device memory")
    if packed and not t.is_contiguous():
        raise ValueError(f"{what}: must be contiguous")
    if not packed and t.shape[-1] > 1 and t.stride()[-1] != 1:
        raise ValueError(f"{what}: its last dimension must be contiguous")
    return _addr(t)


def _strides(t):
    """Strides of a tensor, 0 where a dimension has nothing to step to (torch puts anything there)."""
    return tuple(s if n > 1 else 0 for n, s in zip(t.shape, t.stride()))


class _Request:
    """A descriptor of the C boundary, the tensors it names, and its address for the calls."""

    def _hold(self, desc, *tensors):
        self.desc = desc
        self._tensors = tensors
        self.at = ctypes.addressof(desc)

    def use_workspace(self, workspace) -> None:
        """Device memory of at least the size the *_workspace function gives, filled with zeros before its first use."""
        if getattr(workspace, "is_cuda", True) is False or not workspace.is_contiguous():
            raise ValueError("workspace: contiguous device memory")
        self._workspace = workspace
        self.desc.workspace = _addr(workspace)
        self.desc.workspace_bytes = workspace.numel() * workspace.element_size()


class KvCache(_Request):
    """A paged cache (dl_kv_cache): codes of keys and values as [pages, page_tokens, heads, head_dim] tensors of float8_e4m3fn or
    int8, scales as [pages, page_tokens, heads] tensors of float32; any strides, the same for keys and values."""

    def __init__(self, k, v, k_scale, v_scale):
        shape = tuple(int(n) for n in k.shape)
        if len(shape) != 4:
            raise ValueError("codes have four dimensions: pages, page_tokens, heads, head_dim")
        d = KvCacheDesc(k=_expect(k, "k", _FORMATS, shape), v=_expect(v, "v", _dtype(k), shape), format=_FORMATS[_dtype(k)], heads=shape[2],
                        head_dim=shape[3], page_tokens=shape[1], pages=shape[0])
        for name, s in (("k_scale", k_scale), ("v_scale", v_scale)):
            if _dtype(s) != "float32" or tuple(s.shape) != shape[:3] or getattr(s, "is_cuda", True) is False:
                raise ValueError(f"{name}: float32 of shape {shape[:3]} in device memory")
            setattr(d, name, _addr(s))
        if _strides(k) != _strides(v) or _strides(k_scale) != _strides(v_scale):
            raise ValueError("keys and values have different strides")
        d.page_stride, d.token_stride, d.head_stride = _strides(k)[:3]
        d.scale_page_stride, d.scale_token_stride, d.scale_head_stride = _strides(k_scale)
        self._hold(d, k, v, k_scale, v_scale)


class KvRows(_Request):
    """Rows outside a cache and the slots they belong to (dl_kv_rows): k and v [tokens, heads, head_dim] of float32, bfloat16 or
    float16, either may be None; slots [tokens] of int64."""

    def __init__(self, k, v, slots):
        some = k if k is not None else v
        if some is None:
            raise ValueError("neither keys nor values")
        shape = tuple(int(n) for n in some.shape)
        if len(shape) != 3:
            raise ValueError("rows have three dimensions: tokens, heads, head_dim")
        d = KvRowsDesc(slots=_expect(slots, "slots", "int64", shape[:1], packed=True), tokens=shape[0], type=_TYPES.get(_dtype(some), -1))
        for name, t in (("k", k), ("v", v)):
            if t is not None:
                setattr(d, name, _expect(t, name, _TYPES if t is some else _dtype(some), shape))
                setattr(d, name + "_token_stride", t.stride()[0])
                setattr(d, name + "_head_stride", t.stride()[1])
        self.shape = shape
        self._hold(d, k, v, slots)


class PrefixAttention(_Request):
    """A call of dl_prefix_attention: q and out [batch, q_tokens, q_heads, head_dim] of bfloat16 or float16, pages [batch, max_pages], lens and
    q_lens [batch] and prefix_pages [n] of int32, lse [batch, q_tokens, q_heads] of float32.  scale: 1 / sqrt(head_dim) if None."""

    def __init__(self, cache, q, out, pages, lens, prefix_pages=None, prefix_tokens=0, q_lens=None, lse=None, scale=None):
        shape = tuple(int(n) for n in q.shape)
        if len(shape) != 4:
            raise ValueError("q has four dimensions: batch, q_tokens, q_heads, head_dim")
        B, M, H, D = shape
        if D != cache.desc.head_dim:
            raise ValueError(f"q: head_dim {D}, the cache has {cache.desc.head_dim}")
        prefix_tokens = int(prefix_tokens)
        have = 0 if prefix_pages is None else int(prefix_pages.shape[0]) * cache.desc.page_tokens
        if prefix_tokens > have:
            raise ValueError(f"prefix_tokens {prefix_tokens}, but prefix_pages hold {have}")
        d = PrefixAttentionDesc(
            q=_expect(q, "q", ("bfloat16", "float16"), shape), out=_expect(out, "out", _dtype(q), shape), type=_TYPES[_dtype(q)],
            pages=_expect(pages, "pages", "int32", (B, None)), lens=_expect(lens, "lens", "int32", (B,), packed=True),
            prefix_tokens=prefix_tokens, max_pages=int(pages.shape[1]), pages_stride=pages.stride()[0], batch=B, q_tokens=M, q_heads=H,
            scale=D ** -0.5 if scale is None else float(scale))
        if prefix_pages is not None:
            d.prefix_pages = _expect(prefix_pages, "prefix_pages", "int32", (None,), packed=True)
        if q_lens is not None:
            d.q_lens = _expect(q_lens, "q_lens", "int32", (B,), packed=True)
        if lse is not None:
            d.lse = _expect(lse, "lse", "float32", (B, M, H), packed=True)
        d.q_seq_stride, d.q_token_stride, d.q_head_stride = q.stride()[:3]
        d.out_seq_stride, d.out_token_stride, d.out_head_stride = out.stride()[:3]
        self.cache = cache
        self._hold(d, q, out, pages, lens, prefix_pages, q_lens, lse)


class DraftVerify(_Request):
    """A call of dl_verify_draft: target [batch, drafts + 1, vocab] and draft_probs [batch, drafts, vocab] of float32, bfloat16 or float16,
    draft_tokens [batch, drafts], draft_lens [batch], tokens [batch, drafts + 1] and accepted [batch] of int32, uniform [batch, drafts] and
    race [batch, vocab] of float32."""

    def __init__(self, target, draft_tokens, uniform, race, tokens, accepted, draft_probs=None, draft_lens=None):
        shape = tuple(int(n) for n in target.shape)
        if len(shape) != 3 or shape[1] < 1:
            raise ValueError("target has three dimensions: batch, drafts + 1, vocab")
        B, n, V = shape[0], shape[1] - 1, shape[2]
        d = VerifyDraftDesc(
            target=_expect(target, "target", _TYPES, shape), type=_TYPES[_dtype(target)], batch=B, drafts=n, vocab=V,
            draft_tokens=_expect(draft_tokens, "draft_tokens", "int32", (B, n), packed=True),
            uniform=_expect(uniform, "uniform", "float32", (B, n), packed=True), race=_expect(race, "race", "float32", (B, V)),
            tokens=_expect(tokens, "tokens", "int32", (B, n + 1), packed=True), accepted=_expect(accepted, "accepted", "int32", (B,), packed=True))
        if draft_probs is not None:
            d.draft = _expect(draft_probs, "draft_probs", _dtype(target), (B, n, V))
            d.draft_seq_stride, d.draft_row_stride = draft_probs.stride()[:2]
        if draft_lens is not None:
            d.draft_lens = _expect(draft_lens, "draft_lens", "int32", (B,), packed=True)
        d.target_seq_stride, d.target_row_stride = target.stride()[:2]
        d.race_stride = race.stride()[0]
        self._hold(d, target, draft_tokens, uniform, race, tokens, accepted, draft_probs, draft_lens)


def _rows_fit(cache, rows):
    c = cache.desc
    if rows.shape[1:] != (c.heads, c.head_dim):
        raise ValueError(f"rows of {rows.shape[1]} heads and {rows.shape[2]} elements, the cache has {c.heads} and {c.head_dim}")


def dl_kv_write(cache: KvCache, rows: KvRows, stream=None) -> None:
    """Quantise rows into their slots of the cache, which differ from each other (but for those that are none)."""
    _rows_fit(cache, rows)
    _check(lib().dl_kv_write(cache.at, rows.at, _stream(stream)), "dl_kv_write")


def dl_kv_read(cache: KvCache, rows: KvRows, stream=None) -> None:
    """What the slots of the cache hold, into rows."""
    _rows_fit(cache, rows)
    _check(lib().dl_kv_read(cache.at, rows.at, _stream(stream)), "dl_kv_read")


def _size(n: int, what: str) -> int:
    if n < 0:
        raise DlError(int(n), what)
    return int(n)


def dl_prefix_attention_workspace(request: PrefixAttention) -> int:
    """Bytes of workspace a call needs."""
    return _size(lib().dl_prefix_attention_workspace(request.cache.at, request.at), "dl_prefix_attention_workspace")


def dl_prefix_attention(request: PrefixAttention, stream=None) -> None:
    _check(lib().dl_prefix_attention(request.cache.at, request.at, _stream(stream)), "dl_prefix_attention")


def dl_verify_draft_workspace(request: DraftVerify) -> int:
    """Bytes of workspace a call needs."""
    return _size(lib().dl_verify_draft_workspace(request.at), "dl_verify_draft_workspace")


def dl_verify_draft(request: DraftVerify, stream=None) -> None:
    _check(lib().dl_verify_draft(request.at, _stream(stream)), "dl_verify_draft")


# -------------------------------------------------------------------- prelaunch

def dl_prelaunch_start() -> None:
    _check(lib().dl_prelaunch_start(), "dl_prelaunch_start")


def dl_prelaunch_stop() -> None:
    _check(lib().dl_prelaunch_stop(), "dl_prelaunch_stop")


def dl_last_ticket() -> int:
    return _native().last_ticket()


def dl_trigger(ticket: int | None = None) -> None:
    t = dl_last_ticket() if ticket is None else ticket
    status = _native().trigger(t)
    _check(lib().dl_trigger(t) if status is NotImplemented else status, "dl_trigger")


def dl_wait(ticket: int | None = None, timeout_ns: int = 5_000_000_000) -> None:
    t = dl_last_ticket() if ticket is None else ticket
    status = _native().wait(t, timeout_ns)
    _check(lib().dl_wait(t, timeout_ns) if status is NotImplemented else status, "dl_wait")


def dl_wait_armed(ticket: int | None = None, timeout_ns: int = 5_000_000_000) -> None:
    t = dl_last_ticket() if ticket is None else ticket
    _check(lib().dl_wait_armed(t, timeout_ns), "dl_wait_armed")


def dl_set_trace(on: bool) -> None:
    _check(lib().dl_set_trace(1 if on else 0), "dl_set_trace")


def dl_get_trace(ticket: int | None = None) -> dict:
    t = Trace()
    _check(lib().dl_get_trace(dl_last_ticket() if ticket is None else ticket, ctypes.byref(t)), "dl_get_trace")
    return {f[0]: int(getattr(t, f[0])) for f in Trace._fields_}


def dl_trace_clock():
    """(device ticks per microsecond, host CLOCK_MONOTONIC nanoseconds at device tick 0)."""
    a, b = ctypes.c_double(0), ctypes.c_double(0)
    _check(lib().dl_trace_clock(ctypes.byref(a), ctypes.byref(b)), "dl_trace_clock")
    return a.value, b.value


# --------------------------------------------------------------------- lowering

def _items_out(call):
    n = call(None, 0)
    if n < 0:
        raise DlError(int(n), "dl_plan")
    arr = (PlanItem * max(n, 1))()
    m = call(arr, n)
    assert m == n
    return [dict(src=arr[i].src or 0, bytes=arr[i].bytes, k=arr[i].k,
                 dst=[arr[i].dst[j] or 0 for j in range(arr[i].k)]) for i in range(n)]


def dl_plan_allgather(ins, outs, bytes_per_rank: int, fuse_broadcast: bool = True):
    ins, outs = list(ins), list(outs)
    a, b = _ptr_array(ins), _ptr_array(outs)
    return _items_out(lambda arr, cap: lib().dl_plan_allgather(a, b, len(ins), int(bytes_per_rank),
                                                               1 if fuse_broadcast else 0, arr, cap))


def dl_plan_alltoall(ins, outs, chunk_bytes):
    ins, outs = list(ins), list(outs)
    a, b, c = _ptr_array(ins), _ptr_array(outs), _chunk_array(chunk_bytes, len(ins))
    return _items_out(lambda arr, cap: lib().dl_plan_alltoall(a, b, len(ins), c, arr, cap))


def dl_plan_broadcast(src, dsts, nbytes: int):
    dsts = list(dsts)
    d = _ptr_array(dsts)
    return _items_out(lambda arr, cap: lib().dl_plan_broadcast(_addr(src), d, len(dsts), int(nbytes), arr, cap))


def dl_plan_batch(descs):
    descs = list(descs)
    d = _desc_array(descs)
    return _items_out(lambda arr, cap: lib().dl_plan_batch(d, len(descs), arr, cap))


def dl_plan_token_dispatch(ins, outs, tokens, row_bytes: int, dest):
    a, b, W, tok, d = _dispatch_args(ins, outs, tokens, dest)
    return _items_out(lambda arr, cap: lib().dl_plan_token_dispatch(a, b, W, tok, int(row_bytes), d, arr, cap))


def dl_plan_batch_inferred(descs):
    descs = list(descs)
    d = _desc_array(descs)
    return _items_out(lambda arr, cap: lib().dl_plan_batch_inferred(d, len(descs), arr, cap))


def dl_plan_alltoall_inplace(bufs, chunk_bytes: int):
    """The (a, b, bytes) swaps an in-place all-to-all lowers to."""
    bufs = list(bufs)
    p = _ptr_array(bufs)
    n = lib().dl_plan_alltoall_inplace(p, len(bufs), int(chunk_bytes), None, 0)
    if n < 0:
        raise DlError(int(n), "dl_plan_alltoall_inplace")
    arr = (SwapDesc * max(n, 1))()
    assert lib().dl_plan_alltoall_inplace(p, len(bufs), int(chunk_bytes), arr, n) == n
    return [(arr[i].a or 0, arr[i].b or 0, arr[i].bytes) for i in range(n)]


def dl_plan_swap_first_hazard(descs) -> int:
    descs = list(descs)
    return int(lib().dl_plan_swap_first_hazard(_swap_array(descs), len(descs)))


def _items_in(items):
    arr = (PlanItem * max(len(items), 1))()
    for i, it in enumerate(items):
        arr[i].src, arr[i].bytes, arr[i].k = it["src"] or None, it["bytes"], len(it["dst"])
        for j, d in enumerate(it["dst"]):
            arr[i].dst[j] = d or None
    return arr


def dl_plan_first_hazard(items) -> int:
    return int(lib().dl_plan_first_hazard(_items_in(items), len(items)))


def dl_plan_tiles(items, tile_bytes: int) -> int:
    return int(lib().dl_plan_tiles(_items_in(items), len(items), tile_bytes))
