"""Python binding of the C ABI in ``include/aqua.h`` (ctypes).

Argument marshalling only: every byte of a swap is moved by the library's
HIP kernels.  The low-level functions carry the C names and return the
C status (plus the ticket where the C call writes one); ``KVPool`` wraps
them for torch tensors and raises ``AquaError`` on a failed call.

torch is imported before the library is loaded so that the library binds
to the HIP runtime torch already holds (both carry the same soname), and
pointers and streams from torch are valid in it.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libaqua.so")

AQUA_OK = 0
AQUA_ERR_INVALID = -1
AQUA_ERR_RANGE = -2
AQUA_ERR_DUPLICATE = -3
AQUA_ERR_CAPACITY = -4
AQUA_ERR_HIP = -5
AQUA_ERR_STATE = -6

AQUA_F16, AQUA_BF16, AQUA_FP8_E4M3, AQUA_INT4 = 1, 2, 3, 4
AQUA_TARGET_DEVICE, AQUA_TARGET_HOST = 0, 1
AQUA_HOST_ZERO_COPY, AQUA_HOST_STAGED = 0, 1
AQUA_LINK_RUNTIME, AQUA_LINK_AUTO = -1, -2
AQUA_YARDSTICK_COPY, AQUA_YARDSTICK_READ, AQUA_YARDSTICK_WRITE = 0, 1, 2

EXPORTS = (
    "aqua_kv_pool_create", "aqua_kv_pool_destroy", "aqua_swap_out",
    "aqua_swap_in", "aqua_swap_out_ex", "aqua_swap_in_ex", "aqua_migrate",
    "aqua_sync", "aqua_stream_wait", "aqua_query",
    "aqua_kv_pool_set_max_workgroups", "aqua_kv_pool_set_host_path",
    "aqua_kv_pool_set_link_engine", "aqua_kv_pool_get_link_engine",
    "aqua_pool_stats_get", "aqua_status_str", "aqua_cfs_partition",
    "aqua_swap_space_create", "aqua_swap_space_destroy", "aqua_swap_alloc", "aqua_swap_free",
    "aqua_swap_locate", "aqua_swap_reclaim", "aqua_swap_restore", "aqua_swap_usage",
    "aqua_hbm_yardstick", "aqua_swap_noalloc",
    "aqua_kv_batch_create", "aqua_kv_batch_destroy", "aqua_kv_batch_set", "aqua_kv_append",
    "aqua_kv_attend",
)


class aqua_kv_desc(ctypes.Structure):
    _fields_ = [
        ("num_layers", ctypes.c_uint32),
        ("num_blocks", ctypes.c_uint32),
        ("num_kv_heads", ctypes.c_uint32),
        ("block_tokens", ctypes.c_uint32),
        ("head_dim", ctypes.c_uint32),
        ("dtype", ctypes.c_int32),
    ]


class aqua_swap_range(ctypes.Structure):
    _fields_ = [
        ("img_blocks", ctypes.c_void_p),
        ("first_layer", ctypes.c_uint32),
        ("num_layers", ctypes.c_uint32),
    ]


class aqua_pool_stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in (
        "calls_out", "calls_in", "bytes_out", "bytes_in", "bytes_host",
        "descriptors", "waits_inserted", "waits_elided", "calls_migrate",
        "bytes_migrated", "host_ns", "wait_ns")] + [
        ("hip_error", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("launches", ctypes.c_uint64)]


class aqua_cfs_request(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint32) for n in (
        "prompt_tokens", "prefill_done", "generated", "held_blocks")]


class aqua_cfs_params(ctypes.Structure):
    _fields_ = [("batch_tokens", ctypes.c_uint32), ("decode_slots", ctypes.c_uint32),
                ("block_tokens", ctypes.c_uint32), ("reserved", ctypes.c_uint32),
                ("capacity_blocks", ctypes.c_uint64)]


class aqua_kv_batch_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint32) for n in (
        "num_q_heads", "max_seqs", "max_tokens", "max_blocks")]


class aqua_kv_append_args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "q", "q_out")] + \
        [(n, ctypes.c_uint64) for n in ("k_stride", "v_stride", "q_stride", "q_out_stride")] + \
        [("dtype", ctypes.c_int32), ("interleaved", ctypes.c_int32),
         ("rope", ctypes.c_void_p), ("rope_rows", ctypes.c_uint32),
         ("rope_dim", ctypes.c_uint32), ("k_scale", ctypes.c_float),
         ("v_scale", ctypes.c_float)]


class aqua_kv_attend_args(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p),
                ("q_stride", ctypes.c_uint64), ("out_stride", ctypes.c_uint64),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float)]


class AquaError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {aqua_status_str(status)} ({status})")
        self.status = status


_lib: Optional[ctypes.CDLL] = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Loads the library; fails loudly when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} is missing: build it with "
            "`python -m paper_2407_21255_amd.build` (hipcc, gfx950)")
    L = ctypes.CDLL(path)
    P, u32, u64, i32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int32
    L.aqua_kv_pool_create.argtypes = [ctypes.POINTER(aqua_kv_desc), P, u64,
                                      ctypes.POINTER(P)]
    L.aqua_kv_pool_destroy.argtypes = [P]
    L.aqua_swap_out.argtypes = [P, u32, P, P, P, u64, P, i32, P, ctypes.POINTER(u64)]
    L.aqua_swap_in.argtypes = [P, u32, P, P, P, u64, P, i32, P, ctypes.POINTER(u64)]
    R = ctypes.POINTER(aqua_swap_range)
    L.aqua_swap_out_ex.argtypes = [P, u32, P, P, P, u64, P, R, i32, P, ctypes.POINTER(u64)]
    L.aqua_swap_in_ex.argtypes = [P, u32, P, P, P, u64, P, R, i32, P, ctypes.POINTER(u64)]
    L.aqua_migrate.argtypes = [P, P, u64, i32, P, u64, i32, u32, P, P, P, P,
                               ctypes.POINTER(u64)]
    L.aqua_sync.argtypes = [P, u64]
    L.aqua_stream_wait.argtypes = [P, u64, P]
    L.aqua_query.argtypes = [P, u64]
    L.aqua_kv_pool_set_max_workgroups.argtypes = [P, i32, u32]
    L.aqua_kv_pool_set_host_path.argtypes = [P, i32]
    L.aqua_kv_pool_set_link_engine.argtypes = [P, i32, i32]
    L.aqua_kv_pool_get_link_engine.argtypes = [P, i32, ctypes.POINTER(i32)]
    L.aqua_pool_stats_get.argtypes = [P, ctypes.POINTER(aqua_pool_stats)]
    L.aqua_cfs_partition.argtypes = [P, u32, ctypes.POINTER(aqua_cfs_params), P, P,
                                     ctypes.POINTER(u32), ctypes.POINTER(u64)]
    L.aqua_swap_space_create.argtypes = [P, u64, u64, ctypes.POINTER(P)]
    L.aqua_swap_space_destroy.argtypes = [P]
    L.aqua_swap_alloc.argtypes = [P, u64, ctypes.POINTER(u64)]
    L.aqua_swap_free.argtypes = [P, u64]
    L.aqua_swap_locate.argtypes = [P, u64, ctypes.POINTER(P), ctypes.POINTER(u64),
                                   ctypes.POINTER(i32)]
    L.aqua_swap_reclaim.argtypes = [P, u64, P, ctypes.POINTER(u64)]
    L.aqua_swap_restore.argtypes = [P, P, ctypes.POINTER(u64)]
    L.aqua_swap_usage.argtypes = [P] + [ctypes.POINTER(u64)] * 4
    L.aqua_hbm_yardstick.argtypes = [i32, P, P, u64, P]
    L.aqua_swap_noalloc.argtypes = [P, i32, u32, P, P, P, u64, P, i32, P, ctypes.POINTER(u64)]
    L.aqua_kv_batch_create.argtypes = [P, ctypes.POINTER(aqua_kv_batch_desc), ctypes.POINTER(P)]
    L.aqua_kv_batch_destroy.argtypes = [P]
    L.aqua_kv_batch_set.argtypes = [P, u32, P, P, P, P, P]
    L.aqua_kv_append.argtypes = [P, u32, ctypes.POINTER(aqua_kv_append_args), P]
    L.aqua_kv_attend.argtypes = [P, u32, ctypes.POINTER(aqua_kv_attend_args), P]
    L.aqua_status_str.argtypes = [i32]
    L.aqua_status_str.restype = ctypes.c_char_p
    for n in EXPORTS:
        if n != "aqua_status_str":
            getattr(L, n).restype = i32
    _lib = L
    return L


# -- the C entry points, one to one ------------------------------------------

def aqua_kv_pool_create(desc: aqua_kv_desc, pool_base: int, pool_bytes: int):
    h = ctypes.c_void_p()
    st = load().aqua_kv_pool_create(ctypes.byref(desc), pool_base, pool_bytes,
                                    ctypes.byref(h))
    return st, h


def aqua_kv_pool_destroy(pool) -> int:
    return load().aqua_kv_pool_destroy(pool)


def aqua_swap_out(pool, num_seqs, block_ids, seq_offsets, dst, dst_bytes,
                  img_offsets, target, stream):
    t = ctypes.c_uint64(0)
    st = load().aqua_swap_out(pool, num_seqs, block_ids, seq_offsets, dst, dst_bytes,
                              img_offsets, target, stream, ctypes.byref(t))
    return st, t.value


def aqua_swap_in(pool, num_seqs, block_ids, seq_offsets, src, src_bytes,
                 img_offsets, target, stream):
    t = ctypes.c_uint64(0)
    st = load().aqua_swap_in(pool, num_seqs, block_ids, seq_offsets, src, src_bytes,
                             img_offsets, target, stream, ctypes.byref(t))
    return st, t.value


def aqua_swap_out_ex(pool, num_seqs, block_ids, seq_offsets, dst, dst_bytes,
                     img_offsets, rng, target, stream):
    t = ctypes.c_uint64(0)
    st = load().aqua_swap_out_ex(pool, num_seqs, block_ids, seq_offsets, dst, dst_bytes,
                                 img_offsets, rng, target, stream, ctypes.byref(t))
    return st, t.value


def aqua_swap_in_ex(pool, num_seqs, block_ids, seq_offsets, src, src_bytes,
                    img_offsets, rng, target, stream):
    t = ctypes.c_uint64(0)
    st = load().aqua_swap_in_ex(pool, num_seqs, block_ids, seq_offsets, src, src_bytes,
                                img_offsets, rng, target, stream, ctypes.byref(t))
    return st, t.value


def aqua_swap_noalloc(pool, direction, num_seqs, block_ids, seq_offsets, buf, buf_bytes,
                      img_offsets, target, stream):
    t = ctypes.c_uint64(0)
    st = load().aqua_swap_noalloc(pool, direction, num_seqs, block_ids, seq_offsets, buf,
                                  buf_bytes, img_offsets, target, stream, ctypes.byref(t))
    return st, t.value


def aqua_migrate(pool, src, src_bytes, src_target, dst, dst_bytes, dst_target, n,
                 src_offsets, dst_offsets, lengths, stream):
    t = ctypes.c_uint64(0)
    st = load().aqua_migrate(pool, src, src_bytes, src_target, dst, dst_bytes, dst_target, n,
                             src_offsets, dst_offsets, lengths, stream, ctypes.byref(t))
    return st, t.value


def aqua_sync(pool, ticket: int = 0) -> int:
    return load().aqua_sync(pool, ticket)


def aqua_stream_wait(pool, ticket: int, stream) -> int:
    return load().aqua_stream_wait(pool, ticket, stream)


def aqua_query(pool, ticket: int) -> int:
    return load().aqua_query(pool, ticket)


def aqua_kv_pool_set_max_workgroups(pool, target: int, n: int) -> int:
    return load().aqua_kv_pool_set_max_workgroups(pool, target, n)


def aqua_kv_pool_set_host_path(pool, path: int) -> int:
    return load().aqua_kv_pool_set_host_path(pool, path)


def aqua_kv_pool_set_link_engine(pool, direction: int, engine: int) -> int:
    return load().aqua_kv_pool_set_link_engine(pool, direction, engine)


def aqua_kv_pool_get_link_engine(pool, direction: int):
    e = ctypes.c_int32(0)
    st = load().aqua_kv_pool_get_link_engine(pool, direction, ctypes.byref(e))
    return st, e.value


def aqua_pool_stats_get(pool):
    s = aqua_pool_stats()
    st = load().aqua_pool_stats_get(pool, ctypes.byref(s))
    return st, s


def aqua_hbm_yardstick(kind: int, dst, src, nbytes: int, stream) -> int:
    return load().aqua_hbm_yardstick(kind, dst, src, nbytes, stream)


def hbm_yardstick(kind: int, dst: torch.Tensor, src: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> None:
    """Enqueues one HBM yardstick pass (AQUA_YARDSTICK_COPY / _READ / _WRITE)
    over src's bytes (dst's for a write) on ``stream``; raises AquaError on
    a failed call."""
    nbytes = (src if kind != AQUA_YARDSTICK_WRITE else dst).numel() * \
        (src if kind != AQUA_YARDSTICK_WRITE else dst).element_size()
    st = aqua_hbm_yardstick(kind, dst.data_ptr(), src.data_ptr() if src is not None else None,
                            nbytes, stream.cuda_stream if stream is not None else None)
    if st != AQUA_OK:
        raise AquaError(st, "aqua_hbm_yardstick")


def aqua_status_str(status: int) -> str:
    try:
        return load().aqua_status_str(status).decode()
    except FileNotFoundError:
        return f"status {status}"


def aqua_cfs_partition(requests: np.ndarray, params: aqua_cfs_params,
                       batch_index: np.ndarray, batch_tokens: np.ndarray):
    """requests: uint32 array [n, 4] (the fields of aqua_cfs_request);
    batch_index / batch_tokens: uint32 arrays of n entries.  Returns
    (status, batch size, blocks taken)."""
    n = len(requests)
    size, taken = ctypes.c_uint32(0), ctypes.c_uint64(0)
    st = load().aqua_cfs_partition(
        requests.ctypes.data if n else None, n, ctypes.byref(params),
        batch_index.ctypes.data if n else None, batch_tokens.ctypes.data if n else None,
        ctypes.byref(size), ctypes.byref(taken))
    return st, size.value, taken.value


def cfs_partition(requests, batch_tokens: int, decode_slots: int, capacity_blocks: int,
                  block_tokens: int):
    """One iteration's fair batch (section 7): ``requests`` rows are
    (prompt_tokens, prefill_done, generated, held_blocks).  Returns
    (index array, token array, blocks taken), admission order."""
    req = np.ascontiguousarray(np.asarray(requests, dtype=np.uint32).reshape(-1, 4))
    n = len(req)
    idx = np.zeros(n, dtype=np.uint32)
    tok = np.zeros(n, dtype=np.uint32)
    prm = aqua_cfs_params(batch_tokens, decode_slots, block_tokens, 0, capacity_blocks)
    st, size, taken = aqua_cfs_partition(req, prm, idx, tok)
    if st != AQUA_OK:
        raise AquaError(st, "aqua_cfs_partition")
    return idx[:size], tok[:size], taken


def aqua_swap_space_create(pool, device_bytes: int, host_bytes: int):
    h = ctypes.c_void_p()
    st = load().aqua_swap_space_create(pool, device_bytes, host_bytes, ctypes.byref(h))
    return st, h.value


def aqua_swap_space_destroy(space) -> int:
    return load().aqua_swap_space_destroy(space)


def aqua_swap_alloc(space, nbytes: int):
    h = ctypes.c_uint64(0)
    st = load().aqua_swap_alloc(space, nbytes, ctypes.byref(h))
    return st, h.value


def aqua_swap_free(space, handle: int) -> int:
    return load().aqua_swap_free(space, handle)


def aqua_swap_locate(space, handle: int):
    """(status, pointer, bytes, target)."""
    ptr, nb, tg = ctypes.c_void_p(), ctypes.c_uint64(0), ctypes.c_int32(0)
    st = load().aqua_swap_locate(space, handle, ctypes.byref(ptr), ctypes.byref(nb),
                                 ctypes.byref(tg))
    return st, ptr.value, nb.value, tg.value


def aqua_swap_reclaim(space, nbytes: int, stream):
    t = ctypes.c_uint64(0)
    st = load().aqua_swap_reclaim(space, nbytes, stream, ctypes.byref(t))
    return st, t.value


def aqua_swap_restore(space, stream):
    t = ctypes.c_uint64(0)
    st = load().aqua_swap_restore(space, stream, ctypes.byref(t))
    return st, t.value


def aqua_swap_usage(space):
    """(status, device free bytes, host free bytes, device tensors, host tensors)."""
    v = [ctypes.c_uint64(0) for _ in range(4)]
    st = load().aqua_swap_usage(space, *[ctypes.byref(x) for x in v])
    return (st, *[x.value for x in v])


def aqua_kv_batch_create(pool, desc: aqua_kv_batch_desc):
    h = ctypes.c_void_p()
    st = load().aqua_kv_batch_create(pool, ctypes.byref(desc), ctypes.byref(h))
    return st, h.value


def aqua_kv_batch_destroy(batch) -> int:
    return load().aqua_kv_batch_destroy(batch)


def aqua_kv_batch_set(batch, num_seqs, block_ids, seq_offsets, context_tokens, new_tokens,
                      stream) -> int:
    return load().aqua_kv_batch_set(batch, num_seqs, block_ids, seq_offsets, context_tokens,
                                    new_tokens, stream)


def aqua_kv_append(batch, layer: int, args: aqua_kv_append_args, stream) -> int:
    return load().aqua_kv_append(batch, layer, ctypes.byref(args), stream)


def aqua_kv_attend(batch, layer: int, args: aqua_kv_attend_args, stream) -> int:
    return load().aqua_kv_attend(batch, layer, ctypes.byref(args), stream)


# -- torch-facing wrapper ------------------------------------------------------

class RawBuffer:
    """A byte buffer the library placed (a swap-space tensor), usable where
    the swap calls take a tensor."""

    def __init__(self, ptr: int, nbytes: int, target: int):
        self.ptr, self.nbytes, self.aqua_target = ptr, nbytes, target

    def data_ptr(self) -> int:
        return self.ptr

    def numel(self) -> int:
        return self.nbytes

    def element_size(self) -> int:
        return 1


def _addr(a: Optional[np.ndarray]) -> Optional[int]:
    """Address of an array's data (``a.ctypes.data`` without its wrapper)."""
    return None if a is None else a.__array_interface__["data"][0]


_INT32, _INT64, _UINT64 = (np.dtype(t) for t in (np.int32, np.int64, np.uint64))


def _whole(a, dtype: np.dtype, status: int, what: str) -> np.ndarray:
    """Numbers in a row as an array of `dtype`, none of them wrapped or cut on the way."""
    a = np.asarray(a)
    if a.dtype is not dtype:
        with np.errstate(invalid="ignore"):
            b = a.astype(dtype)
        if not np.array_equal(b, a):
            raise AquaError(status, what)
        a = b
    if a.ndim != 1:
        raise AquaError(AQUA_ERR_INVALID, what)
    return np.ascontiguousarray(a)


def _csr(tables):
    """(int32 ids, uint64 offsets) from a list of tables or an (ids, offs) pair."""
    if isinstance(tables, tuple) and len(tables) == 2 and isinstance(tables[0], np.ndarray):
        ids = _whole(tables[0], _INT32, AQUA_ERR_RANGE, "block ids")
        offs = _whole(tables[1], _UINT64, AQUA_ERR_INVALID, "table offsets")
        if not len(offs) or offs.item(-1) > len(ids):
            raise AquaError(AQUA_ERR_INVALID, "table offsets")
        return ids, offs
    ids = np.asarray([b for t in tables for b in t], dtype=np.int32)
    offs = np.zeros(len(tables) + 1, dtype=np.uint64)
    if len(tables):
        offs[1:] = np.cumsum([len(t) for t in tables])
    return _whole(ids, _INT32, AQUA_ERR_RANGE, "block ids"), offs


# The current device's current stream as a handle, without the Stream object
# that torch.cuda.current_stream() builds around it (0.15 against 2.6 us, of
# the 10 us that a small call costs its caller).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_cur_device = getattr(torch._C, "_cuda_getDevice", None)
_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing",
                     torch.cuda.is_current_stream_capturing)


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None and _cur_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_cur_device()) or None
        stream = torch.cuda.current_stream()
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _target_of(t) -> int:
    if isinstance(t, RawBuffer):
        return t.aqua_target
    if t.is_cuda:
        return AQUA_TARGET_DEVICE
    if t.is_pinned():
        return AQUA_TARGET_HOST
    raise AquaError(AQUA_ERR_INVALID, "offload buffer must be a device or pinned host tensor")


class KVPool:
    """A paged KV pool bound to a caller-owned uint8 device tensor."""

    def __init__(self, shape: Sequence[int], pool: torch.Tensor):
        L, N, H, T, D, dtype = shape
        self.desc = aqua_kv_desc(L, N, H, T, D, dtype)
        self.pool = pool
        st, h = aqua_kv_pool_create(self.desc, pool.data_ptr(),
                                    pool.numel() * pool.element_size())
        if st != AQUA_OK:
            raise AquaError(st, "aqua_kv_pool_create")
        self.handle = h
        self._spaces = []      # swap spaces and batches on this pool, closed before it
        self._held = {}        # ticket -> the tensors its call names, until it completes
        self._prune_at = 64    # prune completed entries when this many are held

    def _hold(self, ticket: int, *tensors) -> None:
        """Keeps the tensors that a call reads or writes alive until the call
        completes: the library only borrows their memory, and a tensor freed
        early could be handed out again while a kernel or a copy engine still
        uses it."""
        if len(self._held) >= self._prune_at:
            done = [t for t in self._held if aqua_query(self.handle, t) == 1]
            for t in done:
                del self._held[t]
            # Amortised: the next pass waits until the held set has doubled.
            self._prune_at = max(64, 2 * len(self._held))
        self._held[ticket] = tensors

    def _swap(self, is_in, tables, buf, img_offsets, stream, target, img_blocks, layers):
        ids, offs = _csr(tables)
        io = None
        if img_offsets is not None:
            io = np.ascontiguousarray(img_offsets, dtype=np.uint64)
        tgt = _target_of(buf) if target is None else target
        args = (self.handle, len(offs) - 1, _addr(ids), _addr(offs),
                buf.data_ptr(), buf.numel() * buf.element_size(), _addr(io))
        if img_blocks is None and layers is None:
            fn, name = (aqua_swap_in, "aqua_swap_in") if is_in else (aqua_swap_out, "aqua_swap_out")
            st, ticket = fn(*args, tgt, _stream_handle(stream))
        else:
            ib = None if img_blocks is None else np.ascontiguousarray(img_blocks, dtype=np.uint64)
            l0, nl = (0, 0) if layers is None else layers
            rng = aqua_swap_range(None if ib is None else ib.ctypes.data, l0, nl)
            fn, name = ((aqua_swap_in_ex, "aqua_swap_in_ex") if is_in
                        else (aqua_swap_out_ex, "aqua_swap_out_ex"))
            st, ticket = fn(*args, ctypes.byref(rng), tgt, _stream_handle(stream))
        if st != AQUA_OK:
            raise AquaError(st, name)
        self._hold(ticket, buf)
        return ticket

    def swap_out(self, tables, dst: torch.Tensor, img_offsets=None, stream=None,
                 target=None, img_blocks=None, layers=None) -> int:
        """Gather; ``img_blocks`` (blocks per layer of each image) and
        ``layers`` = (first, count) select the extended form."""
        return self._swap(False, tables, dst, img_offsets, stream, target, img_blocks, layers)

    def swap_in(self, tables, src: torch.Tensor, img_offsets=None, stream=None,
                target=None, img_blocks=None, layers=None) -> int:
        return self._swap(True, tables, src, img_offsets, stream, target, img_blocks, layers)

    def swap_noalloc(self, direction: int, tables, buf: torch.Tensor, img_offsets=None,
                     stream=None, target=None) -> int:
        """aqua_swap_noalloc: swap-out (direction 0) or swap-in (1) that
        allocates nothing."""
        ids, offs = _csr(tables)
        io = None
        if img_offsets is not None:
            io = np.ascontiguousarray(img_offsets, dtype=np.uint64)
        tgt = _target_of(buf) if target is None else target
        st, ticket = aqua_swap_noalloc(
            self.handle, direction, len(offs) - 1, _addr(ids), _addr(offs),
            buf.data_ptr(), buf.numel() * buf.element_size(), _addr(io), tgt,
            _stream_handle(stream))
        if st != AQUA_OK:
            raise AquaError(st, "aqua_swap_noalloc")
        self._hold(ticket, buf)
        return ticket

    def migrate(self, src: torch.Tensor, dst: torch.Tensor, src_offsets, dst_offsets,
                lengths, stream=None) -> int:
        """Copy byte ranges between offload buffers (device or pinned host)."""
        so, do, ln = (np.ascontiguousarray(x, dtype=np.uint64)
                      for x in (src_offsets, dst_offsets, lengths))
        st, ticket = aqua_migrate(self.handle, src.data_ptr(), src.numel() * src.element_size(),
                                  _target_of(src), dst.data_ptr(),
                                  dst.numel() * dst.element_size(), _target_of(dst), len(ln),
                                  so.ctypes.data, do.ctypes.data, ln.ctypes.data,
                                  _stream_handle(stream))
        if st != AQUA_OK:
            raise AquaError(st, "aqua_migrate")
        self._hold(ticket, src, dst)
        return ticket

    def sync(self, ticket: int = 0) -> None:
        st = aqua_sync(self.handle, ticket)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_sync")
        if ticket == 0:
            self._held.clear()
        else:
            self._held.pop(ticket, None)

    def stream_wait(self, ticket: int, stream=None) -> None:
        st = aqua_stream_wait(self.handle, ticket, _stream_handle(stream))
        if st != AQUA_OK:
            raise AquaError(st, "aqua_stream_wait")

    def query(self, ticket: int) -> bool:
        st = aqua_query(self.handle, ticket)
        if st < 0:
            raise AquaError(st, "aqua_query")
        return st == 1

    def set_max_workgroups(self, target: int, n: int) -> None:
        st = aqua_kv_pool_set_max_workgroups(self.handle, target, n)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_kv_pool_set_max_workgroups")

    def set_host_path(self, path: int) -> None:
        st = aqua_kv_pool_set_host_path(self.handle, path)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_kv_pool_set_host_path")

    def set_link_engine(self, direction: int, engine: int) -> None:
        """Carrier of the staged path's link copies for one direction (0:
        swap-out, 1: swap-in): an SDMA engine index, AQUA_LINK_RUNTIME or
        AQUA_LINK_AUTO."""
        st = aqua_kv_pool_set_link_engine(self.handle, direction, engine)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_kv_pool_set_link_engine")

    def link_engine(self, direction: int) -> int:
        st, e = aqua_kv_pool_get_link_engine(self.handle, direction)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_kv_pool_get_link_engine")
        return e

    def stats(self) -> dict:
        st, s = aqua_pool_stats_get(self.handle)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_pool_stats_get")
        return {n: getattr(s, n) for n, _ in s._fields_ if n != "reserved"}

    def close(self) -> None:
        for sp in list(getattr(self, "_spaces", [])):
            sp.close()
        if getattr(self, "handle", None):
            st = aqua_kv_pool_destroy(self.handle)
            self.handle = None
            self._held.clear()   # destroy waited for every call
            if st != AQUA_OK:
                raise AquaError(st, "aqua_kv_pool_destroy")

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


class SwapSpace:
    """Offload tensors with a device region and a pinned-host fallback, on a
    pool (see aqua_swap_space_create)."""

    def __init__(self, pool: "KVPool", device_bytes: int, host_bytes: int):
        st, h = aqua_swap_space_create(pool.handle, device_bytes, host_bytes)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_swap_space_create")
        self.handle = h
        self.pool = pool
        pool._spaces.append(self)

    def alloc(self, nbytes: int) -> int:
        st, h = aqua_swap_alloc(self.handle, nbytes)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_swap_alloc")
        return h

    def free(self, tensor: int) -> None:
        st = aqua_swap_free(self.handle, tensor)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_swap_free")

    def locate(self, tensor: int):
        """(pointer, bytes, target) of a tensor now."""
        st, ptr, nb, tg = aqua_swap_locate(self.handle, tensor)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_swap_locate")
        return ptr, nb, tg

    def buffer(self, tensor: int) -> RawBuffer:
        """The tensor's current bytes, for KVPool.swap_out / swap_in."""
        return RawBuffer(*self.locate(tensor))

    def reclaim(self, nbytes: Optional[int] = None, stream=None) -> int:
        st, t = aqua_swap_reclaim(self.handle, (1 << 64) - 1 if nbytes is None else nbytes,
                                  _stream_handle(stream))
        if st != AQUA_OK:
            raise AquaError(st, "aqua_swap_reclaim")
        return t

    def restore(self, stream=None) -> int:
        st, t = aqua_swap_restore(self.handle, _stream_handle(stream))
        if st != AQUA_OK:
            raise AquaError(st, "aqua_swap_restore")
        return t

    def usage(self) -> dict:
        st, df, hf, dn, hn = aqua_swap_usage(self.handle)
        if st != AQUA_OK:
            raise AquaError(st, "aqua_swap_usage")
        return {"device_free": df, "host_free": hf, "device_tensors": dn, "host_tensors": hn}

    def close(self) -> None:
        if getattr(self, "handle", None):
            st = aqua_swap_space_destroy(self.handle)
            self.handle = None
            self.pool._spaces.remove(self)
            if st != AQUA_OK:
                raise AquaError(st, "aqua_swap_space_destroy")

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


_DTYPES = {torch.float16: AQUA_F16, torch.bfloat16: AQUA_BF16}


class KVBatch:
    """One step's sequences on a pool, and the operators of its layers (see
    aqua_kv_batch_create): ``set`` once a step, then ``append`` and ``attend`` for
    every layer.  Tensors are [tokens, heads, head_dim] device tensors of one 16-bit
    type, their heads contiguous, the new tokens of all sequences packed in
    sequence order.  There is no backward pass: tensors that require a gradient are
    refused where gradients are on.  Closed with its pool at the latest."""

    def __init__(self, pool: "KVPool", num_q_heads: int, max_seqs: int, max_tokens: int,
                 max_blocks: int):
        if not all(0 <= x < 1 << 32 for x in (num_q_heads, max_seqs, max_tokens, max_blocks)):
            raise AquaError(AQUA_ERR_INVALID, "aqua_kv_batch_create")
        st, h = aqua_kv_batch_create(
            pool.handle, aqua_kv_batch_desc(num_q_heads, max_seqs, max_tokens, max_blocks))
        if st != AQUA_OK:
            raise AquaError(st, "aqua_kv_batch_create")
        self.handle = h
        self.pool = pool
        self.device = pool.pool.device.index
        self.num_q_heads = num_q_heads
        self.head_dim = pool.desc.head_dim
        self.num_layers, self.num_kv_heads = pool.desc.num_layers, pool.desc.num_kv_heads
        self.max_tokens = max_tokens
        self.tokens = 0
        pool._spaces.append(self)

    def set(self, tables, context, new, stream=None) -> None:
        """``tables`` as for swaps; ``context``: tokens of each sequence, the new ones
        among them; ``new``: how many of them are new."""
        if isinstance(tables, list) and tables and \
                all(isinstance(t, np.ndarray) for t in tables):
            # (As _csr does, without a Python number for every block.)
            try:
                ids = np.concatenate(tables)
            except ValueError:   # tables that are not rows of numbers all
                raise AquaError(AQUA_ERR_INVALID, "aqua_kv_batch_set") from None
            ids = _whole(ids, _INT32, AQUA_ERR_RANGE, "aqua_kv_batch_set")
            offs = np.zeros(len(tables) + 1, dtype=np.uint64)
            offs[1:] = np.cumsum([len(t) for t in tables])
        else:
            ids, offs = _csr(tables)
        ctx, fresh = (_whole(x, _INT64, AQUA_ERR_INVALID, "aqua_kv_batch_set")
                      for x in (context, new))
        if not len(ctx) == len(fresh) == len(offs) - 1 or \
                (len(ctx) and (min(ctx.min(), fresh.min()) < 0 or ctx.max() >= 1 << 32)):
            raise AquaError(AQUA_ERR_INVALID, "aqua_kv_batch_set")
        ctx32, fresh32 = ctx.astype(np.uint32), np.minimum(fresh, (1 << 32) - 1).astype(np.uint32)
        st = aqua_kv_batch_set(self.handle, len(ctx), _addr(ids), _addr(offs), _addr(ctx32),
                               _addr(fresh32), self._stream(stream))
        if st != AQUA_OK:
            raise AquaError(st, "aqua_kv_batch_set")
        self.tokens = int(fresh.sum())

    @staticmethod
    def _no_gradients(what: str, *tensors) -> None:
        """The operators have no backward pass: a result that silently has no gradient
        would cut the caller's graph."""
        for t in tensors:
            if t is not None and t.requires_grad:
                raise AquaError(AQUA_ERR_INVALID, what + ", which makes no gradient, of a "
                                "tensor that requires one (detach it, or use torch.no_grad())")

    def _stream(self, stream) -> Optional[int]:
        """A call's stream as a handle: unless given the current one of the pool's device,
        which need not be the current device."""
        if stream is None:
            if _raw_stream is not None:
                return _raw_stream(self.device) or None
            stream = torch.cuda.current_stream(self.device)
        return _stream_handle(stream)

    def _stream_object(self, stream):
        return torch.cuda.ExternalStream(stream, device=self.device) \
            if isinstance(stream, int) else stream

    def _needed(self, stream) -> int:
        """Rows that a call's tensors have: the step's, or, for a call that is being
        captured, as many as a step can ever have."""
        if stream is not None:
            with torch.cuda.stream(self._stream_object(stream)):
                capturing = _capturing()
        elif _cur_device is None or _cur_device() != self.device:
            with torch.cuda.device(self.device):
                capturing = _capturing()
        else:
            capturing = _capturing()
        return self.max_tokens if capturing else self.tokens

    def _stride(self, t: torch.Tensor, heads: int, rows: int, what: str) -> int:
        """The row stride of a tensor that a call may name, after the checks that need
        its shape (the library sees an address)."""
        n, s, D = t.shape, t.stride(), self.head_dim
        if (len(n) != 3 or n[0] < rows or n[1] != heads or n[2] != D or s[2] != 1
                or (heads > 1 and s[1] != D) or not t.is_cuda):
            raise AquaError(AQUA_ERR_INVALID, what)
        return s[0] if n[0] > 1 else heads * D     # (a single row's stride says nothing)

    def _used(self, stream, *tensors) -> None:
        """Tensors of torch's allocator that another than the current stream uses are
        not handed out again before it is done with them."""
        s = self._stream_object(stream)
        if s.cuda_stream != torch.cuda.current_stream(s.device).cuda_stream:
            for t in tensors:
                if t is not None:
                    t.record_stream(s)

    def _result(self, stream, like: torch.Tensor, dtype=None) -> torch.Tensor:
        """A new tensor like `like` that a call on `stream` fills.  It is the memory of that
        stream: what the current one has let go may still be in use there."""
        if stream is None:   # (1.2 us; new_empty takes 1.8)
            return torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)
        s = self._stream_object(stream)
        current = torch.cuda.current_stream(like.device)
        with torch.cuda.stream(s):
            t = torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)
        if s.cuda_stream != current.cuda_stream:
            t.record_stream(current)
        return t

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor,
               q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               rope: Optional[torch.Tensor] = None, interleaved: bool = False,
               k_scale: float = 1.0, v_scale: float = 1.0,
               stream=None) -> Optional[torch.Tensor]:
        """aqua_kv_append.  ``rope``: float32 [positions, rotated part of a head], cosines
        and then sines.  Returns the rotated queries (``q_out``, which may be ``q``
        itself, or a new tensor), None without ``q``."""
        name, H = "aqua_kv_append", self.num_kv_heads
        if not 0 <= layer < self.num_layers:   # (ctypes takes a number's low bits)
            raise AquaError(AQUA_ERR_INVALID, name)
        if torch.is_grad_enabled():
            self._no_gradients(name, k, v, q, q_out, rope)
        dtype = _DTYPES.get(k.dtype)
        if dtype is None or v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
            raise AquaError(AQUA_ERR_INVALID, name)
        rows = self._needed(stream)
        a = aqua_kv_append_args(k=k.data_ptr(), v=v.data_ptr(),
                                k_stride=self._stride(k, H, rows, name),
                                v_stride=self._stride(v, H, rows, name), dtype=dtype,
                                interleaved=int(bool(interleaved)), k_scale=k_scale,
                                v_scale=v_scale)
        if q is not None:
            a.q_stride = self._stride(q, self.num_q_heads, rows, name)
            if q_out is None:
                q_out = self._result(stream, q)
            if q_out.dtype != q.dtype:
                raise AquaError(AQUA_ERR_INVALID, name)
            a.q_out_stride = self._stride(q_out, self.num_q_heads, rows, name)
            a.q, a.q_out = q.data_ptr(), q_out.data_ptr()
        elif q_out is not None:
            raise AquaError(AQUA_ERR_INVALID, name)
        if rope is not None:
            if rope.dtype != torch.float32 or rope.dim() != 2 or not rope.is_contiguous() \
                    or not rope.is_cuda:
                raise AquaError(AQUA_ERR_INVALID, name)
            a.rope, a.rope_rows, a.rope_dim = rope.data_ptr(), rope.shape[0], rope.shape[1]
        st = aqua_kv_append(self.handle, layer, a, self._stream(stream))
        if st != AQUA_OK:
            raise AquaError(st, name)
        if stream is not None:
            self._used(stream, k, v, q, q_out, rope)
        return q_out

    def attend(self, layer: int, q: torch.Tensor, out: Optional[torch.Tensor] = None,
               lse=None, scale: Optional[float] = None, k_scale: float = 1.0,
               v_scale: float = 1.0, stream=None):
        """aqua_kv_attend.  ``scale`` is 1 / sqrt(head_dim) unless given.  ``lse``: True, or
        a contiguous float32 tensor [tokens, query heads] to fill; then (out, lse) is
        returned, else out."""
        name = "aqua_kv_attend"
        if not 0 <= layer < self.num_layers:
            raise AquaError(AQUA_ERR_INVALID, name)
        if torch.is_grad_enabled():
            self._no_gradients(name, q, out, None if isinstance(lse, bool) else lse)
        dtype = _DTYPES.get(q.dtype)
        if dtype is None:
            raise AquaError(AQUA_ERR_INVALID, name)
        rows = self._needed(stream)
        stride = self._stride(q, self.num_q_heads, rows, name)
        if out is None:
            out = self._result(stream, q)
        if out.dtype != q.dtype:
            raise AquaError(AQUA_ERR_INVALID, name)
        if lse is True:
            lse = self._result(stream, q[:, :, 0], torch.float32)
        elif lse is False:
            lse = None
        if lse is not None and (lse.dtype != torch.float32 or lse.dim() != 2
                                or lse.shape[0] < rows
                                or lse.shape[1] != self.num_q_heads or not lse.is_contiguous()):
            raise AquaError(AQUA_ERR_INVALID, name)
        a = aqua_kv_attend_args(
            q=q.data_ptr(), out=out.data_ptr(), lse=None if lse is None else lse.data_ptr(),
            q_stride=stride, out_stride=self._stride(out, self.num_q_heads, rows, name), dtype=dtype,
            scale=self.head_dim ** -0.5 if scale is None else scale,
            k_scale=k_scale, v_scale=v_scale)
        st = aqua_kv_attend(self.handle, layer, a, self._stream(stream))
        if st != AQUA_OK:
            raise AquaError(st, name)
        if stream is not None:
            self._used(stream, q, out, lse)
        return out if lse is None else (out, lse)

    def close(self) -> None:
        if getattr(self, "handle", None):
            st = aqua_kv_batch_destroy(self.handle)
            self.handle = None
            self.pool._spaces.remove(self)
            if st != AQUA_OK:
                raise AquaError(st, "aqua_kv_batch_destroy")

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()
