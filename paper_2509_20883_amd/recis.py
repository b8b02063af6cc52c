"""Python binding of librecis_mi355x.so (ctypes; argument marshalling only).

Every step of the embedding path runs in the library's HIP kernels; PyTorch is
used here only for device memory and the current HIP stream.  There is no
fallback: if the library is not built, or no GPU is present, calls raise.

Names follow the C ABI (include/recis_mi355x.h): ht_create, ht_find_or_insert,
lookup_pool_fwd, lookup_pool_bwd, sparse_opt_step, lookup_pool_bwd_opt,
ids_partition, fused_bucketize, fused_mod, layer_norm_fwd, layer_norm_bwd,
seq_attention_fwd, seq_attention_bwd, seq_cache_append, seq_cache_read,
seq_cache_attention, seq_cache_select.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import NamedTuple, Optional, Tuple

import torch

PKG = os.path.dirname(os.path.abspath(__file__))
# RS_LIB names another build of the library (e.g. a variant being measured)
LIB_PATH = os.environ.get("RS_LIB") or os.path.join(PKG, "librecis_mi355x.so")
HEADER = os.path.join(os.path.dirname(PKG), "include", "recis_mi355x.h")

OK, EINVAL, ENOMEM, EFULL, EKEY, EHIP = 0, 1, 2, 3, 4, 5
STATUS_NAMES = {0: "RS_OK", 1: "RS_EINVAL", 2: "RS_ENOMEM", 3: "RS_EFULL", 4: "RS_EKEY", 5: "RS_EHIP"}
SUM, MEAN, NONE, TAIL = 0, 1, 2, 3
F32, BF16 = 0, 1
ADAGRAD, ADAM, ADAMW, ADAM_TF, ADAGRAD_RW, ADAM_RW = 0, 1, 2, 3, 4, 5
# kernel ids of rs_set_kernel_events ("occ" and "init_rows" bracket the same
# launch; "bwd_long" brackets the hot-key unit sums and their finish)
KERNELS = {"tile_dedup": 0, "partition": 1, "compact_insert": 2, "init_rows": 3, "pool": 4,
           "bwd_short": 5, "bwd_long": 6, "opt": 7, "occ": 8, "occ_list": 9}


class RecisError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class TableDesc(C.Structure):
    _fields_ = [("dim", C.c_int32), ("row_dtype", C.c_int32), ("optimizer", C.c_int32),
                ("init_lo", C.c_float), ("init_hi", C.c_float), ("seed", C.c_uint64),
                ("capacity_slots", C.c_int64), ("max_load", C.c_float), ("block_rows", C.c_int64),
                ("auto_grow", C.c_int32), ("evictable", C.c_int32)]


ALLOC_FN = C.CFUNCTYPE(C.c_void_p, C.c_size_t, C.c_void_p)
FREE_FN = C.CFUNCTYPE(None, C.c_void_p, C.c_void_p)


class Allocator(C.Structure):
    _fields_ = [("alloc", ALLOC_FN), ("free", FREE_FN), ("ctx", C.c_void_p)]


class TorchAllocator:
    """rs_allocator backed by PyTorch's caching allocator (current stream).

    fail_after: return NULL from the (fail_after + 1)-th allocation on (tests
    of the RS_ENOMEM path)."""

    def __init__(self, device=None, fail_after: Optional[int] = None):
        self.device = torch.cuda.current_device() if device is None else device
        self.fail_after = fail_after
        self.calls = 0
        self.live = {}
        self._a = ALLOC_FN(self._alloc)
        self._f = FREE_FN(self._free)
        self.struct = Allocator(self._a, self._f, None)

    def _alloc(self, nbytes, ctx):
        self.calls += 1
        if self.fail_after is not None and self.calls > self.fail_after:
            return None
        try:
            p = torch.cuda.caching_allocator_alloc(int(nbytes), self.device)
        except Exception:  # an exception must not cross the C callback
            return None
        self.live[p] = int(nbytes)
        return p

    def _free(self, ptr, ctx):
        if ptr in self.live:
            del self.live[ptr]
            torch.cuda.caching_allocator_delete(ptr)


class OptParams(C.Structure):
    _fields_ = [("lr", C.c_double), ("eps", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double),
                ("weight_decay", C.c_double)]


class RsCtx(C.Structure):
    _fields_ = [("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
                ("unique", C.c_void_p), ("inverse", C.c_void_p), ("rows", C.c_void_p),
                ("scalars", C.c_void_p), ("offsets", C.c_void_p), ("table", C.c_void_p),
                ("n", C.c_int64), ("bags", C.c_int64), ("pad_len", C.c_int64),
                ("mode", C.c_int32), ("dim", C.c_int32), ("priv", C.c_int64 * 16)]


class AttnDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("heads_q", C.c_int32), ("heads_kv", C.c_int32), ("head_dim", C.c_int32),
                ("causal", C.c_int32), ("reserved", C.c_int32), ("seqs", C.c_int64), ("q_rows", C.c_int64),
                ("kv_rows", C.c_int64), ("q_pad", C.c_int64), ("kv_pad", C.c_int64), ("max_q", C.c_int64),
                ("q_stride", C.c_int64), ("q_head_stride", C.c_int64), ("k_stride", C.c_int64),
                ("k_head_stride", C.c_int64), ("v_stride", C.c_int64), ("v_head_stride", C.c_int64),
                ("scale", C.c_double), ("softcap", C.c_double)]


class CacheDesc(C.Structure):
    _fields_ = [("codes", C.c_int32), ("dtype", C.c_int32), ("heads_kv", C.c_int32), ("head_dim", C.c_int32),
                ("page_len", C.c_int32), ("reserved", C.c_int32), ("pages", C.c_int64), ("slots", C.c_int64),
                ("data", C.c_void_p), ("scales", C.c_void_p), ("open", C.c_void_p), ("bounds", C.c_void_p),
                ("units", C.c_void_p)]


class CacheBatch(C.Structure):
    _fields_ = [("seqs", C.c_int64), ("rows", C.c_int64), ("pad", C.c_int64), ("table_width", C.c_int64),
                ("offsets", C.c_void_p), ("lens", C.c_void_p), ("table", C.c_void_p), ("slots", C.c_void_p)]


class CacheRows(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("q", C.c_void_p), ("q_out", C.c_void_p),
                ("k_stride", C.c_int64), ("k_head_stride", C.c_int64), ("v_stride", C.c_int64),
                ("v_head_stride", C.c_int64), ("q_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("heads_q", C.c_int32), ("rotary", C.c_int32), ("interleaved", C.c_int32), ("reserved", C.c_int32),
                ("turns", C.c_void_p), ("new_lens", C.c_void_p)]


class CacheQuery(C.Structure):
    _fields_ = [("heads_q", C.c_int32), ("causal", C.c_int32), ("count", C.c_int32), ("reserved", C.c_int32),
                ("max_q", C.c_int64), ("max_len", C.c_int64), ("q_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("scale", C.c_double), ("softcap", C.c_double)]


_lib = None


def lib() -> C.CDLL:
    """Load the HIP library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RecisError(EHIP, f"{LIB_PATH} is not built; run paper_2509_20883_amd/build.py")
    L = C.CDLL(LIB_PATH)
    p, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    sig = {
        "rs_version": (C.c_int, []),
        "rs_last_error": (C.c_char_p, []),
        "ht_create": (C.c_int, [C.POINTER(TableDesc), C.POINTER(Allocator), p, C.POINTER(p)]),
        "ht_destroy": (C.c_int, [p]),
        "ht_find_or_insert": (C.c_int, [p, p, i64, p, p, p]),
        "ht_find": (C.c_int, [p, p, i64, p, p]),
        "ht_size": (C.c_int, [p, C.POINTER(i64), p]),
        "rs_table_check": (C.c_int, [p, p]),
        "ht_capacity": (C.c_int, [p, C.POINTER(i64)]),
        "ht_export": (C.c_int, [p, p, p, i64, p, p]),
        "ht_read_rows": (C.c_int, [p, p, i64, p, p, p]),
        "ht_reserve": (C.c_int, [p, i64, p]),
        "lookup_workspace_bytes": (C.c_size_t, [i64, i64, i64, p]),
        "lookup_pool_fwd": (C.c_int, [p, p, p, i64, i64, i32, i64, p, p, C.POINTER(RsCtx), i32, p]),
        "lookup_prepare": (C.c_int, [p, p, p, i64, i64, i32, i64, C.POINTER(RsCtx), i32, p]),
        "lookup_pool_prepared": (C.c_int, [p, C.POINTER(RsCtx), p, p, p]),
        "lookup_pool_bwd": (C.c_int, [p, C.POINTER(RsCtx), p, p, p]),
        "sparse_opt_step": (C.c_int, [p, C.POINTER(RsCtx), p, C.POINTER(OptParams), p]),
        "lookup_pool_bwd_opt": (C.c_int, [p, C.POINTER(RsCtx), p, C.POINTER(OptParams), p]),
        "rs_set_kernel_events": (C.c_int, [p, i32, p, p]),
        "ht_evict": (C.c_int, [p, C.c_uint32, C.POINTER(i64), p]),
        "ht_compact": (C.c_int, [p, C.POINTER(i64), C.POINTER(i64), p]),
        "ids_partition_workspace_bytes": (C.c_size_t, [i64, i32]),
        "ids_partition": (C.c_int, [p, i64, i32, C.c_uint64, p, p, p, p, p, C.c_size_t, p]),
        "fused_bucketize": (C.c_int, [p, i64, p, i32, p, p, p, i32, p]),
        "fused_mod": (C.c_int, [p, i64, p, i32, p, p, i32, p]),
        "rs_bandwidth_probe": (C.c_int, [i32, p, i64, p, i64, p, i64, i32, p]),
        "ids_partition_static": (C.c_int, [p, i64, i32, C.c_uint64, p, p, p, p, p]),
        "layer_norm_fwd": (C.c_int, [p, i64, i64, i64, i32, p, p, i32, C.c_double, p, p, i64, p, p, p]),
        "layer_norm_bwd_workspace_bytes": (C.c_size_t, [i64, i64]),
        "layer_norm_bwd": (C.c_int, [p, i64, p, i64, i64, i64, i32, p, i32, p, p, p, p, i64, p, p, p, C.c_size_t, p]),
        "seq_attention_workspace_bytes": (C.c_size_t, [C.POINTER(AttnDesc), i32]),
        "seq_attention_fwd": (C.c_int, [C.POINTER(AttnDesc)] + [p] * 11 + [C.c_size_t, i32, p]),
        "seq_attention_bwd": (C.c_int, [C.POINTER(AttnDesc)] + [p] * 16 + [C.c_size_t, i32, p]),
        "rs_rotation_turns": (C.c_int, [p, C.c_double, i32, p]),
        "seq_cache_append": (C.c_int, [C.POINTER(CacheDesc), C.POINTER(CacheBatch), C.POINTER(CacheRows), i32, p]),
        "seq_cache_read": (C.c_int, [C.POINTER(CacheDesc), C.POINTER(CacheBatch), p, p, p, i32, i32, p]),
        "seq_cache_attention_workspace_bytes": (C.c_size_t, [C.POINTER(CacheDesc), C.POINTER(CacheBatch),
                                                             C.POINTER(CacheQuery)]),
        "seq_cache_attention": (C.c_int, [C.POINTER(CacheDesc), C.POINTER(CacheBatch), C.POINTER(CacheQuery)] + [p] * 5
                                + [C.c_size_t, i32, p]),
        "seq_cache_select_workspace_bytes": (C.c_size_t, [C.POINTER(CacheDesc), C.POINTER(CacheBatch),
                                                          C.POINTER(CacheQuery)]),
        "seq_cache_select": (C.c_int, [C.POINTER(CacheDesc), C.POINTER(CacheBatch), C.POINTER(CacheQuery)] + [p] * 3
                             + [C.c_size_t, i32, p]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def _check(st: int):
    if st != OK:
        raise RecisError(st, lib().rs_last_error().decode())


# Per-call costs on the host count for the smallest calls (a kernel there takes
# 4-9 us): torch.cuda.current_stream() builds a Stream object (2.9 us); the raw
# handle of the same stream is 0.3 us.  Addresses are passed as plain ints.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    """hipStream_t of the current stream of the current device."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


# The current device without torch.cuda's own checks; a tensor on the GPU has passed them.
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream_of(device: int) -> int:
    """hipStream_t of the current stream of a device."""
    return torch.cuda.current_stream(device).cuda_stream if _raw_stream is None else _raw_stream(device)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dev(t: torch.Tensor, dtype: torch.dtype) -> torch.Tensor:
    if not t.is_cuda:
        raise RecisError(EINVAL, "tensors must be on the GPU")
    if t.dtype != dtype:
        raise RecisError(EINVAL, f"expected {dtype}, got {t.dtype}")
    return t.contiguous()


class Ctx:
    """Forward context: the caller-owned workspace plus the rs_ctx struct."""

    def __init__(self):
        self.ws: Optional[torch.Tensor] = None
        self.c = RsCtx()
        self.keep = ()

    def ensure(self, nbytes: int, device):
        if self.ws is None or self.ws.numel() < nbytes:
            self.ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        self.c.workspace = self.ws.data_ptr()
        self.c.workspace_bytes = self.ws.numel()

    def _view(self, ptr: int, count: int, dtype: torch.dtype) -> torch.Tensor:
        off = ptr - self.ws.data_ptr()
        return self.ws[off:off + count * dtype.itemsize].view(dtype)

    def scalars(self) -> torch.Tensor:
        """Device int64[4]: U, inserted, occurrences kept, live rows before."""
        return self._view(self.c.scalars, 4, torch.int64)

    def unique(self, U: int) -> torch.Tensor:
        return self._view(self.c.unique, U, torch.int64)

    def inverse(self) -> torch.Tensor:
        return self._view(self.c.inverse, self.c.n, torch.int32)

    def rows(self, U: int) -> torch.Tensor:
        return self._view(self.c.rows, U, torch.int64)


def ids_partition_workspace_bytes(n: int, nshards: int) -> int:
    return int(lib().ids_partition_workspace_bytes(n, nshards))


class IdsPartition:
    """Ids partition (dedup + split by owner shard) with a reusable workspace.

    ``__call__(values, nshards, owner_seed)`` enqueues the call on the current
    stream and returns device tensors (keys int64 [n], shard_offsets int64
    [nshards+1], inverse int32 [n], info int64 [2] = {U, error bits}); the
    first U keys are valid, shard s holds keys[offsets[s]:offsets[s+1]].
    """

    def __init__(self):
        self.ws: Optional[torch.Tensor] = None

    def __call__(self, values: torch.Tensor, nshards: int, owner_seed: int = 0, keys=None, shard_offsets=None,
                 inverse=None, info=None):
        v = _dev(values, torch.int64)
        n = v.numel()
        need = ids_partition_workspace_bytes(n, nshards)
        if need == 0:
            raise RecisError(EINVAL, "n must be in [0, 2^28] and nshards in [1, 1024]")
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device=v.device)
        if keys is None:
            keys = torch.empty(max(n, 1), dtype=torch.int64, device=v.device)
        if shard_offsets is None:
            shard_offsets = torch.empty(nshards + 1, dtype=torch.int64, device=v.device)
        if inverse is None:
            inverse = torch.empty(max(n, 1), dtype=torch.int32, device=v.device)
        if info is None:
            info = torch.empty(2, dtype=torch.int64, device=v.device)
        _check(lib().ids_partition(_ptr(v), n, nshards, owner_seed & 0xFFFFFFFFFFFFFFFF, _ptr(keys),
                                   _ptr(shard_offsets), _ptr(inverse), _ptr(info), _ptr(self.ws), self.ws.numel(),
                                   _stream()))
        return keys[:max(n, 0)], shard_offsets, inverse[:n], info


IDS_STATIC_MAX_IDS = 1 << 20


def ids_partition_static(values: torch.Tensor, nshards: int, owner_seed: int, keys: torch.Tensor,
                         shard_offsets: torch.Tensor, inverse: torch.Tensor, info: torch.Tensor) -> None:
    """ids_partition with the library's own fixed workspace: allocates nothing.

    Every tensor is the caller's (contiguous, on the GPU): keys int64 [>= n],
    shard_offsets int64 [nshards + 1], inverse int32 [>= n], info int64 [2];
    n = values.numel() <= IDS_STATIC_MAX_IDS.  Calls on one GPU share the
    workspace: overlapping calls race.
    """
    for t, dt in ((values, torch.int64), (keys, torch.int64), (shard_offsets, torch.int64), (inverse, torch.int32),
                  (info, torch.int64)):
        if not t.is_cuda or t.dtype != dt or not t.is_contiguous():
            raise RecisError(EINVAL, f"expected a contiguous GPU {dt} tensor")
    n = values.numel()
    if keys.numel() < n or inverse.numel() < n or shard_offsets.numel() < nshards + 1 or info.numel() < 2:
        raise RecisError(EINVAL, "output tensors too small")
    _check(lib().ids_partition_static(_ptr(values), n, nshards, owner_seed & 0xFFFFFFFFFFFFFFFF, _ptr(keys),
                                      _ptr(shard_offsets), _ptr(inverse), _ptr(info), _stream()))


def ids_partition(values: torch.Tensor, nshards: int, owner_seed: int = 0):
    """One-off ids partition (allocates its workspace); see IdsPartition."""
    return IdsPartition()(values, nshards, owner_seed)


def fused_bucketize(values: torch.Tensor, col_offsets: torch.Tensor, boundaries: torch.Tensor,
                    bnd_offsets: torch.Tensor, out: Optional[torch.Tensor] = None,
                    validate: bool = False) -> torch.Tensor:
    """Bucket (int64) of every fp32 value of every column; one launch."""
    v = _dev(values, torch.float32)
    co = _dev(col_offsets, torch.int64)
    b = _dev(boundaries, torch.float32)
    bo = _dev(bnd_offsets, torch.int64)
    if out is None:
        out = torch.empty(v.numel(), dtype=torch.int64, device=v.device)
    _check(lib().fused_bucketize(_ptr(v), v.numel(), _ptr(co), co.numel() - 1, _ptr(b), _ptr(bo), _ptr(out),
                                 int(validate), _stream()))
    return out


def fused_mod(values: torch.Tensor, col_offsets: torch.Tensor, moduli: torch.Tensor,
              out: Optional[torch.Tensor] = None, validate: bool = False) -> torch.Tensor:
    """Floor modulus (int64) of every id by its column's modulus; one launch."""
    v = _dev(values, torch.int64)
    co = _dev(col_offsets, torch.int64)
    m = _dev(moduli, torch.int64)
    if out is None:
        out = torch.empty(v.numel(), dtype=torch.int64, device=v.device)
    _check(lib().fused_mod(_ptr(v), v.numel(), _ptr(co), co.numel() - 1, _ptr(m), _ptr(out), int(validate),
                           _stream()))
    return out


_SEQ_TYPES = {torch.float32: F32, torch.bfloat16: BF16}


def _seq_type(t: torch.Tensor, what: str) -> int:
    """rs_dtype of a GPU tensor of a sequence operator."""
    if not t.is_cuda:
        raise RecisError(EINVAL, "tensors must be on the GPU")
    dt = _SEQ_TYPES.get(t.dtype)
    if dt is None:
        raise RecisError(EINVAL, f"{what} must be float32 or bfloat16, got {t.dtype}")
    return dt


def _rows(t: torch.Tensor) -> Tuple[torch.Tensor, int]:
    """The tensor as equally spaced rows of its last axis, and their stride in
    elements (a copy is made where its strides do not allow that)."""
    if t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= t.shape[1]:
        return t, t.stride(0)
    if not t.is_contiguous():
        t = t.contiguous()
    return t, t.shape[-1]


class _Workspace:
    """A buffer that grows with the calls of an object.  What a captured graph
    works on stays with the object when a larger call replaces it; any other
    goes back to the caching allocator, for use once the current stream is past
    the calls so far."""

    def __init__(self):
        self.ws: Optional[torch.Tensor] = None
        self._captured: list = []

    def _take(self, need: int, like: torch.Tensor) -> torch.Tensor:
        ws = self.ws
        if ws is None or ws.numel() < need or ws.device != like.device:
            if ws is not None:
                ws.record_stream(torch.cuda.current_stream(ws.device))
            self.ws = ws = torch.empty(max(need, 256), dtype=torch.uint8, device=like.device)
        if torch.cuda.is_current_stream_capturing() and not any(t is ws for t in self._captured):
            self._captured.append(ws)
        return ws


def _like(t: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor of t's shape and type (empty_like takes half the host time of empty)."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _packed(t: torch.Tensor) -> torch.Tensor:
    """Contiguous and 16-byte aligned (a copy where it is not)."""
    t = t.contiguous()
    return t.clone() if t.data_ptr() % 16 else t


class LayerNorm(_Workspace):
    """Layer norm over the last axis, with a reusable backward workspace.

    ``forward(x, weight, bias, mask)`` returns (y, mean, rstd); ``backward``
    takes the output gradient, x and those statistics and returns (dx,
    dweight, dbias).  x: float32 or bfloat16 [..., dim]; weight, bias [dim] in
    either type or None (1 and 0); mask: uint8 or bool [...], rows of mask 0
    are never read and give y = dx = 0.  Calls of one object share its
    workspace: issue them on one stream, or order the streams, and keep the
    object as long as a graph that captured its calls.
    """

    def __init__(self, eps: float = 1e-5):
        super().__init__()
        self.eps = float(eps)

    @staticmethod
    def _params(x, weight, bias):
        pt = None
        for t, what in ((weight, "weight"), (bias, "bias")):
            if t is None:
                continue
            dt = _seq_type(t, what)
            if pt is not None and dt != pt:
                raise RecisError(EINVAL, "weight and bias must have one type")
            if t.dim() != 1 or t.shape[0] != x.shape[-1] or not t.is_contiguous():
                raise RecisError(EINVAL, f"{what} must be a contiguous [{x.shape[-1]}] tensor")
            pt = dt
        return F32 if pt is None else pt

    @staticmethod
    def _mask(x, mask):
        if mask is None:
            return None
        if not mask.is_cuda or mask.dtype not in (torch.uint8, torch.bool):
            raise RecisError(EINVAL, "mask must be a uint8 or bool GPU tensor")
        if mask.numel() * x.shape[-1] != x.numel():
            raise RecisError(EINVAL, "mask must have one element per row of x")
        return mask.contiguous()

    def forward(self, x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                mask: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None):
        dt = _seq_type(x, "x")
        if x.dim() < 1 or x.shape[-1] < 1:
            raise RecisError(EINVAL, "x needs a last axis of at least one element")
        pt = self._params(x, weight, bias)
        m = self._mask(x, mask)
        dim = x.shape[-1]
        rows = x.numel() // dim
        xr, xs = _rows(x)
        if out is None:
            out = _like(x)
        elif out.shape != x.shape or out.dtype != x.dtype or not out.is_cuda or not out.is_contiguous():
            raise RecisError(EINVAL, "out must be a contiguous GPU tensor of x's shape and type")
        mean = x.new_empty(x.shape[:-1], dtype=torch.float32)
        rstd = torch.empty_like(mean)
        _check(lib().layer_norm_fwd(xr.data_ptr(), rows, dim, xs, dt, _ptr(weight), _ptr(bias), pt, self.eps, _ptr(m),
                                    out.data_ptr(), dim, mean.data_ptr(), rstd.data_ptr(), _stream()))
        return out, mean, rstd

    def backward(self, grad_out: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                 weight: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None):
        dt = _seq_type(x, "x")
        if x.dim() < 1 or x.shape[-1] < 1:
            raise RecisError(EINVAL, "x needs a last axis of at least one element")
        if grad_out.shape != x.shape or grad_out.dtype != x.dtype or not grad_out.is_cuda:
            raise RecisError(EINVAL, "grad_out must be a GPU tensor of x's shape and type")
        pt = self._params(x, weight, None)
        m = self._mask(x, mask)
        dim = x.shape[-1]
        rows = x.numel() // dim
        mean, rstd = _dev(mean, torch.float32), _dev(rstd, torch.float32)
        if mean.numel() != rows or rstd.numel() != rows:
            raise RecisError(EINVAL, "mean and rstd must have one element per row of x")
        xr, xs = _rows(x)
        gr, gs = _rows(grad_out)
        dx = _like(x)
        dw = x.new_empty((dim,), dtype=torch.bfloat16 if pt == BF16 else torch.float32)
        db = torch.empty_like(dw)
        ws = self._take(lib().layer_norm_bwd_workspace_bytes(rows, dim), x)
        _check(lib().layer_norm_bwd(gr.data_ptr(), gs, xr.data_ptr(), rows, dim, xs, dt, _ptr(weight), pt, _ptr(m),
                                    mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), dim, dw.data_ptr(),
                                    db.data_ptr(), ws.data_ptr(), ws.numel(), _stream()))
        return dx, dw, db


class AttnStats(NamedTuple):
    """What SeqAttention.forward keeps for the backward: lse (float32 [...,
    heads_q], the log of each query's softmax sum, -inf where it sees no key)
    and rest (bf16, out's shape: what rounding took from out; None in fp32)."""
    lse: torch.Tensor
    rest: Optional[torch.Tensor]


class SeqAttention(_Workspace):
    """Attention over ragged sequences, with a reusable workspace.

    q [rows, heads_q, d] packed with q_offsets (int64 [seqs + 1]), or the
    padded [seqs, pad, heads_q, d]; k, v [rows, heads_kv, d] or [seqs, pad,
    heads_kv, d] with kv_offsets (default: q_offsets).  Packed offsets run from
    0 to the number of rows: rows that they leave out are written neither in
    the output nor in the gradients.  float32 or bfloat16,
    d a multiple of 8 up to 128.  The last axis must be contiguous; other
    strides are taken as they are where they are multiples of 16 bytes, else
    the tensor is copied.  ``forward`` returns (out, stats); ``backward`` takes
    the output gradient and both and returns (dq, dk, dv, dslopes).

    causal: query i of Lq sees key j of Lk when j <= i + Lk - Lq, or j <
    prefix[s] (int64 [seqs]); softcap: scores capped by softcap * tanh(x /
    softcap); slopes (float32 [heads_q]): the score falls by slope * |i + Lk -
    Lq - j|, and the backward returns their gradient.  max_q: a bound of the
    query lengths where the caller knows one (0: none).  It only shapes the
    launches; rows past a bound that does not hold are right, but slow.  Give
    it for single tokens and short chunks: packed queries without it are
    planned as if one sequence held them all, which takes up to 256 MiB of
    workspace, and past that the keys are not split (one token for each of 128
    users with up to 8192 keys of 128 bf16: 132 us with a bound, 201 without).
    Calls of one object share its workspace: issue them on one stream, or
    order the streams, and keep the object as long as a graph that captured its
    calls.
    """

    def __init__(self, scale: Optional[float] = None, softcap: float = 0.0, causal: bool = True):
        super().__init__()
        self.scale, self.softcap, self.causal = scale, float(softcap), bool(causal)

    @staticmethod
    def _layout(t: torch.Tensor, what: str):
        """The tensor (copied if its strides do not serve), rows, pad, row and head strides."""
        if t.dim() not in (3, 4):
            raise RecisError(EINVAL, f"{what} must be [rows, heads, d] or [seqs, pad, heads, d]")
        unit = 16 // t.element_size()
        st = t.stride()
        if (st[-1] != 1 or st[-2] % unit or st[-3] % unit or max(st[-2], st[-3]) >= 1 << 23 or
                64 * st[-3] + t.shape[-2] * st[-2] >= 1 << 29 or (t.dim() == 4 and st[0] != t.shape[1] * st[1]) or
                t.data_ptr() % 16):
            t = _packed(t)
            st = t.stride()
        if t.dim() == 4:
            return t, t.shape[0] * t.shape[1], t.shape[1], st[1], st[2]
        return t, t.shape[0], 0, st[0], st[1]

    def _desc(self, q, k, v, q_offsets, kv_offsets, prefix, slopes, max_q):
        dt = _seq_type(q, "q")
        if not (k.is_cuda and v.is_cuda) or k.dtype != q.dtype or v.dtype != q.dtype:
            raise RecisError(EINVAL, "q, k and v must be GPU tensors of one type")
        q, q_rows, q_pad, qs, qh = self._layout(q, "q")
        k, kv_rows, kv_pad, ks, kh = self._layout(k, "k")
        v, v_rows, v_pad, vs, vh = self._layout(v, "v")
        if k.shape != v.shape or q.shape[-1] != k.shape[-1]:
            raise RecisError(EINVAL, "k and v must have one shape, and q their last axis")
        qo = _dev(q_offsets, torch.int64)
        ko = qo if kv_offsets is None else _dev(kv_offsets, torch.int64)
        seqs = qo.numel() - 1
        if seqs < 0 or ko.numel() - 1 != seqs:
            raise RecisError(EINVAL, "q_offsets and kv_offsets must both be [seqs + 1]")
        if (q_pad and q.shape[0] != seqs) or (kv_pad and k.shape[0] != seqs):
            raise RecisError(EINVAL, "a padded tensor must have one block per sequence")
        if prefix is not None:
            prefix = _dev(prefix, torch.int64)
            if prefix.numel() != seqs:
                raise RecisError(EINVAL, "prefix must have one length per sequence")
        if slopes is not None:
            slopes = _dev(slopes, torch.float32)
            if slopes.numel() != q.shape[-2]:
                raise RecisError(EINVAL, "slopes must have one value per query head")
        d = q.shape[-1]
        scale = self.scale if self.scale is not None else (d ** -0.5 if d else 1.0)
        desc = AttnDesc(dt, q.shape[-2], k.shape[-2], d, int(self.causal), 0, seqs, q_rows, kv_rows, q_pad, kv_pad,
                        max_q, qs, qh, ks, kh, vs, vh, scale, self.softcap)
        return desc, q, k, v, qo, ko, prefix, slopes

    def forward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_offsets: torch.Tensor,
                kv_offsets: Optional[torch.Tensor] = None, prefix: Optional[torch.Tensor] = None,
                slopes: Optional[torch.Tensor] = None, max_q: int = 0, out: Optional[torch.Tensor] = None,
                validate: bool = False):
        shape = q.shape
        desc, q, k, v, qo, ko, prefix, slopes = self._desc(q, k, v, q_offsets, kv_offsets, prefix, slopes, max_q)
        if out is None:
            out = _like(q)
        elif out.shape != shape or out.dtype != q.dtype or not out.is_cuda or not out.is_contiguous():
            raise RecisError(EINVAL, "out must be a contiguous GPU tensor of q's shape and type")
        stats = AttnStats(q.new_empty(shape[:-1], dtype=torch.float32),
                          torch.empty_like(out) if desc.dtype == BF16 else None)
        need = lib().seq_attention_workspace_bytes(C.byref(desc), 0)
        ws = self._take(need, q) if need else None
        _check(lib().seq_attention_fwd(C.byref(desc), q.data_ptr(), k.data_ptr(), v.data_ptr(), qo.data_ptr(),
                                       ko.data_ptr(), _ptr(prefix), _ptr(slopes), out.data_ptr(), _ptr(stats.rest),
                                       stats.lse.data_ptr(), _ptr(ws), ws.numel() if need else 0, int(validate),
                                       _stream()))
        return out, stats

    def backward(self, grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                 stats: AttnStats, q_offsets: torch.Tensor, kv_offsets: Optional[torch.Tensor] = None,
                 prefix: Optional[torch.Tensor] = None, slopes: Optional[torch.Tensor] = None, max_q: int = 0,
                 validate: bool = False):
        lse, rest = stats
        for t, what in ((grad_out, "grad_out"), (out, "out"), (out if rest is None else rest, "stats.rest")):
            if t.shape != q.shape or t.dtype != q.dtype or not t.is_cuda:
                raise RecisError(EINVAL, f"{what} must be a GPU tensor of q's shape and type")
        if lse.shape != q.shape[:-1] or lse.dtype != torch.float32 or not lse.is_cuda:
            raise RecisError(EINVAL, "stats.lse must be the forward's float32 [..., heads_q]")
        dq, dk, dv = _like(q), _like(k), _like(v)
        desc, q, k, v, qo, ko, prefix, slopes = self._desc(q, k, v, q_offsets, kv_offsets, prefix, slopes, max_q)
        grad_out, out, lse = _packed(grad_out), _packed(out), lse.contiguous()
        rest = None if rest is None else _packed(rest)
        dslopes = None if slopes is None else torch.empty_like(slopes)
        ws = self._take(lib().seq_attention_workspace_bytes(C.byref(desc), 1), q)
        _check(lib().seq_attention_bwd(C.byref(desc), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                       _ptr(rest), lse.data_ptr(), grad_out.data_ptr(), qo.data_ptr(), ko.data_ptr(),
                                       _ptr(prefix), _ptr(slopes), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                       _ptr(dslopes), ws.data_ptr(), ws.numel(), int(validate), _stream()))
        return dq, dk, dv, dslopes


class SeqCache(_Workspace):
    """A paged cache of the keys and values of sequences, full pages in 8 bits.

    pages of `page` tokens (32, 64, 128 or 256) and `slots` sequences' open
    pages are allocated on the current GPU; which sequence has which pages and
    slot is the caller's: table int32 [seqs, width] names the page of each of a
    sequence's page numbers, slots int32 [seqs] its slot (default: its index),
    lens int64 [seqs] the tokens it holds.  codes "i8" (scale max / 127 of a
    page and head, the more exact for values without outliers) or "e4m3"
    (power-of-two scale).  bounds: keep what ``select`` needs.

    rotary columns of keys and queries are turned by their position when they
    are appended, with frequencies base^(-2 i / rotary) or `freqs` (radians a
    position, rotary / 2 of them), pairs (i, i + rotary / 2) or, interleaved,
    (2 i, 2 i + 1).

    ``append(k, v, offsets, lens, table, q=...)`` writes new tokens (packed
    [rows, heads_kv, d] with CSR offsets, or padded [seqs, pad, heads_kv, d])
    and returns (lens afterwards, q turned).  ``attend`` is SeqAttention over
    the tokens held (inference only), with `pages` over the listed ones;
    ``select`` lists the pages of the highest score for each row and key head
    (a row of a causal chunk sees its own page, once the chunk has filled it,
    only where the list names it); ``read`` returns tokens as rows.  scale, softcap, causal and slopes are
    SeqAttention's.  max_q and max_len bound a sequence's queries and tokens
    where the caller knows: they only shape the launches, but packed rows of many
    sequences want max_q (a token of 256 users: 74 us with it, 126 without).

    Calls of one object share its workspace: issue them on one stream, or order
    the streams, and keep the object as long as a graph that captured its calls.
    """

    def __init__(self, pages: int, slots: int, heads_kv: int, head_dim: int, page: int = 64, codes: str = "i8",
                 dtype: torch.dtype = torch.bfloat16, bounds: bool = False, rotary: int = 0, base: float = 10000.0,
                 freqs=None, interleaved: bool = False, scale: Optional[float] = None, softcap: float = 0.0,
                 causal: bool = True):
        super().__init__()
        if codes not in ("i8", "e4m3"):
            raise RecisError(EINVAL, "codes must be 'i8' or 'e4m3'")
        if dtype not in _SEQ_TYPES:
            raise RecisError(EINVAL, f"dtype must be float32 or bfloat16, got {dtype}")
        if page not in (32, 64, 128, 256):
            raise RecisError(EINVAL, "page must be 32, 64, 128 or 256")
        if not 1 <= heads_kv <= 1024 or not 8 <= head_dim <= 128 or head_dim % 8:
            raise RecisError(EINVAL, "heads_kv must be in [1, 1024] and head_dim a multiple of 8 in [8, 128]")
        if pages < 0 or slots < 0:
            raise RecisError(EINVAL, "pages and slots must be >= 0")
        if rotary < 0 or rotary > head_dim or rotary % 2:
            raise RecisError(EINVAL, "rotary must be even and at most head_dim")
        host = (C.c_uint64 * max(rotary // 2, 1))()
        own = None
        if freqs is not None:
            freqs = [float(f) for f in freqs]
            if len(freqs) != rotary // 2:
                raise RecisError(EINVAL, "freqs must have rotary / 2 values")
            own = (C.c_double * max(len(freqs), 1))(*freqs)
        _check(lib().rs_rotation_turns(own, base, rotary, host))
        dev = torch.device("cuda", torch.cuda.current_device())
        self.heads_kv, self.head_dim, self.page, self.dtype = heads_kv, head_dim, page, dtype
        self.rotary, self.interleaved = rotary, bool(interleaved)
        self.scale, self.softcap, self.causal = scale, float(softcap), bool(causal)
        width = 32 if head_dim <= 32 else 64 if head_dim <= 64 else 128
        self.codes = torch.empty(pages, heads_kv, 2, page * width, dtype=torch.uint8, device=dev)
        self.scales = torch.empty(pages, heads_kv, 2, dtype=torch.float32, device=dev)
        self.open = torch.empty(slots, 2, heads_kv, 2, page, head_dim, dtype=dtype, device=dev)
        self.bounds = torch.empty(pages, heads_kv, 2, width, dtype=torch.int8, device=dev) if bounds else None
        self.units = torch.empty(pages, heads_kv, dtype=torch.float32, device=dev) if bounds else None
        # 64-bit fractions as signed words of the same bits
        turns = [t - (1 << 64) if t >> 63 else t for t in host[:rotary // 2]]
        self.turns = torch.tensor(turns, dtype=torch.int64, device=dev) if rotary else None
        self._desc = CacheDesc(1 if codes == "e4m3" else 0, _SEQ_TYPES[dtype], heads_kv, head_dim, page, 0, pages, slots,
                               self.codes.data_ptr(), self.scales.data_ptr(), self.open.data_ptr(), _ptr(self.bounds),
                               _ptr(self.units))
        self._ref = C.byref(self._desc)
        self._index, self._slots, self._turns = dev.index, slots, _ptr(self.turns)
        self._odd = 16 // self.open.element_size() - 1

    # The host time of a call counts for the smallest (kernels there take 4 to 10 us): device numbers are compared, not
    # device objects, and structs are filled by position.
    def _layout(self, t: torch.Tensor, what: str, heads: int = 0):
        """The tensor (copied if its strides do not serve), its address, rows, pad, row and head strides."""
        if t.get_device() != self._index:
            raise RecisError(EINVAL, "tensors must be on the GPU, the cache's")
        if t.dtype != self.dtype:
            raise RecisError(EINVAL, f"{what} must be {self.dtype}, got {t.dtype}")
        shape, st = t.shape, t.stride()
        n = len(shape)
        if n not in (3, 4) or shape[-1] != self.head_dim or (heads and shape[-2] != heads):
            raise RecisError(EINVAL, f"{what} must be [rows, heads, {self.head_dim}] or [seqs, pad, heads, {self.head_dim}]"
                             + (f" with {heads} heads" if heads else ""))
        at = t.data_ptr()
        if (st[-1] != 1 or (st[-2] | st[-3]) & self._odd or st[-2] >> 31 or st[-3] >> 31 or at & 15 or
                (n == 4 and st[0] != shape[1] * st[1])):
            t = _packed(t)
            st, at = t.stride(), t.data_ptr()
        if n == 4:
            return t, at, shape[0] * shape[1], shape[1], st[1], st[2]
        return t, at, shape[0], 0, st[0], st[1]

    def _same(self, t: torch.Tensor, dtype: torch.dtype, what: str) -> torch.Tensor:
        if t.get_device() != self._index or t.dtype != dtype:
            raise RecisError(EINVAL, f"{what} must be {dtype} on the cache's GPU")
        return t if t.is_contiguous() else t.contiguous()

    def _batch(self, rows, pad, padded, offsets, lens, table, slots, own_slots=True):
        if _device() != self._index:
            raise RecisError(EINVAL, "the cache's GPU must be the current one")
        offsets = self._same(offsets, torch.int64, "offsets")
        lens = self._same(lens, torch.int64, "lens")
        table = self._same(table, torch.int32, "table")
        seqs, shape = offsets.numel() - 1, table.shape
        if seqs < 0 or lens.numel() != seqs or len(shape) != 2 or shape[0] != seqs:
            raise RecisError(EINVAL, "offsets must be [seqs + 1], lens [seqs] and table [seqs, width]")
        if padded is not None and padded != seqs:
            raise RecisError(EINVAL, "a padded tensor must have one block per sequence")
        if slots is not None:
            slots = self._same(slots, torch.int32, "slots")
            if slots.numel() != seqs:
                raise RecisError(EINVAL, "slots must have one slot per sequence")
        elif own_slots and self._slots < seqs:
            raise RecisError(EINVAL, "more sequences than slots")
        return CacheBatch(seqs, rows, pad, shape[1], offsets.data_ptr(), lens.data_ptr(), table.data_ptr(),
                          None if slots is None else slots.data_ptr()), (offsets, lens, table, slots)

    def append(self, k: Optional[torch.Tensor], v: Optional[torch.Tensor], offsets: torch.Tensor, lens: torch.Tensor,
               table: torch.Tensor, q: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
               validate: bool = False):
        """Writes k and v as the sequences' tokens from lens on; returns (lens afterwards, q turned by the same
        positions or None).  k = v = None turns q alone (candidates that are not kept): lens then come back as they
        would be with the rows kept, nothing is written, and neither table nor slots are looked at."""
        if (k is None) != (v is None) or (k is None and q is None):
            raise RecisError(EINVAL, "append takes k and v, q, or all three")
        q_out, ka, va, qa, oa, heads = None, None, None, None, None, 0
        ks = kh = vs = vh = qs = qh = 0
        if k is not None:
            k, ka, rows, pad, ks, kh = self._layout(k, "k", self.heads_kv)
            v, va, _, _, vs, vh = self._layout(v, "v", self.heads_kv)
            shape = k.shape
            if shape != v.shape:
                raise RecisError(EINVAL, "k and v must have one shape")
        if q is not None:
            q, qa, rows, pad, qs, qh = self._layout(q, "q")
            if k is not None and q.shape[:-2] != shape[:-2]:
                raise RecisError(EINVAL, "q must have the rows of k")
            q_out, shape = _like(q), q.shape
            oa, heads = q_out.data_ptr(), shape[-2]
        if rows == 0:
            ka = va = qa = oa = None
        b, keep = self._batch(rows, pad, shape[0] if len(shape) == 4 else None, offsets, lens, table, slots, k is not None)
        new_lens = torch.empty_like(keep[1])
        r = CacheRows(ka, va, qa, oa, ks, kh, vs, vh, qs, qh, heads, self.rotary, self.interleaved, 0, self._turns,
                      new_lens.data_ptr())
        st = lib().seq_cache_append(self._ref, b, r, validate, _stream_of(self._index))
        if st:
            _check(st)
        return new_lens, q_out

    def read(self, offsets: torch.Tensor, lens: torch.Tensor, table: torch.Tensor, rows: Optional[int] = None,
             start: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
             dtype: Optional[torch.dtype] = None, validate: bool = False):
        """(k, v) [rows, heads_kv, d] of `dtype` (default: the model's): tokens start[s] (default 0) on, offsets[s + 1] -
        offsets[s] of each sequence.  rows: their number, offsets[seqs], where the caller knows it (else it is read from
        the GPU, which waits for it)."""
        dtype = self.dtype if dtype is None else dtype
        if dtype not in _SEQ_TYPES:
            raise RecisError(EINVAL, f"dtype must be float32 or bfloat16, got {dtype}")
        if rows is None:
            rows = int(offsets[-1])
        b, keep = self._batch(rows, 0, None, offsets, lens, table, slots)
        if start is not None:
            start = self._same(start, torch.int64, "start")
            if start.numel() != b.seqs:
                raise RecisError(EINVAL, "start must have one position per sequence")
        k = torch.empty((rows, self.heads_kv, self.head_dim), dtype=dtype, device=self.codes.device)
        v = torch.empty_like(k)
        st = lib().seq_cache_read(self._ref, b, _ptr(start), k.data_ptr(), v.data_ptr(), _SEQ_TYPES[dtype], validate,
                                  _stream_of(self._index))
        if st:
            _check(st)
        return k, v

    def _query(self, q, offsets, lens, table, slots, count, max_q, max_len, own_slots=True):
        q, at, rows, pad, qs, qh = self._layout(q, "q")
        heads = q.shape[-2]
        if heads < self.heads_kv or heads % self.heads_kv:
            raise RecisError(EINVAL, "q's heads must be a multiple of heads_kv")
        b, keep = self._batch(rows, pad, q.shape[0] if pad or q.dim() == 4 else None, offsets, lens, table, slots, own_slots)
        scale = self.scale if self.scale is not None else self.head_dim ** -0.5
        return q, at, b, keep, CacheQuery(heads, self.causal, count, 0, max_q, max_len, qs, qh, scale, self.softcap)

    def attend(self, q: torch.Tensor, offsets: torch.Tensor, lens: torch.Tensor, table: torch.Tensor,
               pages: Optional[torch.Tensor] = None, slopes: Optional[torch.Tensor] = None,
               slots: Optional[torch.Tensor] = None, max_q: int = 0, max_len: int = 0,
               out: Optional[torch.Tensor] = None, validate: bool = False) -> torch.Tensor:
        shape = q.shape
        count = 0 if pages is None else pages.shape[-1]
        q, at, b, keep, d = self._query(q, offsets, lens, table, slots, count, max_q, max_len)
        if pages is not None:
            pages = self._same(pages, torch.int32, "pages")
            if pages.shape != (*shape[:-2], self.heads_kv, count) or count < 1:
                raise RecisError(EINVAL, "pages must be [rows, heads_kv, count] of q's rows")
        if slopes is not None:
            slopes = self._same(slopes, torch.float32, "slopes")
            if slopes.numel() != shape[-2]:
                raise RecisError(EINVAL, "slopes must have one value per query head")
        if out is None:
            out = _like(q)
        elif out.shape != shape or out.dtype != q.dtype or out.device != q.device or not out.is_contiguous():
            raise RecisError(EINVAL, "out must be a contiguous GPU tensor of q's shape and type")
        elif out.numel():
            es, at_out = out.element_size(), out.data_ptr()
            last = (b.rows - 1) * d.q_stride + (shape[-2] - 1) * d.q_head_stride + self.head_dim
            if at < at_out + out.numel() * es and at_out < at + last * es:
                raise RecisError(EINVAL, "out must not overlap q")
        L = lib()
        need = L.seq_cache_attention_workspace_bytes(self._ref, b, d)
        ws = self._take(need, q) if need else None
        st = L.seq_cache_attention(self._ref, b, d, at, _ptr(pages), _ptr(slopes), out.data_ptr(), _ptr(ws),
                                   ws.numel() if need else 0, validate, _stream_of(self._index))
        if st:
            _check(st)
        return out

    def select(self, q: torch.Tensor, offsets: torch.Tensor, lens: torch.Tensor, table: torch.Tensor, count: int,
               max_q: int = 0, max_len: int = 0, validate: bool = False) -> torch.Tensor:
        """int32 [rows, heads_kv, count] (or [seqs, pad, heads_kv, count]): the numbers of the full pages of the highest
        score, ascending, then -1."""
        if self.bounds is None:
            raise RecisError(EINVAL, "the cache keeps no bounds")
        if count < 1:
            raise RecisError(EINVAL, "count must be >= 1")
        shape = q.shape
        q, at, b, keep, d = self._query(q, offsets, lens, table, None, count, max_q, max_len, False)
        pages = torch.empty((*shape[:-2], self.heads_kv, count), dtype=torch.int32, device=q.device)
        L = lib()
        need = L.seq_cache_select_workspace_bytes(self._ref, b, d)
        ws = self._take(need, q) if need else None
        st = L.seq_cache_select(self._ref, b, d, at, pages.data_ptr(), _ptr(ws), ws.numel() if need else 0, validate,
                                _stream_of(self._index))
        if st:
            _check(st)
        return pages


PROBES = {"read": 0, "write": 1, "copy": 2, "gather": 3, "rmw": 4}


def bandwidth_probe(kind: str, a: torch.Tensor, b: Optional[torch.Tensor] = None, idx: Optional[torch.Tensor] = None,
                    n: Optional[int] = None, row_bytes: int = 0):
    """Enqueue one bandwidth probe (measurement reference) on the current stream.

    read / write / copy: n bytes (default: all of a); gather / rmw: the rows
    of row_bytes of a named by idx (int64), gathered into b or updated in place.
    """
    if not a.is_cuda or (b is not None and not b.is_cuda) or (idx is not None and not idx.is_cuda):
        raise RecisError(EINVAL, "probe buffers must be on the GPU")
    ab = a.numel() * a.element_size()
    bb = 0 if b is None else b.numel() * b.element_size()
    if idx is not None:
        idx = _dev(idx, torch.int64)
    if n is None:
        n = idx.numel() if kind in ("gather", "rmw") else ab
    _check(lib().rs_bandwidth_probe(PROBES[kind], _ptr(a), ab, _ptr(b), bb, _ptr(idx), n, row_bytes, _stream()))


class Table:
    """A dynamic embedding table (IDMap + Blocks) on the current GPU."""

    def __init__(self, dim: int, row_dtype: int = F32, optimizer: int = ADAGRAD, init_lo: float = -0.01,
                 init_hi: float = 0.01, seed: int = 0, capacity_slots: int = 1 << 17, max_load: float = 0.75,
                 block_rows: int = 1 << 16, auto_grow: bool = True, evictable: bool = False,
                 allocator: Optional[TorchAllocator] = None):
        d = TableDesc(dim, row_dtype, optimizer, init_lo, init_hi, seed & 0xFFFFFFFFFFFFFFFF, capacity_slots,
                      max_load, block_rows, int(bool(auto_grow)), int(bool(evictable)))
        h = C.c_void_p()
        self.allocator = allocator  # kept alive for the table's lifetime (its callbacks free the memory)
        _check(lib().ht_create(C.byref(d), C.byref(allocator.struct) if allocator else None, _stream(), C.byref(h)))
        self.h = h
        self.dim, self.row_dtype, self.optimizer = dim, row_dtype, optimizer
        # per-element state vectors; the row-wise optimizers add one scalar per row
        self.nstate = {ADAGRAD: 1, ADAGRAD_RW: 0, ADAM_RW: 1}.get(optimizer, 2)
        self.state_shape = ((self.nstate * dim + 1,) if optimizer in (ADAGRAD_RW, ADAM_RW)
                            else (self.nstate, dim))
        self.device = torch.device("cuda", torch.cuda.current_device())

    def close(self):
        if getattr(self, "h", None) and self.h.value:
            st = lib().ht_destroy(self.h)
            self.h = C.c_void_p()
            _check(st)

    def __del__(self):
        try:
            if getattr(self, "h", None) and self.h.value and _lib is not None:
                _lib.ht_destroy(self.h)
                self.h = C.c_void_p()
        except Exception:
            pass

    # ---------------------------------------------------------------- IDMap
    def find_or_insert(self, keys: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        k = _dev(keys, torch.int64)
        rows = torch.empty_like(k)
        nins = torch.zeros(1, dtype=torch.int64, device=k.device)
        _check(lib().ht_find_or_insert(self.h, _ptr(k), k.numel(), _ptr(rows), _ptr(nins), _stream()))
        return rows, nins

    def find(self, keys: torch.Tensor) -> torch.Tensor:
        k = _dev(keys, torch.int64)
        rows = torch.empty_like(k)
        _check(lib().ht_find(self.h, _ptr(k), k.numel(), _ptr(rows), _stream()))
        return rows

    def size(self) -> int:
        v = C.c_int64()
        _check(lib().ht_size(self.h, C.byref(v), _stream()))
        return v.value

    def evict(self, max_age: int) -> int:
        """Drop the keys not looked up in the last max_age lookup calls; returns the count."""
        v = C.c_int64()
        _check(lib().ht_evict(self.h, max_age & 0xFFFFFFFF, C.byref(v), _stream()))
        return v.value

    def compact(self) -> Tuple[int, int]:
        """Move the live rows above the live count into the free rows below it;
        returns (rows moved, bytes of Blocks memory released).  Synchronizes."""
        m, b = C.c_int64(), C.c_int64()
        _check(lib().ht_compact(self.h, C.byref(m), C.byref(b), _stream()))
        return m.value, b.value

    def check(self):
        _check(lib().rs_table_check(self.h, _stream()))

    def capacity(self) -> int:
        v = C.c_int64()
        _check(lib().ht_capacity(self.h, C.byref(v)))
        return v.value

    def reserve(self, live_upper_bound: int):
        _check(lib().ht_reserve(self.h, live_upper_bound, _stream()))

    def export(self) -> Tuple[torch.Tensor, torch.Tensor]:
        live = self.size()
        keys = torch.empty(max(live, 1), dtype=torch.int64, device=self.device)
        rows = torch.empty(max(live, 1), dtype=torch.int64, device=self.device)
        nd = torch.zeros(1, dtype=torch.int64, device=self.device)
        _check(lib().ht_export(self.h, _ptr(keys), _ptr(rows), live, _ptr(nd), _stream()))
        return keys[:live], rows[:live]

    def read_rows(self, rows: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        r = _dev(rows, torch.int64)
        w = torch.empty(r.numel(), self.dim, dtype=torch.float32, device=r.device)
        s = torch.empty(r.numel(), *self.state_shape, dtype=torch.float32, device=r.device)
        _check(lib().ht_read_rows(self.h, _ptr(r), r.numel(), _ptr(w), _ptr(s), _stream()))
        return w, s

    # ---------------------------------------------------------------- step
    def workspace_bytes(self, n: int, bags: int, pad_len: int = 0) -> int:
        return int(lib().lookup_workspace_bytes(n, bags, pad_len, self.h))

    def forward(self, values: torch.Tensor, offsets: torch.Tensor, mode: int, pad_len: int = 0,
                ctx: Optional[Ctx] = None, out: Optional[torch.Tensor] = None,
                mask: Optional[torch.Tensor] = None, validate: bool = False):
        v = _dev(values, torch.int64)
        o = _dev(offsets, torch.int64)
        n, bags = v.numel(), o.numel() - 1
        ctx = ctx or Ctx()
        ctx.ensure(self.workspace_bytes(n, bags, pad_len), v.device)
        if mode in (NONE, TAIL):
            odt = torch.bfloat16 if self.row_dtype == BF16 else torch.float32
            if out is None:
                out = torch.empty(bags, pad_len, self.dim, dtype=odt, device=v.device)
            if mask is None:
                mask = torch.empty(bags, pad_len, dtype=torch.uint8, device=v.device)
        elif out is None:
            out = torch.empty(bags, self.dim, dtype=torch.float32, device=v.device)
        ctx.keep = (v, o)
        _check(lib().lookup_pool_fwd(self.h, _ptr(v), _ptr(o), n, bags, mode, pad_len, _ptr(out), _ptr(mask),
                                     C.byref(ctx.c), int(validate), _stream()))
        return out, mask, ctx

    def prepare(self, values: torch.Tensor, offsets: torch.Tensor, mode: int, pad_len: int = 0,
                ctx: Optional[Ctx] = None, validate: bool = False, stream=None) -> Ctx:
        """First half of the forward (dedup, find-or-insert, bookkeeping) on `stream`."""
        v = _dev(values, torch.int64)
        o = _dev(offsets, torch.int64)
        n, bags = v.numel(), o.numel() - 1
        ctx = ctx or Ctx()
        ctx.ensure(self.workspace_bytes(n, bags, pad_len), v.device)
        ctx.keep = (v, o)
        st = stream.cuda_stream if stream is not None else _stream()
        _check(lib().lookup_prepare(self.h, _ptr(v), _ptr(o), n, bags, mode, pad_len, C.byref(ctx.c),
                                    int(validate), st))
        return ctx

    def pool(self, ctx: Ctx, out: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None):
        """Second half of the forward: gather + pool of a prepared ctx."""
        c = ctx.c
        dev = ctx.ws.device
        if c.mode in (NONE, TAIL):
            odt = torch.bfloat16 if self.row_dtype == BF16 else torch.float32
            if out is None:
                out = torch.empty(c.bags, c.pad_len, self.dim, dtype=odt, device=dev)
            if mask is None:
                mask = torch.empty(c.bags, c.pad_len, dtype=torch.uint8, device=dev)
        elif out is None:
            out = torch.empty(c.bags, self.dim, dtype=torch.float32, device=dev)
        _check(lib().lookup_pool_prepared(self.h, C.byref(ctx.c), _ptr(out), _ptr(mask), _stream()))
        return out, mask

    def _grad(self, ctx: Ctx, grad_out: torch.Tensor) -> torch.Tensor:
        c = ctx.c
        if c.mode in (NONE, TAIL):
            want, dt = c.bags * c.pad_len * self.dim, (torch.bfloat16 if self.row_dtype == BF16 else torch.float32)
        else:
            want, dt = c.bags * self.dim, torch.float32
        if grad_out.numel() != want or grad_out.dtype != dt or not grad_out.is_cuda:
            raise RecisError(EINVAL, f"grad_out must be a GPU {dt} tensor with {want} elements")
        return grad_out.contiguous()

    def backward(self, ctx: Ctx, grad_out: torch.Tensor, grad_unique: Optional[torch.Tensor] = None):
        g = self._grad(ctx, grad_out)
        if grad_unique is None:
            grad_unique = torch.empty(max(ctx.c.n, 1), self.dim, dtype=torch.float32, device=g.device)
        _check(lib().lookup_pool_bwd(self.h, C.byref(ctx.c), _ptr(g), _ptr(grad_unique), _stream()))
        return grad_unique

    def optimizer_step(self, ctx: Ctx, grad_unique: torch.Tensor, lr: float, eps: float = 1e-8,
                       beta1: float = 0.9, beta2: float = 0.999, weight_decay: float = 0.0):
        p = OptParams(lr, eps, beta1, beta2, weight_decay)
        _check(lib().sparse_opt_step(self.h, C.byref(ctx.c), _ptr(grad_unique), C.byref(p), _stream()))

    def backward_optimizer(self, ctx: Ctx, grad_out: torch.Tensor, lr: float, eps: float = 1e-8,
                           beta1: float = 0.9, beta2: float = 0.999, weight_decay: float = 0.0):
        g = self._grad(ctx, grad_out)
        p = OptParams(lr, eps, beta1, beta2, weight_decay)
        _check(lib().lookup_pool_bwd_opt(self.h, C.byref(ctx.c), _ptr(g), C.byref(p), _stream()))

    def set_kernel_events(self, kernel: str, start, stop):
        """Record torch.cuda.Event `start` / `stop` around every launch of `kernel`."""
        if start is not None and (not start.cuda_event or not stop.cuda_event):
            # torch creates the underlying hipEvent_t on its first record()
            start.record()
            stop.record()
        s = None if start is None else C.c_void_p(start.cuda_event)
        e = None if stop is None else C.c_void_p(stop.cuda_event)
        _check(lib().rs_set_kernel_events(self.h, KERNELS[kernel], s, e))
