"""Thin ctypes binding of ``librocketkv.so`` (see ``include/rocketkv.h``).

Argument marshalling only: every function here forwards device pointers of
torch tensors to the C ABI entry point of the same name and raises
``RocketKVError`` on a non-zero status.  torch is used for device memory and
for the current HIP stream; no computation of the method happens in Python and
there is no fallback: if the native library is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librocketkv.so")

OK, INVALID_ARG, UNSUPPORTED, WORKSPACE_TOO_SMALL, HIP_ERROR = 0, -1, -2, -3, -4
OP_HSA_DECODE, OP_DENSE_DECODE, OP_SNAPKV, OP_ATTEND = 0, 1, 2, 3
OP_APPEND_CHUNK, OP_CHUNK_ATTEND, OP_WEIGHT_EVICT = 4, 5, 6
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BANDS, ROPE_RAMP = 0, 1, 2, 3, 4
MAX_CHUNK = 1 << 24
MAX_PAGES = 32768
V_CHANNEL_MAJOR, V_TOKEN_MAJOR = 0, 1
Q_E4M3, Q_E2M1 = 0, 1

EXPORTS = [
    "rocketkv_workspace_bytes", "rocketkv_workspace_init", "rocketkv_build_page_summaries", "rocketkv_hsa_select",
    "rocketkv_attend", "rocketkv_hsa_decode", "rocketkv_hsa_decode_append", "rocketkv_dense_decode", "rocketkv_append_kv",
    "rocketkv_snapkv_compress", "rocketkv_decompose", "rocketkv_last_error", "rocketkv_version",
    "rocketkv_snapkv_filter", "rocketkv_mt_build_page_summaries", "rocketkv_mt_workspace_bytes", "rocketkv_mt_hsa_decode",
    "rocketkv_mt_append_kv", "rocketkv_mt_hsa_decode_append",
    "rocketkv_stream_read", "rocketkv_stream_read_sink_bytes", "rocketkv_hsa_decode_noalloc",
    "rocketkv_stream_gather", "rocketkv_stream_gather_sink_bytes",
    "rocketkv_rope_frequencies", "rocketkv_rope", "rocketkv_append_chunk", "rocketkv_chunk_attend",
    "rocketkv_accumulate_weights", "rocketkv_weight_evict",
    "rocketkv_q_workspace_bytes", "rocketkv_q_append_chunk", "rocketkv_q_chunk_attend", "rocketkv_q_attend",
    "rocketkv_q_hsa_decode", "rocketkv_quantise", "rocketkv_restore", "rocketkv_tree_mask", "rocketkv_masked_attend",
    "rocketkv_keep_tokens", "rocketkv_q_keep_tokens",
]
NOALLOC_SCRATCH_BYTES = 4 << 20


class RocketKVError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"rocketkv status {status}: {message}")
        self.status = status


class CacheStruct(C.Structure):
    """Mirror of ``rocketkv_cache_t``."""
    _fields_ = [
        ("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("page_size", C.c_int32), ("pages_cap", C.c_int32),
        ("n_phys_pages", C.c_int64), ("stride_page", C.c_int64), ("stride_head", C.c_int64),
        ("seq_lens", C.c_void_p), ("block_table", C.c_void_p),
        ("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("v_layout", C.c_int32),
    ]


class QCacheStruct(C.Structure):
    """Mirror of ``rocketkv_qcache_t``."""
    _fields_ = [
        ("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("page_size", C.c_int32), ("pages_cap", C.c_int32),
        ("n_phys_pages", C.c_int64), ("stride_page", C.c_int64), ("stride_head", C.c_int64),
        ("seq_lens", C.c_void_p), ("block_table", C.c_void_p),
        ("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p),
        ("format", C.c_int32),
    ]


class MaskStruct(C.Structure):
    """Mirror of ``rocketkv_mask_t``."""
    _fields_ = [("bits", C.c_void_p), ("words", C.c_int32)]


class IndexStruct(C.Structure):
    """Mirror of ``rocketkv_index_t``."""
    _fields_ = [("token_index", C.c_void_p), ("n_indexed", C.c_void_p), ("page_size", C.c_int32),
                ("pages_cap", C.c_int32)]


class ChunkStruct(C.Structure):
    """Mirror of ``rocketkv_chunk_t``."""
    _fields_ = [("n_tokens", C.c_int32), ("starts", C.c_void_p)]


class RopeStruct(C.Structure):
    """Mirror of ``rocketkv_rope_t``."""
    _fields_ = [("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("inv_freq", C.c_void_p), ("scale", C.c_float)]


class SplitStruct(C.Structure):
    """Mirror of ``rocketkv_split_t``."""
    _fields_ = [
        ("c", C.c_double), ("r", C.c_double), ("stage1", C.c_double), ("stage2", C.c_double),
        ("head_ratio", C.c_double), ("page_size", C.c_int32), ("keep_budget", C.c_int32),
        ("channel_budget", C.c_int32), ("attend_tokens", C.c_int32),
        ("storage", C.c_double), ("storage_mt", C.c_double), ("traffic", C.c_double),
    ]


_lib = None


def lib():
    """Load the native library (built by ``paper_2502_14051_amd.build``)."""
    global _lib
    if _lib is None:
        # torch first: the library must bind to the HIP runtime torch has already loaded, so that
        # streams and device pointers are shared with it
        import torch  # noqa: F401
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2502_14051_amd.build` "
                              "(or __graft_entry__.build()) first; there is no fallback path")
        L = C.CDLL(LIB_PATH)
        cp = C.POINTER(CacheStruct)
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        L.rocketkv_workspace_bytes.restype = sz
        L.rocketkv_workspace_bytes.argtypes = [i32, cp, i32, i32]
        L.rocketkv_workspace_init.restype = i32
        L.rocketkv_workspace_init.argtypes = [vp, sz, vp]
        L.rocketkv_build_page_summaries.restype = i32
        L.rocketkv_build_page_summaries.argtypes = [cp, vp, vp, i32, i32, vp]
        L.rocketkv_hsa_select.restype = i32
        L.rocketkv_hsa_select.argtypes = [cp, vp, vp, vp, i32, i32, i32, vp, i32, vp, vp, vp]
        L.rocketkv_attend.restype = i32
        L.rocketkv_attend.argtypes = [cp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.rocketkv_hsa_decode.restype = i32
        L.rocketkv_hsa_decode.argtypes = [cp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.rocketkv_stream_gather.restype = i32
        L.rocketkv_stream_gather.argtypes = [cp, vp, i32, vp, vp]
        L.rocketkv_stream_gather_sink_bytes.restype = sz
        L.rocketkv_stream_gather_sink_bytes.argtypes = [cp, i32]
        L.rocketkv_hsa_decode_noalloc.restype = i32
        L.rocketkv_hsa_decode_noalloc.argtypes = [cp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp]
        L.rocketkv_hsa_decode_append.restype = i32
        L.rocketkv_hsa_decode_append.argtypes = [cp, vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.rocketkv_dense_decode.restype = i32
        L.rocketkv_dense_decode.argtypes = [cp, vp, vp, vp, vp, sz, vp]
        L.rocketkv_append_kv.restype = i32
        L.rocketkv_append_kv.argtypes = [cp, vp, vp, vp, vp, vp]
        L.rocketkv_snapkv_compress.restype = i32
        L.rocketkv_snapkv_compress.argtypes = [vp, cp, i32, i32, i32, cp, vp, vp, sz, vp]
        ip = C.POINTER(IndexStruct)
        L.rocketkv_snapkv_filter.restype = i32
        L.rocketkv_snapkv_filter.argtypes = [vp, cp, i32, i32, i32, ip, vp, sz, vp]
        L.rocketkv_mt_build_page_summaries.restype = i32
        L.rocketkv_mt_build_page_summaries.argtypes = [cp, ip, vp, vp, i32, i32, vp]
        L.rocketkv_mt_workspace_bytes.restype = sz
        L.rocketkv_mt_workspace_bytes.argtypes = [cp, ip, i32]
        L.rocketkv_mt_hsa_decode.restype = i32
        L.rocketkv_mt_hsa_decode.argtypes = [cp, ip, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.rocketkv_mt_append_kv.restype = i32
        L.rocketkv_mt_append_kv.argtypes = [cp, ip, vp, vp, vp, vp, vp]
        L.rocketkv_mt_hsa_decode_append.restype = i32
        L.rocketkv_mt_hsa_decode_append.argtypes = [cp, ip, vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        hp, rp, i64, dbl = C.POINTER(ChunkStruct), C.POINTER(RopeStruct), C.c_int64, C.c_double
        L.rocketkv_rope_frequencies.restype = i32
        L.rocketkv_rope_frequencies.argtypes = [i32, i32, dbl, dbl, dbl, dbl, i64, C.POINTER(dbl), C.POINTER(C.c_float)]
        L.rocketkv_rope.restype = i32
        L.rocketkv_rope.argtypes = [rp, vp, i32, i32, vp, i64, vp, i64, vp]
        L.rocketkv_append_chunk.restype = i32
        L.rocketkv_append_chunk.argtypes = [cp, hp, rp, vp, vp, i64, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        L.rocketkv_chunk_attend.restype = i32
        L.rocketkv_chunk_attend.argtypes = [cp, hp, vp, vp, vp, vp, sz, vp]
        L.rocketkv_accumulate_weights.restype = i32
        L.rocketkv_accumulate_weights.argtypes = [cp, hp, vp, vp, vp, vp, vp]
        L.rocketkv_weight_evict.restype = i32
        L.rocketkv_weight_evict.argtypes = [cp, vp, i32, i32, cp, vp, vp, vp, sz, vp]
        qp, mp = C.POINTER(QCacheStruct), C.POINTER(MaskStruct)
        L.rocketkv_q_workspace_bytes.restype = sz
        L.rocketkv_q_workspace_bytes.argtypes = [i32, qp, i32]
        L.rocketkv_q_append_chunk.restype = i32
        L.rocketkv_q_append_chunk.argtypes = [qp, hp, rp, vp, vp, i64, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        L.rocketkv_q_chunk_attend.restype = i32
        L.rocketkv_q_chunk_attend.argtypes = [qp, hp, mp, vp, vp, vp, vp, sz, vp]
        L.rocketkv_q_attend.restype = i32
        L.rocketkv_q_attend.argtypes = [qp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.rocketkv_q_hsa_decode.restype = i32
        L.rocketkv_q_hsa_decode.argtypes = [qp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.rocketkv_quantise.restype = i32
        L.rocketkv_quantise.argtypes = [cp, qp, vp]
        L.rocketkv_restore.restype = i32
        L.rocketkv_restore.argtypes = [qp, cp, vp]
        L.rocketkv_tree_mask.restype = i32
        L.rocketkv_tree_mask.argtypes = [i32, hp, vp, vp, vp, i32, vp, vp]
        L.rocketkv_masked_attend.restype = i32
        L.rocketkv_masked_attend.argtypes = [cp, hp, mp, vp, vp, vp, vp, sz, vp]
        L.rocketkv_keep_tokens.restype = i32
        L.rocketkv_keep_tokens.argtypes = [cp, hp, vp, vp, vp, vp, sz, vp]
        L.rocketkv_q_keep_tokens.restype = i32
        L.rocketkv_q_keep_tokens.argtypes = [qp, hp, vp, vp, vp, vp, sz, vp]
        L.rocketkv_decompose.restype = i32
        L.rocketkv_decompose.argtypes = [C.c_int64, i32, i32, C.POINTER(SplitStruct)]
        L.rocketkv_last_error.restype = C.c_char_p
        L.rocketkv_last_error.argtypes = []
        L.rocketkv_version.restype = i32
        L.rocketkv_version.argtypes = []
        L.rocketkv_stream_read.restype = i32
        L.rocketkv_stream_read.argtypes = [vp, C.c_size_t, vp, vp]
        L.rocketkv_stream_read_sink_bytes.restype = C.c_size_t
        L.rocketkv_stream_read_sink_bytes.argtypes = []
        _lib = L
    return _lib


def last_error() -> str:
    return lib().rocketkv_last_error().decode()


def _check(status: int):
    if status != OK:
        raise RocketKVError(status, last_error())


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch  # (the handle alone: a Stream object around it takes 3 us to make)
        stream = torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


@dataclass
class Cache:
    """A paged KV cache living in torch tensors, plus its C descriptor.

    k_pool: bf16 [n_phys_pages][n_kv_heads][page_size][head_dim]
    v_pool: bf16 [n_phys_pages][n_kv_heads][head_dim][page_size], or
            [n_phys_pages][n_kv_heads][page_size][head_dim] when v_layout is V_TOKEN_MAJOR
    Both may be strided views of one allocation (`interleaved`: the K tile of a (page, head) is
    followed by its V tile), which the C descriptor expresses through its strides.
    seq_lens: int32 [batch]; block_table: int32 [batch][pages_cap] or None (identity).
    """
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    page_size: int
    pages_cap: int
    k_pool: object
    v_pool: object
    seq_lens: object
    block_table: object = None
    v_layout: int = V_CHANNEL_MAJOR

    def struct(self) -> CacheStruct:
        k_pool, table = self.k_pool, self.block_table
        strides = k_pool.stride()
        assert strides[:2] == self.v_pool.stride()[:2], "K and V pools must share strides"
        return CacheStruct(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.page_size, self.pages_cap,
                           k_pool.shape[0], strides[0], strides[1], _ptr(self.seq_lens),
                           None if table is None else table.data_ptr(), k_pool.data_ptr(), self.v_pool.data_ptr(), self.v_layout)

    @property
    def units(self) -> int:
        return self.batch * self.n_kv_heads


def alloc_cache(batch, n_q_heads, n_kv_heads, head_dim, page_size, pages_cap, device,
                block_table=None, n_phys_pages=None, zero=False, v_layout=V_CHANNEL_MAJOR,
                interleaved=False) -> Cache:
    import torch
    pages_cap = (pages_cap + 7) // 8 * 8
    n_phys = n_phys_pages if n_phys_pages is not None else batch * pages_cap
    mk = torch.zeros if zero else torch.empty
    v_shape = (page_size, head_dim) if v_layout == V_TOKEN_MAJOR else (head_dim, page_size)
    if interleaved:
        both = mk((n_phys, n_kv_heads, 2, page_size * head_dim), dtype=torch.bfloat16, device=device)
        k_pool = both[:, :, 0].view(n_phys, n_kv_heads, page_size, head_dim)
        v_pool = both[:, :, 1].view((n_phys, n_kv_heads) + v_shape)
    else:
        k_pool = mk((n_phys, n_kv_heads, page_size, head_dim), dtype=torch.bfloat16, device=device)
        v_pool = mk((n_phys, n_kv_heads) + v_shape, dtype=torch.bfloat16, device=device)
    seq_lens = torch.zeros((batch,), dtype=torch.int32, device=device)
    return Cache(batch, n_q_heads, n_kv_heads, head_dim, page_size, pages_cap, k_pool, v_pool,
                 seq_lens, block_table, v_layout)


def pack_cache(K, V, seq_lens, n_q_heads, page_size, pages_cap=None, block_table=None,
               n_phys_pages=None, v_layout=V_CHANNEL_MAJOR, interleaved=False) -> Cache:
    """Lay token-major bf16 K, V ([B][Hkv][n][D] torch tensors on the device) out as a paged cache.

    Pure data movement (pad, reshape, permute, scatter by the block table)."""
    import torch
    B, Hkv, n, D = K.shape
    need = (n + page_size - 1) // page_size
    pages_cap = max(need, pages_cap or 0, 1)
    cache = alloc_cache(B, n_q_heads, Hkv, D, page_size, pages_cap, K.device, block_table,
                        n_phys_pages, zero=True, v_layout=v_layout, interleaved=interleaved)
    pc = cache.pages_cap
    pad = pc * page_size - n
    Kp = torch.nn.functional.pad(K, (0, 0, 0, pad)) if pad else K
    Vp = torch.nn.functional.pad(V, (0, 0, 0, pad)) if pad else V
    Kt = Kp.reshape(B, Hkv, pc, page_size, D).permute(0, 2, 1, 3, 4)        # [B][pc][Hkv][ps][D]
    Vt = Vp.reshape(B, Hkv, pc, page_size, D).permute(0, 2, 1, 3, 4)        # [B][pc][Hkv][ps][D]
    if v_layout != V_TOKEN_MAJOR:
        Vt = Vt.transpose(3, 4)                                              # [B][pc][Hkv][D][ps]
    v_tile = tuple(cache.v_pool.shape[2:])
    if block_table is None:
        cache.k_pool[:B * pc].copy_(Kt.reshape(B * pc, Hkv, page_size, D))
        cache.v_pool[:B * pc].copy_(Vt.reshape((B * pc, Hkv) + v_tile))
    else:
        idx = block_table.reshape(-1).long()
        cache.k_pool.index_copy_(0, idx, Kt.reshape(B * pc, Hkv, page_size, D).contiguous())
        cache.v_pool.index_copy_(0, idx, Vt.reshape((B * pc, Hkv) + v_tile).contiguous())
    cache.seq_lens.copy_(torch.as_tensor(seq_lens, dtype=torch.int32))
    return cache


def unpack_cache(cache: Cache):
    """Inverse of pack_cache: token-major K, V [B][Hkv][pages_cap*page_size][D] (data movement)."""
    B, Hkv, ps, D, pc = cache.batch, cache.n_kv_heads, cache.page_size, cache.head_dim, cache.pages_cap
    if cache.block_table is None:
        kp, vp = cache.k_pool[:B * pc], cache.v_pool[:B * pc]
    else:
        idx = cache.block_table.reshape(-1).long()
        kp, vp = cache.k_pool[idx], cache.v_pool[idx]
    K = kp.reshape(B, pc, Hkv, ps, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, pc * ps, D)
    if cache.v_layout == V_TOKEN_MAJOR:
        V = vp.reshape(B, pc, Hkv, ps, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, pc * ps, D)
    else:
        V = vp.reshape(B, pc, Hkv, D, ps).permute(0, 2, 1, 4, 3).reshape(B, Hkv, pc * ps, D)
    return K.contiguous(), V.contiguous()


def alloc_summaries(cache: Cache):
    import torch
    shape = (cache.batch, cache.n_kv_heads, cache.head_dim, cache.pages_cap)
    return (torch.zeros(shape, dtype=torch.bfloat16, device=cache.k_pool.device),
            torch.zeros(shape, dtype=torch.bfloat16, device=cache.k_pool.device))


def workspace_bytes(op: int, cache: Cache, a: int = 0, b: int = 0) -> int:
    st = cache.struct()
    n = lib().rocketkv_workspace_bytes(op, C.byref(st), a, b)
    if n == 0 and last_error():
        raise RocketKVError(INVALID_ARG, last_error())
    return int(n)


def workspace_init(workspace, stream=None):
    _check(lib().rocketkv_workspace_init(_ptr(workspace), workspace.numel(), _stream(stream)))


def alloc_workspace(op: int, cache: Cache, a: int = 0, b: int = 0, stream=None):
    """Allocate (torch) and initialise a workspace for `op` on `cache`."""
    import torch
    n = workspace_bytes(op, cache, a, b)
    ws = torch.empty((max(n, 256),), dtype=torch.uint8, device=cache.k_pool.device)
    workspace_init(ws, stream)
    return ws


def build_page_summaries(cache: Cache, kmax, kmin, first_page: int = 0, n_pages: int = -1,
                         stream=None):
    st = cache.struct()
    _check(lib().rocketkv_build_page_summaries(C.byref(st), _ptr(kmax), _ptr(kmin), first_page,
                                               n_pages, _stream(stream)))


def hsa_select(cache: Cache, q, kmax, kmin, channel_budget: int, token_budget: int,
               n_recent_pages: int, out_pages, out_channels=None, out_scores=None, stream=None):
    st = cache.struct()
    _check(lib().rocketkv_hsa_select(C.byref(st), _ptr(q), _ptr(kmax), _ptr(kmin), channel_budget,
                                     token_budget, n_recent_pages, _ptr(out_pages),
                                     int(out_pages.shape[-1]), _ptr(out_channels),
                                     _ptr(out_scores), _stream(stream)))


def attend(cache: Cache, q, pages, out, out_lse, workspace, stream=None):
    st = cache.struct()
    row_len = 0 if pages is None else int(pages.shape[-1])
    _check(lib().rocketkv_attend(C.byref(st), _ptr(q), _ptr(pages), row_len, _ptr(out),
                                 _ptr(out_lse), _ptr(workspace), workspace.numel(),
                                 _stream(stream)))


def hsa_decode(cache: Cache, q, kmax, kmin, channel_budget: int, token_budget: int,
               n_recent_pages: int, out, out_lse, out_pages, out_channels, workspace, stream=None):
    st = cache.struct()
    _check(lib().rocketkv_hsa_decode(C.byref(st), _ptr(q), _ptr(kmax), _ptr(kmin), channel_budget,
                                     token_budget, n_recent_pages, _ptr(out), _ptr(out_lse),
                                     _ptr(out_pages), _ptr(out_channels), _ptr(workspace),
                                     workspace.numel(), _stream(stream)))


def hsa_decode_noalloc(cache: Cache, q, kmax, kmin, channel_budget: int, token_budget: int,
                       n_recent_pages: int, out, out_lse, out_pages, out_channels, stream=None):
    """rocketkv_hsa_decode on the library's own scratch buffer (no workspace, no allocation)."""
    st = cache.struct()
    _check(lib().rocketkv_hsa_decode_noalloc(C.byref(st), _ptr(q), _ptr(kmax), _ptr(kmin), channel_budget,
                                             token_budget, n_recent_pages, _ptr(out), _ptr(out_lse),
                                             _ptr(out_pages), _ptr(out_channels), _stream(stream)))


def hsa_decode_append(cache: Cache, q, k_new, v_new, kmax, kmin, channel_budget: int, token_budget: int,
                      n_recent_pages: int, out, out_lse, out_pages, out_channels, workspace, stream=None):
    st = cache.struct()
    _check(lib().rocketkv_hsa_decode_append(C.byref(st), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(kmax),
                                            _ptr(kmin), channel_budget, token_budget, n_recent_pages,
                                            _ptr(out), _ptr(out_lse), _ptr(out_pages), _ptr(out_channels),
                                            _ptr(workspace), workspace.numel(), _stream(stream)))


def dense_decode(cache: Cache, q, out, out_lse, workspace, stream=None):
    st = cache.struct()
    _check(lib().rocketkv_dense_decode(C.byref(st), _ptr(q), _ptr(out), _ptr(out_lse),
                                       _ptr(workspace), workspace.numel(), _stream(stream)))


def append_kv(cache: Cache, k_new, v_new, kmax, kmin, stream=None):
    st = cache.struct()
    _check(lib().rocketkv_append_kv(C.byref(st), _ptr(k_new), _ptr(v_new), _ptr(kmax), _ptr(kmin),
                                    _stream(stream)))


def snapkv_compress(q_obs, src: Cache, window: int, pool_kernel: int, keep_budget: int,
                    dst: Cache, kept_idx, workspace, stream=None):
    s, d = src.struct(), dst.struct()
    _check(lib().rocketkv_snapkv_compress(_ptr(q_obs), C.byref(s), window, pool_kernel, keep_budget,
                                          C.byref(d), _ptr(kept_idx), _ptr(workspace),
                                          workspace.numel(), _stream(stream)))


@dataclass
class Index:
    """The logical sequence of RocketKV-MT in torch tensors, plus its C descriptor.

    token_index: int32 [batch][n_kv_heads][pages_cap * page_size]; n_indexed: int32 [batch]."""
    token_index: object
    n_indexed: object
    page_size: int
    pages_cap: int

    def struct(self) -> IndexStruct:
        return IndexStruct(_ptr(self.token_index), _ptr(self.n_indexed), self.page_size, self.pages_cap)


def alloc_index(cache: Cache, page_size: int, capacity_tokens: int) -> Index:
    import torch
    pages_cap = ((capacity_tokens + page_size - 1) // page_size + 7) // 8 * 8
    dev = cache.k_pool.device
    return Index(torch.full((cache.batch, cache.n_kv_heads, pages_cap * page_size), -1, dtype=torch.int32, device=dev),
                 torch.zeros((cache.batch,), dtype=torch.int32, device=dev), page_size, pages_cap)


def alloc_index_summaries(cache: Cache, index: Index):
    import torch
    shape = (cache.batch, cache.n_kv_heads, cache.head_dim, index.pages_cap)
    return (torch.zeros(shape, dtype=torch.bfloat16, device=cache.k_pool.device),
            torch.zeros(shape, dtype=torch.bfloat16, device=cache.k_pool.device))


def snapkv_filter(q_obs, src: Cache, window: int, pool_kernel: int, keep_budget: int, index: Index,
                  workspace, stream=None):
    st, ix = src.struct(), index.struct()
    _check(lib().rocketkv_snapkv_filter(_ptr(q_obs), C.byref(st), window, pool_kernel, keep_budget, C.byref(ix),
                                        _ptr(workspace), workspace.numel(), _stream(stream)))


def mt_build_page_summaries(cache: Cache, index: Index, kmax, kmin, first_page: int = 0, n_pages: int = -1,
                            stream=None):
    st, ix = cache.struct(), index.struct()
    _check(lib().rocketkv_mt_build_page_summaries(C.byref(st), C.byref(ix), _ptr(kmax), _ptr(kmin), first_page,
                                                  n_pages, _stream(stream)))


def mt_alloc_workspace(cache: Cache, index: Index, token_budget: int, stream=None):
    import torch
    st, ix = cache.struct(), index.struct()
    n = lib().rocketkv_mt_workspace_bytes(C.byref(st), C.byref(ix), token_budget)
    if n == 0:
        raise RocketKVError(INVALID_ARG, last_error())
    ws = torch.empty((max(int(n), 256),), dtype=torch.uint8, device=cache.k_pool.device)
    workspace_init(ws, stream)
    return ws


def mt_hsa_decode(cache: Cache, index: Index, q, kmax, kmin, channel_budget: int, token_budget: int,
                  n_recent_pages: int, out, out_lse, out_pages, out_channels, workspace, stream=None):
    st, ix = cache.struct(), index.struct()
    _check(lib().rocketkv_mt_hsa_decode(C.byref(st), C.byref(ix), _ptr(q), _ptr(kmax), _ptr(kmin), channel_budget,
                                        token_budget, n_recent_pages, _ptr(out), _ptr(out_lse), _ptr(out_pages),
                                        _ptr(out_channels), _ptr(workspace), workspace.numel(), _stream(stream)))


def mt_append_kv(cache: Cache, index: Index, k_new, v_new, kmax, kmin, stream=None):
    st, ix = cache.struct(), index.struct()
    _check(lib().rocketkv_mt_append_kv(C.byref(st), C.byref(ix), _ptr(k_new), _ptr(v_new), _ptr(kmax), _ptr(kmin),
                                       _stream(stream)))


def mt_hsa_decode_append(cache: Cache, index: Index, q, k_new, v_new, kmax, kmin, channel_budget: int,
                         token_budget: int, n_recent_pages: int, out, out_lse, out_pages, out_channels,
                         workspace, stream=None):
    st, ix = cache.struct(), index.struct()
    _check(lib().rocketkv_mt_hsa_decode_append(C.byref(st), C.byref(ix), _ptr(q), _ptr(k_new), _ptr(v_new),
                                               _ptr(kmax), _ptr(kmin), channel_budget, token_budget,
                                               n_recent_pages, _ptr(out), _ptr(out_lse), _ptr(out_pages),
                                               _ptr(out_channels), _ptr(workspace), workspace.numel(),
                                               _stream(stream)))


@dataclass
class Chunk:
    """The new tokens of all sequences of a cache, packed: rows starts[b] .. starts[b+1]-1 are sequence b's.

    starts: int32 [batch + 1] on the device; n_tokens: rows of the packed tensors."""
    starts: object
    n_tokens: int

    def struct(self, cache: Cache) -> ChunkStruct:
        _tensor("starts", self.starts, "int32", (cache.batch + 1,))
        return ChunkStruct(self.n_tokens, _ptr(self.starts))


@dataclass
class Rope:
    """Rotary positions: inv_freq, float64 [rot_dim / 2] on the device, in radians per position (see rope_frequencies)."""
    inv_freq: object
    interleaved: bool = False
    scale: float = 1.0

    def struct(self) -> RopeStruct:
        _tensor("inv_freq", self.inv_freq, "float64", self.inv_freq.shape[:1] or (0,))
        return RopeStruct(2 * int(self.inv_freq.shape[0]), int(self.interleaved), _ptr(self.inv_freq), self.scale)


_dtypes = {}


def _dtype(name):
    want = _dtypes.get(name)
    if want is None:
        import torch
        want = _dtypes[name] = getattr(torch, name)
    return want


def _tensor(name, t, dtype, shape, rows=False):
    """What a pointer cannot say: type, shape and layout, contiguous or, with `rows`, tokens at any stride."""
    want = _dtypes.get(dtype) or _dtype(dtype)
    have = t.shape
    if t.dtype is not want or have != shape:
        raise RocketKVError(INVALID_ARG, f"{name}: need {dtype} {tuple(shape)}, got {t.dtype} {tuple(have)}")
    if not t.is_contiguous() and not (rows and t.stride()[1:] == (have[2], 1)):
        raise RocketKVError(INVALID_ARG, f"{name}: inner dimensions must be contiguous")


def _here(**tensors):
    """All of them (but for None) on the current GPU."""
    here = None
    for name, t in tensors.items():
        if t is None:
            continue
        device = t.get_device()
        if here is None and device >= 0:
            import torch  # (with a tensor on a GPU, torch.cuda.current_device has nothing left to initialise)
            here = torch._C._cuda_getDevice()
        if device != here:
            raise RocketKVError(INVALID_ARG, f"{name}: on {t.device}, not on the current GPU")


def _here_with(cache, **tensors):
    _here(k_pool=cache.k_pool, v_pool=cache.v_pool, seq_lens=cache.seq_lens, block_table=cache.block_table, **tensors)


def rope_frequencies(rot_dim: int, theta: float, kind: int = ROPE_PLAIN, factor: float = 1.0, low: float = 1.0,
                     high: float = 4.0, original: int = 8192, device=None, interleaved: bool = False) -> Rope:
    """Rotary positions with (stretched) frequencies (host arithmetic in the library); see rocketkv_rope_frequencies."""
    import torch
    if rot_dim < 0:
        raise RocketKVError(INVALID_ARG, f"rot_dim {rot_dim} must not be negative")
    freq, scale = (C.c_double * max(rot_dim // 2, 1))(), C.c_float()
    _check(lib().rocketkv_rope_frequencies(kind, rot_dim, theta, factor, low, high, original, freq, C.byref(scale)))
    return Rope(torch.tensor(list(freq), dtype=torch.float64, device=device), interleaved, scale.value)


def rope(rope: Rope, positions, x, y, stream=None):
    """x, y: bf16 [tokens][heads][128], tokens at any stride; positions: int32 [tokens].  y may be x."""
    _tensor("x", x, "bfloat16", x.shape[:2] + (128,), rows=True)
    n, heads, width = x.shape
    _tensor("y", y, "bfloat16", (n, heads, 128), rows=True)
    _tensor("positions", positions, "int32", (n,))
    r = rope.struct()
    _here(x=x, y=y, positions=positions, inv_freq=rope.inv_freq)
    if n == 0:
        return
    width *= heads  # (a single token's stride may be anything)
    _check(lib().rocketkv_rope(C.byref(r), _ptr(positions), n, heads, _ptr(x), x.stride(0) if n > 1 else width, _ptr(y),
                               y.stride(0) if n > 1 else width, _stream(stream)))


def append_chunk(cache: Cache, chunk: Chunk, k_new, v_new, kmax, kmin, workspace, rope: Optional[Rope] = None,
                 positions=None, q=None, q_out=None, stream=None):
    """k_new, v_new: bf16 [n_tokens][n_kv_heads][128], q: bf16 [n_tokens][n_q_heads][128], tokens at any stride."""
    _append(lib().rocketkv_append_chunk, _here_with, cache, chunk, k_new, v_new, kmax, kmin, workspace, rope, positions, q, q_out,
            stream)


def _append(call, here, cache, chunk, k_new, v_new, kmax, kmin, workspace, rope, positions, q, q_out, stream):
    n = chunk.n_tokens
    _tensor("k_new", k_new, "bfloat16", (n, cache.n_kv_heads, 128), rows=True)
    _tensor("v_new", v_new, "bfloat16", (n, cache.n_kv_heads, 128), rows=True)
    if q is not None:
        _tensor("q", q, "bfloat16", (n, cache.n_q_heads, 128), rows=True)
    if q_out is not None:
        _tensor("q_out", q_out, "bfloat16", (n, cache.n_q_heads, 128))
    if positions is not None:
        _tensor("positions", positions, "int32", (n,))
    _summaries(cache, kmax, kmin)
    st, ch, r = cache.struct(), chunk.struct(cache), rope.struct() if rope is not None else None
    here(cache, k_new=k_new, v_new=v_new, q=q, q_out=q_out, positions=positions, kmax=kmax, kmin=kmin,
         starts=chunk.starts, inv_freq=rope.inv_freq if rope is not None else None, workspace=workspace)
    if n == 0:
        return
    stride = lambda t, heads: t.stride(0) if n > 1 and t is not None else heads * 128
    _check(call(C.byref(st), C.byref(ch), C.byref(r) if r is not None else None, _ptr(positions), _ptr(q),
                stride(q, cache.n_q_heads), _ptr(q_out), _ptr(k_new), stride(k_new, cache.n_kv_heads), _ptr(v_new),
                stride(v_new, cache.n_kv_heads), _ptr(kmax), _ptr(kmin), _ptr(workspace), workspace.numel(), _stream(stream)))


def _summaries(cache, kmax, kmin):
    for name, t in (("kmax", kmax), ("kmin", kmin)):
        if t is not None:
            _tensor(name, t, "bfloat16", (cache.batch, cache.n_kv_heads, cache.head_dim, cache.pages_cap))


def chunk_attend(cache: Cache, chunk: Chunk, q, out, out_lse, workspace, stream=None):
    """q, out: bf16 [n_tokens][n_q_heads][128]; out_lse: float32 [n_tokens][n_q_heads] or None."""
    n = chunk.n_tokens
    _tensor("q", q, "bfloat16", (n, cache.n_q_heads, 128))
    _tensor("out", out, "bfloat16", (n, cache.n_q_heads, 128))
    if out_lse is not None:
        _tensor("out_lse", out_lse, "float32", (n, cache.n_q_heads))
    st, ch = cache.struct(), chunk.struct(cache)
    _here_with(cache, q=q, out=out, out_lse=out_lse, starts=chunk.starts, workspace=workspace)
    if n == 0:
        return
    _check(lib().rocketkv_chunk_attend(C.byref(st), C.byref(ch), _ptr(q), _ptr(out), _ptr(out_lse), _ptr(workspace),
                                       workspace.numel(), _stream(stream)))


def alloc_weights(cache: Cache):
    """Zeroed accumulated weights of a cache."""
    import torch
    return torch.zeros((cache.batch, cache.n_kv_heads, cache.pages_cap * cache.page_size), dtype=torch.float32,
                       device=cache.k_pool.device)


def _weights(name, t, cache):
    _tensor(name, t, "float32", (cache.batch, cache.n_kv_heads, cache.pages_cap * cache.page_size))


def accumulate_weights(cache: Cache, chunk: Chunk, q, lse, weights_in, weights_out, stream=None):
    """q: bf16 [n_tokens][n_q_heads][128], lse: float32 [n_tokens][n_q_heads]; weights as of alloc_weights, weights_in
    None or weights_out itself if it is to be added to."""
    n = chunk.n_tokens
    _tensor("q", q, "bfloat16", (n, cache.n_q_heads, 128))
    _tensor("lse", lse, "float32", (n, cache.n_q_heads))
    if weights_in is not None:
        _weights("weights_in", weights_in, cache)
    _weights("weights_out", weights_out, cache)
    st, ch = cache.struct(), chunk.struct(cache)
    _here_with(cache, q=q, lse=lse, weights_in=weights_in, weights_out=weights_out, starts=chunk.starts)
    _check(lib().rocketkv_accumulate_weights(C.byref(st), C.byref(ch), _ptr(q), _ptr(lse), _ptr(weights_in),
                                             _ptr(weights_out), _stream(stream)))


def weight_evict(src: Cache, weights, n_recent: int, keep_budget: int, dst: Cache, dst_weights, kept_idx, workspace,
                 stream=None):
    _weights("weights", weights, src)
    if dst_weights is not None:
        _weights("dst_weights", dst_weights, dst)
    if kept_idx is not None:
        _tensor("kept_idx", kept_idx, "int32", (src.batch, src.n_kv_heads, keep_budget))
    s, d = src.struct(), dst.struct()
    _here_with(src, weights=weights, dst_weights=dst_weights, kept_idx=kept_idx, workspace=workspace)
    _here_with(dst)
    _check(lib().rocketkv_weight_evict(C.byref(s), _ptr(weights), n_recent, keep_budget, C.byref(d), _ptr(dst_weights),
                                       _ptr(kept_idx), _ptr(workspace), workspace.numel(), _stream(stream)))


@dataclass
class QCache:
    """A paged cache of quantised keys and values in torch tensors, plus its C descriptor (see rocketkv_qcache_t).

    k_codes, v_codes: uint8 [n_phys_pages][n_kv_heads][page_size][128], or [..][64] in Q_E2M1
    k_scales, v_scales: uint8 [n_phys_pages][n_kv_heads][page_size][4]
    Pages and heads may lie at any stride, counted in tokens and the same for all four; a page's tokens are contiguous.
    seq_lens: int32 [batch]; block_table: int32 [batch][pages_cap] or None (identity).
    """
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    page_size: int
    pages_cap: int
    k_codes: object
    v_codes: object
    k_scales: object
    v_scales: object
    seq_lens: object
    block_table: object = None
    format: int = Q_E4M3

    def struct(self) -> QCacheStruct:
        k, v, ks, vs, lens, table = self.k_codes, self.v_codes, self.k_scales, self.v_scales, self.seq_lens, self.block_table
        shape, byte, i32 = k.shape, _dtypes.get("uint8") or _dtype("uint8"), _dtypes.get("int32") or _dtype("int32")
        n, head, width = shape[0], self.page_size, 128 if self.format == Q_E4M3 else 64
        page = head * self.n_kv_heads  # in tokens
        small = (n, self.n_kv_heads, head, 4)
        if not (shape == (n, self.n_kv_heads, head, width) and v.shape == shape and ks.shape == small and vs.shape == small and
                k.dtype is byte and v.dtype is byte and ks.dtype is byte and vs.dtype is byte and
                k.is_contiguous() and v.is_contiguous() and ks.is_contiguous() and vs.is_contiguous()):
            page, head = self._strides()  # (most caches are whole tensors of the right shape, which is quicker to see)
        if lens is not None and not (lens.dtype is i32 and lens.shape == (self.batch,) and lens.is_contiguous()):
            _tensor("seq_lens", lens, "int32", (self.batch,))
        if table is not None and not (table.dtype is i32 and table.shape == (self.batch, self.pages_cap) and table.is_contiguous()):
            _tensor("block_table", table, "int32", (self.batch, self.pages_cap))
        return QCacheStruct(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.page_size, self.pages_cap,
                            n, page, head, _ptr(lens), None if table is None else table.data_ptr(),
                            k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), self.format)

    def _strides(self):
        """Of pages and heads, in tokens; says which of the tensors is none a cache can have."""
        width = q_row_bytes(self.format)
        shape = (self.k_codes.shape[0], self.n_kv_heads, self.page_size)
        pools = (("k_codes", self.k_codes, width), ("v_codes", self.v_codes, width), ("k_scales", self.k_scales, 4),
                 ("v_scales", self.v_scales, 4))
        for name, t, w in pools:
            if t.element_size() != 1 or t.shape != shape + (w,):
                raise RocketKVError(INVALID_ARG, f"{name}: need bytes {shape + (w,)}, got {t.dtype} {tuple(t.shape)}")
        page, head = (x // 4 for x in self.k_scales.stride()[:2])
        for name, t, w in pools:
            if t.stride() != (page * w, head * w, w, 1):
                raise RocketKVError(INVALID_ARG, f"{name}: strides must be those of k_scales in tokens, rows contiguous")
        return page, head


def q_row_bytes(format: int) -> int:
    """Bytes of a token's codes of one head."""
    if format not in (Q_E4M3, Q_E2M1):
        raise RocketKVError(INVALID_ARG, f"unknown format {format}")
    return 128 if format == Q_E4M3 else 64


def alloc_qcache(batch, n_q_heads, n_kv_heads, page_size, pages_cap, device, format=Q_E4M3, block_table=None,
                 n_phys_pages=None) -> QCache:
    """An empty quantised cache."""
    import torch
    pages_cap = (pages_cap + 7) // 8 * 8
    n_phys = n_phys_pages if n_phys_pages is not None else batch * pages_cap
    mk = lambda width: torch.empty((n_phys, n_kv_heads, page_size, width), dtype=torch.uint8, device=device)
    width = q_row_bytes(format)
    return QCache(batch, n_q_heads, n_kv_heads, 128, page_size, pages_cap, mk(width), mk(width), mk(4), mk(4),
                  torch.zeros((batch,), dtype=torch.int32, device=device), block_table, format)


def _here_with_q(cache, **tensors):
    _here(k_codes=cache.k_codes, v_codes=cache.v_codes, k_scales=cache.k_scales, v_scales=cache.v_scales,
          seq_lens=cache.seq_lens, block_table=cache.block_table, **tensors)


def q_workspace_bytes(op: int, cache: QCache, a: int = 0) -> int:
    st = cache.struct()
    n = lib().rocketkv_q_workspace_bytes(op, C.byref(st), a)
    if n == 0 and last_error():
        raise RocketKVError(INVALID_ARG, last_error())
    return int(n)


def q_alloc_workspace(op: int, cache: QCache, a: int = 0, stream=None):
    """Allocate (torch) and initialise a workspace for `op` on a quantised cache."""
    import torch
    ws = torch.empty((max(q_workspace_bytes(op, cache, a), 256),), dtype=torch.uint8, device=cache.k_codes.device)
    workspace_init(ws, stream)
    return ws


def q_append_chunk(cache: QCache, chunk: Chunk, k_new, v_new, kmax, kmin, workspace, rope: Optional[Rope] = None,
                   positions=None, q=None, q_out=None, stream=None):
    """append_chunk into a quantised cache."""
    _append(lib().rocketkv_q_append_chunk, _here_with_q, cache, chunk, k_new, v_new, kmax, kmin, workspace, rope, positions, q,
            q_out, stream)


@dataclass
class Mask:
    """Which of its sequence's rows each row of a chunk sees: bits, int32 [n_tokens][words] (see rocketkv_mask_t)."""
    bits: object

    def struct(self, n: int) -> MaskStruct:
        _tensor("bits", self.bits, "int32", (n, self.bits.shape[-1]))
        return MaskStruct(_ptr(self.bits), int(self.bits.shape[1]))


def alloc_mask(n_tokens: int, most_rows: int, device) -> Mask:
    """A mask for chunks of n_tokens, of sequences that bring at most most_rows each."""
    import torch
    return Mask(torch.zeros((n_tokens, max(1, (most_rows + 31) // 32)), dtype=torch.int32, device=device))


def tree_mask(chunk: Chunk, parents, mask: Mask, base=None, positions=None, stream=None):
    """parents: int32 [n_tokens]; base: int32 [batch] and positions: int32 [n_tokens], or None; see rocketkv_tree_mask."""
    n, batch = chunk.n_tokens, int(chunk.starts.shape[0]) - 1
    _tensor("starts", chunk.starts, "int32", (batch + 1,))
    _tensor("parents", parents, "int32", (n,))
    if base is not None:
        _tensor("base", base, "int32", (batch,))
    if positions is not None:
        _tensor("positions", positions, "int32", (n,))
    m = mask.struct(n)
    _here(starts=chunk.starts, parents=parents, bits=mask.bits, base=base, positions=positions)
    if n == 0:
        return
    ch = ChunkStruct(n, _ptr(chunk.starts))
    _check(lib().rocketkv_tree_mask(batch, C.byref(ch), _ptr(parents), _ptr(base), m.bits, m.words, _ptr(positions),
                                    _stream(stream)))


def _attend_tensors(n, cache, q, out, out_lse):
    _tensor("q", q, "bfloat16", (n, cache.n_q_heads, 128))
    _tensor("out", out, "bfloat16", (n, cache.n_q_heads, 128))
    if out_lse is not None:
        _tensor("out_lse", out_lse, "float32", (n, cache.n_q_heads))


def masked_attend(cache: Cache, chunk: Chunk, mask: Mask, q, out, out_lse, workspace, stream=None):
    """chunk_attend with `mask` in place of the order of the chunk's tokens."""
    n = chunk.n_tokens
    _attend_tensors(n, cache, q, out, out_lse)
    st, ch, m = cache.struct(), chunk.struct(cache), mask.struct(n)
    _here_with(cache, q=q, out=out, out_lse=out_lse, starts=chunk.starts, bits=mask.bits, workspace=workspace)
    if n == 0:
        return
    _check(lib().rocketkv_masked_attend(C.byref(st), C.byref(ch), C.byref(m), _ptr(q), _ptr(out), _ptr(out_lse),
                                        _ptr(workspace), workspace.numel(), _stream(stream)))


def q_chunk_attend(cache: QCache, chunk: Chunk, q, out, out_lse, workspace, mask: Optional[Mask] = None, stream=None):
    """chunk_attend, or with a mask masked_attend, over a quantised cache."""
    n = chunk.n_tokens
    _attend_tensors(n, cache, q, out, out_lse)
    st, ch, m = cache.struct(), chunk.struct(cache), mask.struct(n) if mask is not None else None
    _here_with_q(cache, q=q, out=out, out_lse=out_lse, starts=chunk.starts, bits=mask.bits if mask is not None else None,
                 workspace=workspace)
    if n == 0:
        return
    _check(lib().rocketkv_q_chunk_attend(C.byref(st), C.byref(ch), C.byref(m) if m is not None else None, _ptr(q), _ptr(out),
                                         _ptr(out_lse), _ptr(workspace), workspace.numel(), _stream(stream)))


def q_attend(cache: QCache, q, pages, out, out_lse, workspace, stream=None):
    """q, out: bf16 [batch][n_q_heads][128]; pages: int32 [batch][n_kv_heads][row_len] or None (every page)."""
    _attend_tensors(cache.batch, cache, q, out, out_lse)
    if pages is not None:
        _tensor("pages", pages, "int32", (cache.batch, cache.n_kv_heads, pages.shape[-1]))
    st = cache.struct()
    _here_with_q(cache, q=q, pages=pages, out=out, out_lse=out_lse, workspace=workspace)
    _check(lib().rocketkv_q_attend(C.byref(st), _ptr(q), _ptr(pages), 0 if pages is None else int(pages.shape[-1]), _ptr(out),
                                   _ptr(out_lse), _ptr(workspace), workspace.numel(), _stream(stream)))


def q_hsa_decode(cache: QCache, q, kmax, kmin, channel_budget: int, token_budget: int, n_recent_pages: int, out, out_lse,
                 out_pages, out_channels, workspace, stream=None):
    """hsa_decode over a quantised cache."""
    _attend_tensors(cache.batch, cache, q, out, out_lse)
    _summaries(cache, kmax, kmin)
    if out_pages is not None:
        _tensor("out_pages", out_pages, "int32", (cache.batch, cache.n_kv_heads, pages_row_len(cache, token_budget)))
    if out_channels is not None:
        _tensor("out_channels", out_channels, "int32", (cache.batch, cache.n_kv_heads, channel_budget))
    st = cache.struct()
    _here_with_q(cache, q=q, kmax=kmax, kmin=kmin, out=out, out_lse=out_lse, out_pages=out_pages, out_channels=out_channels,
                 workspace=workspace)
    _check(lib().rocketkv_q_hsa_decode(C.byref(st), _ptr(q), _ptr(kmax), _ptr(kmin), channel_budget, token_budget,
                                       n_recent_pages, _ptr(out), _ptr(out_lse), _ptr(out_pages), _ptr(out_channels),
                                       _ptr(workspace), workspace.numel(), _stream(stream)))


def quantise(src: Cache, dst: QCache, stream=None):
    """Every token of a bf16 cache into a quantised one."""
    s, d = src.struct(), dst.struct()
    _here_with(src)
    _here_with_q(dst)
    _check(lib().rocketkv_quantise(C.byref(s), C.byref(d), _stream(stream)))


def restore(src: QCache, dst: Cache, stream=None):
    """Every token of a quantised cache into a bf16 one, exactly."""
    s, d = src.struct(), dst.struct()
    _here_with_q(src)
    _here_with(dst)
    _check(lib().rocketkv_restore(C.byref(s), C.byref(d), _stream(stream)))


def _keep(call, here, cache, chunk, keep, kmax, kmin, workspace, stream):
    n = chunk.n_tokens
    if keep.element_size() != 1 or keep.shape != (n,) or not keep.is_contiguous():
        raise RocketKVError(INVALID_ARG, f"keep: need {n} bytes or truth values, got {keep.dtype} {tuple(keep.shape)}")
    _summaries(cache, kmax, kmin)
    st, ch = cache.struct(), chunk.struct(cache)
    here(cache, keep=keep, kmax=kmax, kmin=kmin, starts=chunk.starts, workspace=workspace)
    if n == 0:
        return
    _check(call(C.byref(st), C.byref(ch), _ptr(keep), _ptr(kmax), _ptr(kmin), _ptr(workspace), workspace.numel(),
                _stream(stream)))


def keep_tokens(cache: Cache, chunk: Chunk, keep, kmax, kmin, workspace, stream=None):
    """Of the chunk appended last, the tokens with keep != 0 (uint8 or bool [n_tokens]) stay; see rocketkv_keep_tokens."""
    _keep(lib().rocketkv_keep_tokens, _here_with, cache, chunk, keep, kmax, kmin, workspace, stream)


def q_keep_tokens(cache: QCache, chunk: Chunk, keep, kmax, kmin, workspace, stream=None):
    """keep_tokens on a quantised cache."""
    _keep(lib().rocketkv_q_keep_tokens, _here_with_q, cache, chunk, keep, kmax, kmin, workspace, stream)


def decompose(seq_len: int, token_budget: int, head_dim: int = 128) -> dict:
    """Adaptive compression decomposition (host arithmetic in the library); see rocketkv_decompose."""
    out = SplitStruct()
    _check(lib().rocketkv_decompose(int(seq_len), int(token_budget), int(head_dim), C.byref(out)))
    return {name: getattr(out, name) for name, _ in SplitStruct._fields_}


def pages_row_len(cache: Cache, token_budget: int) -> int:
    """Row length of the page list hsa_decode / hsa_select write for this budget."""
    return max(1, min(cache.pages_cap, (token_budget + cache.page_size - 1) // cache.page_size))


def stream_gather(cache: Cache, pages, sink=None, stream=None):
    """Measurement aid: the K/V tiles of a page list read the way the attention kernels read them, nothing
    computed (see rocketkv_stream_gather).  Returns the sink tensor."""
    import torch
    st = cache.struct()
    if sink is None:
        sink = torch.empty((lib().rocketkv_stream_gather_sink_bytes(C.byref(st), pages.shape[-1]),), dtype=torch.uint8,
                           device=pages.device)
    _check(lib().rocketkv_stream_gather(C.byref(st), _ptr(pages), pages.shape[-1], _ptr(sink), _stream(stream)))
    return sink


def stream_read(buf, sink=None, stream=None):
    """Measurement aid: one streaming read of the whole tensor ``buf`` (see rocketkv_stream_read)."""
    import torch

    nbytes = buf.numel() * buf.element_size()
    if sink is None:
        sink = torch.empty((lib().rocketkv_stream_read_sink_bytes(),), dtype=torch.uint8, device=buf.device)
    _check(lib().rocketkv_stream_read(_ptr(buf), nbytes, _ptr(sink), _stream(stream)))
    return sink
