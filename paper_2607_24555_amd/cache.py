"""Thin ctypes binding of the paged-cache calls of liblocks (include/locks_cache.h):
appends with rotary positions, a cache held in 8 bits, and decode attention over it.

As in `locks`: argument checks and marshalling only, tensors are torch device tensors on
the current device, work goes to the given or current stream, and the prepare_* forms do
the checks once for loops over fixed buffers.  Outputs that a call allocates are allocated on
the stream it runs on, those of a prepare_* form on the current one.
"""
from __future__ import annotations

import contextlib
import ctypes
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

from . import locks as B
from .locks import Config, LocksError, PreparedCall, _Cfg

LOCKS_Q8_INT8 = 0
LOCKS_Q8_E4M3 = 1
_CODE_OF = {torch.int8: LOCKS_Q8_INT8, torch.float8_e4m3fn: LOCKS_Q8_E4M3}


class _Rope(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("n_pos", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("axis_pairs", ctypes.c_int32 * 3)]


class _Rows(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("q_out", ctypes.c_void_p), ("cu_tokens", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64),
                ("v_stride", ctypes.c_int64), ("q_out_stride", ctypes.c_int64),
                ("n_tokens", ctypes.c_int32)]


class _Q8(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("code", ctypes.c_int32)]


_P, _SZ, _I = B._P, B._SZ, B._I
_PC, _PR, _PO, _PQ = (ctypes.POINTER(t) for t in (_Cfg, _Rows, _Rope, _Q8))
_SIGS = {
    "locks_rope_append_kv": (ctypes.c_int, [_PC, _PR, _PO, _P, _P, _P, _P, _P]),
    "locks_q8_append_kv": (ctypes.c_int, [_PC, _PR, _PO, _PQ, _P, _P, _P]),
    "locks_q8_build_summaries": (ctypes.c_int, [_PC, _PQ, _P, _P, _P, _I, _P, _P]),
    "locks_q8_dense_attend": (ctypes.c_int, [_PC, _P, _PQ, _P, _P, _P, _P, _P, _SZ, _P]),
    "locks_q8_sparse_attend": (ctypes.c_int, [_PC, _P, _PQ, _P, _P, _P, _P, _P, _P, _SZ, _P]),
}
_lib = None


def lib():
    """liblocks with the signatures of this header (raises LocksError when not built)."""
    global _lib
    if _lib is None:
        L = B.lib()
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


@dataclass
class Rope:
    """Rotary positions (locks_rope_t): `table` [n_pos][rot_dim] float32, cosines of the
    rot_dim / 2 angles and then their sines (rope_table makes one); pairs (i, i + rot_dim / 2),
    or (2 i, 2 i + 1) where `interleaved`; `axis_pairs` splits the pairs over up to three
    position axes."""
    table: torch.Tensor
    interleaved: bool = False
    axis_pairs: Optional[Sequence[int]] = None


def rope_table(n_pos: int, rot_dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """The [n_pos][rot_dim] table of angles p * base ** (-2 i / rot_dim), formed in 64 bits."""
    i = torch.arange(rot_dim // 2, dtype=torch.float64, device=device)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * base ** (-2.0 * i / rot_dim)
    return torch.cat([a.cos(), a.sin()], 1).float().contiguous()


@dataclass
class Q8Cache:
    """A paged cache in 8 bits (locks_q8_t): codes [num_blocks][num_kv_heads][B][128], int8 or
    float8_e4m3fn, and float32 scales [num_blocks][num_kv_heads]."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor


def alloc_q8_cache(cfg: Config, code=torch.int8, device="cuda") -> Q8Cache:
    if code not in _CODE_OF:
        raise LocksError(f"an 8-bit cache holds int8 or float8_e4m3fn codes, not {code}")
    shape = (cfg.num_blocks, cfg.num_kv_heads, cfg.page_size, cfg.head_dim)
    k, v = (torch.zeros(shape, dtype=torch.uint8, device=device).view(code) for _ in range(2))
    ks, vs = (torch.zeros(shape[:2], dtype=torch.float32, device=device) for _ in range(2))
    return Q8Cache(k, v, ks, vs)


def _current_device(*ts):
    """The tensors' one device, which has to be the current one: the library launches on it."""
    B._same_device(*ts)
    dev = next(t.device for t in ts if t is not None)
    if dev.type != "cuda":
        raise LocksError("liblocks takes device tensors")
    if dev.index != torch.cuda.current_device():
        raise LocksError(f"tensors on {dev}, but the current device is cuda:{torch.cuda.current_device()}")


def _allocating_on(stream):
    """What is allocated within belongs to `stream`: memory of the current one may still be in
    use by the work queued there when a call on another stream writes it."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _q8(cfg: Config, cache: Q8Cache) -> _Q8:
    shape = (cfg.num_blocks, cfg.num_kv_heads, cfg.page_size, cfg.head_dim)
    if cache.k.dtype not in _CODE_OF:
        raise LocksError(f"cache.k: dtype {cache.k.dtype}, expected torch.int8 or torch.float8_e4m3fn")
    B._need("cache.k", cache.k, shape, cache.k.dtype)
    B._need("cache.v", cache.v, shape, cache.k.dtype)
    B._need("cache.k_scale", cache.k_scale, shape[:2], torch.float32)
    B._need("cache.v_scale", cache.v_scale, shape[:2], torch.float32)
    return _Q8(B._ptr(cache.k), B._ptr(cache.v), B._ptr(cache.k_scale), B._ptr(cache.v_scale),
               _CODE_OF[cache.k.dtype])


def _rows_tensor(name: str, t: torch.Tensor, n: int, heads: int, dtype) -> None:
    """[n][heads][128] with any distance between tokens: a slice of a fused projection, say."""
    B._need(name, t, (n, heads, B.HEAD_DIM), dtype)
    if not t.is_cuda:
        raise LocksError("liblocks takes device tensors")
    if t.numel() and (t.stride(2) != 1 or (heads > 1 and t.stride(1) != B.HEAD_DIM) or
                      (n > 1 and t.stride(0) < heads * B.HEAD_DIM)):
        raise LocksError(f"{name}: strides {t.stride()}, expected rows of {heads} x {B.HEAD_DIM} elements in a run")


def _stride(t: torch.Tensor, heads: int) -> int:
    return t.stride(0) if t.shape[0] > 1 else heads * B.HEAD_DIM


def _append_args(cfg: Config, k_new, v_new, page_table, seq_lens, rope, positions, cu_tokens, q, q_out):
    """Checks an append's arguments; returns (rows, rope, q_out, tensors to keep)."""
    kv, qt = B._TORCH_OF[cfg.kv_dtype], B._TORCH_OF[cfg.q_dtype]
    if k_new is None or k_new.dim() != 3:
        raise LocksError("k_new: expected [n_tokens][num_kv_heads][128]")
    n = int(k_new.shape[0])
    B._check_tables(cfg, page_table, seq_lens)
    if cu_tokens is not None:
        B._need("cu_tokens", cu_tokens, (cfg.num_seqs + 1,), torch.int32)
    elif n != cfg.num_seqs:
        raise LocksError(f"k_new: {n} rows without cu_tokens, expected one per sequence ({cfg.num_seqs})")
    _rows_tensor("k_new", k_new, n, cfg.num_kv_heads, kv)
    _rows_tensor("v_new", v_new, n, cfg.num_kv_heads, kv)
    if q is not None:
        _rows_tensor("q", q, n, cfg.num_q_heads, qt)
        if q_out is None:
            q_out = torch.empty(n, cfg.num_q_heads, B.HEAD_DIM, dtype=qt, device=q.device)
        _rows_tensor("q_out", q_out, n, cfg.num_q_heads, qt)
    elif q_out is not None:
        raise LocksError("q_out without q")
    r = None
    if rope is not None:
        t = rope.table
        if t.dtype != torch.float32 or t.dim() != 2:
            raise LocksError(f"rope.table: expected float32 [n_pos][rot_dim], got {t.dtype} {tuple(t.shape)}")
        axes = [int(t.shape[1]) // 2] if rope.axis_pairs is None else [int(a) for a in rope.axis_pairs]
        if not 1 <= len(axes) <= 3:
            raise LocksError(f"rope.axis_pairs: {len(axes)} axes, expected 1 to 3")
        if positions is not None:
            shape = (n,) if len(axes) == 1 and positions.dim() == 1 else (len(axes), n)
            B._need("positions", positions, shape, torch.int32)
        elif len(axes) > 1:
            raise LocksError("positions is required with several axes")
        r = _Rope(B._ptr(t), B._ptr(positions), int(t.shape[0]), int(t.shape[1]),
                  1 if rope.interleaved else 0, len(axes), (ctypes.c_int32 * 3)(*axes))
    elif positions is not None:
        raise LocksError("positions without rope")
    table = None if rope is None else rope.table
    keep = (k_new, v_new, page_table, seq_lens, cu_tokens, q, q_out, positions, table)
    _current_device(*keep)

    def at(t):
        return None if t is None else ctypes.c_void_p(t.data_ptr())
    rows = _Rows(at(q), at(k_new), at(v_new), at(q_out), B._ptr(cu_tokens),
                 0 if q is None else _stride(q, cfg.num_q_heads), _stride(k_new, cfg.num_kv_heads),
                 _stride(v_new, cfg.num_kv_heads), 0 if q is None else _stride(q_out, cfg.num_q_heads), n)
    return rows, r, q_out, keep


class _CacheCall(PreparedCall):
    """A PreparedCall that keeps its structures and tensors alive.  A call of one token costs
    the host more than the GPU, so the arguments are laid out once and the current stream is
    asked for as its raw handle (an append: 7.0 -> 4.2 us of host time)."""

    def __init__(self, fn, cfg_struct, args, outputs, keep):
        super().__init__(fn, cfg_struct, args, None, outputs)
        self._keep = keep
        self._all = (ctypes.byref(cfg_struct), *args)
        self._device = torch.cuda.current_device()

    def __call__(self, stream=None):
        if torch._C._cuda_getDevice() != self._device:
            raise LocksError(f"prepared on cuda:{self._device}, but the current device is "
                             f"cuda:{torch.cuda.current_device()}")
        raw = torch._C._cuda_getCurrentRawStream(self._device) if stream is None else stream.cuda_stream
        rc = self._fn(*self._all, raw)
        if rc:
            B._check(rc)


def prepare_rope_append_kv(cfg: Config, k_new, v_new, k_cache, v_cache, page_table, seq_lens,
                           rope: Optional[Rope] = None, positions=None, cu_tokens=None, q=None,
                           q_out=None) -> PreparedCall:
    """rope_append_kv's checks and marshalling, done once (see PreparedCall)."""
    rows, r, q_out, keep = _append_args(cfg, k_new, v_new, page_table, seq_lens, rope, positions,
                                        cu_tokens, q, q_out)
    B._check_cache(cfg, "k_cache", k_cache)
    B._check_cache(cfg, "v_cache", v_cache)
    B._same_device(k_new, k_cache, v_cache)
    args = (ctypes.byref(rows), None if r is None else ctypes.byref(r), B._ptr(k_cache), B._ptr(v_cache),
            B._ptr(page_table), B._ptr(seq_lens))
    return _CacheCall(lib().locks_rope_append_kv, cfg.c(), args, q_out, (rows, r, keep, k_cache, v_cache))


def rope_append_kv(cfg: Config, k_new, v_new, k_cache, v_cache, page_table, seq_lens,
                   rope: Optional[Rope] = None, positions=None, cu_tokens=None, q=None, q_out=None,
                   stream=None):
    """Rotate the new tokens' queries and keys by their positions and write keys and values
    into the paged caches -- locks_rope_append_kv.  k_new / v_new [n][H_kv][128], q
    [n][H_q][128] with any token stride; cu_tokens [S + 1] for ragged runs (one token per
    sequence without).  Returns the rotated queries (q_out; None without q)."""
    with _allocating_on(stream):
        call = prepare_rope_append_kv(cfg, k_new, v_new, k_cache, v_cache, page_table, seq_lens, rope,
                                      positions, cu_tokens, q, q_out)
    call(stream)
    return call.outputs


def prepare_q8_append_kv(cfg: Config, k_new, v_new, cache: Q8Cache, page_table, seq_lens,
                         rope: Optional[Rope] = None, positions=None, cu_tokens=None, q=None,
                         q_out=None) -> PreparedCall:
    """q8_append_kv's checks and marshalling, done once (see PreparedCall)."""
    rows, r, q_out, keep = _append_args(cfg, k_new, v_new, page_table, seq_lens, rope, positions,
                                        cu_tokens, q, q_out)
    store = _q8(cfg, cache)
    B._same_device(k_new, cache.k, cache.v, cache.k_scale, cache.v_scale)
    args = (ctypes.byref(rows), None if r is None else ctypes.byref(r), ctypes.byref(store),
            B._ptr(page_table), B._ptr(seq_lens))
    return _CacheCall(lib().locks_q8_append_kv, cfg.c(), args, q_out, (rows, r, store, keep, cache))


def q8_append_kv(cfg: Config, k_new, v_new, cache: Q8Cache, page_table, seq_lens,
                 rope: Optional[Rope] = None, positions=None, cu_tokens=None, q=None, q_out=None,
                 stream=None):
    """rope_append_kv into an 8-bit cache -- locks_q8_append_kv."""
    with _allocating_on(stream):
        call = prepare_q8_append_kv(cfg, k_new, v_new, cache, page_table, seq_lens, rope, positions,
                                    cu_tokens, q, q_out)
    call(stream)
    return call.outputs


def q8_build_summaries(cfg: Config, cache: Q8Cache, page_table, seq_lens, summaries,
                       build_list: Optional[torch.Tensor] = None, stream=None):
    """locks.build_summaries from the keys of an 8-bit cache -- locks_q8_build_summaries."""
    B._check_tables(cfg, page_table, seq_lens)
    B._check_summaries(cfg, summaries)
    B._check_list("build_list", build_list)
    if build_list is not None and build_list.shape[0] == 0:
        return                      # an empty list names no page (NULL would mean all)
    store = _q8(cfg, cache)
    _current_device(cache.k, cache.k_scale, page_table, seq_lens, summaries, build_list)
    c = cfg.c()
    B._check(lib().locks_q8_build_summaries(
        ctypes.byref(c), ctypes.byref(store), B._ptr(page_table), B._ptr(seq_lens), B._ptr(build_list),
        0 if build_list is None else int(build_list.shape[0]), B._ptr(summaries), B._stream(stream)))


def _prepare_attend(cfg, q, cache, page_table, seq_lens, page_ids, listed, ws, out, out_lse):
    if out is None:
        out, lse = B.alloc_attend_outputs(cfg, q.device)
        out_lse = lse if out_lse is None else out_lse
    B._check_q(cfg, q)
    B._check_tables(cfg, page_table, seq_lens)
    if listed:
        B._need("page_ids", page_ids, (cfg.num_seqs, cfg.num_kv_heads, cfg.k), torch.int32)
    B._check_ws(ws)
    B._check_attend_out(cfg, out, out_lse)
    store = _q8(cfg, cache)
    keep = (q, cache.k, cache.v, cache.k_scale, cache.v_scale, page_table, seq_lens, page_ids, ws, out, out_lse)
    _current_device(*keep)
    ids = (B._ptr(page_ids),) if listed else ()
    args = (B._ptr(q), ctypes.byref(store), B._ptr(page_table), B._ptr(seq_lens), *ids, B._ptr(out),
            B._ptr(out_lse), B._ptr(ws), ws.numel())
    fn = lib().locks_q8_sparse_attend if listed else lib().locks_q8_dense_attend
    return _CacheCall(fn, cfg.c(), args, (out, out_lse), (store, keep))


def prepare_q8_dense_attend(cfg: Config, q, cache: Q8Cache, page_table, seq_lens, ws, out=None,
                            out_lse=None) -> PreparedCall:
    """q8_dense_attend's checks and marshalling, done once (see PreparedCall)."""
    return _prepare_attend(cfg, q, cache, page_table, seq_lens, None, False, ws, out, out_lse)


def q8_dense_attend(cfg: Config, q, cache: Q8Cache, page_table, seq_lens, ws, out=None, out_lse=None,
                    stream=None):
    """Decode attention over every token of an 8-bit cache -- locks_q8_dense_attend."""
    with _allocating_on(stream):
        call = prepare_q8_dense_attend(cfg, q, cache, page_table, seq_lens, ws, out, out_lse)
    call(stream)
    return call.outputs


def prepare_q8_sparse_attend(cfg: Config, q, cache: Q8Cache, page_table, seq_lens, page_ids, ws,
                             out=None, out_lse=None) -> PreparedCall:
    """q8_sparse_attend's checks and marshalling, done once (see PreparedCall)."""
    return _prepare_attend(cfg, q, cache, page_table, seq_lens, page_ids, True, ws, out, out_lse)


def q8_sparse_attend(cfg: Config, q, cache: Q8Cache, page_table, seq_lens, page_ids, ws, out=None,
                     out_lse=None, stream=None):
    """Decode attention over the listed pages of an 8-bit cache (page_ids as select returns
    them) -- locks_q8_sparse_attend."""
    with _allocating_on(stream):
        call = prepare_q8_sparse_attend(cfg, q, cache, page_table, seq_lens, page_ids, ws, out, out_lse)
    call(stream)
    return call.outputs
