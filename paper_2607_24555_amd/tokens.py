"""Thin ctypes binding of the calls of liblocks on single tokens of the paged cache
(include/locks_tokens.h): attention of several new tokens of a sequence, the attention mass
of every cached token, the tokens to keep by it, and kept tokens moved together.

As in `cache`: argument checks and marshalling only, tensors are torch device tensors on the
current device, work goes to the given or current stream, and the prepare_* forms do the
checks once for loops over fixed buffers.

Speculative decoding over a paged cache:

    mask, depth = tree_mask(parents, cu_tokens)
    # past [num_seqs]: tokens cached before; seq [n]: the sequence of each new token
    q = cache.rope_append_kv(cfg, k, v, k_cache, v_cache, page_table, seq_lens, rope,
                             positions=past[seq] + depth, cu_tokens=cu, q=q)
    out, lse = tree_attend(cfg, q, k_cache, v_cache, page_table, seq_lens, ws, cu_tokens=cu, mask=mask)
    # ... the caller accepts a branch: its tokens' indices in `kept`, padded with -1
    keep_tokens(cfg, kept, k_cache, v_cache, page_table, start=past, out_lens=seq_lens)

A cache of bounded size:

    out, lse = locks.dense_attend(cfg, q, k_cache, v_cache, page_table, seq_lens, ws)
    token_mass(cfg, q, lse, k_cache, page_table, seq_lens, mass, decay=0.98)
    # ... when it is full
    kept = pick_tokens(cfg, mass, seq_lens, n_keep, n_sink, n_recent, pick_ws)
    keep_tokens(cfg, kept, k_cache, v_cache, page_table, mass=mass, out_lens=seq_lens)
"""
from __future__ import annotations

import ctypes
from typing import Sequence

import torch

from . import cache as C
from . import locks as B
from .locks import Config, LocksError, PreparedCall, _Cfg


class _Draft(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("cu_tokens", ctypes.c_void_p), ("mask", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("n_tokens", ctypes.c_int32),
                ("mask_words", ctypes.c_int32)]


_P, _SZ, _I, _F = B._P, B._SZ, B._I, ctypes.c_float
_PC, _PD = ctypes.POINTER(_Cfg), ctypes.POINTER(_Draft)
_SIGS = {
    "locks_tree_workspace_bytes": (_SZ, [_PC, _I]),
    "locks_tree_attend": (ctypes.c_int, [_PC, _PD, _P, _P, _P, _P, _P, _I, _P, _P, _SZ, _P]),
    "locks_token_mass": (ctypes.c_int, [_PC, _PD, _P, _P, _P, _P, _F, _P, _P]),
    "locks_pick_workspace_bytes": (_SZ, [_PC]),
    "locks_pick_tokens": (ctypes.c_int, [_PC, _P, _P, _I, _I, _I, _P, _P, _SZ, _P]),
    "locks_keep_tokens": (ctypes.c_int, [_PC, _P, _I, _I, _P, _P, _P, _P, _P, _P, _P]),
}
_DTYPE_OF = {torch.bfloat16: B.LOCKS_BF16, torch.float32: B.LOCKS_FP32}
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


def tree_workspace_bytes(cfg: Config, n_tokens: int) -> int:
    """locks_tree_workspace_bytes."""
    c = cfg.c()
    n = int(lib().locks_tree_workspace_bytes(ctypes.byref(c), n_tokens))
    if n == 0:
        raise LocksError("invalid configuration or token count")
    return n


def alloc_tree_workspace(cfg: Config, n_tokens: int, device="cuda") -> torch.Tensor:
    """A workspace of tree_attend for up to n_tokens new tokens of up to cfg.num_seqs sequences."""
    return torch.empty(tree_workspace_bytes(cfg, n_tokens), dtype=torch.uint8, device=device)


def alloc_pick_workspace(cfg: Config, device="cuda") -> torch.Tensor:
    """A workspace of pick_tokens for up to cfg.num_seqs sequences."""
    c = cfg.c()
    n = int(lib().locks_pick_workspace_bytes(ctypes.byref(c)))
    if n == 0:
        raise LocksError("invalid configuration")
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_mass(cfg: Config, device="cuda") -> torch.Tensor:
    """Zero mass for every token that the page tables can hold."""
    return torch.zeros(cfg.num_seqs, cfg.num_kv_heads, cfg.max_pages_per_seq * cfg.page_size,
                       dtype=torch.float32, device=device)


def tree_mask(parents: Sequence[int], cu_tokens: Sequence[int], device="cuda"):
    """The mask [n][words] (int32) and depths [n] (int32) of drafted trees: parents[r] is the
    index, among its sequence's new tokens, of row r's parent, an earlier one, or -1 where it
    follows the cached tokens themselves; cu_tokens as tree_attend takes it, on the host.  A loop
    on the host and a copy that waits (8 trees of 48 tokens 0.6 to 1.2 ms, 64 of 64 17 to 30), for
    trees that keep their shape over many steps; where they change with each one, its caller
    builds the mask beside them."""
    parents, cu = [int(p) for p in parents], [int(c) for c in cu_tokens]
    if not cu or cu[0] != 0 or cu[-1] != len(parents) or any(a > b for a, b in zip(cu, cu[1:])):
        raise LocksError("cu_tokens: expected ascending row counts from 0 to the number of parents")
    words = max(1, -(-max([b - a for a, b in zip(cu, cu[1:])] or [1]) // 32))
    bits, depth = [], []
    for a, b in zip(cu, cu[1:]):
        for i, p in enumerate(parents[a:b]):
            if not -1 <= p < i:
                raise LocksError(f"parents[{a + i}] = {p}: expected -1 or one of its sequence's {i} tokens before it")
            bits.append((bits[a + p] if p >= 0 else 0) | 1 << i)
            depth.append(depth[a + p] + 1 if p >= 0 else 0)
    flat = [[x >> (32 * w) & 0xffffffff for w in range(words)] for x in bits]
    mask = torch.tensor([[v - (1 << 32) if v >> 31 else v for v in row] for row in flat],
                        dtype=torch.int32).reshape(len(parents), words)
    return mask.to(device), torch.tensor(depth, dtype=torch.int32, device=device)


def _draft(cfg: Config, q, page_table, seq_lens, cu_tokens, mask):
    """Checks the new tokens; returns (draft, n, tensors to keep)."""
    if q is None or q.dim() != 3:
        raise LocksError("q: expected [n_tokens][num_q_heads][128]")
    n = int(q.shape[0])
    B._check_tables(cfg, page_table, seq_lens)
    if cu_tokens is not None:
        B._need("cu_tokens", cu_tokens, (cfg.num_seqs + 1,), torch.int32)
    elif n != cfg.num_seqs:
        raise LocksError(f"q: {n} rows without cu_tokens, expected one per sequence ({cfg.num_seqs})")
    C._rows_tensor("q", q, n, cfg.num_q_heads, B._TORCH_OF[cfg.q_dtype])
    words = 0
    if mask is not None:
        if mask.dim() != 2 or mask.shape[1] < 1:
            raise LocksError(f"mask: shape {tuple(mask.shape)}, expected [n_tokens][words]")
        words = int(mask.shape[1])
        B._need("mask", mask, (n, words), torch.int32)
    keep = (q, page_table, seq_lens, cu_tokens, mask)
    C._current_device(*keep)
    return _Draft(ctypes.c_void_p(q.data_ptr()), B._ptr(cu_tokens), B._ptr(mask), C._stride(q, cfg.num_q_heads),
                  n, words), n, keep


def prepare_tree_attend(cfg: Config, q, k_cache, v_cache, page_table, seq_lens, ws, cu_tokens=None,
                        mask=None, out=None, out_lse=None) -> PreparedCall:
    """tree_attend's checks and marshalling, done once (see PreparedCall)."""
    draft, n, keep = _draft(cfg, q, page_table, seq_lens, cu_tokens, mask)
    B._check_cache(cfg, "k_cache", k_cache)
    B._check_cache(cfg, "v_cache", v_cache)
    B._check_ws(ws)
    if out is None:
        out = torch.empty(n, cfg.num_q_heads, B.HEAD_DIM, dtype=torch.float32, device=q.device)
    if out_lse is None:
        out_lse = torch.empty(n, cfg.num_q_heads, dtype=torch.float32, device=q.device)
    if out.dtype not in _DTYPE_OF:
        raise LocksError(f"out: dtype {out.dtype}, expected torch.float32 or torch.bfloat16")
    B._need("out", out, (n, cfg.num_q_heads, B.HEAD_DIM), out.dtype)
    B._need("out_lse", out_lse, (n, cfg.num_q_heads), torch.float32)
    keep += (k_cache, v_cache, ws, out, out_lse)
    C._current_device(*keep)
    args = (ctypes.byref(draft), B._ptr(k_cache), B._ptr(v_cache), B._ptr(page_table), B._ptr(seq_lens),
            B._ptr(out), _DTYPE_OF[out.dtype], B._ptr(out_lse), B._ptr(ws), ws.numel())
    return C._CacheCall(lib().locks_tree_attend, cfg.c(), args, (out, out_lse), (draft, keep))


def tree_attend(cfg: Config, q, k_cache, v_cache, page_table, seq_lens, ws, cu_tokens=None, mask=None,
                out=None, out_lse=None, stream=None):
    """Attention of every new token over the cached ones and those of the new ones that it
    sees -- locks_tree_attend.  q [n][H_q][128] with any token stride, mask [n][words] int32
    (tree_mask makes one; a run without), out float32 (the default) or bfloat16.  Returns
    (out, out_lse)."""
    with C._allocating_on(stream):
        call = prepare_tree_attend(cfg, q, k_cache, v_cache, page_table, seq_lens, ws, cu_tokens, mask, out,
                                   out_lse)
    call(stream)
    return call.outputs


def _check_mass(cfg: Config, mass):
    B._need("mass", mass, (cfg.num_seqs, cfg.num_kv_heads, cfg.max_pages_per_seq * cfg.page_size),
            torch.float32)


def prepare_token_mass(cfg: Config, q, lse, k_cache, page_table, seq_lens, mass, cu_tokens=None,
                       mask=None, decay: float = 1.0) -> PreparedCall:
    """token_mass's checks and marshalling, done once (see PreparedCall)."""
    draft, n, keep = _draft(cfg, q, page_table, seq_lens, cu_tokens, mask)
    B._need("lse", lse, (n, cfg.num_q_heads), torch.float32)
    B._check_cache(cfg, "k_cache", k_cache)
    _check_mass(cfg, mass)
    keep += (lse, k_cache, mass)
    C._current_device(*keep)
    args = (ctypes.byref(draft), B._ptr(lse), B._ptr(k_cache), B._ptr(page_table), B._ptr(seq_lens),
            float(decay), B._ptr(mass))
    return C._CacheCall(lib().locks_token_mass, cfg.c(), args, mass, (draft, keep))


def token_mass(cfg: Config, q, lse, k_cache, page_table, seq_lens, mass, cu_tokens=None, mask=None,
               decay: float = 1.0, stream=None):
    """Add to `mass` (alloc_mass), in place, the attention weight that every token gets from
    the new ones -- locks_token_mass.  lse [n][H_q] as the attention returned it.  Returns
    mass."""
    call = prepare_token_mass(cfg, q, lse, k_cache, page_table, seq_lens, mass, cu_tokens, mask, decay)
    call(stream)
    return call.outputs


def prepare_pick_tokens(cfg: Config, mass, seq_lens, n_keep: int, n_sink: int, n_recent: int, ws,
                        out=None) -> PreparedCall:
    """pick_tokens' checks and marshalling, done once (see PreparedCall)."""
    _check_mass(cfg, mass)
    B._need("seq_lens", seq_lens, (cfg.num_seqs,), torch.int32)
    B._check_ws(ws)
    if out is None:
        out = torch.empty(cfg.num_seqs, cfg.num_kv_heads, max(0, n_keep), dtype=torch.int32, device=mass.device)
    B._need("out", out, (cfg.num_seqs, cfg.num_kv_heads, n_keep), torch.int32)
    keep = (mass, seq_lens, ws, out)
    C._current_device(*keep)
    args = (B._ptr(mass), B._ptr(seq_lens), n_keep, n_sink, n_recent, B._ptr(out), B._ptr(ws), ws.numel())
    return C._CacheCall(lib().locks_pick_tokens, cfg.c(), args, out, keep)


def pick_tokens(cfg: Config, mass, seq_lens, n_keep: int, n_sink: int, n_recent: int, ws, out=None,
                stream=None):
    """The tokens of every sequence and KV head to keep, ascending, padded with -1
    ([S][H_kv][n_keep] int32): the first n_sink, the last n_recent and the others of largest
    mass -- locks_pick_tokens."""
    with C._allocating_on(stream):
        call = prepare_pick_tokens(cfg, mass, seq_lens, n_keep, n_sink, n_recent, ws, out)
    call(stream)
    return call.outputs


def prepare_keep_tokens(cfg: Config, kept, k_cache, v_cache, page_table, start=None, mass=None,
                        out_lens=None) -> PreparedCall:
    """keep_tokens' checks and marshalling, done once (see PreparedCall)."""
    if kept is None or kept.dim() != 3 or kept.shape[1] not in (1, cfg.num_kv_heads):
        raise LocksError("kept: expected [num_seqs][num_kv_heads or 1][n_keep]")
    B._need("kept", kept, (cfg.num_seqs, kept.shape[1], kept.shape[2]), torch.int32)
    B._check_cache(cfg, "k_cache", k_cache)
    B._check_cache(cfg, "v_cache", v_cache)
    B._need("page_table", page_table, (cfg.num_seqs, cfg.max_pages_per_seq), torch.int32)
    B._need("start", start, (cfg.num_seqs,), torch.int32, optional=True)
    if mass is not None:
        _check_mass(cfg, mass)
    if out_lens is None:
        out_lens = torch.empty(cfg.num_seqs, dtype=torch.int32, device=kept.device)
    B._need("out_lens", out_lens, (cfg.num_seqs,), torch.int32)
    keep = (kept, k_cache, v_cache, page_table, start, mass, out_lens)
    C._current_device(*keep)
    args = (B._ptr(kept), int(kept.shape[1]), int(kept.shape[2]), B._ptr(start), B._ptr(k_cache), B._ptr(v_cache),
            B._ptr(mass), B._ptr(page_table), B._ptr(out_lens))
    return C._CacheCall(lib().locks_keep_tokens, cfg.c(), args, out_lens, keep)


def keep_tokens(cfg: Config, kept, k_cache, v_cache, page_table, start=None, mass=None, out_lens=None,
                stream=None):
    """Move the kept tokens' rows (and mass) together, in place, behind token `start` of each
    sequence (0 without) -- locks_keep_tokens.  kept [S][H_kv or 1][n] as pick_tokens returns
    it.  Returns the new lengths (out_lens, which may be seq_lens)."""
    with C._allocating_on(stream):
        call = prepare_keep_tokens(cfg, kept, k_cache, v_cache, page_table, start, mass, out_lens)
    call(stream)
    return call.outputs
