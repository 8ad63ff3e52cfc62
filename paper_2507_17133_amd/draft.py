"""Thin ctypes binding of the operators of a step with several new tokens of a sequence (see include/brownout_draft.h): attention with sinks, drafted
trees and prompts' chunks over a paged cache, the append of drafted tokens and the move of the accepted ones, log probabilities of given tokens.

As in `layer`: argument marshalling only, no fallback path; tensors on the current device, work on the current stream (`stream`: under that one);
no backward pass, a tensor that requires a gradient is refused unless gradients are off.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from .binding import MOE_OK, _check, lib
from .layer import (KvCache, Rope, _bytes, _heads, _ints, _like, _on, _rows, _table, _under, alloc_attention_workspace,
                    moe_block_table, moe_kv_cache, moe_rope)

MOE_LOGITS_BF16, MOE_LOGITS_FP32 = 0, 1
EXPORTS = ("moe_sink_attention", "moe_rope_append_at", "moe_tree_masks", "moe_tree_window_masks", "moe_chunk_workspace_size", "moe_chunk_attention",
           "moe_cache_move", "moe_logprob_workspace_size", "moe_token_logprobs")


class moe_chunk(C.Structure):
    _fields_ = [("first", C.c_void_p), ("context", C.c_void_p), ("seen", C.c_void_p), ("seen_stride", C.c_int64), ("positions", C.c_void_p),
                ("seen_words", C.c_int32), ("n_seqs", C.c_int32), ("T", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32)]


class moe_logprob_args(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("stride", C.c_int64), ("tokens", C.c_void_p), ("tokens_stride", C.c_int64), ("logprob", C.c_void_p),
                ("rank", C.c_void_p), ("lse", C.c_void_p), ("entropy", C.c_void_p), ("top_id", C.c_void_p), ("top_logprob", C.c_void_p),
                ("T", C.c_int32), ("V", C.c_int32), ("type", C.c_int32), ("n_given", C.c_int32), ("n_top", C.c_int32)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        L, p, i32, i64 = lib(), C.c_void_p, C.c_int32, C.c_int64
        cache, table, size = C.POINTER(moe_kv_cache), C.POINTER(moe_block_table), C.POINTER(C.c_size_t)
        for name, args in {
            "moe_sink_attention": [cache, table, p, i64, i32, i32, p, C.c_float, i32, i32, p, i64, p, p, C.c_size_t, p],
            "moe_rope_append_at": [cache, table, C.POINTER(moe_rope), p, i64, p, i64, p, i64, i32, i32, p, p, p, i64, p],
            "moe_tree_masks": [p, i32, i32, p, p],
            "moe_tree_window_masks": [p, i32, i32, i32, i32, p, p],
            "moe_chunk_workspace_size": [cache, i32, i32, i32, size],
            "moe_chunk_attention": [cache, table, C.POINTER(moe_chunk), p, i64, i32, C.c_float, p, i64, p, p, C.c_size_t, p],
            "moe_cache_move": [cache, table, p, i64, i32, p, p, i32, p],
            "moe_logprob_workspace_size": [i32, i32, i32, i32, size],
            "moe_token_logprobs": [C.POINTER(moe_logprob_args), p, C.c_size_t, p],
        }.items():
            f = getattr(L, name)
            f.restype, f.argtypes = i32, args
        _ready = L
    return _ready


def moe_sink_attention(cache: KvCache, q: torch.Tensor, block_table: torch.Tensor, lengths: torch.Tensor, window: int, sinks: int,
                       table_row: Optional[torch.Tensor] = None, scale: Optional[float] = None, out: Optional[torch.Tensor] = None, want_lse: bool = False,
                       workspace: Optional[torch.Tensor] = None, stream=None):
    """moe_paged_attention over the last `window` positions of each token's sequence (0: all) and the first `sinks` ones."""
    if stream is not None:
        return _under(stream, moe_sink_attention, cache, q, block_table, lengths, window, sinks, table_row, scale, out, want_lse, workspace)
    T, H = q.shape[:2]
    D = cache.dim
    if out is None:
        out, out_stride = _like(q), H * D
    else:
        out_stride = _heads(out, T, H, D)
    lse = q.new_empty((T, H), dtype=torch.float32) if want_lse else None
    if workspace is None:
        workspace = alloc_attention_workspace(cache, T, H)
    st = (_ready or _lib()).moe_sink_attention(
        cache.ref, C.byref(_table(block_table, table_row, T)), q.data_ptr(), _heads(q, T, H, D), H, T, _ints(lengths, T),
        D ** -0.5 if scale is None else scale, window, sinks, out.data_ptr(), out_stride, lse.data_ptr() if want_lse else None, *_bytes(workspace), _on(q))
    if st != MOE_OK:
        _check(st, "moe_sink_attention")
    return (out, lse) if want_lse else out


def moe_rope_append_at(cache: KvCache, rope: Rope, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, places: torch.Tensor,
                       block_table: torch.Tensor, table_row: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """moe_rope_append that turns by `positions` and writes k and v to `places` of the tokens' rows of block_table (negative: nowhere)."""
    if stream is not None:
        return _under(stream, moe_rope_append_at, cache, rope, q, k, v, positions, places, block_table, table_row, out)
    T, H = q.shape[:2]
    Hk, D = cache.heads, cache.dim
    if out is None:
        out, out_stride = _like(q), H * D
    else:
        out_stride = _heads(out, T, H, D)
    st = (_ready or _lib()).moe_rope_append_at(
        cache.ref, C.byref(_table(block_table, table_row, T)), rope.ref, q.data_ptr(), _heads(q, T, H, D), k.data_ptr(), _heads(k, T, Hk, D), v.data_ptr(),
        _heads(v, T, Hk, D), H, T, _ints(positions, T), _ints(places, T), out.data_ptr(), out_stride, _on(q))
    if st != MOE_OK:
        _check(st, "moe_rope_append_at")
    return out


def tree_masks(parents: Sequence[int], words: Optional[int] = None, window: int = 0, sinks: int = 0) -> Tuple[torch.Tensor, torch.Tensor]:
    """(seen [n, words] int32, depth [n] int32) on the CPU of a tree of n tokens; parents[i] < i, or -1 for the context's last token.  With a window, without the
    ancestors that it leaves out; `sinks`: positions behind the context that are sinks yet."""
    n = len(parents)
    words = (n + 31) // 32 if words is None else words
    seen, depth = torch.empty((n, words), dtype=torch.int32), torch.empty(n, dtype=torch.int32)
    up = torch.tensor(list(parents), dtype=torch.int32)
    _check(_lib().moe_tree_window_masks(up.data_ptr(), n, words, window, sinks, seen.data_ptr(), depth.data_ptr()), "moe_tree_window_masks")
    return seen, depth


def chunk_workspace_size(cache: KvCache, n_seqs: int, T: int, n_heads: int) -> int:
    n = C.c_size_t(0)
    _check(_lib().moe_chunk_workspace_size(cache.ref, n_seqs, T, n_heads, C.byref(n)), "moe_chunk_workspace_size")
    return n.value


def alloc_chunk_workspace(cache: KvCache, n_seqs: int, T: int, n_heads: int) -> torch.Tensor:
    """For every call of up to n_seqs sequences and T tokens."""
    return torch.empty(chunk_workspace_size(cache, n_seqs, T, n_heads), dtype=torch.uint8, device=cache.k.device)


def moe_chunk_attention(cache: KvCache, q: torch.Tensor, block_table: torch.Tensor, first: torch.Tensor, context: torch.Tensor,
                        table_row: Optional[torch.Tensor] = None, seen: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                        scale: Optional[float] = None, window: int = 0, sinks: int = 0, out: Optional[torch.Tensor] = None, want_lse: bool = False,
                        workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of q [T, heads, dim], sequence b's new tokens first[b] .. first[b + 1] - 1 behind context[b] cached positions (theirs are in the cache
    already, from position context[b] on).  seen None: each token sees what is before it, with a window and sinks; seen [T, words] int32: bits of the
    sequence's new tokens that it sees, as tree_masks gives them (for a window: with that), at `positions` (None: context + its number).  table_row: each sequence's row."""
    if stream is not None:
        return _under(stream, moe_chunk_attention, cache, q, block_table, first, context, table_row, seen, positions, scale, window, sinks, out, want_lse,
                      workspace)
    T, H = q.shape[:2]
    D, B = cache.dim, context.shape[0]
    words = seen_stride = 0
    if seen is not None:
        words = seen.shape[1]
        seen_stride = _rows(seen, torch.int32, T, words)
    if out is None:
        out, out_stride = _like(q), H * D
    else:
        out_stride = _heads(out, T, H, D)
    lse = q.new_empty((T, H), dtype=torch.float32) if want_lse else None
    if workspace is None:
        workspace = alloc_chunk_workspace(cache, B, T, H)
    a = moe_chunk(_ints(first, B + 1), _ints(context, B), None if seen is None else seen.data_ptr(), seen_stride,
                  None if positions is None else _ints(positions, T), words, B, T, window, sinks)
    st = (_ready or _lib()).moe_chunk_attention(
        cache.ref, C.byref(_table(block_table, table_row, B)), C.byref(a), q.data_ptr(), _heads(q, T, H, D), H, D ** -0.5 if scale is None else scale,
        out.data_ptr(), out_stride, lse.data_ptr() if want_lse else None, *_bytes(workspace), _on(q))
    if st != MOE_OK:
        _check(st, "moe_chunk_attention")
    return (out, lse) if want_lse else out


def moe_cache_move(cache: KvCache, block_table: torch.Tensor, sources: torch.Tensor, start: torch.Tensor, count: torch.Tensor,
                   table_row: Optional[torch.Tensor] = None, stream=None) -> None:
    """For each sequence b and j < count[b]: position sources[b, j] of the cache goes to position start[b] + j (sources [B, most] int32, increasing, none
    before its target).  table_row: each sequence's row of block_table."""
    if stream is not None:
        return _under(stream, moe_cache_move, cache, block_table, sources, start, count, table_row)
    B, most = sources.shape
    st = (_ready or _lib()).moe_cache_move(cache.ref, C.byref(_table(block_table, table_row, B)), sources.data_ptr(), _rows(sources, torch.int32, B, most), most,
                                           _ints(start, B), _ints(count, B), B, _on(sources))
    if st != MOE_OK:
        _check(st, "moe_cache_move")


class Logprobs(NamedTuple):
    logprob: Optional[torch.Tensor] = None    # [T][given] fp32
    rank: Optional[torch.Tensor] = None       # [T][given] int32
    lse: Optional[torch.Tensor] = None        # [T] fp32
    entropy: Optional[torch.Tensor] = None    # [T] fp32
    top_id: Optional[torch.Tensor] = None     # [T][top] int32
    top_logprob: Optional[torch.Tensor] = None  # [T][top] fp32


def alloc_logprobs(T: int, given: int, top: int, device="cuda") -> Logprobs:
    """What moe_token_logprobs takes as `out`: outputs that a program makes once."""
    f32, i32 = (dict(dtype=t, device=device) for t in (torch.float32, torch.int32))
    return Logprobs(torch.empty((T, given), **f32) if given else None, torch.empty((T, given), **i32) if given else None, torch.empty(T, **f32),
                    torch.empty(T, **f32), torch.empty((T, top), **i32) if top else None, torch.empty((T, top), **f32) if top else None)


def logprob_workspace_size(T: int, V: int, given: int, top: int) -> int:
    n = C.c_size_t(0)
    _check(_lib().moe_logprob_workspace_size(T, V, given, top, C.byref(n)), "moe_logprob_workspace_size")
    return n.value


def alloc_logprob_workspace(T: int, V: int, given: int, top: int, device="cuda") -> torch.Tensor:
    """For every call of up to T rows, V entries, and as many given tokens and alternatives."""
    return torch.empty(logprob_workspace_size(T, V, given, top), dtype=torch.uint8, device=device)


def _dense(t: Optional[torch.Tensor], dtype, *shape):
    if t is None:
        return None
    assert t.is_cuda and t.dtype is dtype and t.shape == shape and t.is_contiguous()
    return t.data_ptr()


def moe_token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0, workspace: Optional[torch.Tensor] = None,
                       out: Optional[Logprobs] = None, stream=None) -> Logprobs:
    """Of logits [T, V] (bf16 or fp32): log probabilities and ranks of `tokens` [T, given] int32 (outside [0, V): no token), log of the sum of exponentials,
    entropy, and the `top` best entries.  What `out` leaves None is not written."""
    if stream is not None:
        return _under(stream, moe_token_logprobs, logits, tokens, top, workspace, out)
    T, V = logits.shape
    f32, i32 = torch.float32, torch.int32
    fp32 = logits.dtype is f32
    G = tokens_stride = 0
    if tokens is not None:
        G = tokens.shape[1]
        tokens_stride = _rows(tokens, i32, T, G)
    if out is None:
        new = logits.new_empty
        out = Logprobs(new((T, G), dtype=f32) if G else None, new((T, G), dtype=i32) if G else None, new(T, dtype=f32), new(T, dtype=f32),
                       new((T, top), dtype=i32) if top else None, new((T, top), dtype=f32) if top else None)
        to = [None if t is None else t.data_ptr() for t in out]
    else:
        to = [_dense(out.logprob, f32, T, G), _dense(out.rank, i32, T, G), _dense(out.lse, f32, T), _dense(out.entropy, f32, T),
              _dense(out.top_id, i32, T, top), _dense(out.top_logprob, f32, T, top)]
    if workspace is None:
        workspace = alloc_logprob_workspace(T, V, G, top, logits.device)
    a = moe_logprob_args(logits.data_ptr(), _rows(logits, f32 if fp32 else torch.bfloat16, T, V), tokens.data_ptr() if G else None, tokens_stride,
                         *to, T, V, MOE_LOGITS_FP32 if fp32 else MOE_LOGITS_BF16, G, top)
    st = (_ready or _lib()).moe_token_logprobs(C.byref(a), *_bytes(workspace), _on(logits))
    if st != MOE_OK:
        _check(st, "moe_token_logprobs")
    return out
