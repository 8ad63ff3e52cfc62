"""Thin ctypes binding of the operators around the MoE layer (see include/brownout_layer.h): the norm with its residual and
8-bit output, the 8-bit linear layer, rotary positions with the append to a paged key-value cache, attention over it.

Like `binding`: argument marshalling only, no fallback path.  Tensors are on the current device; work goes to the
current stream.  A call with `stream` is the same call under torch.cuda.stream(stream): what it allocates belongs to that stream.
Tensors of other streams are the caller's to order before it, and to keep until it has run (Tensor.record_stream).
There is no backward pass: a tensor that requires a gradient is refused unless gradients are off (torch.no_grad).
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import NamedTuple, Optional, Tuple

import torch

from .binding import MOE_OK, _check, _ptr, lib

E4M3 = torch.float8_e4m3fn
MOE_KV_BF16, MOE_KV_E4M3 = 0, 1
MOE_ERR_WORKSPACE = -4
NO_BACKWARD = "these operators have no backward pass: call them under torch.no_grad()"
ROPE_SCALINGS = ("none", "linear", "ntk", "yarn")
EXPORTS = ("moe_rms_norm", "moe_quantize_rows", "moe_quantize_weight", "moe_linear_workspace_size", "moe_linear_workspace_bound",
           "moe_linear_e4m3", "moe_rope_frequencies", "moe_rope_append", "moe_attention_workspace_size", "moe_paged_attention")


class moe_norm_args(C.Structure):
    _fields_ = [("x", C.c_void_p), ("x_stride", C.c_int64), ("residual", C.c_void_p), ("residual_stride", C.c_int64),
                ("weight", C.c_void_p), ("residual_out", C.c_void_p), ("residual_out_stride", C.c_int64),
                ("y", C.c_void_p), ("y_stride", C.c_int64), ("y8", C.c_void_p), ("y8_stride", C.c_int64),
                ("scale", C.c_void_p), ("scale_stride", C.c_int64), ("T", C.c_int32), ("d", C.c_int32), ("eps", C.c_float)]


class moe_linear_args(C.Structure):
    _fields_ = [("x8", C.c_void_p), ("x_stride", C.c_int64), ("x_scale", C.c_void_p), ("x_scale_stride", C.c_int64),
                ("w8", C.c_void_p), ("w_scale", C.c_void_p), ("out", C.c_void_p), ("out_stride", C.c_int64),
                ("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32), ("exact", C.c_int32)]


class moe_kv_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64), ("token_stride", C.c_int64),
                ("head_stride", C.c_int64), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("type", C.c_int32),
                ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class moe_block_table(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("row_stride", C.c_int64), ("token_row", C.c_void_p), ("n_rows", C.c_int32),
                ("max_pages", C.c_int32)]


class moe_rope(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("factor", C.c_float)]


class moe_rope_scaling(C.Structure):
    _fields_ = [("kind", C.c_int32), ("factor", C.c_double), ("original_length", C.c_double), ("beta_fast", C.c_double),
                ("beta_slow", C.c_double)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        L, p, i32, i64 = lib(), C.c_void_p, C.c_int32, C.c_int64
        size = C.POINTER(C.c_size_t)
        for name, args in {
            "moe_rms_norm": [C.POINTER(moe_norm_args), p],
            "moe_quantize_rows": [C.POINTER(moe_norm_args), p],
            "moe_quantize_weight": [p, i32, i32, p, p, p],
            "moe_linear_workspace_size": [i32, i32, i32, size],
            "moe_linear_workspace_bound": [i32, i32, i32, size],
            "moe_linear_e4m3": [C.POINTER(moe_linear_args), p, C.c_size_t, p],
            "moe_rope_frequencies": [i32, C.c_double, C.POINTER(moe_rope_scaling), C.POINTER(C.c_double), C.POINTER(C.c_float)],
            "moe_rope_append": [C.POINTER(moe_kv_cache), C.POINTER(moe_block_table), C.POINTER(moe_rope), p, i64, p, i64, p, i64,
                                i32, i32, p, p, i64, p],
            "moe_attention_workspace_size": [C.POINTER(moe_kv_cache), i32, i32, size],
            "moe_paged_attention": [C.POINTER(moe_kv_cache), C.POINTER(moe_block_table), p, i64, i32, i32, p, C.c_float, i32, p,
                                    i64, p, p, C.c_size_t, p],
        }.items():
            f = getattr(L, name)
            f.restype, f.argtypes = i32, args
        _ready = L
    return _ready


# The calls below are a few microseconds of GPU time for a single token, so the Python around them is kept short: a raw stream handle (a
# torch.cuda.Stream object costs as much as a launch), no checks of what was allocated here, no error path on the way to success.
_current_stream = torch._C._cuda_getCurrentRawStream


def _on(t: torch.Tensor):
    return _current_stream(t.get_device())


def _under(stream, call, *args):
    with torch.cuda.stream(stream):
        return call(*args)


def _rows(t: torch.Tensor, dtype, rows: int, cols: int):
    """A [rows, cols] tensor whose rows are contiguous; returns its row stride."""
    assert t.is_cuda and t.dtype is dtype and t.shape == (rows, cols)
    assert not (t.requires_grad and torch.is_grad_enabled()), NO_BACKWARD
    if t.is_contiguous():
        return cols
    assert cols == 1 or t.stride(1) == 1
    return t.stride(0)


def _bytes(workspace: torch.Tensor):
    """Where a workspace is and how large."""
    assert workspace.is_cuda and workspace.is_contiguous()
    return workspace.data_ptr(), workspace.nbytes


def _like(t: torch.Tensor, dtype=torch.bfloat16) -> torch.Tensor:
    return torch.empty_like(t, dtype=dtype) if t.is_contiguous() else t.new_empty(t.shape, dtype=dtype)


def _groups(d: int) -> int:
    return (d + 127) // 128


# ---------------------------------------------------------------- norm, 8-bit rows and weights

class NormOut(NamedTuple):
    y: Optional[torch.Tensor] = None          # [T][d] bf16
    y8: Optional[torch.Tensor] = None         # [T][d] e4m3
    scale: Optional[torch.Tensor] = None      # [ceil(d/128)][T] fp32
    residual: Optional[torch.Tensor] = None   # [T][d] bf16


def alloc_norm_out(T: int, d: int, want=("y",), residual: bool = False, device="cuda") -> NormOut:
    """What moe_rms_norm and moe_quantize_rows take as `out`: outputs that a program makes once."""
    bf, f32 = torch.bfloat16, torch.float32
    q = "y8" in want
    return NormOut(torch.empty((T, d), dtype=bf, device=device) if "y" in want else None,
                   torch.empty((T, d), dtype=E4M3, device=device) if q else None,
                   torch.empty(((d + 127) // 128, T), dtype=f32, device=device) if q else None,
                   torch.empty((T, d), dtype=bf, device=device) if residual else None)


def _norm(call, x, weight, eps, residual, want, out) -> NormOut:
    T, d = x.shape
    bf = torch.bfloat16
    xs, xp = _rows(x, bf, T, d), x.data_ptr()
    r = rs = w = y = ys = y8 = y8s = s = ss = ro = ros = None
    if residual is not None:
        r, rs = residual.data_ptr(), _rows(residual, bf, T, d)
    if weight is not None:
        assert weight.is_cuda and weight.dtype is bf and weight.shape == (d,) and weight.is_contiguous()
        assert not (weight.requires_grad and torch.is_grad_enabled()), NO_BACKWARD
        w = weight.data_ptr()
    if out is None:
        q = "y8" in want
        out = NormOut(_like(x) if "y" in want else None, _like(x, E4M3) if q else None,
                      x.new_empty(((d + 127) // 128, T), dtype=torch.float32) if q else None,
                      _like(x) if residual is not None else None)
        ys = y8s = ros = d
        ss = T
    else:
        if out.y is not None:
            ys = _rows(out.y, bf, T, d)
        if out.y8 is not None:
            y8s, ss = _rows(out.y8, E4M3, T, d), _rows(out.scale, torch.float32, (d + 127) // 128, T)
        if out.residual is not None:
            ros = _rows(out.residual, bf, T, d)
    if out.y is not None:
        y = out.y.data_ptr()
    if out.y8 is not None:
        y8, s = out.y8.data_ptr(), out.scale.data_ptr()
    if out.residual is not None:
        ro = out.residual.data_ptr()
    st = call(C.byref(moe_norm_args(xp, xs, r, rs or 0, w, ro, ros or 0, y, ys or 0, y8, y8s or 0, s, ss or 0, T, d, eps)), _on(x))
    if st != MOE_OK:
        _check(st, call.__name__)
    return out


def moe_rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor], eps: float = 1e-6, residual: Optional[torch.Tensor] = None,
                 want=("y",), out: Optional[NormOut] = None, stream=None) -> NormOut:
    """Norm of x + residual; `want`: "y" (bf16), "y8" (e4m3 with scales), or both.  The sum comes back as `residual` if one was given."""
    if stream is not None:
        return _under(stream, moe_rms_norm, x, weight, eps, residual, want, out)
    return _norm((_ready or _lib()).moe_rms_norm, x, weight, eps, residual, want, out)


def moe_quantize_rows(x: torch.Tensor, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream=None):
    """(x8 [T][d] e4m3, scale [ceil(d/128)][T])."""
    if stream is not None:
        return _under(stream, moe_quantize_rows, x, out)
    o = _norm((_ready or _lib()).moe_quantize_rows, x, None, 0.0, None, ("y8",), None if out is None else NormOut(y8=out[0], scale=out[1]))
    return o.y8, o.scale


def moe_quantize_weight(w: torch.Tensor, stream=None):
    """(w8 [N][K] e4m3, w_scale [ceil(N/128)][ceil(K/128)]) of a bf16 weight [N][K]."""
    if stream is not None:
        return _under(stream, moe_quantize_weight, w)
    N, K = w.shape
    assert w.is_cuda and w.dtype is torch.bfloat16 and w.is_contiguous()
    assert not (w.requires_grad and torch.is_grad_enabled()), NO_BACKWARD
    w8 = torch.empty((N, K), dtype=E4M3, device=w.device)
    scale = torch.empty((_groups(N), _groups(K)), dtype=torch.float32, device=w.device)
    _check(_lib().moe_quantize_weight(_ptr(w), N, K, _ptr(w8), _ptr(scale), _on(w)), "moe_quantize_weight")
    return w8, scale


def linear_workspace_size(M: int, N: int, K: int) -> int:
    """Bytes for exactly this product; not monotone in M."""
    n = C.c_size_t(0)
    _check(_lib().moe_linear_workspace_size(M, N, K, C.byref(n)), "moe_linear_workspace_size")
    return n.value


def linear_workspace_bound(M_max: int, N: int, K: int) -> int:
    """Bytes for every product of up to M_max rows."""
    n = C.c_size_t(0)
    _check(_lib().moe_linear_workspace_bound(M_max, N, K, C.byref(n)), "moe_linear_workspace_bound")
    return n.value


def alloc_linear_workspace(M: int, N: int, K: int, device="cuda") -> torch.Tensor:
    """A workspace for every product of up to M rows with a weight [N, K]."""
    return torch.empty(linear_workspace_bound(M, N, K), dtype=torch.uint8, device=device)


def moe_linear_e4m3(x8: torch.Tensor, x_scale: torch.Tensor, w8: torch.Tensor, w_scale: torch.Tensor, out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None, exact: bool = False) -> torch.Tensor:
    """x8 * x_scale times (w8 * w_scale) transposed, [M, N] bf16.  Beyond K = 512 the 8-bit matrix instructions cut products off at 2^-13 of the largest
    of 8 neighbouring columns, which shows where a column is far larger than the rest; `exact`: products in full, sums in fp32, for up to 2.2 times the time."""
    if stream is not None:
        return _under(stream, moe_linear_e4m3, x8, x_scale, w8, w_scale, out, workspace, None, exact)
    M, K = x8.shape
    N = w8.shape[0]
    G = (K + 127) // 128
    assert w8.is_cuda and w8.dtype is E4M3 and w8.shape[1] == K and w8.is_contiguous()
    assert w_scale.is_cuda and w_scale.dtype is torch.float32 and w_scale.shape == (_groups(N), G) and w_scale.is_contiguous()
    assert not ((w8.requires_grad or w_scale.requires_grad) and torch.is_grad_enabled()), NO_BACKWARD
    L = _ready or _lib()
    if out is None:
        out, out_stride = x8.new_empty((M, N), dtype=torch.bfloat16), N
    else:
        out_stride = _rows(out, torch.bfloat16, M, N)
    a = moe_linear_args(x8.data_ptr(), _rows(x8, E4M3, M, K), x_scale.data_ptr(), _rows(x_scale, torch.float32, G, M), w8.data_ptr(),
                        w_scale.data_ptr(), out.data_ptr(), out_stride, M, N, K, 1 if exact else 0)
    st = L.moe_linear_e4m3(C.byref(a), *((None, 0) if workspace is None else _bytes(workspace)), _on(x8))
    if st == MOE_ERR_WORKSPACE and workspace is None:      # most products need none
        workspace = x8.new_empty(linear_workspace_size(M, N, K), dtype=torch.uint8)
        st = L.moe_linear_e4m3(C.byref(a), *_bytes(workspace), _on(x8))
    if st != MOE_OK:
        _check(st, "moe_linear_e4m3")
    return out


# ---------------------------------------------------------------- paged cache, rotary positions, attention

class KvCache:
    """k and v of a paged cache as [page, token, head, head_dim] tensors or views of one (head by head pages: a transposed view)
    with equal strides, bf16 or e4m3 (then with k_scale and v_scale [head] fp32)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None):
        e4m3 = k.dtype == E4M3
        assert k.is_cuda and v.is_cuda and k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype
        assert k.stride(3) == 1 and (e4m3 or k.dtype == torch.bfloat16)
        assert not ((k.requires_grad or v.requires_grad) and torch.is_grad_enabled()), NO_BACKWARD
        for s in (k_scale, v_scale):
            assert (s is not None) == e4m3, "scales belong to an e4m3 cache, and only to one"
            assert s is None or (s.is_cuda and s.dtype == torch.float32 and s.shape == (k.shape[2],) and s.is_contiguous())
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        n, page, heads, dim = k.shape
        self.struct = moe_kv_cache(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2),
                                   None if k_scale is None else k_scale.data_ptr(), None if v_scale is None else v_scale.data_ptr(),
                                   MOE_KV_E4M3 if e4m3 else MOE_KV_BF16, n, page, heads, dim)
        self.heads, self.dim, self.ref = heads, dim, C.byref(self.struct)


def alloc_kv_cache(n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, k_scale=None, v_scale=None, heads_first: bool = False,
                   device="cuda") -> KvCache:
    """An empty cache; e4m3 if scales are given.  heads_first: pages are stored head by head."""
    dtype = torch.bfloat16 if k_scale is None else E4M3
    shape = (n_pages, n_kv_heads, page_size, head_dim) if heads_first else (n_pages, page_size, n_kv_heads, head_dim)
    k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
    return KvCache(k.transpose(1, 2), v.transpose(1, 2), k_scale, v_scale) if heads_first else KvCache(k, v, k_scale, v_scale)


def _table(block_table: torch.Tensor, table_row: Optional[torch.Tensor], T: int) -> moe_block_table:
    rows, pages = block_table.shape
    return moe_block_table(block_table.data_ptr(), _rows(block_table, torch.int32, rows, pages), None if table_row is None else _ints(table_row, T), rows, pages)


def rope_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original_length: float = 0.0,
                     beta_fast: float = 32.0, beta_slow: float = 1.0) -> Tuple[torch.Tensor, float]:
    """Whole turns per position of each pair (CPU, fp64 [rotary_dim/2]) and the factor on cos and sin."""
    turns = (C.c_double * max(rotary_dim // 2, 1))()
    f = C.c_float(0.0)
    s = moe_rope_scaling(ROPE_SCALINGS.index(scaling), factor, original_length, beta_fast, beta_slow)
    _check(_lib().moe_rope_frequencies(rotary_dim, base, C.byref(s), turns, C.byref(f)), "moe_rope_frequencies")
    return torch.tensor(list(turns), dtype=torch.float64), float(f.value)


@dataclass
class Rope:
    """Rotary positions of a model: turns on the device, as rope_frequencies gives them."""
    turns: Optional[torch.Tensor]
    rotary_dim: int
    interleaved: bool = False
    factor: float = 1.0

    def __post_init__(self):
        if self.rotary_dim:
            assert self.turns.is_cuda and self.turns.dtype == torch.float64 and self.turns.shape == (self.rotary_dim // 2,)
            assert self.turns.is_contiguous()
        self.struct = moe_rope(self.turns.data_ptr() if self.rotary_dim else None, self.rotary_dim, 1 if self.interleaved else 0, self.factor)
        self.ref = C.byref(self.struct)


def make_rope(rotary_dim: int, interleaved: bool = False, device="cuda", **frequencies) -> Rope:
    """Rope of rope_frequencies(rotary_dim, **frequencies)."""
    turns, factor = rope_frequencies(rotary_dim, **frequencies)
    return Rope(turns.to(device), rotary_dim, interleaved, factor)


def _heads(t: torch.Tensor, T: int, heads: int, dim: int) -> int:
    """A [T, heads, dim] tensor whose heads are next to each other; returns its token stride."""
    assert t.is_cuda and t.dtype is torch.bfloat16 and t.shape == (T, heads, dim)
    assert not (t.requires_grad and torch.is_grad_enabled()), NO_BACKWARD
    if t.is_contiguous():
        return heads * dim
    stride = t.stride()
    assert stride[2] == 1 and (heads == 1 or stride[1] == dim)
    return stride[0]


def _ints(t: torch.Tensor, T: int):
    assert t.is_cuda and t.dtype is torch.int32 and t.shape == (T,) and t.is_contiguous()
    return t.data_ptr()


def moe_rope_append(cache: KvCache, rope: Rope, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor,
                    block_table: torch.Tensor, table_row: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """Rotates q [T, heads, dim] and k [T, kv heads, dim] (views of one projection's output as they are), writes k and v to the cache at
    `positions` of the tokens' rows of block_table (table_row; None: row t), and returns the rotated q (`out`; may be q)."""
    if stream is not None:
        return _under(stream, moe_rope_append, cache, rope, q, k, v, positions, block_table, table_row, out)
    T, H = q.shape[:2]
    Hk, D = cache.heads, cache.dim
    if out is None:
        out, out_stride = _like(q), H * D
    else:
        out_stride = _heads(out, T, H, D)
    st = (_ready or _lib()).moe_rope_append(
        cache.ref, C.byref(_table(block_table, table_row, T)), rope.ref, q.data_ptr(), _heads(q, T, H, D), k.data_ptr(),
        _heads(k, T, Hk, D), v.data_ptr(), _heads(v, T, Hk, D), H, T, _ints(positions, T), out.data_ptr(), out_stride, _on(q))
    if st != MOE_OK:
        _check(st, "moe_rope_append")
    return out


def attention_workspace_size(cache: KvCache, T_max: int, n_heads: int) -> int:
    n = C.c_size_t(0)
    _check(_lib().moe_attention_workspace_size(C.byref(cache.struct), T_max, n_heads, C.byref(n)), "moe_attention_workspace_size")
    return n.value


def alloc_attention_workspace(cache: KvCache, T_max: int, n_heads: int) -> torch.Tensor:
    return torch.empty(attention_workspace_size(cache, T_max, n_heads), dtype=torch.uint8, device=cache.k.device)


def moe_paged_attention(cache: KvCache, q: torch.Tensor, block_table: torch.Tensor, lengths: torch.Tensor,
                        table_row: Optional[torch.Tensor] = None, scale: Optional[float] = None, window: int = 0,
                        out: Optional[torch.Tensor] = None, want_lse: bool = False, workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of q [T, heads, dim] over the first `lengths` positions of the tokens' sequences (the last `window` of them if that
    is not 0); scale None: 1 / sqrt(dim).  Returns out (which may not be q), or (out, lse [T, heads]) with want_lse."""
    if stream is not None:
        return _under(stream, moe_paged_attention, cache, q, block_table, lengths, table_row, scale, window, out, want_lse, workspace)
    T, H = q.shape[:2]
    D = cache.dim
    if out is None:
        out, out_stride = _like(q), H * D
    else:
        out_stride = _heads(out, T, H, D)
    lse = q.new_empty((T, H), dtype=torch.float32) if want_lse else None
    if workspace is None:
        workspace = alloc_attention_workspace(cache, T, H)
    st = (_ready or _lib()).moe_paged_attention(
        cache.ref, C.byref(_table(block_table, table_row, T)), q.data_ptr(), _heads(q, T, H, D), H, T, _ints(lengths, T),
        D ** -0.5 if scale is None else scale, window, out.data_ptr(), out_stride, lse.data_ptr() if want_lse else None,
        *_bytes(workspace), _on(q))
    if st != MOE_OK:
        _check(st, "moe_paged_attention")
    return (out, lse) if want_lse else out
