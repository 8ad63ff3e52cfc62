"""Inputs and 64-bit forms for the tests of the operators of a step with several new tokens."""
import math

import torch

from tests._layer_util import E4M3


def make_cache(g, n_pages, page, heads, dim, e4m3=False, heads_first=False, extra=0):
    """k and v (views [page, token, head, dim] whichever way they are stored; `extra` elements between a token's or head's rows) and their scales."""
    import paper_2507_17133_amd as A
    shape = (n_pages, heads, page, dim + extra) if heads_first else (n_pages, page, heads, dim + extra)
    kv, scales = [], [None, None]
    for i in range(2):
        t = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        if e4m3:
            t = (t * 64).to(E4M3)
            scales[i] = torch.empty(heads, device="cuda").uniform_(0.01, 0.03, generator=g)
        t = t[..., :dim]
        kv.append(t.transpose(1, 2) if heads_first else t)
    return A.KvCache(kv[0], kv[1], *scales)


def values(cache, which):
    """[page, token, head, dim] in 64 bits on the CPU."""
    t, s = (cache.k, cache.k_scale) if which == "k" else (cache.v, cache.v_scale)
    d = (t.contiguous().view(torch.uint8).cpu().view(E4M3) if t.dtype == E4M3 else t.cpu()).double()
    return d if s is None else d * s.double().cpu()[None, None, :, None]


def rows_of(cache, table):
    """k and v [rows, positions, heads, dim] in 64 bits, and which positions are there, of a block table's rows (CPU)."""
    t = table.cpu().long()
    ok = (t >= 0) & (t < cache.k.shape[0])
    page = cache.k.shape[1]
    k, v = (values(cache, w)[t.clamp(0, cache.k.shape[0] - 1)].flatten(1, 2) for w in "kv")
    return k, v, ok.repeat_interleave(page, 1)


def seen_of(seen, j):
    """Bit j of each row of a mask [T, words] (CPU)."""
    words = seen.long() & 0xFFFFFFFF
    return (words[:, j // 32] >> (j % 32) & 1).bool() if j // 32 < seen.shape[1] else torch.zeros(len(seen), dtype=torch.bool)


def visible(first, context, positions_there, T, seen=None, positions=None, window=0, sinks=0, rows=None):
    """[T, L] of truth values, and each token's row of the table (-1: of no sequence), from the definition."""
    L = positions_there.shape[1]
    see, row_of = torch.zeros((T, L), dtype=torch.bool), torch.full((T,), -1)
    p = torch.arange(L)
    for b, c in enumerate(context):
        c = max(c, 0)
        lo, hi = min(max(first[b], 0), T), min(max(first[b + 1], 0), T)
        row = b if rows is None else rows[b]
        for t in range(lo, hi):
            row_of[t] = row
            if not 0 <= row < positions_there.shape[0]:
                continue
            at = c + t - lo
            if seen is not None and positions is not None:
                at = max(positions[t], c)
            old = (p > at - window) | (p < sinks) if window else torch.ones(L, dtype=torch.bool)
            if seen is None:
                see[t] = (p <= at) & old
            else:
                see[t] = (p < c) & old
                for j in range(hi - lo):
                    if c + j < L and bool(seen_of(seen[t:t + 1], j)[0]):
                        see[t, c + j] = True
            see[t] &= positions_there[row]
    return see, row_of


def attend(q, k, v, see, row_of, scale):
    """out, lse in 64 bits and the bounds on both: scores and sums of fp32, a probability rounded to bf16 for the product with v, the result rounded to bf16."""
    T, H, D = q.shape
    group = H // k.shape[2]
    out, tol = torch.zeros((2, T, H, D), dtype=torch.float64)
    lse, tol_lse = torch.full((T, H), -math.inf, dtype=torch.float64), torch.zeros((T, H), dtype=torch.float64)
    half = 2.0 ** -8
    for t in range(T):
        at = see[t].nonzero()[:, 0]
        if row_of[t] < 0 or len(at) == 0:
            continue
        kt, vt = (x[row_of[t], at].transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))
        s = (kt @ q[t][:, :, None])[..., 0] * scale
        size = (kt.abs() @ q[t].abs()[:, :, None])[..., 0] * abs(scale)
        lse[t] = torch.logsumexp(s, 1)
        pr = torch.softmax(s, 1)[:, None]
        out[t], near_v = (pr @ vt)[:, 0], (pr @ vt.abs())[:, 0]
        # fp32 sums of D products and of the probabilities, the hardware's exponential and logarithm
        ds = (D + 8) * 2.0 ** -24 * size.amax(1) + 2e-6 + len(at) * 2.0 ** -24 / 8
        tol[t] = half * (out[t].abs() + near_v) + 2 * ds[:, None] * near_v + 1e-30
        tol_lse[t] = ds + 1e-6 * lse[t].abs()
    return out, lse, tol, tol_lse


def random_tree(r, n):
    return [r.randint(max(-1, j - 6), j - 1) for j in range(n)]
