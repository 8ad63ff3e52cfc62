"""Chunk attention of sequences of up to 128 rows, and over an 8-bit cache, to the precision of its fp32 sums: beside a bf16 cache a probability goes to the product with v as
two bf16, so beyond its own rounding to bf16 a result is off by little, and a lost or swapped step of v shows in long sequences too."""
import pytest
import torch

import paper_2507_17133_amd as A
from tests._draft_util import rows_of, visible
from tests._layer_util import HALF_BF16, near
from tests.test_gpu_chunk import _dev, _setup

gpu = pytest.mark.gpu
ULP = 2.0 ** -24


def _exact(q, k, v, see, row_of, scale, e4m3=False, rounded=None):
    """out in 64 bits and how far the kernel may be from it; q [T, H, D], k and v [rows, L, Hk, D], see [T, L].  `rounded`: probabilities through it."""
    T, H, D = q.shape
    out, tol = torch.zeros((2, T, H, D), dtype=torch.float64)
    for t in range(T):
        at = see[t].nonzero()[:, 0]
        n = len(at)
        if row_of[t] < 0 or n == 0:
            continue
        kt, vt = (x[row_of[t], at].transpose(0, 1).repeat_interleave(H // k.shape[2], 0) for x in (k, v))     # [H, positions, D]
        s = (kt @ q[t][:, :, None])[..., 0] * scale
        size = (kt.abs() @ q[t].abs()[:, :, None])[..., 0] * abs(scale)
        p = torch.softmax(s, 1)[:, None]
        near_v = (p @ vt.abs())[:, 0]
        out[t] = ((p if rounded is None else rounded(p)) @ vt)[:, 0]
        # a score: an fp32 sum of D products, its factor, the hardware's exponential
        ds = (D + 8) * ULP * size.amax(1) + 2e-6
        # a probability beside v: two bf16 parts (what is left below bf16's bits is at most 2^-7 of it, and rounded to bf16: 2^-8 of that); or one fp16 (2^-11), of 2^11 times
        # the probability, whose steps below fp16's normal numbers are 2^-24 (half a step: 2^-25 of at least 2^11)
        part = 2.0 ** -11 if e4m3 else 2.0 ** -15
        small = n * 2.0 ** -36 * vt.abs().amax(1) if e4m3 else 0.0
        # the result's rounding and the sum of the probabilities, a lane's half of them one after the other; fp32 sums of 16 products at a time, two of each at most
        tol[t] = (HALF_BF16 + n / 2 * ULP) * out[t].abs() + (part + 2 * ds[:, None] + (n / 8 + 64) * ULP) * near_v + small + 1e-30
    return out, tol


def _check(setup, window=0, sinks=0, scale=None):
    cache, table, first, context, q, seen, positions = setup
    scale = q.shape[2] ** -0.5 if scale is None else scale
    out = A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context), seen=_dev(seen), positions=_dev(positions), scale=scale, window=window, sinks=sinks)
    k, v, there = rows_of(cache, table)
    see, row_of = visible(first, context, there, q.shape[0], seen, None if positions is None else positions.tolist(), window, sinks)
    near(out, *_exact(q.double().cpu(), k, v, see, row_of, scale, cache.k_scale is not None), "out")


# tiles of 32, 64 and 128 rows of every head width, half full and full
@gpu
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new,heads,kv", [(1, 3, 3), (4, 16, 2), (8, 8, 2), (16, 4, 1), (20, 12, 2), (32, 4, 1)])
def test_few_rows(dim, e4m3, new, heads, kv):
    for tree in (True, False):
        _check(_setup(dim + new, [new, new, max(1, new // 2)], [150, 0, 777], heads, kv, dim, 16, e4m3, heads_first=new % 8 == 0, tree=tree))


@gpu
@pytest.mark.parametrize("context,new,heads,kv,dim", [([20000], 8, 8, 2, 128), ([9000, 3], 16, 8, 1, 64), ([20000] + [3] * 20, 4, 8, 1, 128), ([6000] * 5, 9, 12, 2, 96),
                                                      ([4097, 12000], 6, 16, 2, 192), ([4097, 9000], 5, 16, 2, 256)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_long_sequences(context, new, heads, kv, dim, e4m3):
    """Sequences that many shares have a part of."""
    _check(_setup(3, [new] * len(context), context, heads, kv, dim, e4m3=e4m3, tree=True))


@gpu
@pytest.mark.parametrize("window,sinks", [(17, 3), (128, 0), (1000, 70)])
def test_window_and_sinks(window, sinks):
    for tree in (True, False):
        _check(_setup(window, [6, 6, 6], [100, 500, 3000], 8, 2, 128, tree=tree), window, sinks)


@gpu
@pytest.mark.parametrize("spread,scale", [(30.0, 1.0), (1e-3, 1.0), (5.0, -0.7), (1.0, 0.0)])
def test_sharp_and_flat_scores(spread, scale):
    s = _setup(6, [7, 7, 7], [700, 65, 0], 8, 2, 128)
    s[4].mul_(spread)
    _check(s, scale=scale)


@gpu
@pytest.mark.parametrize("new", [900, 333])
def test_an_8_bit_cache_and_many_rows(new):
    _check(_setup(7, [new], [1000], 2, 1, 128, e4m3=True))


def _cancel(k, v, g):
    """Neighbouring positions with nearly the same key and opposite values (k, v [..., positions, heads, dim]): what is left of the values is small, and so is its rounding."""
    n = k.shape[-3] // 2 * 2
    k[..., 1:n:2, :, :] = k[..., 0:n:2, :, :] + 0.02 * torch.randn(k[..., 0:n:2, :, :].shape, generator=g, device=k.device).to(k.dtype)
    v[..., 1:n:2, :, :] = -v[..., 0:n:2, :, :]


@gpu
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("new,heads,kv", [(4, 16, 2), (16, 4, 1), (31, 4, 1)])
def test_values_that_cancel(dim, new, heads, kv):
    s = _setup(dim, [new, new], [16, 64], heads, kv, dim, tree=True)
    g = torch.Generator(device="cuda").manual_seed(dim)
    cache, table = s[0], s[1].long()
    k, v = (t[table].flatten(1, 2).clone() for t in (cache.k, cache.v))
    _cancel(k, v, g)
    cache.k[table], cache.v[table] = (t.unflatten(1, (table.shape[1], -1)) for t in (k, v))
    s[4].mul_(0.1)
    _check(s)


def test_the_bound_notices_rounded_probabilities_and_lost_steps():
    """On the CPU: the 64-bit form with probabilities of one bf16, or without 32 positions of v, is beyond the bound in most results."""
    g = torch.Generator().manual_seed(1)
    rounded = lambda p: p.to(torch.bfloat16).double()
    for n in (32, 2000):
        q, k, v = (torch.randn(s, generator=g).to(torch.bfloat16).double() for s in ((1, 8, 128), (1, n, 1, 128), (1, n, 1, 128)))
        see, row_of = torch.ones((1, n), dtype=torch.bool), torch.zeros(1, dtype=torch.long)
        if n == 32:
            _cancel(k, v, g)
            q = 0.1 * q
        want, tol = _exact(q, k, v, see, row_of, 128 ** -0.5)
        bad = v.clone()
        bad[:, n // 2:n // 2 + 32] = 0
        got = _exact(q, k, v, see, row_of, 128 ** -0.5, rounded=rounded)[0] if n == 32 else _exact(q, k, bad, see, row_of, 128 ** -0.5)[0]
        assert float(((got - want).abs() > tol).double().mean()) > 0.5, n
