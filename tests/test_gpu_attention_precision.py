"""Attention over the paged cache to the precision of its fp32 sums: the probabilities keep 16 bits in the product with v, so beyond its own rounding to bf16 a
result is off by little, and a lost or swapped tile of v shows in long sequences too."""
import math

import pytest
import torch

import paper_2507_17133_amd as P
from tests._layer_util import E4M3, HALF_BF16, near
from tests.test_gpu_attention import _case

gpu = pytest.mark.gpu


def _exact(q, k, v, lengths, scale, window=0):
    """q [T, H, D], k and v [T, L, Hk, D] in 64 bits: out, and how far the kernel may be from it."""
    T, H, D = q.shape
    out, tol = torch.zeros((2, T, H, D), dtype=torch.float64)
    for t in range(T):
        n = int(lengths[t])
        if n == 0:
            continue
        kt, vt = (x[t, max(n - window, 0) if window else 0:n].transpose(0, 1).repeat_interleave(H // k.shape[2], 0) for x in (k, v))     # [H, positions, D]
        s = (kt @ q[t][:, :, None])[..., 0] * scale
        size = (kt.abs() @ q[t].abs()[:, :, None])[..., 0] * abs(scale)
        p = torch.softmax(s, 1)[:, None]
        out[t], near_v = (p @ vt)[:, 0], (p @ vt.abs())[:, 0]
        ulp = 2.0 ** -24
        ds = (D + 8) * ulp * size.amax(1) + 2e-6           # a score: an fp32 sum of D products, its factor, the hardware's exponential
        # the result's rounding and the sum of the probabilities, a lane's four in sixteen one after the other; of each product with v two bf16 parts
        # (what is left below bf16's bits is at most 2^-7, and rounded to bf16), and fp32 sums of 32 products at a time
        tol[t] = (HALF_BF16 + n / 4 * ulp) * out[t].abs() + (2.0 ** -15 + 2 * ds[:, None] + (n / 32 + 64) * ulp) * near_v + 1e-30
    return out, tol


def _check(lengths, H, Hk, D, page, window=0, scale=None, **kw):
    q, cache, table, k, v = _case(lengths, H, Hk, D, page, **kw)
    scale = D ** -0.5 if scale is None else scale
    n = torch.tensor(lengths)
    out = P.moe_paged_attention(cache, q.cuda(), table.cuda(), n.to(torch.int32).cuda(), scale=scale, window=window)
    near(out, *_exact(q.double(), k, v, n, scale, window), "out")


@gpu
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("H,Hk", [(4, 4), (8, 2), (24, 1)])
@pytest.mark.parametrize("e4m3,heads_first,page", [(False, False, 16), (True, True, 7), (True, False, 64)])
def test_heads_and_types(D, H, Hk, e4m3, heads_first, page):
    _check([1, 2, 0, 31, 33, 129, 300, 777], H, Hk, D, page, e4m3=e4m3, heads_first=heads_first, seed=D + H)


@gpu
@pytest.mark.parametrize("lengths,H,Hk,D", [([20000], 8, 1, 128), ([9000, 3], 8, 2, 64), ([20000] + [3] * 20, 8, 1, 128), ([6000] * 5, 16, 2, 96), ([4097, 12000], 32, 2, 256)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_long_sequences(lengths, H, Hk, D, e4m3):
    """Sequences that many shares have a part of."""
    _check(lengths, H, Hk, D, 16, e4m3=e4m3, seed=3)


@gpu
@pytest.mark.parametrize("window", [17, 128, 1000])
def test_window(window):
    _check([5, 100, 500, 3000], 8, 2, 128, 16, window=window, seed=window)


@gpu
@pytest.mark.parametrize("std,scale", [(30.0, 1.0), (1e-3, 1.0), (5.0, -0.7), (1.0, 0.0)])
def test_sharp_and_flat_scores(std, scale):
    _check([700, 65, 1], 8, 4, 128, 16, std=std, scale=scale, seed=6)


@gpu
@pytest.mark.parametrize("lengths", [[40], [700, 5], [9000]])
def test_an_infinite_value_stays_one(lengths):
    """v of an attended position infinite: so is the result in that column, with its sign, and the others are what they were."""
    H, Hk, D = 8, 2, 64
    q, cache, table, k, v = _case(lengths, H, Hk, D, 16, seed=7)
    q = q * 0.1                                            # every probability well above 2^-100
    n = torch.tensor(lengths)
    want, tol = _exact(q.double(), k, v, n, D ** -0.5)
    last = lengths[0] - 1
    cache.v[table[0, last // 16].item(), last % 16, 0, 5] = math.inf
    cache.v[table[0, 2 // 16].item(), 2, 1, 9] = -math.inf
    out = P.moe_paged_attention(cache, q.cuda(), table.cuda(), n.to(torch.int32).cuda()).cpu()
    assert bool((out[0, :4, 5] == math.inf).all()) and bool((out[0, 4:, 9] == -math.inf).all())
    out[0, :4, 5], out[0, 4:, 9] = want[0, :4, 5].to(out.dtype), want[0, 4:, 9].to(out.dtype)
    near(out, want, tol, "out")


@pytest.mark.parametrize("n,lost", [(20000, 128), (9000, 8)])
def test_the_bound_notices_lost_and_swapped_rows(n, lost):
    """On the CPU: the 64-bit form with some rows of v missing, or those of another place in their stead, is beyond the bound in most results."""
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(s, generator=g).to(torch.bfloat16).double() for s in ((1, 8, 128), (1, n, 1, 128), (1, n, 1, 128)))
    want, tol = _exact(q, k, v, [n], 128 ** -0.5)
    at = n // 2
    zeroed, swapped = v.clone(), v.clone()
    zeroed[:, at:at + lost] = 0
    swapped[:, at:at + lost] = v[:, :lost]
    for bad in (zeroed, swapped):
        off = (_exact(q, k, bad, [n], 128 ** -0.5)[0] - want).abs() > tol
        assert float(off.double().mean()) > 0.5
