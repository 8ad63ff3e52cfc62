"""The 8-bit linear layer where one column in 128 is far larger than the rest, as activations have them.

Beyond K = 512 the product goes through the 8-bit matrix instructions.  They add up 8 neighbouring columns at a time: each product is cut off (toward zero) at 2^-13
of 2^e, e the largest sum of two exponents among the 8; what a group of 8 gives is added in fp32.  So the error of a result is at most what that cuts off.  With
`exact` products are whole and the sums fp32, for every K."""
import math

import pytest
import torch

import paper_2507_17133_amd as P
from tests._layer_util import E4M3, FLOOR, groups, near, spread
from tests.test_gpu_linear8 import _case, _exact

gpu = pytest.mark.gpu


def _outliers(M, N, K, times, seed):
    """Rows with one column in 128 `times` larger, in 8 bits with a scale per 128 columns; an ordinary weight."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((M, K), generator=g, device="cuda")
    x[:, 5::128] *= times
    y = groups(x)
    s = y.abs().amax(2).clamp_min(FLOOR) / 448.0
    x8 = (y / s[:, :, None]).to(E4M3).reshape(M, -1)[:, :K].contiguous()
    _, _, w8, ws = _case(1, N, K, seed)
    return x8, s.t().contiguous(), w8, ws


def _exponent(v):
    """Of e4m3 values; those below 2^-6 have the least one."""
    return torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6)))


def _cut_off(x8, xs, w8, ws):
    """[M, N] the most that the groups of 8 lose, in 64 bits."""
    K, N = x8.shape[1], w8.shape[0]
    x, w = x8.double(), w8.double()
    ex, ew = (torch.where(v == 0, -math.inf, _exponent(v)) for v in (x, w))
    wide = ws.double().repeat_interleave(128, 0)[:N]
    lost = torch.zeros((x.shape[0], N), dtype=torch.float64, device=x.device)
    for k in range(0, K, 8):
        p = (x[:, None, k:k + 8] * w[None, :, k:k + 8]).abs()
        at = torch.exp2((ex[:, None, k:k + 8] + ew[None, :, k:k + 8]).amax(2, keepdim=True) - 13)
        lost += torch.minimum(p, at).sum(2) * xs[k // 128].double()[:, None] * wide[None, :, k // 128]
    return lost


# a row's blocks of 16 and of 32 columns, tiles from 64 x 64 to 256 x 256, with and without slices of K
SHAPES = [(1, 300, 1040), (16, 6144, 1024), (33, 200, 4112), (64, 6160, 640), (65, 300, 2048), (130, 512, 4096), (300, 1408, 1040), (1000, 1408, 528), (1500, 2100, 640),
          (2048, 4100, 528)]


@gpu
@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("times", [100.0, 500.0])
def test_what_the_instructions_cut_off(M, N, K, times):
    case = _outliers(M, N, K, times, M + N)
    want, tol = _exact(*case)
    got = P.moe_linear_e4m3(*case)
    at = torch.arange(0, M, max(1, M // 40), device="cuda")            # rows that the bound is worked out for
    x8, xs, w8, ws = case
    lost = _cut_off(x8.view(torch.uint8)[at].view(E4M3), xs[:, at], w8, ws)
    near(got[at], want[at], tol[at] + lost, "out")
    # every row: no group loses more than 7 times 2^-13 of its largest product
    a, b = (v.double().abs() * s for v, s in ((x8, spread(xs.double(), K)), (w8, ws.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K])))
    most = sum(a[:, k:k + 8].amax(1)[:, None] * b[:, k:k + 8].amax(1)[None] for k in range(0, K, 8))
    near(got, want, tol + 7 * 2.0 ** -13 * most, "out")


@gpu
@pytest.mark.parametrize("M,N,K", SHAPES + [(20, 16, 65536), (20, 6144, 4096), (3600, 1027, 1488), (256, 6144, 4096)])
@pytest.mark.parametrize("times", [1.0, 500.0])
def test_exact(M, N, K, times):
    """Within fp32 sums of exact products, whatever the sizes of the columns; no workspace needed."""
    case = _outliers(M, N, K, times, M + K)
    want, tol = _exact(*case)
    wide = torch.full((M, N + 9), 7.0, dtype=torch.bfloat16, device="cuda")
    near(P.moe_linear_e4m3(*case, exact=True, out=wide[:, 1:1 + N], workspace=torch.empty(0, dtype=torch.uint8, device="cuda")), want, tol, "out")
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, 1 + N:] == 7).all())
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = P.moe_linear_e4m3(*case, exact=True, stream=s)
    s.synchronize()
    assert torch.equal(got, wide[:, 1:1 + N])


@gpu
def test_short_k_is_exact_either_way():
    case = _outliers(100, 300, 512, 500.0, 3)
    want, tol = _exact(*case)
    near(P.moe_linear_e4m3(*case), want, tol, "out")
    assert torch.equal(P.moe_linear_e4m3(*case), P.moe_linear_e4m3(*case, exact=True))


def test_the_model_on_an_example():
    """On the CPU: the rule's bound is above what cutting off at it loses, and such rows lose more than fp32 sums may."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn((16, 128), generator=g)
    x[:, 5] *= 500
    x8, w8 = (x * (448 / x.abs().amax(1, keepdim=True))).to(E4M3), (torch.randn((16, 128), generator=g) * 60).clamp(-448, 448).to(E4M3)
    one = torch.ones((1, 16)), torch.ones((1, 1))
    p = x8.double()[:, None] * w8.double()[None]
    e = torch.where(p == 0, -math.inf, _exponent(x8.double())[:, None] + _exponent(w8.double())[None]).view(16, 16, 16, 8)
    at = torch.exp2(e.amax(3, keepdim=True) - 13)
    got = (torch.trunc(p.view(16, 16, 16, 8) / at) * at).sum((2, 3))
    off = (got - p.sum(2)).abs()
    assert bool((off <= _cut_off(x8, one[0], w8, one[1])).all())
    assert bool((off > 128 * 2.0 ** -24 * p.abs().sum(2)).any())
