"""The norm with residual and 8-bit output, the 8-bit rows alone and the 8-bit weight, against 64 bits."""
import math

import pytest
import torch

import paper_2507_17133_amd as P
from tests._layer_util import E4M3, FLOOR, HALF_BF16, HALF_E4M3, near, scales_of, spread

pytestmark = pytest.mark.gpu

# sums of d squares in fp32: at most 8 x 8 terms one after the other and a tree, halved by the square root; a few roundings of factors
REL = 5e-6


def _x(T, d, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, d), generator=g) * std
    x[:, ::7] *= 30
    return x.to(torch.bfloat16)


def _exact(x, r, w, eps):
    h = x.double() if r is None else x.double() + r.double()
    y = h / (h.square().mean(1, keepdim=True) + eps).sqrt()
    return h, y if w is None else y * w.double()


def _check8(y8, scale, y):
    s = scales_of(y)
    near(scale, s, REL * s, "scale")
    s = spread(scale.double().cpu(), y.shape[1])
    near(y8.float().double().cpu() * s, y, (HALF_E4M3 * y.abs()).clamp_min(2.0 ** -10 * s) + 2 * REL * y.abs(), "y8")


@pytest.mark.parametrize("T,d", [(1, 8), (3, 64), (5, 136), (2, 512), (1, 520), (7, 1024), (4, 1032), (1, 2048), (9, 2056), (3, 4096), (2, 5632),
                                 (5, 7168), (2, 8200), (1, 16384), (700, 256)])
@pytest.mark.parametrize("with_residual,with_weight", [(True, True), (False, True), (True, False)])
def test_norm(T, d, with_residual, with_weight):
    x, r = _x(T, d, 1), _x(T, d, 2, 3.0) if with_residual else None
    w = (1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(3))).to(torch.bfloat16) if with_weight else None
    c = lambda t: None if t is None else t.cuda()
    got = P.moe_rms_norm(c(x), c(w), 1e-5, residual=c(r), want=("y", "y8"))
    h, y = _exact(x, r, w, 1e-5)
    near(got.y, y, (HALF_BF16 + REL) * y.abs(), "y")
    _check8(got.y8, got.scale, y)
    if with_residual:
        assert torch.equal(got.residual.cpu(), (x.float() + r.float()).to(torch.bfloat16))
    else:
        assert got.residual is None
    only = P.moe_rms_norm(c(x), c(w), 1e-5, residual=c(r), want=("y8",))
    assert only.y is None and torch.equal(only.y8.view(torch.uint8), got.y8.view(torch.uint8)) and torch.equal(only.scale, got.scale)
    only = P.moe_rms_norm(c(x), c(w), 1e-5, residual=c(r))
    assert only.y8 is None and torch.equal(only.y, got.y)


@pytest.mark.parametrize("T,d", [(1, 8), (6, 128), (5, 264), (3, 2048), (2, 4096), (4, 5640), (1, 16384)])
def test_quantize_rows(T, d):
    x = _x(T, d, 4)
    x[0, : min(128, d)] = 0                         # a group of zeros
    x8, scale = P.moe_quantize_rows(x.cuda())
    y = x.double()
    s = (scales_of(x.float())).double()             # the same fp32 division
    near(scale, s, 2.0 ** -23 * s, "scale")
    _check8(x8, scale, y)
    assert float(scale[0, 0]) == float(torch.tensor(FLOOR) / 448) and not bool(x8[0, : min(128, d)].float().any())


def test_extreme_rows():
    """Rows of zeros, tiny rows, the type's largest values, infinities and NaN."""
    big = torch.finfo(torch.bfloat16).max
    x = torch.zeros((6, 256))
    x[1] = 1e-38
    x[2] = big
    x[3, 5] = math.inf
    x[4, 200] = math.nan
    x[5, 0], x[5, 128] = 1e-30, -2.0
    x = x.to(torch.bfloat16)
    x8, scale = P.moe_quantize_rows(x.cuda())
    stands = x8.float().cpu() * spread(scale.cpu(), 256)
    near(stands[[0, 1, 2, 5]], x[[0, 1, 2, 5]].double(), (HALF_E4M3 * x[[0, 1, 2, 5]].double().abs()).clamp_min(2.0 ** -110), "quantised")
    assert bool(stands[3, :128].isnan().all()) and not bool(stands[3, 128:].any())
    assert not bool(stands[4, :128].any()) and bool(stands[4, 128:].isnan().all())
    got = P.moe_rms_norm(x.cuda(), None, 0.0, want=("y", "y8"))
    y = got.y.float().cpu()
    assert bool(y[0].isnan().all())                 # 0 / 0
    assert bool(y[4].isnan().all()) and bool(y[3, 5].isnan()) and not bool(y[3, :5].any())
    assert bool((got.scale[:, 0].isnan() | (got.y8[0].float().isnan().all())).all())
    zero = P.moe_rms_norm(x[:1].cuda(), None, 1e-6, want=("y", "y8"))
    assert not bool(zero.y.any()) and not bool(zero.y8.float().any())


def test_strided_rows_and_outputs():
    T, d = 37, 640
    wide = _x(T, 2000, 5).cuda()
    x, r = wide[:, 16:16 + d], wide[:, 1000:1000 + d]
    dense = P.moe_rms_norm(x.contiguous(), None, 1e-6, residual=r.contiguous(), want=("y", "y8"))
    out = P.NormOut(torch.full((T, 800), 7.0, dtype=torch.bfloat16, device="cuda")[:, 8:8 + d],
                    torch.zeros((T, 704), dtype=torch.uint8, device="cuda").view(E4M3)[:, 8:8 + d],
                    torch.full((5, 64), 7.0, device="cuda")[:, 3:3 + T], torch.empty((T, 1000), dtype=torch.bfloat16, device="cuda")[:, :d])
    got = P.moe_rms_norm(x, None, 1e-6, residual=r, out=out)
    for a, b in zip(got, dense):
        assert torch.equal(a.view(torch.uint8) if a.dtype == E4M3 else a, b.view(torch.uint8) if b.dtype == E4M3 else b)
    assert bool((out.y._base[:, :8] == 7).all()) and bool((out.y._base[:, 8 + d:] == 7).all())
    assert bool((out.scale._base[:, :3] == 7).all()) and bool((out.scale._base[:, 3 + T:] == 7).all())


def test_residual_in_place_and_a_stream_of_its_own():
    T, d = 300, 2048
    x, r = _x(T, d, 6).cuda(), _x(T, d, 7).cuda()
    want = P.moe_rms_norm(x, None, 1e-6, residual=r)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    mine = r.clone()
    torch.cuda.synchronize()
    got = P.moe_rms_norm(x, None, 1e-6, residual=mine, out=P.NormOut(y=torch.empty_like(x), residual=mine), stream=s)
    s.synchronize()
    assert torch.equal(got.y, want.y) and torch.equal(mine, want.residual)


def test_no_rows():
    got = P.moe_rms_norm(torch.empty((0, 256), dtype=torch.bfloat16, device="cuda"), None, want=("y", "y8"))
    assert got.y.shape == (0, 256) and got.scale.shape == (2, 0)


@pytest.mark.parametrize("N,K", [(1, 16), (130, 144), (128, 128), (257, 2048), (1408, 336)])
def test_quantize_weight(N, K):
    w = _x(N, K, 8)
    w[:, :16] *= 100
    w8, scale = P.moe_quantize_weight(w.cuda())
    big = torch.nn.functional.pad(w.float(), (0, -K % 128, 0, -N % 128))
    s = big.reshape(-(-N // 128), 128, -(-K // 128), 128).abs().amax((1, 3)).clamp_min(FLOOR) / 448
    near(scale, s, 2.0 ** -23 * s, "scale")
    full = scale.cpu().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K].double()
    near(w8.float().cpu().double() * full, w.double(), (HALF_E4M3 * w.double().abs()).clamp_min(2.0 ** -10 * full) * (1 + 1e-5), "w8")


@pytest.mark.parametrize("T,d", [(9001, 504), (5003, 1000), (1100, 4096), (700, 8000), (333, 16384)])
def test_results_too_large_for_the_caches(T, d):
    """More than 8 MiB of bf16 rows: they go past the caches."""
    x, r = _x(T, d, 5), _x(T, d, 6)
    got = P.moe_rms_norm(x.cuda(), None, 1e-5, residual=r.cuda(), want=("y", "y8"))
    _, y = _exact(x, r, None, 1e-5)
    near(got.y, y, (HALF_BF16 + REL) * y.abs(), "y")
    _check8(got.y8, got.scale, y)
    assert torch.equal(got.residual.cpu(), (x.float() + r.float()).to(torch.bfloat16))
    _check8(*P.moe_quantize_rows(x.cuda()), x.double())
