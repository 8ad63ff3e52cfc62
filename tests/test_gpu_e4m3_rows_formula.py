"""The 8-bit form bit for bit: s = max(largest |y|, 2^-100) / 448 and e4m3(y / s) are fp32 divisions, each rounded once, so elementary fp32 arithmetic
gives the same scales and codes, those whose quotient lies next to a midpoint included.  (y times a rounded 1 / s does not.)"""
import pytest
import torch

import paper_2507_17133_amd as P
from tests._layer_util import E4M3, FLOOR, groups

pytestmark = pytest.mark.gpu


def _values(rows, cols, seed):
    """Columns of very different sizes, and small integers over powers of two, whose quotients by a scale often lie at a midpoint."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g)
    x[:, ::7] *= 30
    x[:, 3::11] = -0.0
    x[rows // 2:] = torch.randint(-256, 257, x[rows // 2:].shape, generator=g) / 64.0
    x[rows // 4: rows // 2] *= torch.exp2(torch.randint(-110, 90, (rows // 2 - rows // 4, 1), generator=g).float())     # groups around 2^-100 among them
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("T,d", [(64, 128), (300, 504), (200, 1000), (257, 4096), (1500, 4104), (60, 16384)])
def test_rows(T, d):
    x = _values(T, d, T + d)
    y = groups(x.float())
    s = y.abs().amax(2).clamp_min(FLOOR) / 448.0
    want = (y / s[:, :, None]).to(E4M3).reshape(T, -1)[:, :d]
    got, scale = P.moe_quantize_rows(x.cuda())
    assert torch.equal(scale.cpu(), s.t())
    assert torch.equal(got.cpu().view(torch.uint8), want.contiguous().view(torch.uint8))


@pytest.mark.parametrize("N,K", [(128, 128), (300, 2064), (1408, 4096)])
def test_weight(N, K):
    w = _values(N, K, N + K)
    b = torch.nn.functional.pad(w.float(), (0, -K % 128, 0, -N % 128)).reshape(-(-N // 128), 128, -(-K // 128), 128)
    s = b.abs().amax((1, 3)).clamp_min(FLOOR) / 448.0
    want = (b / s[:, None, :, None]).to(E4M3).reshape(b.shape[0] * 128, -1)[:N, :K]
    got, scale = P.moe_quantize_weight(w.cuda())
    assert torch.equal(scale.cpu(), s)
    assert torch.equal(got.cpu().view(torch.uint8), want.contiguous().view(torch.uint8))


@pytest.mark.parametrize("T,d", [(100, 1000), (7, 8200), (5, 16384)])
def test_rows_of_the_norm(T, d):
    """y is known where the norm only scales by a power of two: rows of +-a have a mean square of a^2 and eps 0, so 1 / rms is exact and y is
    the weight with a sign."""
    g = torch.Generator().manual_seed(T)
    sign = torch.randint(0, 2, (T, d), generator=g) * 2.0 - 1
    x = (sign * torch.exp2(torch.randint(-3, 4, (T, 1), generator=g).float())).to(torch.bfloat16)
    w = _values(8, d, 9)[1]
    y = groups(sign * w.float())
    s = y.abs().amax(2).clamp_min(FLOOR) / 448.0
    want = (y / s[:, :, None]).to(E4M3).reshape(T, -1)[:, :d]
    got = P.moe_rms_norm(x.cuda(), w.cuda(), 0.0, want=("y8",))
    assert torch.equal(got.scale.cpu(), s.t())
    assert torch.equal(got.y8.cpu().view(torch.uint8), want.contiguous().view(torch.uint8))


def test_every_pair_of_significands():
    """A group's largest value with each of the 128 significands that bf16 has, the other values with each of them and at many sizes below it."""
    most, value = (1 + torch.arange(128) / 128.0 for _ in range(2))
    below = [1, 2, 7, 8, 9, 13, 14, 15, 16, 17, 18, 19]
    # rows: largest x size; columns: two groups of a largest value and half the significands
    x = torch.zeros((128, len(below), 2, 128))
    x[..., 0] = most[:, None, None]
    for i, e in enumerate(below):
        x[:, i, 0, 1:65], x[:, i, 1, 1:65] = value[:64] * 2.0 ** -e, value[64:] * 2.0 ** -e
    x = x.reshape(-1, 256)
    for size in (0, -90, -98, 100, 120):                   # whole rows scaled: the floor of a group's magnitude is 2^-100
        rows = (x * 2.0 ** size).to(torch.bfloat16)
        y = groups(rows.float())
        s = y.abs().amax(2).clamp_min(FLOOR) / 448.0
        got, scale = P.moe_quantize_rows(rows.cuda())
        assert torch.equal(scale.cpu(), s.t())
        assert torch.equal(got.cpu().view(torch.uint8), (y / s[:, :, None]).to(E4M3).reshape(-1, 256).view(torch.uint8))
