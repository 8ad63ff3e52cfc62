"""norm -> 8-bit rows -> product with an 8-bit weight, as a decoder layer uses them: what one call writes is what the next one reads."""
import math

import pytest
import torch

import paper_2507_17133_amd as P
from tests._layer_util import groups, near
from tests.test_gpu_linear8 import _exact

# An e4m3 rounding moves a value by at most 2^-4 of it; as a uniform error 2^-4 / sqrt(3) in the mean square, of rows and weights together sqrt(2) of that.
# Independent errors add up in a product like its terms do, so its norm is off by that share of itself.
OFF = math.sqrt(2 / 3) * 2.0 ** -4


def _inputs(T, d, N):
    g = torch.Generator().manual_seed(T + d)
    x = torch.randn((T, d), generator=g)
    x[:, ::5] *= 3
    return x.to(torch.bfloat16), (torch.randn((N, d), generator=g) / math.sqrt(d)).to(torch.bfloat16)


def _unquantised(x, w):
    y = x.double() / (x.double().square().mean(1, keepdim=True) + 1e-6).sqrt()
    return y, y @ w.double().t()


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,N", [(1, 1024, 384), (70, 1024, 384), (300, 2064, 1000), (129, 5632, 2050)])
def test_rows_of_the_norm_times_a_quantised_weight(T, d, N):
    x, w = _inputs(T, d, N)
    n = P.moe_rms_norm(x.cuda(), None, 1e-6, want=("y8",))
    w8, ws = P.moe_quantize_weight(w.cuda())
    got = P.moe_linear_e4m3(n.y8, n.scale, w8, ws)
    # the codes and scales that came back, multiplied in 64 bits
    near(got, *_exact(n.y8, n.scale, w8, ws), "product")
    y, want = _unquantised(x, w)
    assert float((got.double().cpu() - want).norm() / want.norm()) < OFF
    # and for the rows alone
    x8, xs = P.moe_quantize_rows(x.cuda())
    got = P.moe_linear_e4m3(x8, xs, w8, ws).double().cpu()
    assert float((got - x.double() @ w.double().t()).norm() / (x.double() @ w.double().t()).norm()) < OFF


def test_the_bound_notices_a_lost_block():
    """On the CPU: a product without one of its blocks of 128, with the scales of two neighbouring rows or groups exchanged, or a tenth too large is out of bounds."""
    x, w = _inputs(70, 1024, 384)
    y, want = _unquantised(x, w)
    s = groups(y).abs().amax(2) / 448
    units = groups(y) / s[:, :, None]
    lost = groups(y).clone()
    lost[:, 3] = 0
    other_rows, other_groups = s.clone(), s.clone()
    other_rows[0::2], other_rows[1::2] = s[1::2], s[0::2]
    other_groups[:, 0::2], other_groups[:, 1::2] = s[:, 1::2], s[:, 0::2]
    for wrong in (lost.reshape(70, -1), (units * other_rows[:, :, None]).reshape(70, -1), (units * other_groups[:, :, None]).reshape(70, -1), 1.1 * y):
        assert float((wrong @ w.double().t() - want).norm() / want.norm()) > OFF


@pytest.mark.gpu
@pytest.mark.parametrize("want,residual", [(("y",), False), (("y8",), True), (("y", "y8"), True)])
def test_outputs_made_once(want, residual):
    """alloc_norm_out's tensors take what a call would allocate, call after call."""
    T, d = 37, 1000
    out = P.alloc_norm_out(T, d, want, residual)
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x, r = (torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        r = r if residual else None
        fresh = P.moe_rms_norm(x, None, 1e-6, residual=r, want=want)
        got = P.moe_rms_norm(x, None, 1e-6, residual=r, out=out)
        assert got is out
        for a, b in zip(got, fresh):
            assert (a is None) == (b is None) and (a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)))
