"""The operators around the layer have no backward pass: a tensor that requires a gradient is refused, not taken with its gradient lost, unless gradients are off."""
import pytest
import torch

import paper_2507_17133_amd as P
from tests._layer_util import E4M3

pytestmark = pytest.mark.gpu

D, H, Hk, T = 64, 4, 2, 5


def _made():
    g = torch.Generator(device="cuda").manual_seed(1)
    bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    x8, xs = P.moe_quantize_rows(bf(T, 256))
    w8, ws = P.moe_quantize_weight(bf(128, 256))
    t = dict(x=bf(T, 256), residual=bf(T, 256), weight=bf(256), w=bf(128, 256), x8=x8, xs=xs, w8=w8, ws=ws, q=bf(T, H, D), k=bf(T, Hk, D), v=bf(T, Hk, D))
    cache = P.alloc_kv_cache(2, 16, Hk, D)
    cache.k.zero_(), cache.v.zero_()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    rest = (cache, P.make_rope(D), i32([[0, 1]]), i32([0] * T), torch.arange(T, dtype=torch.int32, device="cuda"))
    return t, rest


CALLS = {
    "norm": (("x", "residual", "weight"), lambda t, r: P.moe_rms_norm(t["x"], t["weight"], residual=t["residual"]).y),
    "rows": (("x",), lambda t, r: P.moe_quantize_rows(t["x"])[1]),
    "weight": (("w",), lambda t, r: P.moe_quantize_weight(t["w"])[1]),
    "linear": (("x8", "xs", "w8", "ws"), lambda t, r: P.moe_linear_e4m3(t["x8"], t["xs"], t["w8"], t["ws"])),
    "rope": (("q", "k", "v"), lambda t, r: P.moe_rope_append(r[0], r[1], t["q"], t["k"], t["v"], r[4], r[2], table_row=r[3])),
    "attention": (("q",), lambda t, r: P.moe_paged_attention(r[0], t["q"], r[2], r[4] + 1, table_row=r[3])),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_a_lost_gradient_is_refused(name):
    t, rest = _made()
    inputs, call = CALLS[name]
    want = call(t, rest)
    for i in inputs:
        with_grad = dict(t, **{i: t[i].detach().requires_grad_()})
        with pytest.raises(AssertionError):
            call(with_grad, rest)
        with torch.no_grad():
            assert torch.equal(call(with_grad, rest), want)
        with torch.inference_mode():
            assert torch.equal(call(with_grad, rest), want)


def test_a_cache_that_requires_a_gradient():
    k = torch.zeros((2, 16, Hk, D), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(AssertionError):
        P.KvCache(k.requires_grad_(), torch.zeros_like(k))
    with torch.no_grad():
        P.KvCache(k, torch.zeros_like(k))
