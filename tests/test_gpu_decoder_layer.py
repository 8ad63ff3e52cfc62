"""The example's decoder layer (norm, 8-bit projections, rotary append, paged attention, MoE layer) against the same layer in 64 bits on the
unquantised weights, and its decode steps against the same tokens as part of the prompt."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import decoder_layer as E
from paper_2507_17133_amd import workloads as WL


def _norm(x):
    return x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()


def _attention_half(layer, x):
    """[tokens, d] of one sequence -> what attention adds, 64 bits."""
    D, H, Hk = layer.D, layer.H, layer.Hk
    n = x.shape[0]
    qkv = (_norm(x) @ layer.qkv_weight.double().t()).view(n, H + 2 * Hk, D)
    t = torch.arange(n, device="cuda").double()[:, None] * layer.rope.turns
    ang = (t - t.round()) * 2 * math.pi
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    a, b = qkv[:, :H + Hk, :D // 2].clone(), qkv[:, :H + Hk, D // 2:].clone()
    qkv[:, :H + Hk, :D // 2], qkv[:, :H + Hk, D // 2:] = a * c - b * s, b * c + a * s
    q, k, v = qkv.split((H, Hk, Hk), 1)
    k, v = (z.repeat_interleave(H // Hk, 1).transpose(0, 1).contiguous() for z in (k, v))       # [H, n, D]
    score = q.transpose(0, 1).contiguous() @ k.transpose(1, 2).contiguous() / D ** 0.5
    score = score.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), -math.inf)
    o = (torch.softmax(score, 2) @ v).transpose(0, 1).reshape(n, H * D)
    return o @ layer.o_weight.double().t()


@pytest.mark.parametrize("kv8", [False, True])
def test_residual_stream_behind_attention(kv8):
    """Four 8-bit roundings (rows and weights of two products), each within 1/16 of a value and 2.6 % on average, and one more of k and v in
    the 8-bit cache: what attention adds is within 5 * 2.6 % of its norm even if all of them pull the same way."""
    cfg = WL.CONFIGS["tiny"].with_(d=512)
    layer, _, x, out, res, _, _ = E.serve(cfg, batch=3, prompt=70, steps=5, kv8=kv8, chunk=64, page_size=16)
    assert bool(out.isfinite().all())
    for b in range(3):
        want = _attention_half(layer, x[b].double())
        got = res[b].double() - x[b].double()
        assert float((got - want).norm() / want.norm()) < 0.13


def test_steps_give_what_a_longer_prompt_gives():
    """The same tokens, once decoded step by step from a graph and once as part of the prompt: the cache is the same up to the sums' order in the
    projections, so the residual stream agrees to its roundings to bf16 and e4m3 (a value at an edge may fall to the other side)."""
    cfg = WL.CONFIGS["tiny"].with_(d=512)
    one = E.serve(cfg, batch=4, prompt=40, steps=6, chunk=64)
    all_ = E.serve(cfg, batch=4, prompt=46, steps=0, chunk=64)
    assert torch.equal(one[2], all_[2])
    a, b = one[4].double(), all_[4].double()
    assert float((a - b).norm() / b.norm()) < 4e-3


def test_the_moe_half_is_the_layers():
    """The layer's output is moe_forward of the normed residual stream, up to the rounding of that stream."""
    import paper_2507_17133_amd as P
    cfg = WL.CONFIGS["tiny"].with_(d=512)
    layer, _, x, out, res, _, _ = E.serve(cfg, batch=1, prompt=50, steps=0, threshold=0.5)
    n = P.moe_rms_norm(res[0], layer.norm2)
    y = P.moe_forward(layer.moe_cfg, n.y, layer.gate, layer.gate_b, layer.experts, layer.united, layer.shared, 0.5)
    rel = float((y.double() - out[0].double()).norm() / y.double().norm())
    # the layer norms the unrounded sum, here its bf16 rounding is normed: 2^-9 of a value, which may move a token across a routing edge
    assert rel < 0.05
