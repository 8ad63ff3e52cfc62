"""Attention's output may not lie over its queries: blocks read q of heads that others have written already.  Refused by the host; rows that merely alternate
with those of q in a wider tensor are taken."""
import pytest

from tests.test_layer_abi import INVALID, OK, P, _attention_call

FAR = P + (1 << 30)
W = 4096 * 2                                   # bytes of a token's row: 32 heads of 128 in bf16
# (q, q's stride, out, out's stride, tokens)
OVER = [(P, 4096, P, 4096, 8), (P, 4096, P, 4096, 1), (P, 4096, P + W // 2, 4096, 1), (P + 16, 4096, P, 4096, 1), (P, 4096, P + 3 * W, 4096, 8),
        (P, 0, P, 4096, 8), (P, 4096, P + 7 * W + 128, 8192, 8), (P, 8192, P + W + 16, 8192, 8), (P, 8192, P + 8, 12288, 3), (P + 5 * W, 8, P, 4096, 8)]
APART = [(P, 4096, FAR, 4096, 8), (FAR, 4096, P, 4096, 8), (P, 4096, P + 8 * W, 4096, 8), (P, 8192, P + W, 8192, 8), (P + W, 8192, P, 8192, 8),
         (P, 0, P + W, 4096, 8), (P, 8192, P + W, 16384, 8), (P, 24576, P + W, 12288, 3)]


@pytest.mark.parametrize("q,qs,out,os,T", OVER)
def test_over_the_queries(q, qs, out, os, T):
    assert _attention_call(q=q, qs=qs, out=out, os=os, T=T) == INVALID
    assert _attention_call(q=q, qs=qs, out=out, os=os, T=0) == OK


def test_pairs_by_hand():
    """The lists above against every pair of rows."""
    over = lambda q, qs, out, os, T: any(q + 2 * qs * i < out + 2 * os * j + W and out + 2 * os * j < q + 2 * qs * i + W for i in range(T) for j in range(T))
    assert all(over(*c) for c in OVER) and not any(over(*c) for c in APART)


@pytest.mark.gpu
@pytest.mark.parametrize("q,qs,out,os,T", APART)
def test_beside_the_queries(q, qs, out, os, T):
    """On the device, with real memory in the same places."""
    import torch

    import paper_2507_17133_amd as A
    if max(q, out) >= FAR:
        q, out = (x - FAR + P + 16 * W if x >= FAR else x for x in (q, out))
    g = torch.Generator(device="cuda").manual_seed(3)
    cache = A.alloc_kv_cache(4, 16, 8, 128)
    cache.k.normal_(generator=g), cache.v.normal_(generator=g)
    wide = torch.empty(1 << 18, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    at = lambda p, s: wide.as_strided((T, 32, 128), (s, 128, 1), (p - P) // 2)
    queries = at(q, qs).clone()
    table = torch.randperm(4, generator=g, device="cuda").to(torch.int32).expand(T, 4).contiguous()
    lengths = torch.randint(0, 65, (T,), generator=g, device="cuda").to(torch.int32)
    want = A.moe_paged_attention(cache, queries, table, lengths)
    assert torch.equal(A.moe_paged_attention(cache, at(q, qs), table, lengths, out=at(out, os)), want)
    assert torch.equal(at(q, qs), queries)
