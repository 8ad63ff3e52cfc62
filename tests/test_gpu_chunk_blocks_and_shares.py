"""Long chunks of every head width, where the device decides between a block for each item and shares of their steps, against the definition in 64 bits: the values of a column
tell which of the positions' stretches of 32 were weighed, and the log of the sum which were counted, so one lost or doubled shows in thousands."""
import math

import pytest
import torch

import paper_2507_17133_amd as A
from tests._layer_util import E4M3, HALF_BF16, near
from tests.test_gpu_chunk import _check as check_all, _dev, _setup

pytestmark = pytest.mark.gpu
ULP = 2.0 ** -24


def _marked(cache, table, contexts, new):
    """v = 1 in the one column that a stretch of 32 positions of the sequence has, 0 in the others."""
    page, D = cache.v.shape[1], cache.v.shape[3]
    for b, (c, n) in enumerate(zip(contexts, new)):
        p = torch.arange(table.shape[1] * page, device="cuda")
        rows = torch.nn.functional.one_hot(p // 32 % D, D).to(torch.bfloat16)[:, None].expand(-1, cache.v.shape[2], -1)
        cache.v[table[b].long()[p // page], p % page] = rows.to(E4M3) if cache.v.dtype is E4M3 else rows


def _sample(setup, tokens, got, lse, window, sinks):
    cache, table, first, context, q, _, _ = setup
    page, H, Hk, D = cache.k.shape[1], q.shape[1], cache.k.shape[2], cache.k.shape[3]
    for t in tokens:
        b = max(i for i in range(len(context)) if first[i] <= t)
        at = context[b] + t - first[b]
        p = torch.arange(at + 1, device="cuda")
        if window:
            p = p[(p > at - window) | (p < sinks)]
        page_of, place, n = table[b].long()[p // page], p % page, len(p)
        for h in range(Hk):
            kh, vh = ((x.view(torch.uint8)[page_of, place, h].view(E4M3).double() * s[h].double()) if s is not None else x[page_of, place, h].double()
                      for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
            heads = slice(h * H // Hk, (h + 1) * H // Hk)
            qh = q[t, heads].double()
            s = qh @ kh.t().contiguous() * D ** -0.5
            # a score is an fp32 sum of D products; sums of probabilities and of 16 products at a time one after the other
            ds = (D + 8) * ULP * float((qh.abs() @ kh.abs().t().contiguous()).max()) * D ** -0.5 + 2e-6
            want = torch.logsumexp(s, 1)
            near(lse[t, heads], want, ds + (n / 2 + 64) * ULP + 2.0 ** -22 * want.abs().cpu(), f"lse of token {t}")
            out = torch.softmax(s, 1) @ vh
            # nothing cancels: the rounding of each probability to bf16 and the result's
            near(got[t, heads], out, ((2 * HALF_BF16 + 2 * ds + n * ULP + 64 * ULP) * out + 1e-30).cpu(), f"token {t}")


# sequences of as many new tokens, contexts of a length: a block for each item; one of them far longer: shares
@pytest.mark.parametrize("contexts", [(0, 0, 40), (9000, 0, 70), (100, 0, 12000)])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("e4m3", [False, True])
def test_long_chunks(dim, e4m3, contexts):
    new = [700, 701, 699]
    setup = _setup(dim, new, contexts, 32, 4 if dim > 96 else 16, dim, e4m3=e4m3)
    cache, table, first, context, q, _, _ = setup
    _marked(cache, table, contexts, new)
    for window, sinks in ((0, 0), (1500, 40)):
        got, lse = A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context), window=window, sinks=sinks, want_lse=True)
        _sample(setup, [0, 1, 63, 350, 699, 700, 1399, 1401, 1733, 2099], got, lse, window, sinks)


@pytest.mark.parametrize("dim", [96, 128, 192, 256])
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_block_for_each_of_many_sequences(dim, e4m3):
    each = [1] * 1030
    each[5], each[77], each[1029] = 0, 40, 3
    context = [b % 50 for b in range(1030)]
    context[9] = 700
    setup = _setup(dim, each, context, 4, 2, dim, e4m3=e4m3)
    check_all(setup)
