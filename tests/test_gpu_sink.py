"""Attention with a window and sinks of single tokens against the definition in 64 bits; without sinks it is moe_paged_attention to the bit."""
import math

import pytest
import torch

import paper_2507_17133_amd as A
from tests._draft_util import attend, make_cache, rows_of
from tests._layer_util import near

pytestmark = pytest.mark.gpu


def _setup(seed, lengths, heads, kv, dim, page=16, e4m3=False, heads_first=False, missing=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, pages = len(lengths), max(1, -(-max(lengths) // page))
    cache = make_cache(g, T * pages + 1, page, kv, dim, e4m3, heads_first)
    table = torch.randperm(T * pages + 1, generator=g, device="cuda")[: T * pages].reshape(T, pages).to(torch.int32)
    if missing:
        table = torch.where(torch.rand((T, pages), generator=g, device="cuda") < missing, -1, table).to(torch.int32)
    q = torch.empty((T, heads, dim), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    return cache, table, q, torch.tensor(lengths, dtype=torch.int32, device="cuda")


def _check(setup, window, sinks):
    cache, table, q, n = setup
    out, lse = A.moe_sink_attention(cache, q, table, n, window, sinks, want_lse=True)
    k, v, there = rows_of(cache, table)
    p, n = torch.arange(k.shape[1])[None, :], n.cpu().clamp(0, k.shape[1])[:, None]
    see = (p < n) & there
    if window:
        see &= (p >= n - window) | (p < sinks)
    want, want_lse, tol, tol_lse = attend(q.double().cpu(), k, v, see, torch.arange(q.shape[0]), q.shape[2] ** -0.5)
    near(out, want, tol, "out")
    assert torch.equal(lse.cpu() == -math.inf, want_lse == -math.inf)
    fine = want_lse != -math.inf
    near(lse.cpu()[fine], want_lse[fine], tol_lse[fine], "lse")


@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 8), (24, 1), (32, 4)])
def test_widths_types_and_heads(dim, e4m3, heads, kv):
    _check(_setup(dim, [0, 1, 7, 300, 129, 64], heads, kv, dim, 16, e4m3, heads_first=heads == 8), 50, 5)


@pytest.mark.parametrize("window", [1, 5, 31, 32, 33, 128, 500, 1 << 30, (1 << 31) - 1])
@pytest.mark.parametrize("sinks", [0, 1, 4, 31, 32, 129, 400, (1 << 31) - 1])
def test_borders(window, sinks):
    _check(_setup(window % 1000 + sinks % 1000, [0, 1, 2, 31, 32, 33, 127, 128, 129, 160, 400, 700], 8, 2, 64, 16), window, sinks)


@pytest.mark.parametrize("page", [1, 7, 64, 128])
def test_pages(page):
    _check(_setup(page, [500, 3, 129, 260], 8, 2, 128, page, missing=0.3), 100, 20)
    _check(_setup(page, [500, 3, 129, 260], 8, 2, 128, page, True, missing=1.0), 100, 20)


def test_a_long_sequence_among_short_ones():
    _check(_setup(1, [60000, 5, 90, 0], 8, 2, 64, 16), 30000, 2000)


def test_without_sinks_it_is_the_other_call():
    cache, table, q, n = _setup(2, [0, 1, 7, 3000, 129, 64], 8, 2, 128)
    for window in (0, 1, 100, 5000):
        a, b = A.moe_sink_attention(cache, q, table, n, window, 0, want_lse=True), A.moe_paged_attention(cache, q, table, n, window=window, want_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # a window of 0 sees everything, with sinks or without
    assert torch.equal(A.moe_sink_attention(cache, q, table, n, 0, 9), A.moe_paged_attention(cache, q, table, n))


def test_what_is_left_out_does_not_matter():
    cache, table, q, n = _setup(3, [400, 300], 8, 2, 128)
    want = A.moe_sink_attention(cache, q, table, n, 64, 16)
    for b in range(2):
        p = torch.arange(16, int(n[b]) - 64, device="cuda")
        for t in (cache.k, cache.v):
            t[table[b].long()[p // 16], p % 16] = math.nan
    assert torch.equal(A.moe_sink_attention(cache, q, table, n, 64, 16), want)


def test_a_graph():
    cache, table, q, n = _setup(4, [400, 300, 90], 8, 2, 128)
    ws, out = A.alloc_attention_workspace(cache, 3, 8), torch.empty_like(q)
    A.moe_sink_attention(cache, q, table, n, 64, 4, out=out, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.moe_sink_attention(cache, q, table, n, 64, 4, out=out, workspace=ws)
    for turn in range(4):
        n.sub_(31)
        q.normal_()
        graph.replay()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, A.moe_sink_attention(cache, q, table, n, 64, 4))
