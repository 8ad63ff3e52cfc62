"""The append of drafted tokens at places of their own, and the move of accepted ones, against the definitions."""
import math
import random

import pytest
import torch

import paper_2507_17133_amd as A
from tests._draft_util import make_cache

pytestmark = pytest.mark.gpu


def _bits(cache):
    return tuple(t.contiguous().view(torch.uint8 if t.dtype == A.layer.E4M3 else torch.int16).clone() for t in (cache.k, cache.v))


def _append_inputs(seed, T, heads, kv, dim, e4m3, R=None, interleaved=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = make_cache(g, 40, 16, kv, dim, e4m3)
    qkv = torch.empty((T, heads + 2 * kv, dim), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    table = torch.randperm(40, generator=g, device="cuda")[:36].reshape(3, 12).to(torch.int32)
    return cache, A.Rope(None, 0) if R == 0 else A.make_rope(dim if R is None else R, interleaved), qkv.split((heads, kv, kv), 1), table


@pytest.mark.parametrize("dim,e4m3,R,interleaved", [(64, False, None, False), (96, True, 48, True), (128, False, 64, True), (128, True, None, False), (256, True, 16, False),
                                                   (192, False, 0, False)])
def test_places_apart_from_positions(dim, e4m3, R, interleaved):
    """Each token's q, and what lies at its place, are those of an append at its position; nothing else changes."""
    T, heads, kv = 23, 6, 2
    cache, rope, (q, k, v), table = _append_inputs(dim, T, heads, kv, dim, e4m3, R, interleaved)
    r = random.Random(dim)
    row = torch.tensor([r.randrange(3) for _ in range(T)], dtype=torch.int32, device="cuda")
    positions = torch.tensor([r.randrange(190) for _ in range(T)], dtype=torch.int32, device="cuda")
    places = torch.tensor(r.sample(range(190), T), dtype=torch.int32, device="cuda")
    before = _bits(cache)
    got = A.moe_rope_append_at(cache, rope, q, k, v, positions, places, table, table_row=row)
    after = _bits(cache)
    want = [t.clone() for t in before]
    for t in range(T):
        one = lambda x: x[t:t + 1].contiguous()
        assert torch.equal(A.moe_rope_append(cache, rope, one(q), one(k), one(v), positions[t:t + 1], table, table_row=row[t:t + 1])[0], got[t])
        at, pos = int(places[t]), int(positions[t])
        page = table[int(row[t])]
        for w, h in zip(want, _bits(cache)):
            w[int(page[at // 16]), at % 16] = h[int(page[pos // 16]), pos % 16]
    assert all(torch.equal(a, w) for a, w in zip(after, want))


@pytest.mark.parametrize("e4m3", [False, True])
def test_the_positions_as_places_are_the_other_call(e4m3):
    cache, rope, (q, k, v), table = _append_inputs(1, 30, 8, 2, 128, e4m3)
    row = torch.arange(30, device="cuda").to(torch.int32) % 3
    positions = torch.arange(30, device="cuda").to(torch.int32) * 5
    a = A.moe_rope_append(cache, rope, q, k, v, positions, table, table_row=row)
    bits = _bits(cache)
    cache.k.zero_(), cache.v.zero_()
    cache2, *_ = _append_inputs(1, 30, 8, 2, 128, e4m3)
    b = A.moe_rope_append_at(cache2, rope, q, k, v, positions, positions, table, table_row=row)
    assert torch.equal(a, b) and all(torch.equal(x, y) for x, y in zip(bits, _bits(cache2)))


def test_places_that_are_not_followed():
    cache, rope, (q, k, v), table = _append_inputs(2, 6, 4, 2, 64, False)
    table[1, 3] = 99
    row = torch.tensor([0, 0, 1, 7, 0, 0], dtype=torch.int32, device="cuda")
    positions = torch.tensor([5, 6, 50, 8, -1, 9], dtype=torch.int32, device="cuda")
    places = torch.tensor([-1, 12 * 16, 50, 8, 3, -(1 << 31)], dtype=torch.int32, device="cuda")
    before = _bits(cache)
    got = A.moe_rope_append_at(cache, rope, q, k, v, positions, places, table, table_row=row)
    assert all(torch.equal(a, b) for a, b in zip(before, _bits(cache)))
    assert not bool(got[4].any()) and bool(got[[0, 1, 2, 3, 5]].any(2).all())


# ---------------------------------------------------------------- move

def _moved(cache, table, sources, start, count, rows=None):
    """The cache's bits after the move, from the definition: all sources read first."""
    bits = [b.cpu() for b in _bits(cache)]
    want = [b.clone() for b in bits]
    t, (pages, page) = table.cpu(), cache.k.shape[:2]

    def place(b, p):
        row = b if rows is None else rows[b]
        if not 0 <= row < t.shape[0] or not 0 <= p < t.shape[1] * page or not 0 <= int(t[row, p // page]) < pages:
            return None
        return int(t[row, p // page]), p % page
    for b, src in enumerate(sources):
        last = -1
        for j in range(min(max(count[b], 0), len(src))):
            follows = src[j] > last and src[j] >= start[b] + j
            last = max(last, src[j])
            a, z = place(b, src[j]), place(b, start[b] + j)
            if follows and a is not None and z is not None:
                for w, h in zip(want, bits):
                    w[z] = h[a]
    return want


def _check_move(cache, table, sources, start, count, rows=None):
    want = _moved(cache, table, sources, start, count, rows)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    A.moe_cache_move(cache, table, i32(sources), i32(start), i32(count), table_row=None if rows is None else i32(rows))
    assert all(torch.equal(a.cpu(), w) for a, w in zip(_bits(cache), want))


@pytest.mark.parametrize("dim,kv,e4m3,page,heads_first,extra", [(64, 1, False, 16, False, 0), (128, 8, False, 16, True, 0), (96, 3, True, 1, False, 0), (16, 2, True, 5, False, 16),
                                                               (256, 4, True, 64, True, 0), (128, 40, False, 16, False, 8)])
def test_accepted_paths(dim, kv, e4m3, page, heads_first, extra):
    g, r = torch.Generator(device="cuda").manual_seed(dim), random.Random(dim)
    cache = make_cache(g, 5 * (-(-140 // page)) + 1, page, kv, dim, e4m3, heads_first, extra)
    pages = -(-140 // page)
    table = torch.randperm(5 * pages, generator=g, device="cuda").reshape(5, pages).to(torch.int32)
    start = [0, 7, 31, 64, 99]
    sources = [sorted(r.sample(range(s, s + 40), 21)) for s in start]
    _check_move(cache, table, sources, start, [21, 0, 1, 9, 20])
    _check_move(cache, table, [[s + j for j in range(21)] for s in start], start, [21] * 5)           # in place already
    _check_move(cache, table, [[s + 1 + j for j in range(21)] for s in start], start, [21, 5, 8, 9, 16])     # every one one place down


def test_entries_that_are_not_followed():
    g = torch.Generator(device="cuda").manual_seed(5)
    cache = make_cache(g, 30, 16, 2, 64)
    table = torch.randperm(30, generator=g, device="cuda")[:20].reshape(4, 5).to(torch.int32)
    table[1, 2], table[2, 0] = -1, 30
    _check_move(cache, table, [[5, 5, 9, 8, -3, 20, 19, 30, 79, 80, 90, 2000], [40, 41, 50, 60, 61, 62, 63, 64, 65, 66, 67, 68], [3, 20, 21, 22, 23, 24, 25, 26, 27, 28, 29, 30],
                                    [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12]], [2, 33, 10, 20], [12, 12, 50, 12])
    _check_move(cache, table, [[30, 40], [30, 40], [30, 40]], [10, -1, 79], [2, 2, 2], rows=[3, 0, 9])
    _check_move(cache, table, [[(1 << 31) - 1, 3], [70, 71]], [(1 << 31) - 2, 5], [-4, 2], rows=[0, 3])


def test_a_graph_and_a_stream():
    g = torch.Generator(device="cuda").manual_seed(6)
    cache = make_cache(g, 8, 16, 4, 128)
    table = torch.arange(8, dtype=torch.int32, device="cuda").reshape(2, 4)
    sources, start, count = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([[10, 13], [20, 21]], [9, 20], [2, 1]))
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.moe_cache_move(cache, table, sources, start, count)
    for turn in range(4):
        cache.k.normal_(), cache.v.normal_()
        sources += 1
        want = _moved(cache, table, sources.tolist(), start.tolist(), count.tolist())
        if turn == 2:
            side.wait_stream(torch.cuda.current_stream())
            A.moe_cache_move(cache, table, sources, start, count, stream=side)
            torch.cuda.current_stream().wait_stream(side)
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.cpu(), w) for a, w in zip(_bits(cache), want))


def test_nan_is_moved_as_it_is():
    g = torch.Generator(device="cuda").manual_seed(7)
    cache = make_cache(g, 4, 16, 1, 64)
    cache.k[0, 9] = math.nan
    table = torch.arange(4, dtype=torch.int32, device="cuda").reshape(1, 4)
    _check_move(cache, table, [[9]], [3], [1])
