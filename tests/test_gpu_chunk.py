"""Attention of several new tokens of a sequence (drafted trees, prompts' chunks) over a paged cache against the definition in 64 bits."""
import math
import random

import pytest
import torch

import paper_2507_17133_amd as A
from tests._draft_util import attend, make_cache, random_tree, rows_of, visible
from tests._layer_util import near

pytestmark = pytest.mark.gpu


def _setup(seed, each, context, heads, kv, dim, page=16, e4m3=False, heads_first=False, tree=False, missing=0.0, blank=0.0, extra=0, more_pages=0):
    g, r = torch.Generator(device="cuda").manual_seed(seed), random.Random(seed)
    B, T = len(each), sum(each)
    pages = max(1, -(-max(c + n for c, n in zip(context, each)) // page)) + more_pages
    cache = make_cache(g, B * pages + 2, page, kv, dim, e4m3, heads_first, extra)
    table = torch.randperm(B * pages + 2, generator=g, device="cuda")[: B * pages].reshape(B, pages).to(torch.int32)
    if missing:
        lost = torch.rand((B, pages), generator=g, device="cuda") < missing
        table = torch.where(lost, torch.where(torch.rand((B, pages), generator=g, device="cuda") < 0.5, -1, 1 << 30), table).to(torch.int32)
    first = [0]
    for n in each:
        first.append(first[-1] + n)
    q = torch.empty((T, heads, dim), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    seen = positions = None
    if tree:
        words = max(1, -(-max(each) // 32))
        parts = [A.tree_masks(random_tree(r, n), words) for n in each]
        seen = torch.cat([s for s, _ in parts])
        positions = torch.cat([c + d for c, (_, d) in zip(context, parts)]).to(torch.int32)
        if blank:
            seen[torch.rand(T) < blank] = 0
    return cache, table, first, list(context), q, seen, positions


def _dev(x):
    return None if x is None else torch.as_tensor(x, dtype=torch.int32).cuda()


def _check(setup, window=0, sinks=0, scale=None, rows=None, what=""):
    cache, table, first, context, q, seen, positions = setup
    scale = q.shape[2] ** -0.5 if scale is None else scale
    out, lse = A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context), table_row=_dev(rows), seen=_dev(seen), positions=_dev(positions), scale=scale,
                                     window=window, sinks=sinks, want_lse=True)
    k, v, there = rows_of(cache, table)
    see, row_of = visible(first, context, there, q.shape[0], seen, None if positions is None else positions.tolist(), window, sinks, rows)
    want, want_lse, tol, tol_lse = attend(q.double().cpu(), k, v, see, row_of, scale)
    own = row_of >= 0
    near(out[own.cuda()], want[own], tol[own], what + " out")
    got_lse = lse.double().cpu()[own]
    assert torch.equal(got_lse == -math.inf, want_lse[own] == -math.inf), what
    fine = want_lse[own] != -math.inf
    near(got_lse[fine], want_lse[own][fine], tol_lse[own][fine], what + " lse")
    return out, lse


def _same_within_roundings(a, b, what):
    """Two ways to the same result: each may round its probabilities to bf16 (off by at most half a step, 2^-8 of them, so 2^-8 of sum p |v| <= max |v| < 6 for these inputs)
    and rounds its result (2^-8 of it)."""
    near(a, b.double(), 2 * 2.0 ** -8 * b.double().abs().cpu() + 2 * 2.0 ** -8 * 6, what)


# every head width, type and height of tiles: rows of a sequence from 1 to several tiles
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new,heads,kv", [(1, 3, 3), (7, 8, 2), (33, 4, 2), (40, 8, 1)])
def test_trees(dim, e4m3, new, heads, kv):
    each = [new, max(1, new // 2), new]
    _check(_setup(dim + new, each, [150, 0, 77], heads, kv, dim, 16, e4m3, heads_first=new % 2 == 1, tree=True))


@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new,heads,kv", [(1, 2, 1), (9, 7, 7), (70, 7, 1), (200, 4, 2)])
def test_chunks(dim, e4m3, new, heads, kv):
    _check(_setup(dim + new, [new, 3], [0, 131], heads, kv, dim, 48, e4m3))


@pytest.mark.parametrize("page", [1, 3, 16, 64, 128])
@pytest.mark.parametrize("context", [0, 1, 15, 31, 32, 33, 63, 64, 65, 127, 128, 129, 400])
def test_borders(page, context):
    _check(_setup(context, [5, 1, 30], [context, context + 1, max(0, context - 1)], 4, 2, 64, page, tree=True))
    _check(_setup(context, [5, 1, 30], [context, context + 1, max(0, context - 1)], 4, 2, 64, page))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (32, 4), (33, 40), (64, 64), (100, 1), (200, 500), (1 << 30, 7), (0, 9)])
@pytest.mark.parametrize("tree", [False, True])
def test_window_and_sinks(window, sinks, tree):
    _check(_setup(window, [40, 3, 129, 1], [300, 5, 37, 500], 4, 2, 64, 16, tree=tree), window, sinks)
    _check(_setup(window, [8, 3], [190, 700], 8, 2, 128, 16, e4m3=True, tree=tree), window, sinks)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 20)])
def test_missing_pages_and_blank_rows(tree, window, sinks):
    _check(_setup(1, [20, 6, 33], [200, 90, 300], 4, 2, 64, 16, tree=tree, missing=0.4, blank=0.3), window, sinks)
    _check(_setup(2, [20, 6, 33], [200, 90, 300], 4, 2, 96, 1, True, tree=tree, missing=0.5, blank=0.3), window, sinks)
    _check(_setup(3, [2, 3], [0, 0], 8, 2, 128, 16, tree=tree, missing=1.0), window, sinks)


def test_nothing_to_see():
    s = _setup(4, [6, 6], [0, 40], 4, 2, 64, tree=True)
    s[5][:] = 0
    out, lse = _check(s)
    assert not bool(out[:6].any()) and bool((lse[:6] == -math.inf).all())
    out, lse = _check(_setup(5, [6, 6], [0, 40], 4, 2, 64), rows=[7, -1])          # rows that the table does not have
    assert not bool(out.any()) and bool((lse == -math.inf).all())


def test_empty_sequences_and_tokens_of_none():
    cache, table, first, context, q, _, _ = _setup(6, [3, 0, 5, 0, 0, 1, 4], [10, 20, 0, 5, 7, 64, 33], 4, 2, 64)
    _check((cache, table, first, context, q, None, None))
    # tokens before the first and behind the last sequence, and a first beyond the call's tokens
    for at in ([2, 3, 3, 8, 8, 9, 9, 11], [0, 3, 3, 8, 8, 9, 10, 10], [0, 3, 3, 8, 8, 9, 12, 99]):
        out = torch.full_like(q, 7.0)
        n = table.shape[1] * 16
        A.moe_chunk_attention(cache, q, table, _dev(at), _dev(context), out=out)
        own = torch.zeros(q.shape[0], dtype=torch.bool)
        own[at[0]:min(at[-1], q.shape[0])] = True
        assert bool((out[~own.cuda()] == 7.0).all()) and not bool((out[own.cuda()] == 7.0).all(2).any())
        _check((cache, table, at, context, q, None, None))
    assert n > 0


def test_rows_of_the_table_and_odd_contexts():
    s = _setup(7, [4, 9, 2], [50, 20, 30], 4, 2, 64, more_pages=1)
    _check(s, rows=[2, 0, 0])
    cache, table, first, _, q, _, _ = s
    cap = table.shape[1] * 16
    _check((cache, table, first, [-5, cap, cap - 3], q, None, None))               # behind the table's last position nothing is there
    _check((cache, table, first, [cap + 100, 1 << 30, 0], q, None, None), window=1 << 29)


@pytest.mark.parametrize("n_seqs,new,context", [(1030, 1, 3), (300, 2, 40), (1, 900, 0), (2, 500, 600)])
def test_many_items(n_seqs, new, context):
    """A block for each item where there are many sequences or items; long chunks in shares."""
    each = [new - (b % 2 if new > 1 else 0) for b in range(n_seqs)]
    _check(_setup(n_seqs, each, [context + b % 3 for b in range(n_seqs)], 8 if n_seqs == 300 else 2, 8 if n_seqs == 300 else 1, 64))


@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 4)])
def test_a_block_for_each_item_of_long_chunks(window, sinks):
    cache, table, first, context, q, _, _ = _setup(22, [700 - b for b in range(12)], [31 * b for b in range(12)], 64, 32, 64)
    got = A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context), window=window, sinks=sinks)
    row = torch.repeat_interleave(torch.arange(12), torch.tensor([700 - b for b in range(12)]))
    n = torch.tensor([context[b] + t - first[b] + 1 for t, b in enumerate(row.tolist())], dtype=torch.int32)
    want = A.moe_sink_attention(cache, q, table, n.cuda(), window, sinks, table_row=row.to(torch.int32).cuda())
    _same_within_roundings(got, want, "single tokens")


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("lengths", [(0, 0, 0), (9000, 0, 70), (1000, 0, 9000)])
def test_long_chunks_of_very_different_contexts(lengths, e4m3):
    """A block for each item if they are of a length, shares of their steps if one sequence has most of them: the device decides."""
    new = [400, 401, 399]
    cache, table, first, context, q, _, _ = _setup(23, new, list(lengths), 64, 32, 64, e4m3=e4m3)
    got, lse = A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context), want_lse=True)
    row = torch.repeat_interleave(torch.arange(3), torch.tensor(new))
    n = torch.tensor([context[b] + t - first[b] + 1 for t, b in enumerate(row.tolist())], dtype=torch.int32)
    want = A.moe_sink_attention(cache, q, table, n.cuda(), 0, 0, table_row=row.to(torch.int32).cuda())
    _same_within_roundings(got, want, "single tokens")
    assert bool(torch.isfinite(lse).all())


def test_captured_chunks_whose_contexts_change():
    """One graph and one workspace: a block for each item, then shares, then blocks again, as the lengths of the replay say."""
    new, lengths = [400, 401, 399], [(0, 0, 0), (9000, 0, 70), (30, 60, 0), (0, 9000, 1000), (0, 0, 0)]
    cache, table, first, _, q, _, _ = _setup(24, new, [9000, 9000, 9000], 64, 32, 64)
    first, context = _dev(first), _dev([0, 0, 0])
    ws = A.alloc_chunk_workspace(cache, 3, q.shape[0], 64)
    call = lambda workspace: A.moe_chunk_attention(cache, q, table, first, context, want_lse=True, workspace=workspace)
    eager = []
    for n in lengths:
        context.copy_(torch.tensor(n, dtype=torch.int32))
        eager.append(call(A.alloc_chunk_workspace(cache, 3, q.shape[0], 64)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = call(ws)
    for n, (want, want_lse) in zip(lengths, eager):
        context.copy_(torch.tensor(n, dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse), n


def test_one_long_sequence_among_short_ones():
    _check(_setup(8, [5, 5, 5, 5], [20000, 3, 50, 0], 8, 2, 64, 64, tree=True))
    _check(_setup(9, [30, 1], [30000, 9], 8, 2, 128, 16, e4m3=True), window=25000, sinks=5)


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-6])
def test_scales(scale):
    _check(_setup(10, [20, 3], [100, 7], 4, 2, 64, tree=True), scale=scale)
    _check(_setup(11, [20, 3], [100, 7], 4, 2, 64, e4m3=True), scale=scale)


def test_strides():
    cache, table, first, context, q, seen, positions = _setup(12, [20, 9], [60, 5], 4, 2, 64, tree=True, extra=8)
    want, want_lse = A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context), seen=_dev(seen), positions=_dev(positions), want_lse=True)
    T, wide = q.shape[0], torch.zeros((q.shape[0], 7, 64), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:5] = q
    out = torch.full((T, 6, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    masks = torch.full((T, 3), -1, dtype=torch.int32, device="cuda")
    masks[:, :1] = _dev(seen)
    table2 = torch.full((2, table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    table2[:, : table.shape[1]] = table
    got, lse = A.moe_chunk_attention(cache, wide[:, 1:5], table2[:, : table.shape[1]], _dev(first), _dev(context), seen=masks[:, :1], positions=_dev(positions),
                                     out=out[:, 1:5], want_lse=True)
    assert torch.equal(got, want) and torch.equal(lse, want_lse) and bool((out[:, 0] == 5.0).all()) and bool((out[:, 5] == 5.0).all())
    _check((cache, table, first, context, q, seen, positions))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("new,heads,kv,dim", [(6, 8, 2, 64), (12, 8, 2, 128), (20, 4, 1, 96), (45, 8, 2, 128), (24, 4, 1, 256)])
def test_what_a_token_does_not_see_does_not_matter(bad, which, new, heads, kv, dim):
    """Values that are not finite at a drafted token's place reach the tokens that see it and no others; places that nobody sees may hold anything."""
    for tree in (True, False):
        cache, table, first, context, q, seen, positions = _setup(13, [new, 5], [70, 100], heads, kv, dim, tree=tree, more_pages=1)
        call = lambda: A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context), seen=_dev(seen), positions=_dev(positions))
        clean = call()
        held = cache.k if which == "k" else cache.v
        # behind the last token, and in pages of nobody
        used = torch.zeros(held.shape[:2], dtype=torch.bool, device="cuda")
        for b, (c, n) in enumerate(zip(context, (new, 5))):
            p = torch.arange(c + n, device="cuda")
            used[table[b].long()[p // 16], p % 16] = True
        held[~used] = bad
        assert torch.equal(call(), clean)
        j = new // 2
        p = context[0] + j
        held[table[0, p // 16].long(), p % 16] = bad
        got = call()
        reaches = torch.tensor([t < new and (bool(seen[t, j // 32].item() >> (j % 32) & 1) if tree else t >= j) for t in range(q.shape[0])])
        assert bool(reaches.any()) and not bool(reaches.all())
        _same_within_roundings(got[~reaches.cuda()], clean[~reaches.cuda()], "others")
        hit = got[reaches.cuda()].float()
        if which == "v":
            assert bool((hit.isnan() if bad != bad else hit == bad).all())
        elif bad != bad:
            assert bool(hit.isnan().all())


def test_nan_of_an_8_bit_cache_and_of_q():
    cache, table, first, context, q, seen, positions = _setup(14, [12, 5], [70, 100], 8, 2, 128, e4m3=True, tree=True)
    call = lambda: A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context), seen=_dev(seen), positions=_dev(positions))
    clean = call()
    cache.v.view(torch.uint8)[table[0, 76 // 16].long(), 76 % 16] = 0x7F                # NaN, at the place of token 6
    got = call()
    reaches = torch.tensor([t < 12 and bool(seen[t, 0].item() >> 6 & 1) for t in range(17)]).cuda()
    assert bool(got[reaches].isnan().all()) and not bool(got[~reaches].isnan().any())
    _same_within_roundings(got[~reaches], clean[~reaches], "others")
    cache.v.view(torch.uint8)[table[0, 76 // 16].long(), 76 % 16] = 0
    before = call()
    q[3, 5] = math.nan
    after = call()
    assert bool(after[3, 5].isnan().all())
    q[3, 5] = 0
    keep = torch.ones(17, 8, dtype=torch.bool, device="cuda")
    keep[3, 5] = False
    _same_within_roundings(after[keep], before[keep], "other rows")


def test_large_scores_and_values():
    """Scores that grow along the cache move the maximum step by step; probabilities of far ones vanish; large values of v overflow nothing."""
    cache, table, first, context, q, _, _ = _setup(15, [6, 40], [500, 900], 4, 2, 128)
    p = torch.arange(960, device="cuda")
    for b in range(2):
        at = p[: context[b] + (6, 40)[b]]
        cache.k[table[b].long()[at // 16], at % 16] *= (1 + at / 40.0)[:, None, None].to(torch.bfloat16)
    cache.v.mul_(1e30)
    _check((cache, table, first, context, q, None, None))


def test_the_same_call_gives_the_same_bits():
    for s in (_setup(16, [30] * 9, [700 + 50 * b for b in range(9)], 8, 2, 128, tree=True), _setup(17, [900], [100], 8, 2, 64)):
        cache, table, first, context, q, seen, positions = s
        ws = A.alloc_chunk_workspace(cache, 9, 270, 8)
        call = lambda: A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context), seen=_dev(seen), positions=_dev(positions), want_lse=True, workspace=ws)
        a = call()
        ws.fill_(255)                                     # needs no initialisation
        b = call()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_another_stream_and_a_graph():
    cache, table, first, context, q, seen, positions = _setup(18, [20, 11], [300, 90], 8, 2, 128, tree=True, more_pages=2)
    f, c, s, p = _dev(first), _dev(context), _dev(seen), _dev(positions)
    ws, out = A.alloc_chunk_workspace(cache, 2, 31, 8), torch.empty_like(q)
    want = A.moe_chunk_attention(cache, q, table, f, c, seen=s, positions=p, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = A.moe_chunk_attention(cache, q, table, f, c, seen=s, positions=p, workspace=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graphs = []
    for _ in range(2):                                    # two graphs that share a workspace, replayed by turns
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            A.moe_chunk_attention(cache, q, table, f, c, seen=s, positions=p, workspace=ws, out=out)
        graphs.append(graph)
    for turn in range(6):
        c.copy_(torch.tensor([300 - 7 * turn, 90 + turn], dtype=torch.int32))
        p.copy_(_dev(positions) + torch.tensor([-7 * turn] * 20 + [turn] * 11, dtype=torch.int32, device="cuda"))
        q.normal_()
        graphs[turn % 2].replay()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, A.moe_chunk_attention(cache, q, table, f, c, seen=s, positions=p))


def test_single_tokens_agree_with_the_other_attention():
    """One new token a sequence: what moe_sink_attention gives for its length, within the roundings of both."""
    cache, table, first, context, q, _, _ = _setup(19, [1] * 12, [60 * b for b in range(12)], 8, 2, 128)
    n = _dev([c + 1 for c in context])
    for window, sinks in ((0, 0), (100, 4)):
        a = A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context), window=window, sinks=sinks)
        b = A.moe_sink_attention(cache, q, table, n, window, sinks)
        _same_within_roundings(a, b, "both")


def test_a_tensor_that_requires_a_gradient_is_refused():
    cache, table, first, context, q, _, _ = _setup(20, [2], [5], 2, 1, 64)
    q.requires_grad_()
    with pytest.raises(AssertionError):
        A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context))
    with torch.no_grad():
        A.moe_chunk_attention(cache, q, table, _dev(first), _dev(context))


def test_no_tokens():
    cache, table, first, context, q, _, _ = _setup(21, [2], [5], 2, 1, 64)
    assert A.moe_chunk_attention(cache, q[:0], table, _dev([0, 0]), _dev([5])).shape == (0, 2, 64)
    assert A.moe_chunk_attention(cache, q[:0], table[:0], _dev([0]), _dev([])).shape == (0, 2, 64)
