"""Attention of new tokens over the paged cache against 64 bits."""
import math

import pytest
import torch

import paper_2507_17133_amd as P
from tests._layer_util import E4M3, attention, near

pytestmark = pytest.mark.gpu


def _case(lengths, H, Hk, D, page, e4m3=False, heads_first=False, seed=0, std=1.0, spare=3, garbage=True):
    """q, a cache with pages in random order (unused places hold NaN), its block table, and what the table leads to [T, L, Hk, D]."""
    g = torch.Generator().manual_seed(seed)
    T, most = len(lengths), max(1, -(-max(lengths) // page))
    n_pages = T * most + spare
    table = torch.randperm(n_pages, generator=g)[: T * most].reshape(T, most).to(torch.int32)
    shape = (n_pages, page, Hk, D)
    scales = [torch.rand(Hk, generator=g) * 0.01 + 0.005 for _ in range(2)] if e4m3 else [None, None]
    raw, seen = [], []
    used = torch.zeros((n_pages, page), dtype=torch.bool)
    for t, n in enumerate(lengths):
        at = torch.arange(n)
        used[table[t, at // page].long(), at % page] = True
    for i in range(2):
        x = torch.randn(shape, generator=g) * std
        x = (x * 64).to(E4M3) if e4m3 else x.to(torch.bfloat16)
        if garbage:
            bits = x.view(torch.uint8) if e4m3 else x.view(torch.int16)
            bits[~used] = 0x7F if e4m3 else 0x7FC0             # NaN
        raw.append(x)
        full = x.float().double()
        if e4m3:
            full = full * scales[i].double()[None, None, :, None]
        seen.append(full[table.long()].reshape(T, most * page, Hk, D))
    dev = [x.transpose(1, 2).contiguous().cuda().transpose(1, 2) if heads_first else x.cuda() for x in raw]
    cache = P.KvCache(*dev, *(None if s is None else s.cuda() for s in scales))
    q = (torch.randn((T, H, D), generator=g)).to(torch.bfloat16)
    return q, cache, table, seen[0], seen[1]


def _check(lengths, H, Hk, D, page, window=0, scale=None, **kw):
    q, cache, table, k, v = _case(lengths, H, Hk, D, page, **kw)
    scale = D ** -0.5 if scale is None else scale
    n = torch.tensor(lengths)
    out, lse = P.moe_paged_attention(cache, q.cuda(), table.cuda(), n.to(torch.int32).cuda(), scale=scale, window=window, want_lse=True)
    want, want_lse, tol, tol_lse = attention(q.double(), k, v, n, scale, window)
    near(out, want, tol, "out")
    empty = want_lse == -math.inf
    assert torch.equal(lse.cpu() == -math.inf, empty)
    near(torch.where(empty, 0.0, lse.cpu().double()), torch.where(empty, 0.0, want_lse), tol_lse, "lse")
    return out, lse


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("H,Hk", [(4, 4), (8, 2), (5, 1), (24, 1), (32, 2)])
@pytest.mark.parametrize("e4m3,heads_first,page", [(False, False, 16), (True, True, 7), (True, False, 64), (False, True, 1)])
def test_heads_types_and_pages(D, H, Hk, e4m3, heads_first, page):
    _check([1, 0, 31, 32, 33, 127, 128, 129, 300, 257], H, Hk, D, page, e4m3=e4m3, heads_first=heads_first, seed=D + H)


@pytest.mark.parametrize("lengths", [[0], [1], [2], [0, 0, 0], [128], [4097], [0, 9000, 0, 5], [1] * 700, [0] * 3 + [640] * 300, [3000, 1] * 40])
@pytest.mark.parametrize("e4m3", [False, True])
def test_lengths(lengths, e4m3):
    _check(lengths, 8, 2, 64, 16, e4m3=e4m3, seed=len(lengths))


@pytest.mark.parametrize("window", [1, 16, 100, 128, 1000])
def test_window(window):
    _check([0, 1, 15, 16, 17, 99, 100, 101, 500, 1500], 8, 2, 128, 16, window=window, seed=window)


def test_one_long_sequence_among_short_ones():
    _check([20000] + [3] * 20, 8, 1, 128, 64, seed=5)


@pytest.mark.parametrize("std,scale", [(30.0, 1.0), (1e-3, 1.0), (5.0, -0.7), (1.0, 0.0)])
def test_sharp_and_flat_scores(std, scale):
    _check([700, 65, 1], 8, 4, 128, 16, std=std, scale=scale, seed=6)


def test_pages_and_rows_that_are_not_there():
    """Positions whose page is outside the pool do not take part; a token whose row is outside the table has none; lengths end with the
    table's row, and below 0 there is none."""
    lengths = [100, 100, 100, 100, 100]
    q, cache, table, k, v = _case(lengths, 8, 2, 128, 16, seed=7, garbage=False)
    n_pages = cache.k.shape[0]
    table[0, 1], table[0, 3], table[1, 0], table[2, :] = -1, n_pages, 2 ** 31 - 1, -5
    gone = ((table < 0) | (table >= n_pages)).repeat_interleave(16, 1)
    n = torch.tensor([100, 112, 100, 2 ** 31 - 1, -4])
    rows = torch.tensor([0, 1, 2, 3, 4])
    out, lse = P.moe_paged_attention(cache, q.cuda(), table.cuda(), n.to(torch.int32).cuda(), table_row=rows.to(torch.int32).cuda(), want_lse=True)
    want, want_lse, tol, _ = attention(q.double(), k, v, n, 128 ** -0.5, left_out=gone)
    near(out, want, tol, "out")
    assert torch.equal(lse.cpu() == -math.inf, want_lse == -math.inf) and not bool(out[2].any()) and not bool(out[4].any())
    rows = torch.tensor([3, 9, -1, 0, 3])
    out, lse = P.moe_paged_attention(cache, q.cuda(), table.cuda(), n.to(torch.int32).cuda(), table_row=rows.to(torch.int32).cuda(), want_lse=True)
    at = rows.clone()
    at[1] = at[2] = 0
    n = torch.tensor([100, 0, 0, 2 ** 31 - 1, 0])
    want, want_lse, tol, _ = attention(q.double(), k[at], v[at], n, 128 ** -0.5, left_out=gone[at])
    near(out, want, tol, "out")
    assert torch.equal(lse.cpu() == -math.inf, want_lse == -math.inf)


def test_infinities_and_nan_inside_the_sequence():
    """A NaN score makes its heads NaN; a key whose score is -infinity has no weight; other tokens stay as they are."""
    q, cache, table, k, v = _case([200, 200, 200], 4, 2, 64, 16, seed=8)
    q = q.abs()
    cache.k[table[0, 3].item(), 5, 1, 0] = math.nan
    cache.k[table[1, 2].item(), 4, 0, :] = -math.inf
    k[1, 36, 0] = -1e6                                     # weight 0 all the same
    n = torch.tensor([200, 200, 200])
    out, lse = P.moe_paged_attention(cache, q.cuda(), table.cuda(), n.to(torch.int32).cuda(), want_lse=True)
    want, _, tol, _ = attention(q.double(), k, v, n, 64 ** -0.5)
    assert bool(out[0, 2:].isnan().all()) and bool(lse[0, 2:].isnan().all())
    near(out[0, :2], want[0, :2], tol[0, :2])
    tol[1, :2] = attention(q.double(), k.clamp_min(-100), v, n, 64 ** -0.5)[2][1, :2]
    near(out[1:], want[1:], tol[1:])


def test_strided_q_and_out_no_lse_own_stream_and_repeatable():
    lengths = [900, 40, 0, 77]
    q, cache, table, k, v = _case(lengths, 8, 2, 128, 16, seed=9)
    n = torch.tensor(lengths, dtype=torch.int32).cuda()
    wide = torch.zeros((4, 8 * 128 + 64), dtype=torch.bfloat16, device="cuda")
    wide[:, 16:16 + 1024] = q.reshape(4, -1).cuda()
    qv = wide[:, 16:16 + 1024].unflatten(1, (8, 128))
    ov = torch.full((4, 1200), 3.0, dtype=torch.bfloat16, device="cuda")
    dense = P.moe_paged_attention(cache, q.cuda(), table.cuda(), n)
    ws = P.alloc_attention_workspace(cache, 4, 8)
    t = table.cuda()
    for i in range(3):
        ws.fill_(255)                                      # nothing an earlier call left is read
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        out = P.moe_paged_attention(cache, qv, t, n, out=ov[:, 4:4 + 1024].unflatten(1, (8, 128)), workspace=ws, stream=s)
        s.synchronize()
        assert torch.equal(out, dense)
    assert bool((ov[:, :4] == 3).all()) and bool((ov[:, 1028:] == 3).all())


def test_tokens_of_one_sequence_share_its_row():
    """A prompt's chunk: all tokens name one row, each sees the positions up to its own."""
    q, cache, table, k, v = _case([77], 8, 2, 64, 16, seed=10)
    T = 77
    q = torch.randn((T, 8, 64), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    n = torch.arange(1, T + 1)
    out = P.moe_paged_attention(cache, q.cuda(), table.cuda(), n.to(torch.int32).cuda(), table_row=torch.zeros(T, dtype=torch.int32, device="cuda"))
    want, _, tol, _ = attention(q.double(), k.expand(T, -1, -1, -1), v.expand(T, -1, -1, -1), n, 64 ** -0.5)
    near(out, want, tol, "out")


def test_graph_replays():
    lengths = [5000, 40, 0, 77, 300]
    q, cache, table, k, v = _case(lengths, 8, 2, 128, 16, seed=11)
    qd, t, n = q.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
    out, ws = torch.empty_like(qd), P.alloc_attention_workspace(cache, 5, 8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.moe_paged_attention(cache, qd, t, n, out=out, workspace=ws)
    for i in range(4):
        n.copy_(torch.tensor([5000 - 1000 * i, 40 + i, i, 77, 300 * i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        # bit for bit, NaN of places beyond what the case filled included
        assert torch.equal(out.view(torch.int16), P.moe_paged_attention(cache, qd, t, n).view(torch.int16))
        qd.mul_(0.9)


def test_places_beyond_32_bits():
    """A cache of more than 2^31 elements (and 2^32 bytes): the sequence's pages lie at its far end."""
    n_pages, page, Hk, D = 2300, 1024, 8, 128              # 2.4e9 elements, 4.8 GB each
    k, v = (torch.empty((n_pages, page, Hk, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(12)
    kc, vc = (torch.randn((2, page, Hk, D), generator=g).to(torch.bfloat16) for _ in range(2))
    k[-2:], v[-2:] = kc.cuda(), vc.cuda()
    cache = P.KvCache(k, v)
    q = torch.randn((1, 8, D), generator=g).to(torch.bfloat16)
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    out = P.moe_paged_attention(cache, q.cuda(), table, torch.tensor([1500], dtype=torch.int32, device="cuda"))
    seen = [x[[1, 0]].reshape(1, 2 * page, Hk, D).double() for x in (kc, vc)]
    want, _, tol, _ = attention(q.double(), *seen, torch.tensor([1500]), D ** -0.5)
    near(out, want, tol, "out")
    # and the append writes there
    x = torch.randn((1, 24, D), generator=g).to(torch.bfloat16).cuda()
    P.moe_rope_append(cache, P.layer.Rope(None, 0), x[:, :8], x[:, 8:16], x[:, 16:], torch.tensor([1023], dtype=torch.int32, device="cuda"), table)
    assert torch.equal(k[-1, 1023], x[0, 8:16]) and torch.equal(v[-1, 1023], x[0, 16:])
