"""Rotary positions and the append to the paged cache against 64 bits."""
import math

import pytest
import torch

import paper_2507_17133_amd as P
from tests._layer_util import E4M3, HALF_BF16, HALF_E4M3, near

pytestmark = pytest.mark.gpu


def _rotate(x, pos, turns, factor, R, interleaved):
    """64 bits, and the size that errors of cos and sin (an fp32 angle of at most half a turn, 2 ulp) are relative to."""
    x = x.double().clone()
    i = torch.arange(R // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    t = pos.double()[:, None] * turns[None]
    ang = (t - t.round()) * 2 * math.pi
    c, s = ang.cos()[:, None] * factor, ang.sin()[:, None] * factor
    xa, xb = x[..., a], x[..., b]
    size = x.abs()
    size[..., a] = size[..., b] = (xa.abs() + xb.abs()) * factor
    x[..., a], x[..., b] = xa * c - xb * s, xb * c + xa * s
    return x, size


def _case(T, H, Hk, D, seed, lead=0):
    """q, k, v as views of one projection's output."""
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn((T, (H + 2 * Hk) * D + lead), generator=g).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, lead:].view(T, H + 2 * Hk, D).split((H, Hk, Hk), 1) if lead == 0 else (
        qkv[:, lead:lead + H * D].unflatten(1, (H, D)), qkv[:, lead + H * D:lead + (H + Hk) * D].unflatten(1, (Hk, D)),
        qkv[:, lead + (H + Hk) * D:].unflatten(1, (Hk, D)))
    return q, k, v


SCALINGS = {"none": {}, "linear": dict(scaling="linear", factor=4.0), "ntk": dict(scaling="ntk", factor=8.0),
            "yarn": dict(scaling="yarn", factor=8.0, original_length=4096.0)}


@pytest.mark.parametrize("D,R,H,Hk", [(128, 128, 32, 8), (128, 64, 4, 4), (64, 16, 8, 1), (96, 96, 3, 3), (256, 256, 16, 2), (192, 64, 5, 1), (16, 0, 2, 1),
                                      (80, 48, 6, 2)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("e4m3,heads_first,page,scaling", [(False, False, 16, "none"), (True, True, 7, "yarn"), (False, True, 1, "linear"), (True, False, 64, "ntk")])
def test_rope_append(D, R, H, Hk, interleaved, e4m3, heads_first, page, scaling):
    T, S, far = 45, 4, 200000
    q, k, v = _case(T, H, Hk, D, 11)
    g = torch.Generator().manual_seed(12)
    rows = torch.randint(0, S, (T,), generator=g)
    pos = torch.randperm(4 * T, generator=g)[:T] + torch.tensor([0, 1, 3000, far])[rows]      # different in each row
    max_pages = int(pos.max()) // page + 1
    used = sorted({(int(r), int(p) // page) for r, p in zip(rows, pos)})
    n_pages = len(used) + 2
    perm = torch.randperm(n_pages, generator=g)
    table = torch.full((S, max_pages), -1, dtype=torch.int32)
    for (r, pg), at in zip(used, perm):
        table[r, pg] = int(at)
    scales = [torch.rand(Hk, generator=g) * 0.02 + 0.004 for _ in range(2)] if e4m3 else [None, None]
    cache = P.alloc_kv_cache(n_pages, page, Hk, D, *(s.cuda() if e4m3 else None for s in scales), heads_first=heads_first)
    cache.k.view(torch.uint8 if e4m3 else torch.int16).fill_(0x55)
    cache.v.view(torch.uint8 if e4m3 else torch.int16).fill_(0x55)
    rope = P.make_rope(R, interleaved, **SCALINGS[scaling]) if R else P.layer.Rope(None, 0)
    turns = rope.turns.cpu() if R else torch.zeros(0, dtype=torch.float64)
    i32 = lambda t: t.to(torch.int32).cuda()
    got = P.moe_rope_append(cache, rope, q, k, v, i32(pos), table.cuda(), table_row=i32(rows))
    want, size = _rotate(q.cpu(), pos, turns, rope.factor, R, interleaved)
    near(got, want, HALF_BF16 * want.abs() + 1e-6 * size, "q")
    kept = torch.zeros((n_pages, page), dtype=torch.bool)
    for name, x in (("k", _rotate(k.cpu(), pos, turns, rope.factor, R, interleaved)), ("v", (v.cpu().double(), v.cpu().double().abs()))):
        stored = getattr(cache, name).float().cpu()
        at = table[rows, pos // page].long(), pos % page
        want, size = x
        if e4m3:
            s = scales[name == "v"].double()[None, :, None]
            want = (want / s).clamp(-448, 448)
            near(stored[at], want, (HALF_E4M3 * want.abs()).clamp_min(2.0 ** -10) + 2e-6 * size / s, name)
        else:
            near(stored[at], want, HALF_BF16 * want.abs() + 1e-6 * size, name)
        kept[at] = True
    for t in (cache.k, cache.v):                    # nothing else was written
        raw = t.view(torch.uint8 if e4m3 else torch.int16).cpu()
        assert bool((raw[~kept] == 0x55).all())


def test_padding_and_places_that_are_not_there():
    T, H, Hk, D, page = 8, 4, 2, 64, 16
    q, k, v = _case(T, H, Hk, D, 13)
    cache = P.alloc_kv_cache(6, page, Hk, D)
    cache.k.zero_(), cache.v.zero_()
    table = torch.tensor([[3, -1, 9], [2, 5, 0]], dtype=torch.int32, device="cuda")
    rows = torch.tensor([0, 0, 0, 0, 1, 7, -1, 1], dtype=torch.int32, device="cuda")
    pos = torch.tensor([4, -1, 16, 40, 48, 0, 0, 47], dtype=torch.int32, device="cuda")     # there, padding, page -1, page 9, beyond, no row, no row, there
    rope = P.make_rope(D)
    got = P.moe_rope_append(cache, rope, q, k, v, pos, table, table_row=rows)
    want, size = _rotate(q.cpu(), pos.cpu().clamp_min(0), rope.turns.cpu(), 1.0, D, False)
    want[1] = 0
    near(got, want, HALF_BF16 * want.abs() + 1e-6 * size, "q")
    written = cache.v.cpu().abs().sum((2, 3)) > 0
    assert written.nonzero().tolist() == [[0, 15], [3, 4]]
    assert torch.equal(cache.v[3, 4], v[0]) and torch.equal(cache.v[0, 15], v[7])


def test_values_beyond_the_8_bit_range_and_nan():
    cache = P.alloc_kv_cache(1, 4, 1, 64, *(torch.full((1,), 0.5, device="cuda") for _ in range(2)))
    q = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    v = q.clone()
    v[0, 0, :6] = torch.tensor([1000.0, -1000.0, 224.0, math.inf, -math.inf, math.nan])
    P.moe_rope_append(cache, P.layer.Rope(None, 0), q, v.clone(), v, torch.zeros(1, dtype=torch.int32, device="cuda"),
                      torch.zeros((1, 1), dtype=torch.int32, device="cuda"))
    for t in (cache.k, cache.v):
        assert t[0, 0, 0, :5].float().tolist() == [448.0, -448.0, 448.0, 448.0, -448.0] and bool(t[0, 0, 0, 5].float().isnan())


def test_in_place_with_strides_and_a_stream():
    T, H, Hk, D = 19, 8, 2, 128
    q, k, v = _case(T, H, Hk, D, 14, lead=8)
    rope = P.make_rope(D, interleaved=True)
    table = torch.arange(2, dtype=torch.int32, device="cuda")[None].contiguous()
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    zero = torch.zeros(T, dtype=torch.int32, device="cuda")
    caches = [P.alloc_kv_cache(2, 16, Hk, D) for _ in range(2)]
    for c in caches:
        c.k.zero_(), c.v.zero_()
    want = P.moe_rope_append(caches[0], rope, q, k, v, pos, table, table_row=zero)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = P.moe_rope_append(caches[1], rope, q, k, v, pos, table, table_row=zero, out=q, stream=s)
    s.synchronize()
    assert got.data_ptr() == q.data_ptr() and torch.equal(q, want)
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)
    empty = P.moe_rope_append(caches[0], rope, q[:0], k[:0], v[:0], pos[:0], table, table_row=zero[:0])
    assert empty.shape == (0, H, D)


@pytest.mark.parametrize("pos", [0, 1, 131071, 1 << 20, (1 << 31) - 17])
def test_far_positions_keep_their_angle(pos):
    """The cosine itself: q = (1, 0) in every pair, so q_out is cos and sin; one bf16 rounding away from 64 bits however far.  The page
    is not in the table that far, which leaves q as it is."""
    D = 128
    q = torch.zeros((1, 1, D), dtype=torch.bfloat16, device="cuda")
    q[..., : D // 2] = 1
    cache = P.alloc_kv_cache(1, 16, 1, D)
    rope = P.make_rope(D)
    got = P.moe_rope_append(cache, rope, q, q, q, torch.tensor([pos], dtype=torch.int32, device="cuda"),
                            torch.zeros((1, 1), dtype=torch.int32, device="cuda"))
    t = pos * rope.turns.cpu()
    ang = (t - t.round()) * 2 * math.pi
    want = torch.cat((ang.cos(), ang.sin()))[None, None]
    # pos * turns in 64 bits is itself off by 2^-53 of the turns made
    near(got, want, HALF_BF16 * want.abs() + 1e-6 + pos * 2.0 ** -50, "cos, sin")


@pytest.mark.parametrize("e4m3", [False, True])
def test_q_too_large_for_the_caches(e4m3):
    """More than 8 MiB of q: it goes past the caches; two sequences' prompts in one call."""
    T, H, Hk, D, page = 1301, 32, 4, 128, 16
    q, k, v = _case(T, H, Hk, D, 31)
    rows = (torch.arange(T) >= 600).to(torch.int32)
    pos = torch.where(rows == 0, torch.arange(T), torch.arange(T) - 600).to(torch.int32)
    n = -(-701 // page)
    table = torch.randperm(2 * n, generator=torch.Generator().manual_seed(32)).to(torch.int32).view(2, n)
    scale = torch.full((Hk,), 0.02) if e4m3 else None
    cache = P.alloc_kv_cache(2 * n, page, Hk, D, *(None if scale is None else scale.cuda() for _ in range(2)))
    rope = P.make_rope(D)
    got = P.moe_rope_append(cache, rope, q, k, v, pos.cuda(), table.cuda(), table_row=rows.cuda())
    turns = rope.turns.cpu()
    want, size = _rotate(q.cpu(), pos, turns, rope.factor, D, False)
    near(got, want, HALF_BF16 * want.abs() + 1e-6 * size, "q")
    at = table[rows.long(), pos.long() // page].long(), pos.long() % page
    want, size = _rotate(k.cpu(), pos, turns, rope.factor, D, False)
    if e4m3:
        want, size = (want / 0.02).clamp(-448, 448), size / 0.02
        near(cache.k.float().cpu()[at], want, (HALF_E4M3 * want.abs()).clamp_min(2.0 ** -10) + 2e-6 * size, "k")
    else:
        near(cache.k.float().cpu()[at], want, HALF_BF16 * want.abs() + 1e-6 * size, "k")
