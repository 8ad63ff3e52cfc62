"""Host side, no GPU: chunk attention's workspace goes by the call's tokens, and holds what the launch of every call up to its arguments writes."""
import ctypes as C
import os

import pytest

from paper_2507_17133_amd import binding as B
from paper_2507_17133_amd import draft as M
from tests._fake_hip_draft import trace

if not os.path.exists(B.LIB_PATH):
    from paper_2507_17133_amd import build as _build
    _build.build()


def _size(n_seqs, T, heads, kv, dim, e4m3):
    size = C.c_size_t(0)
    cache = M.moe_kv_cache(k=4096, v=4096, page_stride=16 * kv * dim, token_stride=kv * dim, head_stride=dim, k_scale=4096, v_scale=4096, type=1 if e4m3 else 0, n_pages=10,
                           page_size=16, n_kv_heads=kv, head_dim=dim)
    assert M._lib().moe_chunk_workspace_size(C.byref(cache), n_seqs, T, heads, C.byref(size)) == 0
    return size.value


@pytest.mark.parametrize("e4m3", [False, True])
def test_small_calls_ask_for_little(e4m3):
    """Two parts of a tile's rows, 128 columns and two numbers each, for 512 blocks of 32 rows, 256 of 128, and 256 of 256."""
    for T, rows, blocks in ((1, 32, 512), (8, 32, 512), (26, 128, 256), (32, 128, 256), (33, 256, 256), (4096, 256, 256)):
        assert _size(1, T, 32, 8, 128, e4m3) <= 2 * blocks * rows * 130 * 4 + 16384, T
    assert _size(1, 1, 32, 8, 128, e4m3) < _size(1, 26, 32, 8, 128, e4m3) < _size(1, 4096, 32, 8, 128, e4m3)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_every_smaller_call_fits(dim, e4m3, tmp_path):
    up = lambda n: -(-n // 256) * 256
    heads, kv = 16, 4
    calls = [dict(entry="chunk", T=T, seqs=s, heads=heads, kv_heads=kv, dim=dim, page=16, max_pages=m, e4m3=e4m3, tree=t)
             for T in (1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 64, 100, 512, 2000) for s in (1, 2, 5, 16, 64, 400, 1024, 1025) if s <= 2 * T for m in (1, 20, 600) for t in (False, True)]
    need = []
    for c, r in zip(calls, trace(calls, tmp_path)):
        assert r["status"] == 0, c
        if len(r["launches"]) == 2:
            rows = 32 * r["launches"][0]["args"][2]
            shares = r["launches"][1]["grid"][0]
            need.append((c["T"], c["seqs"], up(16 * shares) + 4 * 2 * shares * rows * (dim + 2)))
    assert len(need) > 50
    for T in sorted({t for t, _, _ in need}):
        sizes = {s: _size(s, T, heads, kv, dim, e4m3) for s in (1, 2, 5, 16, 64, 400, 1024, 1025)}
        for t, s, n in need:
            if t <= T:
                assert all(n <= have for most, have in sizes.items() if s <= most), (t, s, T)
