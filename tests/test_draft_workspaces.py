"""Host side, no GPU: what the launches of the log probabilities and of chunk attention write to their workspaces stays within the sizes that are asked for, also
of a workspace that was made for larger calls; and the slices of a row hold all of it."""
import os

import pytest

from paper_2507_17133_amd import binding as B
from paper_2507_17133_amd import draft as M
from tests._fake_hip_draft import trace

if not os.path.exists(B.LIB_PATH):
    from paper_2507_17133_amd import build as _build
    _build.build()

up = lambda n: -(-n // 256) * 256


def _need(T, slices, G, N):
    parts = T * slices
    return up(16 * parts) + up(4 * parts * G) + up(8 * parts * N)


CASES = [dict(T=T, V=V, given=G, top=min(N, V), fp32=f, off=o)
         for T in (1, 2, 67, 500, 767, 2112, 70000) for V in (1, 7, 100, 2041, 8192, 8193, 50021, 131072, 1 << 20) for G, N in ((0, 0), (1, 5), (4, 0), (64, 64))
         for f, o in ((False, 0), (False, 2), (True, 0), (True, 4)) if T * V <= 1 << 32]


def test_log_probabilities(tmp_path):
    out = trace([dict(c, entry="logprob") for c in CASES], tmp_path)
    for c, r in zip(CASES, out):
        assert r["status"] == 0, c
        first, T, V = r["launches"][0], c["T"], c["V"]
        slices, each = first["grid"][0] // T, first["args"][-1]
        assert first["name"] == "slice_kernel" and first["grid"] == [T * slices, 1, 1] and first["block"] == 64
        # a row that begins inside a 16-byte line has its first slice begin before it
        per = 4 if c["fp32"] else 8
        ahead = 0 if c["off"] == 0 and (T == 1 or V % per == 0) else per - 1
        assert slices * each * 64 >= V + ahead
        assert (len(r["launches"]) == 2) == (slices > 1)
        if slices > 1:
            join = r["launches"][1]
            assert join["name"] == "join_rows" and join["grid"] == [T, 1, 1] and join["block"] == 256
        for T_max in (T, T + 1, 3 * T, 100 * T):
            if T_max <= 1 << 21:
                assert M.logprob_workspace_size(T_max, V, c["given"], c["top"]) >= _need(T, slices, c["given"], c["top"]), (c, T_max)


@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_chunk_attention(dim, tmp_path):
    calls = [dict(entry="chunk", T=T, seqs=s, heads=h * k, kv_heads=k, dim=dim, page=16, max_pages=m, e4m3=e, tree=t)
             for T, s in ((1, 1), (26, 1), (40, 40), (2112, 64), (4096, 1), (16384, 4), (65536, 65536), (5000, 3000)) for h, k in ((1, 1), (7, 8), (64, 2))
             for m in (1, 600) for e in (False, True) for t in (False, True)]
    out = trace(calls, tmp_path)
    for c, r in zip(calls, out):
        assert r["status"] == 0, c
        first = r["launches"][0]
        D, e4m3, WM, WK, PB = first["args"]
        rows = 32 * WM
        assert first["name"] == "chunk_kernel" and D == dim and bool(e4m3) == c["e4m3"] and first["block"] == 64 * WM * WK and first["lds"] <= 160 * 1024
        if len(r["launches"]) == 1 and first["grid"][0] > 1:      # a block for each item: room for all tiles of rows, however the tokens are dealt out
            group = c["heads"] // c["kv_heads"]
            assert first["grid"][0] == (c["T"] * group // rows + c["seqs"]) * c["kv_heads"]
        else:                                                     # shares, two parts each; perhaps with blocks enough for the items, too
            shares = first["grid"][0]
            if len(r["launches"]) == 2:
                group, join = c["heads"] // c["kv_heads"], r["launches"][1]
                items = (c["T"] * group // rows + c["seqs"]) * c["kv_heads"]
                shares = join["grid"][0]
                assert join["name"] == "chunk_join" and first["grid"][0] in (shares, max(shares, items)) and (not c["tree"] or first["grid"][0] == shares), c
            size = M.C.c_size_t(0)
            cache = M.moe_kv_cache(k=4096, v=4096, page_stride=16 * c["kv_heads"] * dim, token_stride=c["kv_heads"] * dim, head_stride=dim, k_scale=4096,
                                   v_scale=4096, type=1 if c["e4m3"] else 0, n_pages=10, page_size=16, n_kv_heads=c["kv_heads"], head_dim=dim)
            assert M._lib().moe_chunk_workspace_size(M.C.byref(cache), c["seqs"], c["T"], c["heads"], M.C.byref(size)) == 0
            assert size.value >= up(16 * shares) + 4 * 2 * shares * rows * (dim + 2), c
