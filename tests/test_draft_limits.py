"""Host side, no GPU: no launch of the operators of a step with several new tokens asks for 2^32 threads or more, which a runtime refuses; calls within the documented limits
are launched whole, in several launches where it takes them."""
import os

import pytest

from paper_2507_17133_amd import binding as B
from tests import _fake_hip_rows
from tests._fake_hip_draft import trace

if not os.path.exists(B.LIB_PATH):
    from paper_2507_17133_amd import build as _build
    _build.build()


def _within(launch):
    return launch["grid"][0] * launch["block"] < 1 << 32 and launch["grid"][1] < 65536 and launch["grid"][2] < 65536


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("T,seqs", [(65536, 65536), (1, 65536), (65536, 1025), (65536, 1024), (65536, 1), (3000, 40000)])
def test_chunk_attention(dim, T, seqs, tmp_path):
    calls = [dict(entry="chunk", T=T, seqs=seqs, heads=h * k, kv_heads=k, dim=dim, page=16, max_pages=100, e4m3=e, tree=t)
             for h, k in ((1, 1), (1, 256), (1, 1024), (4, 256), (1024, 1)) for e in (False, True) for t in (False, True)]
    for c, r in zip(calls, trace(calls, tmp_path)):
        assert r["status"] == 0, c
        assert all(_within(l) for l in r["launches"]), c
        if seqs > 1024:                                   # a block for each item, in as many launches as it takes
            rows, group = 32 * r["launches"][0]["args"][2], c["heads"] // c["kv_heads"]
            assert all(l["name"] == "chunk_kernel" for l in r["launches"])
            assert sum(l["grid"][0] for l in r["launches"]) == (T * group // rows + seqs) * c["kv_heads"], c


@pytest.mark.parametrize("T,V", [(1 << 21, 1), (1 << 21, 2048), (1 << 21, 2049), (1 << 21, 70000), (1 << 20, 131072), (1 << 20, 131073), (1 << 21, 1 << 20), (140000, 1 << 20)])
def test_log_probabilities(T, V, tmp_path):
    calls = [dict(entry="logprob", T=T, V=V, given=g, top=min(n, V), fp32=f, off=o) for g, n in ((0, 0), (3, 8)) for f, o in ((False, 0), (True, 4))]
    for c, r in zip(calls, trace(calls, tmp_path)):
        assert r["status"] == 0, c
        assert all(_within(l) for l in r["launches"]), c
        slices = [l for l in r["launches"] if l["name"] == "slice_kernel"]
        each, per = slices[0]["args"][-1] * 64, 4 if c["fp32"] else 8
        n = -(-(V + (0 if c["off"] == 0 and V % per == 0 else per - 1)) // each)
        assert sum(l["grid"][0] for l in slices) == T * n, c
        assert sum(l["grid"][0] for l in r["launches"] if l["name"] == "join_rows") == (T if n > 1 else 0), c


@pytest.mark.parametrize("T,V", [(67, 50021), (1 << 20, 131073), (140000, 1 << 20)])
def test_rows_of_each_launch_of_log_probabilities(T, V, tmp_path):
    """Each launch begins where the one before ends, in every argument."""
    calls = [dict(T=T, V=V, given=g, top=n, fp32=f, stride=V + 5) for g, n in ((0, 0), (3, 0), (0, 7), (3, 7)) for f in (False, True)]
    for c, r in zip(calls, _fake_hip_rows.trace(calls, tmp_path)):
        assert r["status"] == 0, c
        row = dict(logits=(V + 5) * (4 if c["fp32"] else 2), tokens=4 * (c["given"] + 2), logprob=4 * c["given"], rank=4 * c["given"], lse=4, entropy=4, top_id=4 * c["top"],
                   top_logprob=4 * c["top"])
        for name in ("slice", "join"):
            t = 0
            for l in r["launches"]:
                if l["name"] == name:
                    for k, v in row.items():
                        assert l[k] == (r["base"][k] + t * v if r["base"][k] else 0), (c, k, t)
                    t += l["T"]
            assert t == T, c
