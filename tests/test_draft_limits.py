"""Host side, no GPU: no launch of the operators of a step with several new tokens asks for 2^32 threads or more, which a runtime refuses; calls within the documented limits
are launched whole, or refused for what they are."""
import os

import pytest

from paper_2507_17133_amd import binding as B
from tests._fake_hip_draft import trace
from tests.test_layer_abi import UNSUPPORTED

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
