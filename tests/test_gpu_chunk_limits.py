"""Chunk attention at its documented limits."""
import pytest
import torch

import paper_2507_17133_amd as A

pytestmark = pytest.mark.gpu


def test_more_blocks_than_a_launch_takes():
    """65536 sequences of one token, 256 key heads: each sees one position, so its result is the value there."""
    B, H, D = 65536, 256, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.empty((3, 1, H, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    cache = A.KvCache(k, v)
    table = (torch.arange(B, device="cuda") % 3).to(torch.int32).view(B, 1)
    q = torch.empty((B, H, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out = A.moe_chunk_attention(cache, q, table, torch.arange(B + 1, device="cuda").to(torch.int32), torch.zeros(B, dtype=torch.int32, device="cuda"))
    for r in range(3):
        assert bool((out[r::3] == v[r, 0]).all())
