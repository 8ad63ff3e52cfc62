"""A call without tokens is valid and does nothing, the empty batch's block table (no rows, so no memory) included."""
import ctypes as C

import pytest
import torch

import paper_2507_17133_amd as P
from paper_2507_17133_amd import layer as L
from tests.test_layer_abi import OK, INVALID, SHAPE, _attention_call, _cache, _rope_call

TABLES = [dict(pages=None, n_rows=0, token_row=None), dict(n_rows=0, token_row=None), dict(pages=None, n_rows=0, max_pages=0, row_stride=0, token_row=None)]


@pytest.mark.parametrize("table", TABLES)
def test_no_tokens_and_no_table(table):
    assert _rope_call(T=0, table=table, q=None, k=None, v=None, pos=None, out=None) == OK
    assert _attention_call(T=0, table=table, q=None, lengths=None, out=None, ws=None, size=0) == OK
    assert _rope_call(T=1, table=table) in (INVALID, SHAPE) and _attention_call(T=1, table=table) in (INVALID, SHAPE)


def test_what_is_refused_without_tokens():
    """What belongs to the cache and the model is checked all the same."""
    assert _rope_call(T=0, cache=dict(k=None)) == INVALID and _attention_call(T=0, cache=dict(k=None)) == INVALID
    assert _rope_call(T=0, rope=dict(rotary_dim=24)) == SHAPE and _attention_call(T=0, H=12) == SHAPE and _attention_call(T=0, window=-1) == INVALID
    assert _rope_call(T=-1) == INVALID and _attention_call(T=-1) == INVALID
    r = C.byref(_cache())
    assert L._lib().moe_rope_append(r, None, None, None, 0, None, 0, None, 0, 32, 0, None, None, 0, None) == INVALID        # no rotary positions


@pytest.mark.gpu
def test_an_empty_batch_from_python():
    cache, rope = P.alloc_kv_cache(4, 16, 2, 64), P.make_rope(64)
    i32 = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")
    bf = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    assert P.moe_rope_append(cache, rope, bf(0, 4, 64), bf(0, 2, 64), bf(0, 2, 64), i32(0), i32(0, 3)).shape == (0, 4, 64)
    out, lse = P.moe_paged_attention(cache, bf(0, 4, 64), i32(0, 3), i32(0), want_lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
