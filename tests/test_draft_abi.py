"""Host side of the operators of a step with several new tokens, no GPU: the library exports what brownout_draft.h declares, refuses what it cannot do before touching
the device, and tree_masks gives a tree's ancestors."""
import ctypes as C
import math
import os
import random
import re

import pytest
import torch

from paper_2507_17133_amd import binding as B
from paper_2507_17133_amd import draft as M
from paper_2507_17133_amd import layer as L
from tests.test_layer_abi import ALIGN, CACHE_REFUSALS, INVALID, OK, P, SHAPE, TABLE_REFUSALS, UNSUPPORTED, WORKSPACE, _cache
from tests.test_layer_overlap import APART, OVER

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "brownout_draft.h")


def test_every_declared_function_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(moe_[a-z0-9_]+)\s*\(", text))
    assert names == set(M.EXPORTS)
    lib = C.CDLL(B.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


def _table(**kw):
    t = dict(pages=P, row_stride=4, token_row=P, n_rows=2, max_pages=4)
    t.update(kw)
    return C.byref(L.moe_block_table(**t))


def _sink(cache={}, table={}, **kw):
    a = dict(q=P, qs=4096, H=32, T=8, lengths=P, scale=0.1, window=16, sinks=4, out=P + (1 << 30), os=4096, lse=None, ws=P, size=1 << 40)
    a.update(kw)
    return M._lib().moe_sink_attention(C.byref(_cache(**cache)), _table(**table), a["q"], a["qs"], a["H"], a["T"], a["lengths"], a["scale"], a["window"],
                                       a["sinks"], a["out"], a["os"], a["lse"], a["ws"], a["size"], None)


@pytest.mark.parametrize("change,status", [(dict(cache=c), s) for c, s in CACHE_REFUSALS] + [(dict(table=t), s) for t, s in TABLE_REFUSALS] + [
    (dict(T=0), OK), (dict(T=-1), INVALID), (dict(sinks=-1), INVALID), (dict(window=-1), INVALID), (dict(scale=math.nan), INVALID), (dict(lengths=None), INVALID),
    (dict(H=12), SHAPE), (dict(T=65537), UNSUPPORTED), (dict(size=1024), WORKSPACE), (dict(ws=P + 16), ALIGN), (dict(out=P), INVALID)])
def test_sink_refusals(change, status):
    assert _sink(**change) == status


def _append(cache={}, table={}, rope={}, **kw):
    r = dict(turns=P, rotary_dim=128, interleaved=0, factor=1.0)
    r.update(rope)
    a = dict(q=P, qs=4096, k=P, ks=1024, v=P, vs=1024, H=32, T=8, pos=P, places=P, out=P, os=4096)
    a.update(kw)
    return M._lib().moe_rope_append_at(C.byref(_cache(**cache)), _table(**table), C.byref(L.moe_rope(**r)), a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"],
                                       a["H"], a["T"], a["pos"], a["places"], a["out"], a["os"], None)


@pytest.mark.parametrize("change,status", [(dict(cache=c), s) for c, s in CACHE_REFUSALS] + [(dict(table=t), s) for t, s in TABLE_REFUSALS] + [
    (dict(T=0), OK), (dict(T=-1), INVALID), (dict(places=None), INVALID), (dict(pos=None), INVALID), (dict(places=P + 2), ALIGN), (dict(rope=dict(rotary_dim=24)), SHAPE),
    (dict(os=4088), SHAPE), (dict(H=1025), UNSUPPORTED), (dict(T=(1 << 21) + 1), UNSUPPORTED)])
def test_append_refusals(change, status):
    assert _append(**change) == status


FAR = P + (1 << 30)
SEQ_TABLE_REFUSALS = [(t, s) for t, s in TABLE_REFUSALS if t != dict(token_row=None)] + [(dict(token_row=None, n_rows=1), SHAPE)]      # rows of sequences


def _chunk(cache={}, table={}, chunk={}, **kw):
    c = dict(first=P, context=P, seen=None, seen_stride=0, positions=None, seen_words=0, n_seqs=2, T=8, window=0, sinks=0)
    c.update(chunk)
    a = dict(q=P, qs=4096, H=32, scale=0.1, out=FAR, os=4096, lse=None, ws=P, size=1 << 40)
    a.update(kw)
    return M._lib().moe_chunk_attention(C.byref(_cache(**cache)), _table(**table), C.byref(M.moe_chunk(**c)), a["q"], a["qs"], a["H"], a["scale"], a["out"], a["os"],
                                        a["lse"], a["ws"], a["size"], None)


TREE = dict(seen=P, seen_stride=2, seen_words=2)


@pytest.mark.parametrize("change,status", [(dict(cache=c), s) for c, s in CACHE_REFUSALS] + [(dict(table=t), s) for t, s in SEQ_TABLE_REFUSALS] + [
    (dict(chunk=dict(T=0)), OK), (dict(chunk=dict(n_seqs=0)), OK), (dict(chunk=dict(T=-1)), INVALID), (dict(chunk=dict(n_seqs=-1)), INVALID),
    (dict(chunk=dict(window=-1)), INVALID), (dict(chunk=dict(sinks=-1)), INVALID), (dict(scale=math.inf), INVALID), (dict(chunk=dict(first=None)), INVALID),
    (dict(chunk=dict(context=None)), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(chunk=dict(positions=P)), INVALID),
    (dict(chunk=dict(seen_words=2)), INVALID), (dict(chunk=dict(TREE, seen_words=0)), INVALID), (dict(chunk=dict(TREE, seen_words=129, seen_stride=129)), UNSUPPORTED),
    (dict(chunk=dict(TREE, seen_stride=1)), SHAPE), (dict(chunk=dict(TREE, seen=P + 2)), ALIGN), (dict(chunk=dict(TREE, positions=P + 1)), ALIGN),
    (dict(chunk=dict(first=P + 2)), ALIGN), (dict(chunk=dict(T=65537)), UNSUPPORTED), (dict(chunk=dict(n_seqs=65537)), UNSUPPORTED), (dict(H=12), SHAPE),
    (dict(cache=dict(head_dim=80, head_stride=80)), UNSUPPORTED), (dict(os=4092), SHAPE), (dict(os=4094), ALIGN), (dict(out=FAR + 4), ALIGN), (dict(lse=P + 2), ALIGN),
    (dict(qs=4092), ALIGN), (dict(ws=None), WORKSPACE), (dict(size=1024), WORKSPACE), (dict(ws=P + 16), ALIGN)])
def test_chunk_refusals(change, status):
    assert _chunk(**change) == status


@pytest.mark.parametrize("q,qs,out,os,T", OVER)
def test_chunk_over_its_queries(q, qs, out, os, T):
    assert _chunk(q=q, qs=qs, out=out, os=os, chunk=dict(T=T)) == INVALID


def _move(cache={}, table={}, **kw):
    a = dict(src=P, stride=4, most=4, start=P, count=P, n=2)
    a.update(kw)
    return M._lib().moe_cache_move(C.byref(_cache(**cache)), _table(**table), a["src"], a["stride"], a["most"], a["start"], a["count"], a["n"], None)


@pytest.mark.parametrize("change,status", [(dict(cache=c), s) for c, s in CACHE_REFUSALS] + [(dict(table=t), s) for t, s in SEQ_TABLE_REFUSALS] + [
    (dict(n=0), OK), (dict(most=0), OK), (dict(n=-1), INVALID), (dict(most=-1), INVALID), (dict(src=None), INVALID), (dict(start=None), INVALID), (dict(count=None), INVALID),
    (dict(src=P + 2), ALIGN), (dict(start=P + 1), ALIGN), (dict(count=P + 2), ALIGN), (dict(stride=3), SHAPE), (dict(stride=-1), SHAPE),
    (dict(most=4097, stride=4097), UNSUPPORTED), (dict(n=65537), UNSUPPORTED),
    (dict(cache=dict(head_dim=4, head_stride=8)), SHAPE), (dict(cache=dict(head_dim=1024, head_stride=1024, n_kv_heads=1024, token_stride=1 << 20, page_stride=1 << 24)), UNSUPPORTED)])
def test_move_refusals(change, status):
    assert _move(**change) == status


def _logprobs(**kw):
    a = dict(logits=P, stride=1000, tokens=P, tokens_stride=3, logprob=P, rank=P, lse=P, entropy=P, top_id=P, top_logprob=P, T=4, V=1000, type=0, n_given=3, n_top=5)
    ws = {k: kw.pop(k) for k in ("ws", "size") if k in kw}
    a.update(kw)
    return M._lib().moe_token_logprobs(C.byref(M.moe_logprob_args(**a)), ws.get("ws", P), ws.get("size", 1 << 40), None)


@pytest.mark.parametrize("change,status", [
    (dict(T=0), OK), (dict(T=-1), INVALID), (dict(type=2), INVALID), (dict(logits=None), INVALID), (dict(tokens=None), INVALID), (dict(n_given=-1), INVALID),
    (dict(n_top=-1), INVALID), (dict(V=0), SHAPE), (dict(n_top=33, V=32, stride=32), SHAPE), (dict(V=(1 << 20) + 1, stride=1 << 21), UNSUPPORTED),
    (dict(n_top=65), UNSUPPORTED), (dict(n_given=65, tokens_stride=65), UNSUPPORTED), (dict(T=(1 << 21) + 1), UNSUPPORTED), (dict(stride=999), SHAPE), (dict(stride=-1000), SHAPE),
    (dict(tokens_stride=2), SHAPE), (dict(logits=P + 1), ALIGN), (dict(type=1, logits=P + 2), ALIGN), (dict(tokens=P + 2), ALIGN), (dict(logprob=P + 2), ALIGN),
    (dict(rank=P + 1), ALIGN), (dict(lse=P + 2), ALIGN), (dict(entropy=P + 2), ALIGN), (dict(top_id=P + 2), ALIGN), (dict(top_logprob=P + 3), ALIGN),
    (dict(ws=None), WORKSPACE), (dict(size=16), WORKSPACE), (dict(ws=P + 16), ALIGN)])
def test_logprob_refusals(change, status):
    assert _logprobs(**change) == status


def test_tree_masks():
    r = random.Random(3)
    for n in (0, 1, 2, 31, 32, 33, 70, 200):
        parents = [r.randint(-1, j - 1) for j in range(n)]
        for words in ((n + 31) // 32, (n + 31) // 32 + 2):
            seen, depth = M.tree_masks(parents, words)
            for i in range(n):
                up, j = set(), i
                while j >= 0:
                    up.add(j)
                    j = parents[j]
                assert {j for j in range(32 * words) if seen[i, j // 32].item() >> (j % 32) & 1} == up and depth[i] == len(up) - 1


@pytest.mark.parametrize("parents,words", [([0], 1), ([-1, 1], 1), ([-2], 1), ([-1] * 33, 1), ([-1] * 4097, 129)])
def test_tree_masks_refusals(parents, words):
    with pytest.raises(B.MoeError):
        M.tree_masks(parents, words)


