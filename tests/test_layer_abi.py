"""Host side of the operators around the MoE layer, no GPU: the library exports what brownout_layer.h declares, refuses what it cannot do
before touching the device, and rope_frequencies gives the frequencies of the formulas."""
import ctypes as C
import math
import os
import re

import pytest
import torch

from paper_2507_17133_amd import binding as B
from paper_2507_17133_amd import layer as L

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "brownout_layer.h")

if not os.path.exists(B.LIB_PATH):
    from paper_2507_17133_amd import build as _build
    _build.build()

OK, INVALID, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = 0, -1, -2, -3, -4, -5
P = 0x10000                                    # a pointer that is never followed


def test_every_declared_function_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(moe_[a-z0-9_]+)\s*\(", text))
    assert names == set(L.EXPORTS)
    lib = C.CDLL(B.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


def _norm(**kw):
    a = dict(x=P, x_stride=256, weight=P, y=P, y_stride=256, T=4, d=256, eps=1e-6)
    a.update(kw)
    return C.byref(L.moe_norm_args(**a))


def _quant(**kw):
    a = dict(x=P, x_stride=256, y8=P, y8_stride=256, scale=P, scale_stride=4, T=4, d=256)
    a.update(kw)
    return C.byref(L.moe_norm_args(**a))


@pytest.mark.parametrize("change,status", [
    (dict(T=0), OK), (dict(T=0, x=None), OK), (dict(T=-1), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID),
    (dict(d=12), SHAPE), (dict(d=0), SHAPE), (dict(d=16392, x_stride=16392, y_stride=16392), UNSUPPORTED), (dict(eps=-1.0), INVALID), (dict(eps=math.nan), INVALID),
    (dict(x=P + 2), ALIGN), (dict(x_stride=257), ALIGN), (dict(x_stride=-256), ALIGN), (dict(weight=P + 4), ALIGN), (dict(y_stride=128), SHAPE),
    (dict(residual=P + 8), ALIGN), (dict(residual=P, residual_stride=4), ALIGN), (dict(residual_out=P, residual_out_stride=8), SHAPE),
    (dict(y8=P, y8_stride=256), INVALID), (dict(y8=P, y8_stride=256, scale=P, scale_stride=3), SHAPE),
    (dict(y8=P + 4, y8_stride=256, scale=P, scale_stride=4), ALIGN)])
def test_norm_refusals(change, status):
    assert L._lib().moe_rms_norm(_norm(**change), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(T=0), OK), (dict(y8=None), INVALID), (dict(scale=None), INVALID), (dict(y=P, y_stride=256), INVALID), (dict(weight=P), INVALID),
    (dict(residual=P, residual_stride=256), INVALID), (dict(d=9), SHAPE), (dict(scale=P + 2), ALIGN)])
def test_quantize_rows_refusals(change, status):
    assert L._lib().moe_quantize_rows(_quant(**change), None) == status


def test_quantize_weight_refusals():
    f = L._lib().moe_quantize_weight
    assert f(P, 8, 24, P, P, None) == SHAPE and f(P, 0, 32, P, P, None) == SHAPE and f(None, 8, 32, P, P, None) == INVALID
    assert f(P + 8, 8, 32, P, P, None) == ALIGN and f(P, 8, 1 << 21, P, P, None) == UNSUPPORTED


def _linear(**kw):
    a = dict(x8=P, x_stride=256, x_scale=P, x_scale_stride=8, w8=P, w_scale=P, out=P, out_stride=128, M=8, N=128, K=256)
    a.update(kw)
    return C.byref(L.moe_linear_args(**a))


@pytest.mark.parametrize("change,status", [
    (dict(M=0), OK), (dict(M=-1), INVALID), (dict(x8=None), INVALID), (dict(w_scale=None), INVALID), (dict(out=None), INVALID),
    (dict(K=250), SHAPE), (dict(K=0), SHAPE), (dict(N=0), SHAPE), (dict(x8=P + 8), ALIGN), (dict(x_stride=264), ALIGN), (dict(out=P + 1), ALIGN),
    (dict(x_scale=P + 2), ALIGN), (dict(x_scale_stride=7), SHAPE), (dict(out_stride=127), SHAPE), (dict(N=(1 << 20) + 1), UNSUPPORTED),
    (dict(M=(1 << 21) + 1, x_scale_stride=1 << 22), UNSUPPORTED), (dict(x_stride=(1 << 23) + 16), UNSUPPORTED)])
def test_linear_refusals(change, status):
    assert L._lib().moe_linear_e4m3(_linear(**change), P, 1 << 40, None) == status


def test_linear_workspace():
    assert L.linear_workspace_size(1, 4096, 4096) == 0 and L.linear_workspace_size(0, 64, 64) == 0
    sizes = {(M, N, K): L.linear_workspace_size(M, N, K) for M in (1, 65, 200, 1000) for N in (100, 1408, 4096) for K in (128, 2048, 16384)}
    assert all(v % 256 == 0 for v in sizes.values()) and any(sizes.values())
    for (M, N, K), v in sizes.items():
        if v:
            big = dict(M=M, N=N, K=K, x_stride=K, out_stride=N, x_scale_stride=M)
            assert L._lib().moe_linear_e4m3(_linear(**big), P, v - 1, None) == WORKSPACE
            assert L._lib().moe_linear_e4m3(_linear(**big), None, v, None) == WORKSPACE
            assert L._lib().moe_linear_e4m3(_linear(**big), P + 16, v, None) == ALIGN
    with pytest.raises(B.MoeError):
        L.linear_workspace_size(8, 8, 20)


def _cache(**kw):
    a = dict(k=P, v=P, page_stride=16 * 8 * 128, token_stride=8 * 128, head_stride=128, type=0, n_pages=10, page_size=16, n_kv_heads=8,
             head_dim=128)
    a.update(kw)
    return L.moe_kv_cache(**a)


def _rope_call(cache={}, table={}, rope={}, **kw):
    t = dict(pages=P, row_stride=4, token_row=P, n_rows=2, max_pages=4)
    r = dict(turns=P, rotary_dim=128, interleaved=0, factor=1.0)
    t.update(table)
    r.update(rope)
    a = dict(q=P, qs=4096, k=P, ks=1024, v=P, vs=1024, H=32, T=8, pos=P, out=P, os=4096)
    a.update(kw)
    return L._lib().moe_rope_append(C.byref(_cache(**cache)), C.byref(L.moe_block_table(**t)), C.byref(L.moe_rope(**r)), a["q"], a["qs"],
                                    a["k"], a["ks"], a["v"], a["vs"], a["H"], a["T"], a["pos"], a["out"], a["os"], None)


CACHE_REFUSALS = [
    (dict(k=None), INVALID), (dict(type=2), INVALID), (dict(type=1), INVALID), (dict(n_pages=0), SHAPE), (dict(page_size=0), SHAPE),
    (dict(n_kv_heads=0), SHAPE), (dict(k=P + 4), ALIGN), (dict(token_stride=1028), ALIGN), (dict(head_stride=64), SHAPE),
    (dict(type=1, k_scale=P, v_scale=P, head_stride=136), ALIGN), (dict(type=1, k_scale=P, v_scale=P + 1), ALIGN), (dict(page_stride=-16384), ALIGN),
    (dict(n_pages=1 << 22, page_stride=1 << 15), UNSUPPORTED), (dict(page_size=1 << 30, token_stride=1 << 40), UNSUPPORTED)]
TABLE_REFUSALS = [(dict(pages=None), INVALID), (dict(n_rows=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(row_stride=-1), SHAPE),
                  (dict(token_row=None), SHAPE), (dict(pages=P + 2), ALIGN), (dict(token_row=P + 1), ALIGN)]


@pytest.mark.parametrize("change,status", [(dict(cache=c), s) for c, s in CACHE_REFUSALS] + [(dict(table=t), s) for t, s in TABLE_REFUSALS] + [
    (dict(T=0), OK), (dict(T=-1), INVALID), (dict(rope=dict(rotary_dim=24)), SHAPE), (dict(rope=dict(rotary_dim=144)), SHAPE),
    (dict(rope=dict(rotary_dim=-16)), SHAPE), (dict(rope=dict(turns=None)), INVALID), (dict(rope=dict(turns=P + 4)), ALIGN),
    (dict(q=None), INVALID), (dict(pos=None), INVALID), (dict(out=None), INVALID), (dict(q=P + 2), ALIGN), (dict(vs=1028), ALIGN),
    (dict(os=4088), SHAPE), (dict(H=0), SHAPE), (dict(H=1025), UNSUPPORTED),
    (dict(cache=dict(head_dim=120, head_stride=120), rope=dict(rotary_dim=64)), SHAPE),
    (dict(cache=dict(head_dim=512, head_stride=512, token_stride=4096, page_stride=65536)), UNSUPPORTED)])
def test_rope_refusals(change, status):
    assert _rope_call(**change) == status


def _attention_call(cache={}, table={}, **kw):
    t = dict(pages=P, row_stride=4, token_row=P, n_rows=2, max_pages=4)
    t.update(table)
    a = dict(q=P, qs=4096, H=32, T=8, lengths=P, scale=0.1, window=0, out=P, os=4096, lse=None, ws=P, size=1 << 40)
    a.update(kw)
    return L._lib().moe_paged_attention(C.byref(_cache(**cache)), C.byref(L.moe_block_table(**t)), a["q"], a["qs"], a["H"], a["T"],
                                        a["lengths"], a["scale"], a["window"], a["out"], a["os"], a["lse"], a["ws"], a["size"], None)


@pytest.mark.parametrize("change,status", [(dict(cache=c), s) for c, s in CACHE_REFUSALS] + [(dict(table=t), s) for t, s in TABLE_REFUSALS] + [
    (dict(T=0), OK), (dict(T=-1), INVALID), (dict(T=65537), UNSUPPORTED), (dict(H=12), SHAPE), (dict(H=0), SHAPE), (dict(H=2048), UNSUPPORTED),
    (dict(cache=dict(head_dim=80, head_stride=80)), UNSUPPORTED), (dict(window=-1), INVALID), (dict(scale=math.inf), INVALID),
    (dict(lengths=None), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(out=P + 4), ALIGN), (dict(os=4094), ALIGN),
    (dict(os=4092), SHAPE), (dict(lse=P + 2), ALIGN), (dict(ws=None), WORKSPACE), (dict(size=1024), WORKSPACE), (dict(ws=P + 16), ALIGN)])
def test_attention_refusals(change, status):
    assert _attention_call(**change) == status


def test_attention_workspace_never_shrinks():
    n = C.c_size_t(0)
    for dim in (64, 96, 128, 192, 256):
        c = _cache(head_dim=dim, head_stride=dim, token_stride=8 * dim, page_stride=128 * dim)
        for H in (8, 32, 128, 256):
            last = 0
            for T in (0, 1, 7, 512, 65536):
                assert L._lib().moe_attention_workspace_size(C.byref(c), T, H, C.byref(n)) == OK
                assert n.value >= last and n.value % 256 == 0
                last = n.value


def test_frequencies_of_the_formulas():
    for R in (2, 16, 64, 128, 256):
        i = torch.arange(R // 2, dtype=torch.float64)
        for base in (10000.0, 500000.0):
            plain = base ** (-2 * i / R) / (2 * math.pi)
            t, f = L.rope_frequencies(R, base)
            assert f == 1.0 and torch.allclose(t, plain, rtol=1e-14, atol=0)
            t, f = L.rope_frequencies(R, base, "linear", 8.0)
            assert f == 1.0 and torch.allclose(t, plain / 8, rtol=1e-14, atol=0)
            t, f = L.rope_frequencies(R, base, "ntk", 8.0)
            # the fastest pair keeps its frequency; the slowest is stretched by the factor
            assert f == 1.0 and abs(t[0] * 2 * math.pi - 1) < 1e-14 and (R == 2 or abs(float(plain[-1] / t[-1]) - 8.0) < 1e-10)
            t, f = L.rope_frequencies(R, base, "yarn", 8.0, 4096.0)
            made = 4096.0 * plain
            assert abs(f - (0.1 * math.log(8.0) + 1)) < 1e-6 and bool((t <= plain * (1 + 1e-15)).all()) and bool((t >= plain / 8 * (1 - 1e-15)).all())
            assert torch.equal(t[made > 32 * base ** (2 / R)], plain[made > 32 * base ** (2 / R)])
            if R > 2:
                slow = made < base ** (-2 / R)
                assert torch.allclose(t[slow], plain[slow] / 8, rtol=1e-12, atol=0)


@pytest.mark.parametrize("args", [(0,), (7,), (-2,), (64, 1.0), (64, math.nan), (64, 1e4, "linear", 0.5), (64, 1e4, "yarn", 8.0, 0.0),
                                  (64, 1e4, "yarn", 8.0, 4096.0, 1.0, 1.0), (64, 1e4, "yarn", 8.0, 4096.0, 32.0, 0.0), (64, 1e4, "ntk", math.inf)])
def test_frequencies_refusals(args):
    with pytest.raises(B.MoeError):
        L.rope_frequencies(*args)


@pytest.mark.parametrize("rows,status", [((1 << 21) + 1, UNSUPPORTED), ((1 << 31) - 1, UNSUPPORTED)])
def test_more_rows_than_a_launch_takes(rows, status):
    assert L._lib().moe_rms_norm(_norm(T=rows), None) == status
    assert L._lib().moe_quantize_rows(_quant(T=rows, scale_stride=rows), None) == status
    assert _rope_call(T=rows) == status
