"""Every kernel that the rules of the linear layer and of attention choose between, each against 64 bits; which one a case gets is seen on the CPU, from the launches."""
import pytest
import torch

import paper_2507_17133_amd as P
from tests._fake_hip_layer import trace
from tests._layer_util import near
from tests.test_gpu_attention import _case as attention_case
from tests.test_gpu_attention_precision import _exact as attention_exact
from tests.test_gpu_linear8 import _case as linear_case, _exact as linear_exact

gpu = pytest.mark.gpu

# rows kernel: (M, N, K, exact) -> row tiles, column tiles, blocks of K ahead, widened
ROWS = [((10, 300, 640, 0), (1, 1, 4, 0)), ((16, 6144, 640, 0), (1, 2, 3, 0)), ((17, 300, 2064, 0), (2, 1, 4, 0)), ((32, 6144, 4096, 0), (2, 2, 3, 0)),
        ((20, 6150, 1040, 0), (2, 2, 3, 0)), ((50, 300, 640, 0), (4, 1, 2, 0)), ((50, 6160, 528, 0), (4, 2, 2, 0)), ((64, 6300, 528, 0), (4, 2, 2, 0)),
        ((7, 4096, 640, 0), (1, 1, 4, 0)), ((7, 4100, 640, 0), (1, 2, 3, 0)), ((31, 5000, 1040, 0), (2, 2, 3, 0)), ((64, 5100, 512, 0), (4, 2, 1, 1)),
        ((10, 300, 512, 0), (1, 1, 1, 1)), ((3, 6144, 512, 0), (1, 2, 1, 1)), ((20, 300, 400, 0), (2, 1, 1, 1)), ((32, 6200, 272, 0), (2, 2, 1, 1)),
        ((64, 300, 512, 0), (4, 1, 1, 1)), ((50, 6144, 400, 0), (4, 2, 1, 1)), ((10, 300, 1040, 1), (1, 1, 4, 1)), ((10, 6144, 2064, 1), (1, 2, 3, 1)),
        ((20, 300, 4112, 1), (2, 1, 4, 1)), ((32, 6144, 4096, 1), (2, 2, 3, 1)), ((50, 300, 1040, 1), (4, 1, 2, 1)), ((64, 6200, 1552, 1), (4, 2, 2, 1))]


@pytest.mark.parametrize("shape,kernel", ROWS)
@gpu
def test_rows_of_the_linear_layer(shape, kernel):
    M, N, K, exact = shape
    x8, xs, w8, ws = linear_case(M, N, K, M + N + K, ld=K + 32)
    want, tol = linear_exact(x8, xs, w8, ws)
    wide = torch.full((M, N + 9), 7.0, dtype=torch.bfloat16, device="cuda")
    near(P.moe_linear_e4m3(x8, xs, w8, ws, exact=bool(exact), out=wide[:, 1:1 + N]), want, tol, "out")
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, 1 + N:] == 7).all())
    near(P.moe_linear_e4m3(x8.contiguous(), xs, w8, ws, exact=bool(exact)), want, tol, "dense")


def test_rows_get_these_kernels(tmp_path):
    got = trace([dict(entry="linear", M=M, N=N, K=K, exact=e) for (M, N, K, e), _ in ROWS], tmp_path)
    for (shape, kernel), r in zip(ROWS, got):
        assert r["status"] == 0 and [(l["name"], tuple(l["args"])) for l in r["launches"]] == [("linear_rows_kernel", kernel)], shape


SHORT = [1, 0, 31, 32, 33, 127, 128, 129, 300, 257]
LONG = [700, 2000, 5]
MANY = [(7 * i) % 45 for i in range(700)]
# heads, key heads, head_dim, e4m3, lengths, positions that the table has room for -> key heads side by side, shares at most (the rule goes by the room)
SIDES = [(2 * Hk, Hk, D, e4m3, lengths, room, side, 256 if D >= 128 and not e4m3 else 512)
         for D in (64, 96, 128, 192, 256) for e4m3 in (False, True) for Hk, lengths, room, side in ((4, SHORT, 70000, 4), (8, LONG, 120000, 4), (6, SHORT, 70000, 2), (2, LONG, 200000, 2))]
SIDES += [(48, 2, 128, False, LONG, 800000, 2, 256), (96, 4, 64, True, SHORT, 2000000, 4, 512), (20, 4, 128, False, SHORT, 300000, 4, 256),
          (4, 2, 128, False, MANY, 48, 1, 512), (8, 4, 128, False, MANY, 208, 2, 512), (32, 8, 128, False, MANY, 2000, 4, 512)]


def _shape(case):
    H, Hk, D, e4m3, lengths, room, side, shares = case
    return dict(entry="attention", T=len(lengths), heads=H, kv_heads=Hk, dim=D, page=16, max_pages=room // 16, e4m3=e4m3)


@pytest.mark.parametrize("case", SIDES, ids=lambda c: "-".join(map(str, c[:4] + (len(c[4]),) + c[5:])))
@gpu
def test_key_heads_side_by_side(case):
    H, Hk, D, e4m3, lengths, room, side, shares = case
    q, cache, table, k, v = attention_case(lengths, H, Hk, D, 16, e4m3=e4m3, seed=D + Hk)
    full = torch.full((len(lengths), room // 16), -1, dtype=torch.int32)
    full[:, :table.shape[1]] = table
    n = torch.tensor(lengths)
    ws = P.alloc_attention_workspace(cache, len(lengths), H)
    ws.fill_(255)
    out, lse = P.moe_paged_attention(cache, q.cuda(), full.cuda(), n.to(torch.int32).cuda(), want_lse=True, workspace=ws)
    want, tol = attention_exact(q.double(), k, v, n, D ** -0.5)
    near(out, want, tol, "out")
    assert torch.equal((lse == -float("inf")).cpu(), (n == 0)[:, None].expand(-1, H))
    again = P.moe_paged_attention(cache, q.cuda(), full.cuda(), n.to(torch.int32).cuda())
    assert torch.equal(again, out)


def test_attention_gets_these_launches(tmp_path):
    for case, r in zip(SIDES, trace([_shape(c) for c in SIDES], tmp_path)):
        H, Hk, D, e4m3, lengths, room, side, shares = case
        heads = min(H // Hk, 16)
        first, join = r["launches"]
        assert r["status"] == 0 and first["name"] == "attention_kernel" and first["args"] == [D, int(e4m3)] and join["name"] == "join_kernel", case
        assert first["lds"] == (4 - side) * heads * (D + 4) * 4, case          # one row of O for each wave behind the first of its key head
        assert first["grid"][0] == shares, case
        items = len(lengths) * (Hk // side) * -(-H // Hk // 16)
        assert join["args"] == [D, int(items * 4 < shares)] and join["grid"][1] == (heads * side if items * 4 < shares else -(-heads * side // 4)), case
