"""The 8-bit linear layer against 64 bits."""
import math

import pytest
import torch

import paper_2507_17133_amd as P
from tests._layer_util import E4M3, HALF_BF16, near, spread

pytestmark = pytest.mark.gpu


def _case(M, N, K, seed, ld=None, pad_rows=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    G, GN = -(-K // 128), -(-N // 128)
    x8 = (torch.randn((M + pad_rows, ld or K), generator=g, device="cuda") * 60).clamp(-448, 448).to(E4M3)[:M, :K]
    w8 = (torch.randn((N, K), generator=g, device="cuda") * 60).clamp(-448, 448).to(E4M3)
    xs = torch.rand((G, M), generator=g, device="cuda") * 3e-3 + 1e-4
    ws = torch.rand((GN, G), generator=g, device="cuda") * 3e-3 + 1e-4
    return x8, xs, w8, ws


def _exact(x8, xs, w8, ws):
    K, N = x8.shape[1], w8.shape[0]
    a = x8.double() * spread(xs.double(), K)
    w = w8.double() * ws.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    out, size = a @ w.t(), a.abs() @ w.abs().t()
    # fp32 sums of K products, whatever their order, and of the blocks; one rounding to bf16
    return out, HALF_BF16 * out.abs() + (K + 8 * (K // 128 + 2)) * 2.0 ** -24 * size


ROWS = [1, 2, 15, 16, 17, 33, 48, 64, 65, 100, 128, 129, 255, 256, 300, 513]


@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("N,K", [(128, 128), (1, 16), (7, 144), (100, 1040), (300, 2048), (129, 272), (512, 4112)])
def test_linear(M, N, K):
    x8, xs, w8, ws = _case(M, N, K, M + N + K)
    want, tol = _exact(x8, xs, w8, ws)
    near(P.moe_linear_e4m3(x8, xs, w8, ws), want, tol, "out")


@pytest.mark.parametrize("M,N,K", [(1, 6144, 4096), (67, 2816, 2048), (256, 14336, 4096), (1000, 1408, 2048), (3001, 4096, 768), (4096, 4100, 7168), (5000, 8200, 384),
                                   (130, 512, 16384), (20, 16, 65536), (700, 700, 700 // 16 * 16)])
def test_larger(M, N, K):
    x8, xs, w8, ws = _case(M, N, K, 1)
    want, tol = _exact(x8, xs, w8, ws)
    near(P.moe_linear_e4m3(x8, xs, w8, ws), want, tol, "out")


@pytest.mark.parametrize("M,N,K", [(3, 40, 208), (70, 200, 1040), (300, 130, 400)])
def test_strides_and_what_lies_beside(M, N, K):
    """Rows of x8 in a wider tensor whose other columns are NaN, scales in a wider tensor, out of any alignment in a wider one, and a
    stream of its own."""
    x8, xs, w8, ws = _case(M, N, K, 2, ld=K + 160, pad_rows=2)
    x8._base.view(torch.uint8)[:, K:] = 0x7F
    x8._base.view(torch.uint8)[M:] = 0x7F
    wide = torch.full((xs.shape[0], M + 9), math.nan, device="cuda")
    wide[:, 5:5 + M] = xs
    out = torch.full((M, N + 7), 5.0, dtype=torch.bfloat16, device="cuda")
    want, tol = _exact(x8, xs, w8, ws)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = P.moe_linear_e4m3(x8, wide[:, 5:5 + M], w8, ws, out=out[:, 3:3 + N], stream=s)
    s.synchronize()
    near(got, want, tol, "out")
    assert bool((out[:, :3] == 5).all()) and bool((out[:, 3 + N:] == 5).all())
    again = P.moe_linear_e4m3(x8.contiguous(), xs, w8, ws)
    assert torch.equal(again, got)


@pytest.mark.parametrize("M", [4, 200, 700])
def test_nan_stays_in_its_row_and_column(M):
    N, K = 200, 336
    x8, xs, w8, ws = _case(M, N, K, 3)
    want, tol = _exact(x8, xs, w8, ws)
    x8.view(torch.uint8)[2, 330] = 0x7F
    w8.view(torch.uint8)[150, 5] = 0x7F
    got = P.moe_linear_e4m3(x8, xs, w8, ws)
    keep = torch.ones_like(got, dtype=torch.bool)
    keep[2], keep[:, 150] = False, False
    assert bool(got[2].isnan().all()) and bool(got[:, 150].isnan().all())
    near(got[keep], want[keep], tol[keep], "out")


def test_rows_from_the_norm_and_weights_from_bf16():
    """The chain as it is used: norm -> 8 bits -> product, against the unquantised product; each side's e4m3 rounding is at most 2^-4 of a value."""
    T, d, N = 70, 1024, 384
    g = torch.Generator().manual_seed(4)
    x = torch.randn((T, d), generator=g).to(torch.bfloat16)
    w = (torch.randn((N, d), generator=g) / math.sqrt(d)).to(torch.bfloat16)
    n = P.moe_rms_norm(x.cuda(), None, 1e-6, want=("y8",))
    w8, ws = P.moe_quantize_weight(w.cuda())
    got = P.moe_linear_e4m3(n.y8, n.scale, w8, ws)
    y = x.double() / (x.double().square().mean(1, keepdim=True) + 1e-6).sqrt()
    want, size = y @ w.double().t(), y.abs() @ w.double().abs().t()
    near(got, want, (2 * 2.0 ** -4 + 2.0 ** -7) * size + 1e-3, "out")


def test_no_rows_and_graph_replays():
    N, K = 512, 2048
    x8, xs, w8, ws = _case(0, N, K, 5)
    assert P.moe_linear_e4m3(x8, xs, w8, ws).shape == (0, N)
    for M in (3, 100, 600):
        x8, xs, w8, ws = _case(M, N, K, 6)
        out, work = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), P.alloc_linear_workspace(M, N, K)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            P.moe_linear_e4m3(x8, xs, w8, ws, out=out, workspace=work)
        for i in range(3):
            xs.mul_(1.5)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, P.moe_linear_e4m3(x8, xs, w8, ws))


# rows of whole rounds in tiles of 128 x 128, 128 x 256 or 256 x 256, the rest in rows, small tiles with and without slices of K, middle tiles
@pytest.mark.parametrize("M,N,K", [(3600, 1027, 1488), (1056, 15595, 288), (4793, 1675, 1440), (10909, 1283, 304), (8425, 398, 3088), (10825, 1447, 2464),
                                   (723, 10988, 2704), (9229, 2108, 400), (15189, 1055, 272)])
def test_rows_of_whole_rounds_and_the_rest(M, N, K):
    x8, xs, w8, ws = _case(M, N, K, 2, ld=K + 32)
    want, tol = _exact(x8, xs, w8, ws)
    wide = torch.full((M, N + 9), 7.0, dtype=torch.bfloat16, device="cuda")
    near(P.moe_linear_e4m3(x8, xs, w8, ws, out=wide[:, 1:1 + N]), want, tol, "out")
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, 1 + N:] == 7).all())
    near(P.moe_linear_e4m3(x8.contiguous(), xs, w8, ws), want, tol, "dense")


@pytest.mark.parametrize("M,N,K", [(4100, 1000, 256), (2000, 2100, 144), (129, 520, 16)])
def test_many_rows_of_short_k(M, N, K):
    x8, xs, w8, ws = _case(M, N, K, 3)
    want, tol = _exact(x8, xs, w8, ws)
    near(P.moe_linear_e4m3(x8, xs, w8, ws), want, tol, "out")
