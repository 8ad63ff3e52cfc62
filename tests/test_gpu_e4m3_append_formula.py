"""The append to an 8-bit cache code for code: a value that is not rotated is stored as e4m3 of itself divided by its head's scale (one fp32 division),
held within 448 scales."""
import pytest
import torch

import paper_2507_17133_amd as P
from tests._layer_util import E4M3

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,H,Hk,D", [(33, 4, 2, 64), (700, 16, 16, 128), (50, 5, 1, 256), (120, 9, 3, 80)])
@pytest.mark.parametrize("heads_first", [False, True])
def test_codes(T, H, Hk, D, heads_first):
    g = torch.Generator().manual_seed(T + D)
    qkv = torch.randn((T, H + 2 * Hk, D), generator=g)
    qkv[:, :, ::3] = torch.randint(-896, 897, qkv[:, :, ::3].shape, generator=g) * (0.5 * 7 / 512)       # quotients at midpoints, exactly, by 7 / 512
    qkv[:, :, 1::17] = -0.0
    qkv[:, :, 2::19] *= 1e4                                # beyond 448 scales
    q, k, v = qkv.to(torch.bfloat16).split((H, Hk, Hk), 1)
    scales = [torch.randint(128, 256, (Hk,), generator=g) / 32.0 / 448 for _ in range(2)]        # a largest value in bf16 over 448
    scales[0][0], scales[1][-1] = 7 / 512, 2.0 ** -6
    page, n = 16, -(-T // 16)
    cache = P.alloc_kv_cache(n, page, Hk, D, scales[0].cuda(), scales[1].cuda(), heads_first=heads_first)
    P.moe_rope_append(cache, P.layer.Rope(None, 0), q.cuda(), k.cuda(), v.cuda(), torch.arange(T, dtype=torch.int32, device="cuda"),
                      torch.arange(n, dtype=torch.int32, device="cuda").view(1, n), table_row=torch.zeros(T, dtype=torch.int32, device="cuda"))
    for stored, x, s in ((cache.k, k, scales[0]), (cache.v, v, scales[1])):
        want = (x.float() / s[None, :, None]).clamp(-448, 448).to(E4M3)
        got = stored.view(torch.uint8).cpu().reshape(n * page, Hk, D)[:T]
        assert torch.equal(got, want.view(torch.uint8))
