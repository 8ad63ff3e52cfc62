"""A workspace that the device cannot write is refused; one of another type counts by its bytes."""
import pytest
import torch

import paper_2507_17133_amd as P
from tests.test_gpu_linear8 import _case

pytestmark = pytest.mark.gpu


def _attention():
    g = torch.Generator(device="cuda").manual_seed(2)
    cache = P.alloc_kv_cache(4, 16, 2, 64)
    cache.k.normal_(generator=g), cache.v.normal_(generator=g)
    q = torch.randn((3, 8, 64), generator=g, device="cuda").to(torch.bfloat16)
    table = torch.arange(4, dtype=torch.int32, device="cuda").expand(3, 4).contiguous()
    lengths = torch.tensor([64, 1, 40], dtype=torch.int32, device="cuda")
    return cache, P.alloc_attention_workspace(cache, 3, 8), lambda ws: P.moe_paged_attention(cache, q, table, lengths, workspace=ws)


def _linear():
    case = _case(100, 200, 4096, 1)
    work = P.alloc_linear_workspace(100, 200, 4096)
    assert work.numel() > 0
    return None, work, lambda ws: P.moe_linear_e4m3(*case, workspace=ws)


@pytest.mark.parametrize("make", [_attention, _linear])
def test_workspaces(make):
    _, work, call = make()
    want = call(work)
    with pytest.raises(AssertionError):
        call(torch.empty(work.numel(), dtype=torch.uint8))                       # host memory
    with pytest.raises(AssertionError):
        call(torch.empty(4 * work.numel(), dtype=torch.uint8, device="cuda")[::2])
    with pytest.raises(P.MoeError):
        call(work[:0])
    assert torch.equal(call(torch.empty(work.numel() // 4, dtype=torch.float32, device="cuda")), want)
