"""A call on a stream of the caller's: what it allocates belongs to that stream, so the allocator gives it to no one else while the work is under way,
and the results are those of the current stream."""
import pytest
import torch

import paper_2507_17133_amd as P

pytestmark = pytest.mark.gpu


def _owner(t):
    """The stream that the allocator keeps the tensor's memory for."""
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= t.data_ptr() < segment["address"] + segment["total_size"]:
            return segment["stream"]
    raise AssertionError("not found")


def _calls():
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((130, 512), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn((200, 512), generator=g, device="cuda").to(torch.bfloat16)
    w8, ws = P.moe_quantize_weight(w)
    x8, xs = P.moe_quantize_rows(x)
    cache, rope = P.alloc_kv_cache(12, 16, 2, 64), P.make_rope(64)
    cache.k.zero_(), cache.v.zero_()
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(1, 12)
    row, pos = torch.zeros(130, dtype=torch.int32, device="cuda"), torch.arange(130, dtype=torch.int32, device="cuda")
    q, k, v = x.view(130, 8, 64).split((4, 2, 2), 1)
    return {
        "norm": lambda s: P.moe_rms_norm(x, None, residual=x, want=("y", "y8"), stream=s),
        "quantize_rows": lambda s: P.moe_quantize_rows(x, stream=s),
        "quantize_weight": lambda s: P.moe_quantize_weight(w, stream=s),
        "linear": lambda s: (P.moe_linear_e4m3(x8, xs, w8, ws, stream=s),),
        "rope": lambda s: (P.moe_rope_append(cache, rope, q, k, v, pos, table, table_row=row, stream=s),),
        "attention": lambda s: P.moe_paged_attention(cache, q, table, pos + 1, table_row=row, want_lse=True, stream=s),
    }


@pytest.mark.parametrize("name", ["norm", "quantize_rows", "quantize_weight", "linear", "rope", "attention"])
def test_results_belong_to_the_stream(name):
    call = _calls()[name]
    want = call(None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(s)
    s.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
        assert _owner(a) == 0 and _owner(b) == s.cuda_stream
