"""The linear layer looks for its way of cutting a product once per call, and a call without a workspace asks for one only where the product needs it."""
import pytest
import torch

import paper_2507_17133_amd as P
from paper_2507_17133_amd import layer as L


class _Counts:
    """The library with its calls counted."""

    def __init__(self, lib):
        self.lib, self.calls = lib, []

    def __getattr__(self, name):
        f = getattr(self.lib, name)

        def call(*a):
            self.calls.append(name)
            return f(*a)
        call.__name__ = name
        return call


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,calls", [(1, 256, 1024, 1), (4096, 512, 512, 1), (100, 200, 4096, 3)])
def test_calls_without_a_workspace(M, N, K, calls, monkeypatch):
    from tests.test_gpu_linear8 import _case
    case = _case(M, N, K, 1)
    work = P.alloc_linear_workspace(M, N, K)
    want = P.moe_linear_e4m3(*case, workspace=work)
    counts = _Counts(L._lib())
    monkeypatch.setattr(L, "_ready", counts)
    assert torch.equal(P.moe_linear_e4m3(*case), want)
    assert len(counts.calls) == calls
    assert (L.linear_workspace_size(M, N, K) > 0) == (calls == 3)
