"""A workspace of the linear layer that is kept for batches of changing size: enough for every one up to the largest, although the need of one M is not monotone
(products of few tiles are cut along K, larger ones are not)."""
import ctypes as C

import pytest
import torch

from paper_2507_17133_amd import binding as B
from paper_2507_17133_amd import layer as L

SHAPES = [(4096, 4096), (2048, 4096), (1408, 2048), (100, 16384), (512, 8192), (8, 65536), (14336, 4096), (300, 528), (2816, 512)]


@pytest.mark.parametrize("N,K", SHAPES)
def test_enough_for_every_smaller_batch(N, K):
    need = [L.linear_workspace_size(M, N, K) for M in range(2500)]
    so_far = last = 0
    for M in range(2500):
        so_far = max(so_far, need[M])
        have = L.linear_workspace_bound(M, N, K)
        assert have >= so_far and have >= last and have % 256 == 0
        last = have
    assert last <= 2 * max(need) and (last > 0) == (max(need) > 0)
    for M in (5000, 5001, 16384, 100000, 1 << 21):         # rows left over by whole rounds of tiles included
        assert L.linear_workspace_bound(M, N, K) >= max(last, L.linear_workspace_size(M, N, K))


def test_the_need_is_not_monotone():
    assert L.linear_workspace_size(128, 4096, 4096) > L.linear_workspace_size(4096, 4096, 4096) == 0
    assert L.linear_workspace_bound(4096, 4096, 4096) >= L.linear_workspace_size(128, 4096, 4096)


def test_refusals():
    f, n = L._lib().moe_linear_workspace_bound, C.c_size_t(7)
    assert f(-1, 64, 64, C.byref(n)) == -1 and f(8, 0, 64, C.byref(n)) == -2 and f(8, 64, 24, C.byref(n)) == -2 and f(8, 64, 64, None) == -1
    assert f((1 << 21) + 1, 64, 64, C.byref(n)) == -5 and n.value == 7
    with pytest.raises(B.MoeError):
        L.linear_workspace_bound(8, 8, 20)


@pytest.mark.gpu
@pytest.mark.parametrize("N,K", [(512, 4096), (2048, 4096)])
def test_one_workspace_for_a_server(N, K):
    """Allocated once for the largest batch, used for all, results those of calls that bring their own."""
    from tests.test_gpu_linear8 import _case
    most = 1000
    work = L.alloc_linear_workspace(most, N, K)
    for M in (most, 1, 40, 64, 65, 128, 200, 333, 512, most):
        case = _case(M, N, K, M)
        work.fill_(255)
        assert torch.equal(L.moe_linear_e4m3(*case, workspace=work), L.moe_linear_e4m3(*case))
