"""Trees for layers that see a window: the bits of moe_tree_window_masks against the definition (CPU), and a tree's tokens against the same tokens as single ones."""
import random

import pytest
import torch

import paper_2507_17133_amd as A
from paper_2507_17133_amd import draft as M
from tests._draft_util import random_tree
from tests._layer_util import HALF_BF16, near
from tests.test_layer_abi import INVALID, OK, SHAPE, UNSUPPORTED


def _path(parents, i):
    up = []
    while i >= 0:
        up.append(i)
        i = parents[i]
    return up[::-1]


def _chain(n):
    return [j - 1 for j in range(n)]


def test_bits():
    r = random.Random(5)
    for parents in [random_tree(r, n) for n in (1, 2, 31, 33, 70)] + [_chain(n) for n in (3, 40, 130)] + [[-1, -1, 0, 2, 3, 1]]:
        paths = [_path(parents, i) for i in range(len(parents))]
        for window in (0, 1, 2, 5, 31, 32, 33, 64, (1 << 31) - 1):
            for sinks in (0, 1, 3, 40):
                seen, depth = M.tree_masks(parents, -(-len(parents) // 32) + 1, window, sinks)
                for i, path in enumerate(paths):
                    want = {j for d, j in enumerate(path) if window == 0 or len(path) - 1 - d < window or d < sinks}
                    assert {j for j in range(32 * seen.shape[1]) if seen[i, j // 32].item() >> (j % 32) & 1} == want and depth[i] == len(path) - 1


def test_without_a_window_as_before():
    parents = random_tree(random.Random(6), 50)
    a, b = (torch.empty((50, 2), dtype=torch.int32) for _ in range(2))
    up = torch.tensor(parents, dtype=torch.int32)
    assert M._lib().moe_tree_masks(up.data_ptr(), 50, 2, a.data_ptr(), None) == OK and M._lib().moe_tree_window_masks(up.data_ptr(), 50, 2, 0, 9, b.data_ptr(), None) == OK
    assert torch.equal(a, b)


@pytest.mark.parametrize("change,status", [(dict(n=-1), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(words=0), SHAPE), (dict(n=4097), UNSUPPORTED),
                                           (dict(parents=None), INVALID), (dict(n=0, parents=None), OK), (dict(seen=None, words=0, depth=None), OK)])
def test_refusals(change, status):
    up, seen, depth = (torch.zeros(s, dtype=torch.int32) for s in (3, 3, 3))
    up[0] = -1
    a = dict(parents=up.data_ptr(), n=3, words=1, window=2, sinks=1, seen=seen.data_ptr(), depth=depth.data_ptr())
    a.update(change)
    assert M._lib().moe_tree_window_masks(a["parents"], a["n"], a["words"], a["window"], a["sinks"], a["seen"], a["depth"]) == status


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (8, 0), (20, 5), (20, 60), (1000, 4)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_tree_and_its_tokens_one_by_one(window, sinks, e4m3):
    """Each token sees what it would see as the last one of its path behind the context, also where the path is longer than the window or reaches into the sinks."""
    H, Hk, D, page = 4, 2, 64, 16
    g, r = torch.Generator(device="cuda").manual_seed(window), random.Random(window)
    for context, parents in ((50, _chain(30)), (0, _chain(24)), (3, random_tree(r, 40)), (70, random_tree(r, 20)), (20, [-1] + [max(0, j - 2) for j in range(1, 25)])):
        n = len(parents)
        pages = -(-(context + n) // page)
        scale = torch.full((Hk,), 1 / 64, device="cuda") if e4m3 else None
        make = lambda: torch.empty((pages, page, Hk, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        k, v = (((x * 64).to(torch.float8_e4m3fn)) if e4m3 else x for x in (make(), make()))
        q = torch.empty((n, H, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        seen, depth = A.tree_masks(parents, None, window, max(0, sinks - context))
        run = lambda bits: A.moe_chunk_attention(A.KvCache(k, v, scale, scale), q, table, dev([0, n]), dev([context]), seen=bits.cuda(), positions=depth.cuda() + context,
                                                 window=window, sinks=sinks)
        got, most, different = run(seen), float((v.float() / (64 if e4m3 else 1)).abs().max()), False
        unseen = run(A.tree_masks(parents)[0])
        for i in range(n):
            path = torch.tensor(_path(parents, i), device="cuda")
            cache = A.KvCache(k.clone(), v.clone(), scale, scale)
            for held, of in ((cache.k, k), (cache.v, v)):
                held.view(torch.uint8).flatten(0, 1)[context:context + len(path)] = of.view(torch.uint8).flatten(0, 1)[context + path]
            want = A.moe_sink_attention(cache, q[i:i + 1], table, dev([context + len(path)]), window, sinks)[0].double().cpu()
            # each side rounds its result (half a step of bf16); a probability keeps 16 bits, or the 11 of fp16 beside an 8-bit v; scores are fp32 sums
            tol = 2 * HALF_BF16 * want.abs() + (2.0 ** -10 if e4m3 else 2.0 ** -12) * most
            near(got[i], want, tol, f"token {i} of {n} behind {context}")
            different = different or bool(((unseen[i].double().cpu() - want).abs() > tol).any())
        # an ancestor at depth j is left out for the deepest token, at depth d, if j <= d - window and j is no sink
        assert different == (int(depth.max()) - window >= max(0, sinks - context))
