"""A step of drafted trees as a serving program makes it: append at places of their own, attention of the trees, logits, log probabilities of each token's
children, the accepted path moved to its positions -- against the same tokens decoded one after the other, eager and from a graph."""
import random

import pytest
import torch

import paper_2507_17133_amd as A
from tests._draft_util import random_tree
from tests._layer_util import near

pytestmark = pytest.mark.gpu

H, HK, D, V, PAGE = 8, 2, 64, 1000, 16


class _Step:
    """Weights, cache and trees of a few sequences; `draft` is the step up to the log probabilities, `keep` the move."""

    def __init__(self, seed, e4m3, prompts, new):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = random.Random(seed)
        d = H * D
        normal = lambda *s: (torch.randn(s, generator=g, device="cuda") / s[-1] ** 0.5).to(torch.bfloat16)
        self.wqkv, self.head = A.moe_quantize_weight(normal((H + 2 * HK) * D, d)), A.moe_quantize_weight(normal(V, d))
        self.norm = torch.ones(d, dtype=torch.bfloat16, device="cuda")
        self.rope = A.make_rope(D)
        B, self.pages = len(prompts), -(-(max(prompts) + max(new) + 2) // PAGE)
        scale = torch.full((HK,), 1 / 64, device="cuda") if e4m3 else None
        self.cache = A.alloc_kv_cache(B * self.pages, PAGE, HK, D, scale, scale)
        for t in (self.cache.k, self.cache.v):
            t.view(torch.uint8).zero_()
        self.table = torch.randperm(B * self.pages, generator=g, device="cuda").to(torch.int32).view(B, self.pages)
        self.context, self.new = list(prompts), list(new)
        self.parents = [random_tree(r, n) for n in new]
        masks = [A.tree_masks(p, -(-max(new) // 32)) for p in self.parents]
        self.seen, self.depth = torch.cat([m for m, _ in masks]).cuda(), torch.cat([x for _, x in masks]).cuda()
        self.row = torch.repeat_interleave(torch.arange(B), torch.tensor(new)).to(torch.int32).cuda()
        self.first = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32).cuda()
        self.nth = torch.cat([torch.arange(n) for n in new]).to(torch.int32).cuda()
        self.ctx = torch.tensor(prompts, dtype=torch.int32).cuda()
        self.prompt = [torch.randn((n, d), generator=g, device="cuda").to(torch.bfloat16) for n in prompts]
        self.x = torch.randn((sum(new), d), generator=g, device="cuda").to(torch.bfloat16)      # what the drafted tokens stand for
        # each token's children (up to 3), as the numbers of the tokens that they stand for
        self.vocab = torch.randint(0, V, (sum(new),), generator=g, device="cuda").to(torch.int32)
        children = torch.full((sum(new), 3), -1, dtype=torch.int32)
        for b, p in enumerate(self.parents):
            for j, up in enumerate(p):
                if up >= 0:
                    free = (children[int(self.first[b]) + up] == -1).nonzero()
                    if len(free):
                        children[int(self.first[b]) + up, free[0]] = self.vocab[int(self.first[b]) + j].cpu()
        self.children = children.cuda()
        self.ws = A.alloc_chunk_workspace(self.cache, B, sum(new), H)
        self.lws = A.alloc_logprob_workspace(sum(new), V, 3, 5)
        for b, x in enumerate(self.prompt):
            q, k, v = self.qkv(x)
            pos = torch.arange(len(x), device="cuda").to(torch.int32)
            A.moe_rope_append(self.cache, self.rope, q, k, v, pos, self.table, table_row=torch.full_like(pos, b))

    def qkv(self, x):
        n = A.moe_rms_norm(x, self.norm, want=("y8",))
        return A.moe_linear_e4m3(n.y8, n.scale, *self.wqkv).view(-1, H + 2 * HK, D).split((H, HK, HK), 1)

    def draft(self):
        q, k, v = self.qkv(self.x)
        start = self.ctx[self.row.long()]
        positions, places = start + self.depth, start + self.nth
        q = A.moe_rope_append_at(self.cache, self.rope, q, k, v, positions, places, self.table, table_row=self.row)
        o = A.moe_chunk_attention(self.cache, q, self.table, self.first, self.ctx, seen=self.seen, positions=positions, workspace=self.ws)
        logits = A.moe_linear_e4m3(*A.moe_quantize_rows(o.view(-1, H * D)), *self.head)
        return o, logits, A.moe_token_logprobs(logits, self.children, 5, workspace=self.lws)

    def path(self, b, j):
        p = []
        while j >= 0:
            p.append(j)
            j = self.parents[b][j]
        return p[::-1]

    def one_by_one(self, cache, b, path):
        """Attention's outputs of a path's tokens decoded one after the other, and the cache then."""
        got = []
        for i, j in enumerate(path):
            t = int(self.first[b]) + j
            q, k, v = self.qkv(self.x[t:t + 1])
            pos = torch.tensor([self.context[b] + i], dtype=torch.int32, device="cuda")
            row = torch.tensor([b], dtype=torch.int32, device="cuda")
            q = A.moe_rope_append(cache, self.rope, q, k, v, pos, self.table, table_row=row)
            got.append(A.moe_paged_attention(cache, q, self.table, pos + 1, table_row=row)[0])
        return got


def _copy(cache):
    return A.KvCache(cache.k.clone(), cache.v.clone(), cache.k_scale, cache.v_scale)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("prompts,new", [([40, 3, 90], [13, 33, 1]), ([200], [60]), ([17] * 9, [4] * 9)])
def test_a_step(e4m3, prompts, new):
    s = _Step(1, e4m3, prompts, new)
    clean = _copy(s.cache)
    o, logits, lp = s.draft()
    B = len(prompts)
    deepest = [max(range(n), key=lambda j: len(s.path(b, j))) for b, n in enumerate(new)]
    sequential = []
    for b in range(B):
        for j in {deepest[b], new[b] - 1, 0}:
            cache = _copy(clean)
            path = s.path(b, j)
            for i, want in zip(path, s.one_by_one(cache, b, path)):
                # probabilities rounded to bf16 (half a step, 2^-8, of |v| < 8 here) in one of the two ways, the result in both
                near(o[int(s.first[b]) + i], want.double(), 2 * 2.0 ** -8 * want.double().abs().cpu() + 2.0 ** -8 * 8, f"token {i} of sequence {b}")
            if j == deepest[b]:
                sequential.append(cache)
    # log probabilities of what the logits say
    x = logits.double()
    logp = torch.log_softmax(x, 1)
    real = s.children >= 0
    want = torch.where(real, logp.gather(1, s.children.long().clamp_min(0)), 0.0)
    near(lp.logprob, want, 44 * 2.0 ** -24 + 2.0 ** -22 * (want.abs().cpu() + 8), "log probabilities")
    assert torch.equal(lp.top_id[:, 0].long(), x.float().argmax(1)) and bool((lp.rank[real] >= 0).all()) and bool((lp.rank[~real] == -1).all())
    # the accepted paths: one token fewer for every second sequence
    paths = [s.path(b, deepest[b])[: None if b % 2 == 0 else -1] for b in range(B)]
    most = max(len(p) for p in paths)
    sources = torch.tensor([[s.context[b] + j for j in p] + [-1] * (most - len(p)) for b, p in enumerate(paths)], dtype=torch.int32, device="cuda").view(B, most)
    A.moe_cache_move(s.cache, s.table, sources, s.ctx, torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda"))
    for b, p in enumerate(paths):
        at = torch.arange(s.context[b] + len(p), device="cuda")
        page, place = s.table[b].long()[at // PAGE], at % PAGE
        for mine, theirs in ((s.cache.k, sequential[b].k), (s.cache.v, sequential[b].v)):
            assert torch.equal(mine.view(torch.uint8)[page, place], theirs.view(torch.uint8)[page, place])


def test_a_step_from_a_graph():
    s = _Step(2, False, [40, 3, 90], [13, 33, 1])
    accepted, count = torch.zeros((3, 2), dtype=torch.int32, device="cuda"), torch.tensor([2, 1, 0], dtype=torch.int32, device="cuda")

    def step():
        r = s.draft()
        A.moe_cache_move(s.cache, s.table, accepted, s.ctx, count)
        return r
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, logits, lp = step()
    for turn in range(4):
        s.x.normal_()
        s.ctx.copy_(torch.tensor([40 - turn, 3 + turn, 90], dtype=torch.int32))
        accepted.copy_(s.ctx[:, None] + torch.tensor([[0, 2], [1, 5], [0, 0]], dtype=torch.int32, device="cuda"))
        before = _copy(s.cache)
        graph.replay()
        got = [t.clone() for t in (o, logits, *lp)]
        after = _copy(s.cache)
        torch.cuda.synchronize()
        s.cache.k.copy_(before.k), s.cache.v.copy_(before.v)
        o2, logits2, lp2 = step()
        assert all(torch.equal(a, b) for a, b in zip(got, (o2, logits2, *lp2)))
        assert torch.equal(after.k, s.cache.k) and torch.equal(after.v, s.cache.v)
