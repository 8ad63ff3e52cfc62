"""Log probabilities of given tokens, ranks, entropy and the best alternatives against the definitions in 64 bits."""
import math

import pytest
import torch

import paper_2507_17133_amd as A

pytestmark = pytest.mark.gpu

# A sum of exponentials is off by at most 40 roundings of fp32 on the way to it (32 terms of a thread, across 64 lanes, four waves, slices), each term by
# its exponent's rounding and the hardware's exponential (2 and 1 units in the last place, at terms that count)
SUM = 44 * 2.0 ** -24


def _reference(x, tokens, top):
    x = x.double().cpu()
    T, V = x.shape
    logp = torch.log_softmax(x, 1)
    lse = torch.logsumexp(x, 1)
    none = x.isnan().any(1) | (x == math.inf).any(1)
    empty = (x == -math.inf).all(1)
    ent = -(logp.exp() * logp.clamp_min(-1e300)).sum(1)
    ent[empty], lse[empty] = 0.0, -math.inf
    ent[none] = lse[none] = math.nan
    of = lambda r, i: math.nan if none[r] else -math.inf if x[r, i] == -math.inf else float(logp[r, i])
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    r = dict(lse=lse, entropy=ent)
    if tokens is not None:
        tok = tokens.cpu()
        rank, lp = torch.empty(tok.shape, dtype=torch.int64), torch.empty(tok.shape, dtype=torch.float64)
        place = torch.empty_like(order).scatter_(1, order, torch.arange(V).expand(T, V))
        for t in range(T):
            for g in range(tok.shape[1]):
                i = int(tok[t, g])
                ok = 0 <= i < V
                rank[t, g] = -1 if not ok or none[t] else place[t, i]
                lp[t, g] = of(t, i) if ok else 0.0
        r.update(rank=rank, logprob=lp)
    if top:
        ids = order[:, :top].clone()
        r["top_logprob"] = torch.tensor([[of(t, int(i)) for i in ids[t]] for t in range(T)], dtype=torch.float64)
        ids[none] = -1
        r["top_id"] = ids
    return r


def _check(x, tokens=None, top=0, got=None):
    got = A.moe_token_logprobs(x, tokens, top) if got is None else got
    want = _reference(x, tokens, top)
    big = x.double().abs().cpu()
    big[~big.isfinite()] = 0
    big = big.amax(1)
    for name, w in want.items():
        g = getattr(got, name)
        if name in ("rank", "top_id"):
            assert torch.equal(g.cpu().long(), w), name
            continue
        g = g.double().cpu()
        w = torch.where(w < -torch.finfo(torch.float32).max, -math.inf, w)      # fp32 holds nothing below: x_g - lse of 3e38 apart is -infinity there
        assert torch.equal(g.isnan(), w.isnan()), name
        assert torch.equal(g == -math.inf, w == -math.inf), name
        f = w.isfinite()
        # log S, at most log V; the maximum and the value come in exactly, differences and results are rounded
        tol = SUM + 2.0 ** -23 * (w.abs() + math.log(x.shape[1]) + 1)
        if name == "entropy":
            tol = SUM * (2 + 2 * math.log(x.shape[1])) + 2.0 ** -22 * (w.abs() + math.log(x.shape[1]) + 1)
        if name == "lse":
            tol = tol + 2.0 ** -23 * big
        bad = f & ~((g - w).abs() <= tol)
        assert not bool(bad.any()), (name, bad.nonzero()[0].tolist(), g[bad][0].item(), w[bad][0].item(), tol[bad][0].item())
    return got


def _logits(seed, T, V, dtype=torch.bfloat16, std=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((T, V), device="cuda").normal_(0, std, generator=g)
    return x.to(dtype), lambda n: torch.randint(0, V, (T, n), generator=g, device="cuda").to(torch.int32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 64, 65, 100, 2040, 2048, 2049, 8191, 8192, 8200, 20011, 100003])
@pytest.mark.parametrize("T", [1, 5])
def test_sizes(dtype, V, T):
    x, ids = _logits(V + T, T, V, dtype)
    _check(x, ids(3), min(V, 20))


@pytest.mark.parametrize("T,V", [(800, 8200), (3000, 500), (130, 60000)])
def test_many_rows(T, V):
    x, ids = _logits(T, T, V)
    _check(x, ids(2), 5)


@pytest.mark.parametrize("given,top", [(0, 0), (1, 0), (0, 1), (64, 0), (0, 64), (64, 64), (5, 33)])
@pytest.mark.parametrize("V", [64, 70, 5000, 50000])
def test_given_and_top(given, top, V):
    x, ids = _logits(given + top, 3, V)
    _check(x, ids(given) if given else None, top)


def test_the_most_entries():
    x, ids = _logits(1, 1, 1 << 20, torch.float32)
    _check(x, ids(4), 64)
    _check(x.to(torch.bfloat16), ids(4), 64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("off", [1, 3, 5, 7])
def test_rows_that_begin_anywhere(dtype, off):
    wide, ids = _logits(off, 4, 9013, dtype)
    for V in (9, 2050, 9000):
        x = wide[:, off:off + V]
        tokens = ids(3) % V
        _check(x, tokens, 9)
        for t in range(4):                                # a row's neighbours do not matter
            alone = A.moe_token_logprobs(x[t:t + 1].contiguous(), tokens[t:t + 1].contiguous(), 9)
            assert torch.equal(alone.top_id, A.moe_token_logprobs(x, tokens, 9).top_id[t:t + 1])
    around = torch.full((3, 700), math.nan, dtype=dtype, device="cuda")
    around[:, off:off + 600] = wide[:3, :600]
    _check(around[:, off:off + 600], ids(2)[:3] % 600, 5)


@pytest.mark.parametrize("V", [5, 300, 3000, 70001])
def test_ties(V):
    for x in (torch.zeros((2, V), device="cuda"), torch.full((2, V), -3.0, dtype=torch.bfloat16, device="cuda"),
              (torch.arange(V, device="cuda") % 3).float().expand(2, V).contiguous(), torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0).expand(2, V).contiguous(),
              torch.round(_logits(V, 2, V)[0].float())):
        tokens = torch.tensor([[0, V - 1, V // 2], [V // 3, 1 % V, V // 2 + 1 if V > 3 else 0]], dtype=torch.int32, device="cuda")
        _check(x, tokens, min(V, 40))


def test_banned_entries():
    x, ids = _logits(2, 4, 5000)
    x[0, 100:] = -math.inf
    x[1] = -math.inf
    x[2, :4990] = -math.inf
    x[3, ::2] = -math.inf
    tokens = ids(6)
    tokens[:, 0], tokens[:, 1] = 99, 4995
    _check(x, tokens, 30)
    _check(x.float(), tokens, 64)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("V", [50, 30000])
def test_rows_without_a_distribution(bad, V):
    x, ids = _logits(3, 4, V)
    x[1, V - 1], x[2, 0] = bad, bad
    if bad != bad:
        x[2] = bad
    tokens = ids(5)
    tokens[1, 0], tokens[2, 1] = V - 1, -1
    got = _check(x, tokens, 10)
    assert bool(got.lse[1:3].isnan().all()) and bool((got.top_id[1:3] == -1).all()) and float(got.logprob[2, 1]) == 0.0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_and_small_values(dtype):
    x, ids = _logits(4, 8, 4000, torch.float32)
    x[0] *= 1e4
    x[1] *= 1e30
    x[2] = x[2].clamp(-1, 1) * 3e38
    x[3] *= 1e-30
    x[4] += 1000
    x[5] -= 60000
    x[6] = 1e-45
    x[7, 17] = 300.0                                      # all of the probability on one entry
    _check(x.to(dtype), ids(4), 8)


def test_tokens_that_are_none():
    x, _ = _logits(5, 3, 777)
    tokens = torch.tensor([[-1, 777, 776, 0], [1 << 30, -(1 << 31), 5, 5], [3, 3, 3, -7]], dtype=torch.int32, device="cuda")
    _check(x, tokens, 3)


def test_outputs_that_are_not_wanted():
    x, ids = _logits(6, 5, 3000)
    tokens = ids(3)
    want = A.moe_token_logprobs(x, tokens, 7)
    for keep in (("logprob",), ("rank",), ("lse",), ("entropy", "top_id"), ("top_logprob",), ()):
        out = A.alloc_logprobs(5, 3, 7)
        out = A.Logprobs(**{k: getattr(out, k) for k in keep})
        got = A.moe_token_logprobs(x, tokens, 7, out=out)
        assert all(torch.equal(getattr(got, k), getattr(want, k)) for k in keep)


def test_strided_tokens_the_same_bits_a_workspace_of_larger_calls_and_a_stream():
    x, ids = _logits(7, 9, 40000)
    wide = ids(8)
    ws = A.alloc_logprob_workspace(900, 50000, 8, 20)
    want = A.moe_token_logprobs(x, wide[:, 2:5].contiguous(), 11)
    ws.fill_(255)
    side = torch.cuda.Stream()
    for k in range(3):
        side.wait_stream(torch.cuda.current_stream())
        got = A.moe_token_logprobs(x, wide[:, 2:5], 11, workspace=ws, stream=side if k else None)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_graphs_that_share_a_workspace():
    x, ids = _logits(8, 6, 33000)
    tokens, ws, out = ids(2), A.alloc_logprob_workspace(6, 33000, 2, 5), A.alloc_logprobs(6, 2, 5)
    A.moe_token_logprobs(x, tokens, 5, workspace=ws, out=out)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            A.moe_token_logprobs(x, tokens, 5, workspace=ws, out=out)
        graphs.append(g)
    for turn in range(4):
        x.normal_(0, 3)
        graphs[turn % 2].replay()
        got = [t.clone() for t in out]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, A.moe_token_logprobs(x, tokens, 5)))


def test_no_rows_and_a_tensor_that_requires_a_gradient():
    x, ids = _logits(9, 2, 100)
    assert A.moe_token_logprobs(x[:0], ids(2)[:0], 3).top_id.shape == (0, 3)
    with pytest.raises(AssertionError):
        A.moe_token_logprobs(x.requires_grad_(), ids(2))
