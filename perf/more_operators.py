"""Operators of a step with several new tokens of a sequence, and of what a model answers, as they are timed and compared: attention with a
window and sinks for single tokens, attention of drafted trees and of prompts' chunks over the paged cache, the append of drafted tokens at places
of their own, the move of the accepted ones to their positions, and log probabilities of given tokens with entropy and the best alternatives.

A case names an operator in `op`:

  sink      T tokens, each attending to the last `window` positions of its own sequence and to its first `sinks` ones
  chunk     `seqs` sequences with up to `new` new tokens each behind a cached context: a tree of drafted tokens, each seeing the context and its own
            ancestors (`tree`), or a chunk of a prompt, each seeing what is before it, with a window and sinks if `window` is not 0
  append    drafted tokens' q and k rotated by their depth in the tree, k and v written one behind the other
  move      keys and values of accepted drafted tokens moved to the positions that they have in the sequence
  logprob   logits of T rows: log probabilities and ranks of `given` tokens a row, entropy, log of the sum of exponentials, the `top` best

`own` False: the plain form in elementary torch operations; True: the framework's kernels.
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
BIG = 448.0                  # largest e4m3 value

#: A drawn case costs no more than these: elements of k that tokens or sequences attend to (as many of v), products of the attention, elements of
#: scores that the plain form holds, q, k and v of append, elements of the caches of move, logits.
MOST_READ = 256 * 4160 * 4 * 128
MOST_PRODUCTS = 16384 * 56 * 128 * 4000
MOST_SCORES = 4 * 4096 * 56 * 12288
MOST_APPEND = 2112 * 48 * 128
MOST_MOVED = 256 * 1024 * 8 * 128
MOST_LOGITS = 2112 * 131072


def _sink(name, T, heads, kv_heads, D, longest, window, sinks, e4m3, page, heads_first=False, empty=0.0):
    return {"name": name, "op": "sink", "T": T, "heads": heads, "kv_heads": kv_heads, "D": D, "longest": longest, "window": window, "sinks": sinks,
            "e4m3": e4m3, "page": page, "heads_first": heads_first, "empty": empty}


def _chunk(name, tree, seqs, new, heads, kv_heads, D, longest, e4m3, page, heads_first=False, window=0, sinks=0, blank=0.0):
    return {"name": name, "op": "chunk", "tree": tree, "seqs": seqs, "new": new, "heads": heads, "kv_heads": kv_heads, "D": D, "longest": longest,
            "e4m3": e4m3, "page": page, "heads_first": heads_first, "window": window, "sinks": sinks, "blank": blank}


def _append(name, seqs, new, heads, kv_heads, D, R, interleaved, longest, e4m3, page, heads_first=False):
    return {"name": name, "op": "append", "seqs": seqs, "new": new, "heads": heads, "kv_heads": kv_heads, "D": D, "R": R, "interleaved": interleaved,
            "longest": longest, "e4m3": e4m3, "page": page, "heads_first": heads_first}


def _move(name, seqs, new, accepted, kv_heads, D, longest, e4m3, page, heads_first=False):
    return {"name": name, "op": "move", "seqs": seqs, "new": new, "accepted": accepted, "kv_heads": kv_heads, "D": D, "longest": longest, "e4m3": e4m3,
            "page": page, "heads_first": heads_first}


def _logprob(name, T, V, given, top, fp32=False, banned=0.0):
    return {"name": name, "op": "logprob", "T": T, "V": V, "given": given, "top": top, "fp32": fp32, "banned": banned}


def listed():
    return [
        # one request of a stream without end: its last 1024 positions and the first four
        _sink("sink_token_1", 1, 32, 8, 128, 8192, 1024, 4, False, 16),
        # a decode batch of 256 such requests with wide windows, some slots of the batch unused
        _sink("sink_decode_256", 256, 32, 4, 128, 8192, 4096, 64, False, 16, empty=0.05),
        # one request with a small tree of drafted tokens: latency counts
        _chunk("tree_request_1", True, 1, 26, 32, 8, 128, 2048, False, 16),
        # 64 requests with trees of up to 33 tokens, cache in 8 bits, some tokens of a tree without anything to see
        _chunk("tree_batch_64", True, 64, 33, 64, 8, 128, 8192, True, 64, heads_first=True, blank=0.02),
        # prefill of 16384 tokens of four prompts in chunks of 4096 behind up to 8192 earlier positions, hidden size 7168 in 56 heads
        _chunk("chunk_prefill_16384", False, 4, 4096, 56, 8, 128, 8192, False, 16, window=4096, sinks=4),
        # the drafted tree of one request goes to the cache
        _append("append_tree_26", 1, 26, 32, 8, 128, 128, False, 2048, False, 16),
        # the trees of 64 requests go to a cache in 8 bits, half of each head rotated in pairs
        _append("append_trees_64", 64, 33, 32, 8, 128, 64, True, 8192, True, 64, True),
        # one request keeps its accepted path
        _move("move_request_1", 1, 26, 5, 8, 128, 2048, False, 16),
        # 256 requests keep theirs
        _move("move_batch_256", 256, 64, 9, 8, 128, 1000, True, 16),
        # one token's logits over 32000 entries, the token chosen and five alternatives
        _logprob("logprob_token_1", 1, 32000, 1, 5),
        # an odd decode batch over an odd number of entries, logits in 32 bits, a tenth of them banned
        _logprob("logprob_decode_67", 67, 50021, 1, 20, fp32=True, banned=0.1),
        # every token of 64 trees of 33, four children each to be looked up
        _logprob("logprob_trees_2112", 2112, 131072, 4, 8),
    ]


def _log(rng, lo, hi):
    hi = max(lo, hi)
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng, most):
    kv = rng.choice([1, 2, 4, 8, 8, 16])
    return kv * rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8, 16, 24) if g * kv <= most]), kv


def draw(rng):
    op = rng.choice(["sink", "tree", "tree", "chunk", "append", "move", "logprob"])
    D, page, first, e4m3 = rng.choice([64, 96, 128, 128, 128, 192, 256]), rng.choice([1, 16, 16, 48, 64, 128]), rng.random() < 0.5, rng.random() < 0.4
    heads, kv = _heads(rng, 64)
    if op == "sink":
        T = _log(rng, 1, 512)
        most = MOST_READ // (T * kv * D)
        sinks = rng.choice([0, 1, 4, 4, 33, 128])
        window = _log(rng, 1, max(1, min(8192, most - sinks)))
        longest = _log(rng, 1, max(1, min(65536, 2 * most)))
        case = _sink("", T, heads, kv, D, longest, window, sinks, e4m3, page, first, rng.choice([0.0, 0.0, 0.1]))
    elif op in ("tree", "chunk"):
        tree = op == "tree"
        seqs = _log(rng, 1, 128 if tree else 16)
        new = _log(rng, 1, 130 if tree else 4096 // max(1, seqs // 4))
        longest = _log(rng, 1, min(131072, MOST_READ // (seqs * kv * D), MOST_PRODUCTS // (seqs * new * heads * D), MOST_SCORES // (seqs * new * heads)))
        window = rng.choice([0, 0, 0, 100, 1024]) if tree else rng.choice([0, 0, 64, 1000, 4096])
        # new tokens see each other too: what is left of the products goes by both lengths
        new = max(1, min(new, MOST_PRODUCTS // (seqs * new * heads * D), MOST_SCORES // (seqs * (longest + new) * heads)))
        case = _chunk("", tree, seqs, new, heads, kv, D, longest, e4m3, page, first, window, rng.choice([0, 1, 4, 40]) if window else 0,
                      rng.choice([0.0, 0.0, 0.1]) if tree else 0.0)
    elif op == "append":
        seqs = _log(rng, 1, 64)
        new = _log(rng, 1, max(1, min(128, MOST_APPEND // (seqs * (heads + 2 * kv) * D))))
        case = _append("", seqs, new, heads, kv, D, rng.choice([D, D // 2 // 16 * 16, 16 * rng.randint(1, D // 16)]), rng.random() < 0.4,
                       _log(rng, 1, 65536), e4m3, page, first)
    elif op == "move":
        seqs, new = _log(rng, 1, 256), _log(rng, 1, 128)
        accepted = min(new, _log(rng, 1, 32))
        longest = _log(rng, 1, min(2048, max(1, MOST_MOVED // (seqs * kv * D) - new - page)))
        case = _move("", seqs, new, accepted, kv, D, longest, e4m3, page, first)
    else:
        V = _log(rng, 100, 200000)
        T = _log(rng, 1, min(4096, MOST_LOGITS // V))
        case = _logprob("", T, V, rng.choice([0, 1, 1, 3, 8]), rng.choice([0, 1, 5, 20, 32]), rng.random() < 0.3, rng.choice([0.0, 0.3]))
    del case["name"]
    return case


# ---------------------------------------------------------------- inputs

def _normal(gen, shape, std=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _ints(gen, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=torch.int64)


def _cache(case, gen, n_pages):
    """k and v of a paged cache, [page, token, head, D] whichever of the two orders they are stored in; e4m3 with a scale per head."""
    H, P, D = case["kv_heads"], case["page"], case["D"]
    shape = (n_pages, H, P, D) if case["heads_first"] else (n_pages, P, H, D)
    s = {}
    for n in ("k", "v"):
        t = _normal(gen, shape)
        if case["e4m3"]:
            s[n + "_scale"] = torch.empty(H, device="cuda").uniform_(0.01, 0.02, generator=gen)
            t = (t * 64).to(E4M3)                # N(0, 64^2) in units of the scale: inside the type's range
        s[n] = t.transpose(1, 2) if case["heads_first"] else t
    return s


def _table(gen, rows, pages):
    """A block table [rows, pages] that deals out the pages of a pool at random, and the pool's size."""
    n = rows * pages + 3
    return torch.randperm(n, generator=gen, device="cuda")[: rows * pages].reshape(rows, pages).to(torch.int32), n


def _new_tokens(case):
    """How many new tokens each sequence has: the most for the first, down to half as many, now and then one or none."""
    most, half = case["new"], case["new"] // 2
    each = [most - (b * 7919) % (half + 1) if case.get("tree", True) else most for b in range(case["seqs"])]
    if case["seqs"] > 8:
        each[3], each[5] = 1, 0
    return each


def _words(case):
    return -(-case["new"] // 32)


def _trees(case, seed):
    """A random tree for each sequence: its tokens' ancestors and themselves as bits [T, words], and their depths [T]."""
    r, words = torch.Generator().manual_seed(seed * 1000 + 31), _words(case)
    each = _new_tokens(case)
    picks = torch.rand(sum(each), generator=r).tolist()
    blank = (torch.rand(sum(each), generator=r) < case.get("blank", 0.0)).tolist()
    bits, depths, at = [], [], 0
    for n in each:
        seen, depth = [], []
        for j in range(n):
            parent = int(picks[at + j] ** 0.5 * j)   # late tokens are likelier parents: chains with branches
            seen.append(1 << j | (seen[parent] if j else 0))
            depth.append(depth[parent] + 1 if j else 0)
        bits += [0 if blank[at + j] else seen[j] for j in range(n)]
        depths += depth
        at += n
    flat = [(b >> 32 * w) & 0xFFFFFFFF for b in bits for w in range(words)]
    seen = torch.tensor(flat, dtype=torch.int64).reshape(len(bits), words).cuda()
    return (seen - ((seen >> 31) << 32)).to(torch.int32), torch.tensor(depths, dtype=torch.int64).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000 + 29)
    s = {"case": case}
    if case["op"] == "logprob":
        T, V = case["T"], case["V"]
        x = _normal(gen, (T, V), 2.0, torch.float32 if case["fp32"] else torch.bfloat16)
        x[torch.arange(T, device="cuda")[:, None], _ints(gen, 0, V, (T, 8))] += 8           # a few likely tokens
        if case["banned"]:
            x[:, torch.rand(V, generator=gen, device="cuda") < case["banned"]] = -math.inf
        s["logits"] = x
        given = _ints(gen, 0, V, (T, case["given"])) if case["given"] else None
        if given is not None and T > 4:
            given[T // 2, -1] = -1                   # no token
        s["given"] = None if given is None else given.to(torch.int32)
        s["top"] = min(case["top"], V)
        return s
    H, Hk, D, P, longest = (case[k] for k in ("heads", "kv_heads", "D", "page", "longest")) if case["op"] != "move" else (0,) + tuple(
        case[k] for k in ("kv_heads", "D", "page", "longest"))
    if case["op"] == "sink":
        T = case["T"]
        n = _ints(gen, (longest + 1) // 2, longest + 1, (T,))          # between half the longest and the longest
        n = torch.where(torch.rand(T, generator=gen, device="cuda") < case["empty"], 0, n)
        s["lengths"] = n.to(torch.int32)
        s["table"], pages = _table(gen, T, -(-longest // P))
        s["q"] = _normal(gen, (T, H, D))
        s["cache"] = _cache(case, gen, pages)
        s["scale"] = 1.0 / math.sqrt(D)
        return s
    each, B = _new_tokens(case), case["seqs"]
    T = sum(each)
    s["most"] = max(each)                                              # new tokens of a sequence, known to a program that lays them out
    context = _ints(gen, longest // 2, longest + 1, (B,))
    s["context"] = context.to(torch.int32)
    s["table"], pages = _table(gen, B, -(-(longest + case["new"]) // P))
    if case["op"] == "move":
        s["cache"] = _cache(case, gen, pages)
        # accepted: increasing numbers among the sequence's drafted tokens
        order = torch.rand((B, case["new"]), generator=gen, device="cuda").argsort(1)[:, : case["accepted"]].sort(1).values
        s["sources"] = (context[:, None] + order).to(torch.int32)
        s["count"] = _ints(gen, 0, case["accepted"] + 1, (B,)).to(torch.int32)
        s["count"][0] = case["accepted"]
        return s
    sizes = torch.tensor(each, device="cuda")
    s["first"] = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)]).to(torch.int32)
    row = torch.repeat_interleave(torch.arange(B, device="cuda"), sizes)
    nth = torch.arange(T, device="cuda") - s["first"].long()[row]
    if case["op"] == "append" or case["tree"]:
        seen, depth = _trees(case, seed)
        s["positions"] = (context[row] + depth).to(torch.int32)
    if case["op"] == "chunk":
        s["seen"] = seen if case["tree"] else None
        s["q"] = _normal(gen, (T, H, D))
        s["cache"] = _cache(case, gen, pages)
        s["scale"] = 1.0 / math.sqrt(D)
    else:
        s["table_row"], s["places"] = row.to(torch.int32), (context[row] + nth).to(torch.int32)
        s["qkv"] = _normal(gen, (T, (H + 2 * Hk) * D))
        s["turns"] = (10000.0 ** (-2.0 * torch.arange(case["R"] // 2, dtype=torch.float64) / max(case["R"], 1)) / (2 * math.pi)).cuda()
        # only the pages that are written need to be there
        used = torch.zeros_like(s["table"], dtype=torch.bool)
        used[row, s["places"].long() // P] = True
        s["table"] = torch.where(used, used.flatten().cumsum(0).reshape(used.shape), 0).to(torch.int32)
        s["cache"] = {k: v if "scale" in k else torch.zeros_like(v) for k, v in _cache(case, gen, B * (-(-case["new"] // P) + 1) + 1).items()}
    return s


# ---------------------------------------------------------------- the plain forms, in 32 bits

def _held(cache, name, page, at, head):
    """k or v of one head at places (page, at), as the values it stands for."""
    c = cache[name]
    if c.dtype == E4M3:
        return c.view(torch.uint8)[page, at, head].view(E4M3).float() * cache[name + "_scale"][head]
    return c[page, at, head].float()


def _softmax_over(score, seen, v):
    """score and seen [.., q, positions], v [.., positions, D]."""
    score = score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top.clamp_min(-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / total.clamp_min(1e-30), (top + torch.log(total))[..., 0]


def _plain_sink(s):
    case, cache = s["case"], s["cache"]
    T, H, Hk, D, P, W, S = (case[k] for k in ("T", "heads", "kv_heads", "D", "page", "window", "sinks"))
    n = s["lengths"].long()[:, None]
    i = torch.arange(min(S + W, case["longest"]), device="cuda")[None, :]
    lo = (n - W).clamp_min(0)
    sinks = lo.clamp_max(S)
    pos = torch.where(i < sinks, i, i - sinks + lo)
    seen = pos < n
    pos = torch.where(seen, pos, 0)
    page = s["table"].long().gather(1, pos // P)
    k, v = (_held(cache, c, page[:, None], (pos % P)[:, None], torch.arange(Hk, device="cuda")[None, :, None]) if not case["e4m3"] else
            cache[c].view(torch.uint8)[page[:, None], (pos % P)[:, None], torch.arange(Hk, device="cuda")[None, :, None]].view(E4M3).float()
            * cache[c + "_scale"][None, :, None, None] for c in ("k", "v"))                        # [T, Hk, positions, D]
    score = torch.matmul(s["q"].float().reshape(T, Hk, H // Hk, D), k.transpose(2, 3)) * s["scale"]
    out, lse = _softmax_over(score, seen[:, None, None, :], v)
    return {"out": out.reshape(T, H, D).to(torch.bfloat16), "lse": lse.reshape(T, H)}


def _plain_chunk(s):
    case, cache = s["case"], s["cache"]
    H, Hk, D, P, W, S, B = (case[k] for k in ("heads", "kv_heads", "D", "page", "window", "sinks", "seqs"))
    N, T, G = s["most"], s["q"].shape[0], case["heads"] // case["kv_heads"]
    first, context = s["first"].long(), s["context"].long()
    token = first[:-1, None] + torch.arange(N, device="cuda")                                     # [B, N]
    real = token < first[1:, None]
    token = torch.where(real, token, 0)
    p = torch.arange(case["longest"] + N, device="cuda")                                          # [L]
    new = p[None, :] - context[:, None]                                                           # [B, L]: number of the new token there
    at = s["positions"].long()[token] if case["tree"] else context[:, None] + torch.arange(N, device="cuda")
    seen = p[None, None, :] <= at[:, :, None]
    if W:
        seen = seen & ((p[None, None, :] > at[:, :, None] - W) | (p[None, None, :] < S))
    if case["tree"]:
        j = new.clamp(0, 32 * s["seen"].shape[1] - 1)[:, None, :].expand(-1, N, -1)
        bit = (s["seen"].long()[token].gather(2, j // 32) >> (j % 32) & 1).bool()
        seen = torch.where(new[:, None, :] >= 0, bit, seen)
    pos = torch.where(new < N, p[None, :], 0)
    page = s["table"].long().gather(1, pos // P)
    q = s["q"].float()[token].reshape(B, N, Hk, G, D)
    out = torch.zeros((T, Hk, G, D), device="cuda")
    lse = torch.zeros((T, Hk, G), device="cuda")
    mask = seen[:, :, None, :].expand(-1, -1, G, -1).reshape(B, N * G, -1)
    for h in range(Hk):                                                                           # all heads' scores at once would not fit
        k, v = _held(cache, "k", page, pos % P, h), _held(cache, "v", page, pos % P, h)           # [B, L, D]
        o, l = _softmax_over(torch.matmul(q[:, :, h].reshape(B, N * G, D), k.transpose(1, 2)).mul_(s["scale"]), mask, v)
        out[token[real], h], lse[token[real], h] = o.reshape(B, N, G, D)[real], l.reshape(B, N, G)[real]
    return {"out": out.reshape(T, H, D).to(torch.bfloat16), "lse": lse.reshape(T, H)}


def _plain_append(s):
    case, cache = s["case"], s["cache"]
    H, Hk, D, P, R = (case[k] for k in ("heads", "kv_heads", "D", "page", "R"))
    q, k, v = s["qkv"].reshape(-1, H + 2 * Hk, D).float().split((H, Hk, Hk), 1)
    # whole turns are taken off in 64 bits: a position times a frequency leaves few bits of the angle in 32
    turns = s["positions"].double()[:, None] * s["turns"][None, :]
    angle = ((turns - turns.floor()) * (2 * math.pi)).float()
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def rotated(x):
        rot, rest = x[..., :R], x[..., R:]
        a, b = (rot[..., 0::2], rot[..., 1::2]) if case["interleaved"] else (rot[..., : R // 2], rot[..., R // 2:])
        c, d = a * cos - b * sin, b * cos + a * sin
        rot = torch.stack((c, d), -1).flatten(-2) if case["interleaved"] else torch.cat((c, d), -1)
        return torch.cat((rot, rest), -1)

    q, k = rotated(q), rotated(k)
    place = s["places"].long()
    page, at = s["table"].long()[s["table_row"].long(), place // P], place % P
    for name, x in (("k", k), ("v", v)):
        if case["e4m3"]:
            x = (x / cache[name + "_scale"][None, :, None]).clamp(-BIG, BIG).to(E4M3)
            cache[name].view(torch.uint8)[page, at] = x.view(torch.uint8)
        else:
            cache[name][page, at] = x.to(torch.bfloat16)
    return {"q": q.to(torch.bfloat16), "k": cache["k"], "v": cache["v"]}


def _plain_move(s):
    case, cache, P = s["case"], s["cache"], s["case"]["page"]
    j = torch.arange(case["accepted"], device="cuda")
    row, j = torch.nonzero(j[None, :] < s["count"][:, None], as_tuple=True)
    src, dst = s["sources"].long()[row, j], s["context"].long()[row] + j
    table = s["table"].long()
    for name in ("k", "v"):
        c = cache[name].view(torch.uint8) if case["e4m3"] else cache[name]
        c[table[row, dst // P], dst % P] = c[table[row, src // P], src % P]
    return {"k": cache["k"], "v": cache["v"]}


def _plain_logprob(s):
    x, given, n = s["logits"].float(), s["given"], s["top"]
    V = x.shape[1]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    spread = torch.where(e > 0, e * (x - top), 0).sum(1, keepdim=True)
    lse = top + torch.log(total)
    out = {"lse": lse[:, 0], "entropy": (torch.log(total) - spread / total)[:, 0]}
    if given is not None:
        real = given >= 0
        id = torch.where(real, given, 0).long()
        xg = x.gather(1, id)
        out["logprob"] = torch.where(real, xg - top - torch.log(total), 0.0)
        ids = torch.arange(V, device="cuda")
        before = torch.stack([((x > a[:, None]) | ((x == a[:, None]) & (ids < i[:, None]))).sum(1) for a, i in zip(xg.unbind(1), id.unbind(1))], 1)
        out["rank"] = torch.where(real, before, -1).to(torch.int32)
    if n:
        # values in the order of whole numbers, then ids, so that no two are alike
        bits = (x + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -(bits + 2 ** 31), bits) * 2 ** 20 - torch.arange(V, device="cuda")
        id = key.topk(n, 1).indices
        out["top_id"], out["top_logprob"] = id.to(torch.int32), x.gather(1, id) - top - torch.log(total)
    return out


# ---------------------------------------------------------------- the framework's calls

def _kept_cache(L, s):
    """The cache's descriptor, which a program makes once."""
    if "kv" not in s:
        c = s["cache"]
        s["kv"] = L.KvCache(c["k"], c["v"], c.get("k_scale"), c.get("v_scale"))
    return s["kv"]


def _own_sink(L, s):
    if "workspace" not in s:
        s["workspace"] = L.alloc_attention_workspace(_kept_cache(L, s), *s["q"].shape[:2])
    out, lse = L.moe_sink_attention(_kept_cache(L, s), s["q"], s["table"], s["lengths"], s["case"]["window"], s["case"]["sinks"], scale=s["scale"],
                                    want_lse=True, workspace=s["workspace"])
    return {"out": out, "lse": lse}


def _own_chunk(L, s):
    case = s["case"]
    if "workspace" not in s:
        s["workspace"] = L.alloc_chunk_workspace(_kept_cache(L, s), case["seqs"], *s["q"].shape[:2])
    out, lse = L.moe_chunk_attention(_kept_cache(L, s), s["q"], s["table"], s["first"], s["context"], seen=s["seen"], positions=s.get("positions"),
                                     scale=s["scale"], window=case["window"], sinks=case["sinks"], want_lse=True, workspace=s["workspace"])
    return {"out": out, "lse": lse}


def _own_append(L, s):
    case = s["case"]
    H, Hk, D = case["heads"], case["kv_heads"], case["D"]
    if "rope" not in s:
        s["rope"] = L.Rope(s["turns"], case["R"], case["interleaved"])
    q, k, v = s["qkv"].view(-1, H + 2 * Hk, D).split((H, Hk, Hk), 1)
    q = L.moe_rope_append_at(_kept_cache(L, s), s["rope"], q, k, v, s["positions"], s["places"], s["table"], table_row=s["table_row"])
    return {"q": q, "k": s["cache"]["k"], "v": s["cache"]["v"]}


def _own_move(L, s):
    L.moe_cache_move(_kept_cache(L, s), s["table"], s["sources"], s["context"], s["count"])
    return {"k": s["cache"]["k"], "v": s["cache"]["v"]}


def _own_logprob(L, s):
    if "workspace" not in s:
        s["workspace"] = L.alloc_logprob_workspace(*s["logits"].shape, s["case"]["given"], s["top"])
    r = L.moe_token_logprobs(s["logits"], s["given"], s["top"], workspace=s["workspace"])
    return {k: v for k, v in r._asdict().items() if v is not None}


_PLAIN = {"sink": _plain_sink, "chunk": _plain_chunk, "append": _plain_append, "move": _plain_move, "logprob": _plain_logprob}
_OWN = {"sink": _own_sink, "chunk": _own_chunk, "append": _own_append, "move": _own_move, "logprob": _own_logprob}


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2507_17133_amd as framework
        return _OWN[op](framework, state)
    return _PLAIN[op](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "logprob":
        n, e = case["T"] * case["V"], 4 if case["fp32"] else 2
        return {"bytes": e * n + case["T"] * (8 + 12 * case["given"] + 8 * min(case["top"], case["V"])), "flops": 4 * n}
    Hk, D, e = case["kv_heads"], case["D"], 1 if case["e4m3"] else 2
    if case["op"] == "move":
        n = case["seqs"] * (case["accepted"] / 2) if case["seqs"] > 1 else case["accepted"]
        return {"bytes": n * (4 * e * Hk * D + 4) + 8 * case["seqs"], "flops": 0}
    H, longest = case["heads"], case["longest"]
    W, S = case.get("window", 0) or 1 << 40, case.get("sinks", 0)
    if case["op"] == "sink":
        lengths = range((longest + 1) // 2, longest + 1)
        mean = sum(min(n, W) + min(S, max(0, n - W)) for n in lengths) / len(lengths) * (1 - case["empty"])
        return {"bytes": case["T"] * (2 * e * Hk * D + 4.0 / case["page"]) * mean + case["T"] * H * (4 * D + 4), "flops": 4 * case["T"] * H * D * mean}
    each = _new_tokens(case)
    T = sum(each)
    if case["op"] == "append":
        return {"bytes": T * D * (4 * H + 4 * Hk + 2 * e * Hk) + 12 * T + 4 * case["R"], "flops": 3 * T * (H + Hk) * case["R"]}
    c = (longest // 2 + longest) // 2                                       # contexts lie between half the longest and the longest
    if case["tree"]:
        cached = min(c, W) + min(S, max(0, c - W))
        pairs, read = sum(n * (cached + min(n, 2 * n ** 0.5)) for n in each), sum(cached + n for n in each if n)
        masks = 4 * T * _words(case) + 4 * T
    else:
        pairs = sum(min(c + i + 1, W) + min(S, max(0, c + i + 1 - W)) for n in each for i in range(n))
        read = sum(min(c, W) + min(S, max(0, c - W)) + n for n in each if n)
        masks = 0
    return {"bytes": read * (2 * e * Hk * D + 4.0 / case["page"]) + T * H * (4 * D + 4) + masks, "flops": 4 * H * D * pairs}


# ---------------------------------------------------------------- in 64 bits, from the definitions

def _exact_rows(s, row, pos, h):
    """k and v of one head at a sequence's positions."""
    case, P = s["case"], s["case"]["page"]
    page = s["table"][row, pos // P].long()
    got = []
    for c in ("k", "v"):
        if case["e4m3"]:
            got.append(s["cache"][c].view(torch.uint8)[:, :, h][page, pos % P].view(E4M3).double() * s["cache"][c + "_scale"][h].double())
        else:
            got.append(s["cache"][c][:, :, h][page, pos % P].double())
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "logprob":
        parts = []
        for rows in torch.arange(case["T"], device="cuda").split(max(1, (1 << 27) // case["V"])):
            x = s["logits"][rows].double()
            logp = torch.log_softmax(x, 1)
            one = {"lse": torch.logsumexp(x, 1), "entropy": -(logp.exp() * logp.clamp_min(-1e300)).sum(1)}
            if s["given"] is not None:
                g = s["given"][rows].long()
                one["logprob"] = torch.where(g < 0, 0.0, logp.gather(1, g.clamp_min(0)))
                one["rank"] = None
            if s["top"]:
                one["top_id"], one["top_logprob"] = None, logp.sort(1, descending=True).values[:, : s["top"]]
            parts.append(one)
        return {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}
    Hk, D, P = (case[k] for k in ("kv_heads", "D", "page"))
    if case["op"] == "move":
        out = {}
        moves = [(b, int(a), t + j) for b, (n, t, src) in enumerate(zip(s["count"].tolist(), s["context"].tolist(), s["sources"].tolist()))
                 for j, a in enumerate(src[:n])]
        t, at = s["table"].tolist(), lambda i: torch.tensor(i, device="cuda", dtype=torch.int64)
        src, dst = (at([t[b][p // P] * P + p % P for b, *x in moves for p in (x[i],)]) for i in (0, 1))
        for n in ("k", "v"):
            flat = s["cache"][n].float().reshape(-1, Hk, D)      # 8-bit codes as they are, without their scale: so they are returned
            flat[dst] = flat[src].clone()
            out[n] = flat.view(s["cache"][n].shape).double()
        return out
    H = case["heads"]
    if case["op"] == "append":
        R, x = case["R"], s["qkv"].view(-1, H + 2 * Hk, D).double()
        turn = torch.remainder(s["positions"].double()[:, None] * s["turns"], 1.0) * 2 * math.pi
        i = torch.arange(R // 2, device="cuda")
        a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
        z = torch.complex(x[:, : H + Hk, a], x[:, : H + Hk, b]) * torch.polar(torch.ones_like(turn), turn)[:, None]
        x[:, : H + Hk, a], x[:, : H + Hk, b] = z.real, z.imag
        out, place = {"q": x[:, :H].clone()}, s["places"].long()
        slot = s["table"][s["table_row"].long(), place // P].long() * P + place % P
        for n, at in (("k", H), ("v", H + Hk)):
            y = x[:, at: at + Hk]
            if case["e4m3"]:
                y = y / s["cache"][n + "_scale"].double()[:, None]
            c = s["cache"][n]
            full = torch.zeros((c.shape[0] * P, Hk, D), dtype=torch.float64, device="cuda")
            full[slot] = y
            out[n] = full.view(c.shape)
        return out
    G, W, S = H // Hk, case["window"], case["sinks"]
    T = s["q"].shape[0]
    out = torch.zeros((T, H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device="cuda")

    def attend(t0, t1, row, pos, seen):
        """Tokens t0 .. t1 - 1 of a sequence over its positions pos where seen [tokens, positions]."""
        for h in range(Hk):
            k, v = _exact_rows(s, row, pos, h)
            a = (s["q"][t0:t1, h * G: (h + 1) * G].double().reshape(-1, D) @ k.t() * s["scale"]).view(t1 - t0, G, -1)
            a.masked_fill_(~seen[:, None, :], -math.inf)
            lse[t0:t1, h * G: (h + 1) * G] = torch.logsumexp(a, 2)
            p = torch.softmax(a, 2).masked_fill_(~seen.any(1)[:, None, None], 0.0)
            out[t0:t1, h * G: (h + 1) * G] = (p.view((t1 - t0) * G, -1) @ v).view(t1 - t0, G, D)

    if case["op"] == "sink":
        for t, n in enumerate(s["lengths"].tolist()):
            pos = torch.tensor(sorted(set(range(max(0, n - W), n)) | set(range(min(S, n)))), device="cuda", dtype=torch.int64)
            if n:
                attend(t, t + 1, t, pos, torch.ones((1, len(pos)), dtype=torch.bool, device="cuda"))
        return {"out": out, "lse": lse}
    first, context = s["first"].tolist(), s["context"].tolist()
    for b, c in enumerate(context):
        for t0 in range(first[b], first[b + 1], 1024):
            t1 = min(first[b + 1], t0 + 1024)
            if case["tree"]:
                at, pos = s["positions"][t0:t1].long()[:, None], torch.arange(c + first[b + 1] - first[b], device="cuda")
            else:
                at, pos = c + torch.arange(t0 - first[b], t1 - first[b], device="cuda")[:, None], torch.arange(c + t1 - first[b], device="cuda")
            seen = pos <= at
            if W:
                seen = seen & ((pos + W > at) | (pos < S))
            if case["tree"]:
                words = s["seen"][t0:t1].long() & 0xFFFFFFFF
                seen = torch.cat([seen[:, :c], torch.stack([words[:, j // 32] >> (j % 32) & 1 for j in range(first[b + 1] - first[b])], 1).bool()], 1)
            attend(t0, t1, b, pos, seen)
    return {"out": out, "lse": lse}
