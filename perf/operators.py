"""The operators around the MoE layer in a decoder layer, as they are timed and compared: the norm with its 8-bit output, the
8-bit linear layer, rotary positions with the append to the paged key-value cache, and attention of new tokens over that cache.

A case names an operator in `op`:

  norm       root-mean-square norm of T rows of d columns, with the residual's addition (`residual`), output in bf16 (`y`) or in e4m3 with
             a scale for each 128 columns (`y8`); without `norm` the 8-bit output of the rows as they are
  rope       q, k and v of T new tokens out of one fused projection: q and k rotated, k and v written to the pages of the cache
  attention  T new tokens, each attending to its own sequence in the paged cache
  linear     rows in e4m3 with a scale per 128 columns, times a weight in e4m3 with a scale per block of 128 x 128

`own` False: the plain form in elementary torch operations; True: the framework's kernels.
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
BIG = 448.0                  # largest e4m3 value
FLOOR = 2.0 ** -100          # smallest magnitude a group's scale is made for
EPS = 1e-6

#: A drawn case costs no more than these: bytes of the norm and of rope, cache elements of attention (padded and real), products of linear.
MOST_NORM = 16384 * 7168
MOST_ROPE = 16384 * 72 * 128
MOST_CACHE = 3 * 131072 * 8 * 128
MOST_LINEAR = 16384 * 7168 * 7168


def _norm(name, T, d, y8, residual=True, norm=True):
    return {"name": name, "op": "norm", "T": T, "d": d, "y8": y8, "residual": residual, "norm": norm}


def _rope(name, T, seqs, heads, kv_heads, D, R, interleaved, scaling, longest, e4m3, page, heads_first=False):
    return {"name": name, "op": "rope", "T": T, "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "D": D, "R": R,
            "interleaved": interleaved, "scaling": scaling, "longest": longest, "e4m3": e4m3, "page": page, "heads_first": heads_first}


def _attention(name, T, heads, kv_heads, D, longest, e4m3, page, window=0, heads_first=False, empty=0.0):
    return {"name": name, "op": "attention", "T": T, "heads": heads, "kv_heads": kv_heads, "D": D, "longest": longest, "e4m3": e4m3,
            "page": page, "window": window, "heads_first": heads_first, "empty": empty}


def _linear(name, M, N, K):
    return {"name": name, "op": "linear", "M": M, "N": N, "K": K}


def listed():
    return [
        # one request decoding alone, hidden size 2048: the launch is all there is
        _norm("norm_token_1", 1, 2048, False),
        # the attention's output of a decode batch of 256, made ready for the projection behind it
        _norm("quantize_decode_256", 256, 4096, True, residual=False, norm=False),
        # the largest prefill batch of the benchmark, hidden size 7168: residual in and out, 8-bit rows for the projection
        _norm("norm_prefill_16384", 16384, 7168, True),
        # one new token: 32 query heads over 8 key heads of 128
        _rope("rope_token_1", 1, 1, 32, 8, 128, 128, False, "none", 2048, False, 16),
        # an odd chunk of three prompts, half of each head rotated in pairs, positions far beyond the trained length, 8-bit cache
        _rope("rope_chunk_1021", 1021, 3, 16, 16, 128, 64, True, "yarn", 131072, True, 64, True),
        # prefill of 16384 tokens of four prompts, hidden size 7168 in 56 heads
        _rope("rope_prefill_16384", 16384, 4, 56, 8, 128, 128, False, "linear", 16384, False, 16),
        # one request alone, of the paper's longest sequence
        _attention("attention_token_1", 1, 32, 8, 128, 2048, False, 16),
        # the benchmark's decode batch of 256 requests of up to 2048 tokens, some slots of the batch unused
        _attention("attention_decode_256", 256, 32, 4, 128, 2048, False, 16, empty=0.05),
        # three long documents, cache in 8 bits: few rows, all of the work along the cache
        _attention("attention_long_3", 3, 64, 8, 128, 131072, True, 64, heads_first=True),
        # one token through the fused projection of q, k and v (4096 -> 32 + 2 * 8 heads of 128)
        _linear("linear_token_1", 1, 6144, 4096),
        # a small decode batch, expert width 1408 twice: neither side a whole number of tiles
        _linear("linear_decode_67", 67, 2816, 2048),
        # prefill of 16384 tokens at hidden size 7168
        _linear("linear_prefill_16384", 16384, 7168, 7168),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "rope", "attention", "linear"])
    if op == "norm":
        d = rng.choice([256, 2048, 4096, 5632, 7168, 8 * _log(rng, 8, 1024)])
        T = _log(rng, 1, min(16384, MOST_NORM // d))
        norm = rng.random() < 0.8
        case = _norm("", T, d, rng.random() < 0.5 or not norm, residual=norm and rng.random() < 0.7, norm=norm)
    elif op == "rope":
        D = rng.choice([64, 96, 128, 128, 192, 256])
        kv = rng.choice([1, 2, 4, 8, 16])
        heads = kv * rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8, 16) if g * kv <= 64])
        T = _log(rng, 1, min(16384, MOST_ROPE // ((heads + 2 * kv) * D)))
        case = _rope("", T, min(T, _log(rng, 1, 64)), heads, kv, D, rng.choice([D, D // 2, 16 * rng.randint(1, D // 16)]),
                     rng.random() < 0.4, rng.choice(["none", "linear", "ntk", "yarn"]), 0, rng.random() < 0.4,
                     rng.choice([1, 16, 16, 48, 64, 128]), rng.random() < 0.5)
        case["longest"] = _log(rng, -(-T // case["seqs"]) + 16, 262144)
    elif op == "attention":
        D = rng.choice([64, 96, 128, 128, 128, 192, 256])
        kv = rng.choice([1, 2, 4, 8, 8, 16])
        heads = kv * rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8, 16, 24) if g * kv <= 128])
        T = _log(rng, 1, 512)
        longest = _log(rng, 1, min(131072, MOST_CACHE // (T * kv * D)))
        case = _attention("", T, heads, kv, D, longest, rng.random() < 0.4, rng.choice([1, 16, 16, 48, 64, 128]),
                          rng.choice([0, 0, 0, 128, 1000]), rng.random() < 0.5, rng.choice([0.0, 0.0, 0.1]))
    else:
        N, K = _log(rng, 8, 16384), 16 * _log(rng, 8, 1024)
        if rng.random() < 0.5:
            N, K = rng.choice([1408, 2048, 2560, 4096, 6144, 14336]), rng.choice([768, 1408, 2048, 4096, 7168])
        case = _linear("", _log(rng, 1, min(16384, MOST_LINEAR // (N * K))), N, K)
    del case["name"]
    return case


# ---------------------------------------------------------------- inputs

def _normal(gen, shape, std=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=gen)


def _ints(gen, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=torch.int64)


def _cache(case, gen, n_pages, filled):
    """k and v of a paged cache, [page, token, head, D] whichever of the two orders they are stored in; e4m3 with a scale per head."""
    H, P, D = case["kv_heads"], case["page"], case["D"]
    shape = (n_pages, H, P, D) if case["heads_first"] else (n_pages, P, H, D)
    s = {}
    for n in ("k", "v"):
        t = _normal(gen, shape) if filled else torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        if case["e4m3"]:
            s[n + "_scale"] = torch.empty(H, device="cuda").uniform_(0.01, 0.02, generator=gen)
            t = (t * 64).to(E4M3)                # N(0, 64^2) in units of the scale: inside the type's range
        s[n] = t.transpose(1, 2) if case["heads_first"] else t
    return s


def _table(gen, pages_of):
    """A block table [sequences, most pages] that deals out the pages of a pool at random, and the pool's size."""
    most = max(1, int(max(pages_of)))
    n = len(pages_of) * most + 3
    table = torch.randperm(n, generator=gen, device="cuda")[: len(pages_of) * most]
    return table.reshape(len(pages_of), most).to(torch.int32), n


def _turns(case):
    """Turns per position of each rotated pair, and the factor on cos and sin (64 bits; made once by a program)."""
    R, base, factor, original = case["R"], 10000.0, 8.0, 4096.0
    i = torch.arange(R // 2, dtype=torch.float64)
    if case["scaling"] == "ntk" and R > 2:
        base = base * factor ** (R / (R - 2.0))
    f = base ** (-2.0 * i / R) / (2 * math.pi)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "yarn":
        at = lambda turns: R * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))  # pair that makes so many turns
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), R - 1)
        ramp = ((i - low) / max(high - low, 1e-3)).clamp(0, 1)
        f = f * (1 - ramp) + f / factor * ramp
        return f.cuda(), 0.1 * math.log(factor) + 1.0
    return f.cuda(), 1.0


def _rows8(x):
    """x [rows, d] in e4m3 and the scales [groups, rows] (the quantisation that a layer before has done)."""
    T, d = x.shape
    G = -(-d // 128)
    y = torch.nn.functional.pad(x.float(), (0, G * 128 - d)).reshape(T, G, 128)
    s = y.abs().amax(2).clamp_min(FLOOR) / BIG
    return (y / s[:, :, None]).to(E4M3).reshape(T, G * 128)[:, :d].contiguous(), s.t().contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000 + 29)
    s = {"case": case}
    if case["op"] == "norm":
        T, d = case["T"], case["d"]
        s["x"] = _normal(gen, (T, d))
        s["x"][:, :: max(1, d // 5)] *= 20       # some channels are much larger than the rest
        s["weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(torch.bfloat16) if case["norm"] else None
        s["residual"] = _normal(gen, (T, d), 3.0) if case["residual"] else None
    elif case["op"] == "rope":
        T, S, H, Hk, D = case["T"], case["seqs"], case["heads"], case["kv_heads"], case["D"]
        each = [T // S + (1 if i < T % S else 0) for i in range(S)]
        start = [int(v) for v in _ints(gen, 0, max(1, case["longest"] - max(each)), (S,)).tolist()]
        s["positions"] = torch.cat([torch.arange(a, a + n, device="cuda") for a, n in zip(start, each)]).to(torch.int32)
        s["table_row"] = torch.repeat_interleave(torch.arange(S, device="cuda"), torch.tensor(each, device="cuda")).to(torch.int32)
        # a table as long as the longest sequence; pages that hold none of these tokens are all page 0, which no token uses
        used = [(a // case["page"], (a + n - 1) // case["page"] + 1) for a, n in zip(start, each)]
        n_pages = sum(-(-n // case["page"]) + 1 for n in each) + 1
        pages = 1 + torch.randperm(n_pages - 1, generator=gen, device="cuda").to(torch.int32)
        s["table"] = torch.zeros((S, max(b for _, b in used)), dtype=torch.int32, device="cuda")
        at = 0
        for i, (a, b) in enumerate(used):
            s["table"][i, a:b] = pages[at: at + b - a]
            at += b - a
        s["qkv"] = _normal(gen, (T, (H + 2 * Hk) * D))
        s["turns"], s["factor"] = _turns(case)
        s["cache"] = _cache(case, gen, n_pages, False)
    elif case["op"] == "attention":
        T, most = case["T"], case["longest"]
        n = _ints(gen, (most + 1) // 2, most + 1, (T,))          # between half the longest and the longest
        n = torch.where(torch.rand(T, generator=gen, device="cuda") < case["empty"], 0, n)
        s["lengths"] = n.to(torch.int32)
        s["table"], n_pages = _table(gen, [-(-most // case["page"])] * T)
        s["q"] = _normal(gen, (T, case["heads"], case["D"]))
        s["scale"] = 1.0 / math.sqrt(case["D"])
        s["cache"] = _cache(case, gen, n_pages, True)
    else:
        M, N, K = case["M"], case["N"], case["K"]
        s["x8"], s["x_scale"] = _rows8(_normal(gen, (M, K)))
        w = torch.zeros((-(-N // 128) * 128, -(-K // 128) * 128), dtype=torch.bfloat16, device="cuda")
        w[:N, :K] = _normal(gen, (N, K), 1.0 / math.sqrt(K))
        b = w.reshape(w.shape[0] // 128, 128, w.shape[1] // 128, 128)
        s["w_scale"] = b.float().abs().amax((1, 3)).clamp_min(FLOOR) / BIG
        s["w8"] = (b / s["w_scale"][:, None, :, None]).to(E4M3).reshape(w.shape)[:N, :K].contiguous()
    return s


# ---------------------------------------------------------------- the plain forms, in 32 bits

def _plain_norm(s):
    case = s["case"]
    h = s["x"].float()
    out = {}
    if s["residual"] is not None:
        h = h + s["residual"].float()
        out["residual"] = h.to(torch.bfloat16)
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["weight"].float() if case["norm"] else h
    if not case["y8"]:
        out["y"] = y.to(torch.bfloat16)
        return out
    T, d = y.shape
    G = -(-d // 128)
    y = torch.nn.functional.pad(y, (0, G * 128 - d)).reshape(T, G, 128)
    scale = y.abs().amax(2).clamp_min(FLOOR) / BIG
    out["y8"] = (y / scale[:, :, None]).clamp(-BIG, BIG).to(E4M3).reshape(T, G * 128)[:, :d]
    out["scale"] = scale.t()
    return out


def _rotated(x, cos, sin, R, interleaved):
    """x [T, heads, D] in 32 bits with its first R columns rotated."""
    rot, rest = x[..., :R], x[..., R:]
    a, b = (rot[..., 0::2], rot[..., 1::2]) if interleaved else (rot[..., : R // 2], rot[..., R // 2:])
    c, d = a * cos[:, None] - b * sin[:, None], b * cos[:, None] + a * sin[:, None]
    rot = torch.stack((c, d), -1).flatten(-2) if interleaved else torch.cat((c, d), -1)
    return torch.cat((rot, rest), -1)


def _plain_rope(s):
    case, cache = s["case"], s["cache"]
    H, Hk, D, P = case["heads"], case["kv_heads"], case["D"], case["page"]
    q, k, v = s["qkv"].reshape(-1, H + 2 * Hk, D).float().split((H, Hk, Hk), 1)
    # whole turns are taken off in 64 bits: a position times a frequency leaves few bits of the angle in 32
    turns = s["positions"].double()[:, None] * s["turns"][None, :]
    angle = ((turns - turns.floor()) * (2 * math.pi)).float()
    cos, sin = angle.cos() * s["factor"], angle.sin() * s["factor"]
    q, k = (_rotated(x, cos, sin, case["R"], case["interleaved"]) for x in (q, k))
    pos = s["positions"].long()
    page, at = s["table"].long()[s["table_row"].long(), pos // P], pos % P
    for name, x in (("k", k), ("v", v)):
        if case["e4m3"]:
            x = (x / cache[name + "_scale"][None, :, None]).clamp(-BIG, BIG).to(E4M3)
            cache[name].view(torch.uint8)[page, at] = x.view(torch.uint8)
        else:
            cache[name][page, at] = x.to(torch.bfloat16)
    return {"q": q.to(torch.bfloat16), "k": cache["k"], "v": cache["v"]}


def _plain_attention(s):
    case, cache = s["case"], s["cache"]
    T, H, Hk, D = case["T"], case["heads"], case["kv_heads"], case["D"]
    n = s["lengths"].long()
    table = s["table"].long()
    k, v = (cache[c].view(torch.uint8)[table].view(E4M3) if case["e4m3"] else cache[c][table] for c in ("k", "v"))
    k, v = (x.reshape(T, -1, Hk, D).permute(0, 2, 1, 3).float() for x in (k, v))        # [T, Hk, L, D]
    if case["e4m3"]:
        k, v = k * cache["k_scale"][None, :, None, None], v * cache["v_scale"][None, :, None, None]
    score = torch.matmul(s["q"].float().reshape(T, Hk, H // Hk, D), k.transpose(2, 3)) * s["scale"]
    at = torch.arange(score.shape[3], device="cuda")
    seen = at[None, :] < n[:, None]
    if case["window"]:
        seen = seen & (at[None, :] >= n[:, None] - case["window"])
    score = score.masked_fill(~seen[:, None, None, :], -math.inf)
    top = score.amax(3, keepdim=True)
    p = torch.exp(score - top.clamp_min(-1e30))
    total = p.sum(3, keepdim=True)
    out = torch.matmul(p, v) / total.clamp_min(1e-30)
    lse = (top + torch.log(total)).reshape(T, H)
    return {"out": out.reshape(T, H, D).to(torch.bfloat16), "lse": lse}


def _plain_linear(s):
    K, N = s["x8"].shape[1], s["w8"].shape[0]
    a = s["x8"].float() * s["x_scale"].t().repeat_interleave(128, 1)[:, :K]
    w = s["w8"].float() * s["w_scale"].repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    return {"out": torch.matmul(a, w.t()).to(torch.bfloat16)}


# ---------------------------------------------------------------- the framework's calls

def _own_norm(L, s):
    case = s["case"]
    if not case["norm"]:
        y8, scale = L.moe_quantize_rows(s["x"])
        return {"y8": y8, "scale": scale}
    r = L.moe_rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], want=("y8",) if case["y8"] else ("y",))
    out = {"residual": r.residual} if case["residual"] else {}
    return dict(out, y8=r.y8, scale=r.scale) if case["y8"] else dict(out, y=r.y)


def _kept_cache(L, s):
    """The cache's descriptor, which a program makes once."""
    if "kv" not in s:
        c = s["cache"]
        s["kv"] = L.KvCache(c["k"], c["v"], c.get("k_scale"), c.get("v_scale"))
    return s["kv"]


def _own_rope(L, s):
    case = s["case"]
    H, Hk, D = case["heads"], case["kv_heads"], case["D"]
    if "rope" not in s:
        s["rope"] = L.Rope(s["turns"], case["R"], case["interleaved"], s["factor"])
    q, k, v = s["qkv"].view(-1, H + 2 * Hk, D).split((H, Hk, Hk), 1)
    q = L.moe_rope_append(_kept_cache(L, s), s["rope"], q, k, v, s["positions"], s["table"], table_row=s["table_row"])
    return {"q": q, "k": s["cache"]["k"], "v": s["cache"]["v"]}


def _own_attention(L, s):
    if "workspace" not in s:
        s["workspace"] = L.alloc_attention_workspace(_kept_cache(L, s), *s["q"].shape[:2])
    out, lse = L.moe_paged_attention(_kept_cache(L, s), s["q"], s["table"], s["lengths"], scale=s["scale"], window=s["case"]["window"],
                                     want_lse=True, workspace=s["workspace"])
    return {"out": out, "lse": lse}


def _own_linear(L, s):
    if "workspace" not in s:
        s["workspace"] = L.alloc_linear_workspace(s["x8"].shape[0], s["w8"].shape[0], s["x8"].shape[1])
    return {"out": L.moe_linear_e4m3(s["x8"], s["x_scale"], s["w8"], s["w_scale"], workspace=s["workspace"])}


_PLAIN = {"norm": _plain_norm, "rope": _plain_rope, "attention": _plain_attention, "linear": _plain_linear}
_OWN = {"norm": _own_norm, "rope": _own_rope, "attention": _own_attention, "linear": _own_linear}


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2507_17133_amd import layer
        return _OWN[op](layer, state)
    return _PLAIN[op](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "norm":
        n, G = case["T"] * case["d"], -(-case["d"] // 128)
        b = 2 * n + (4 * n if case["residual"] else 0) + (n + 4 * G * case["T"] if case["y8"] else 2 * n) + (2 * case["d"] if case["norm"] else 0)
        return {"bytes": b, "flops": 6 * n}
    T, H, Hk, D = (case.get(k, 0) for k in ("T", "heads", "kv_heads", "D"))
    e = 1 if case.get("e4m3") else 2
    if case["op"] == "rope":
        return {"bytes": T * D * (4 * H + 4 * Hk + 2 * e * Hk) + 8 * T + 4 * case["R"], "flops": 3 * T * (H + Hk) * case["R"]}
    if case["op"] == "attention":
        longest, w = case["longest"], case["window"]
        lengths = range((longest + 1) // 2, longest + 1)
        mean = sum(min(n, w) if w else n for n in lengths) / len(lengths) * (1 - case["empty"])
        return {"bytes": T * (2 * e * Hk * D + 4.0 / case["page"]) * mean + T * H * (4 * D + 4), "flops": 4 * T * H * D * mean}
    M, N, K = case["M"], case["N"], case["K"]
    G = -(-K // 128)
    return {"bytes": M * K + N * K + 2 * M * N + 4 * G * (M + -(-N // 128)), "flops": 2 * M * N * K}


# ---------------------------------------------------------------- in 64 bits, from the definitions

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        outs = []
        for rows in torch.arange(case["T"], device="cuda").split(2048):
            h = s["x"][rows].double()
            one = {}
            if case["residual"]:
                h = one["residual"] = h + s["residual"][rows].double()
            if case["norm"]:
                h = s["weight"].double() * (h / ((h * h).sum(1) / case["d"] + EPS).sqrt()[:, None])
            if case["y8"]:
                one["scale"] = torch.stack([g.abs().max(1).values.clamp_min(FLOOR) / BIG for g in h.split(128, 1)])
                one["y8"] = torch.cat([g / c[:, None] for g, c in zip(h.split(128, 1), one["scale"])], 1)
            else:
                one["y"] = h
            outs.append(one)
        return {k: torch.cat([o[k] for o in outs], 1 if k == "scale" else 0) for k in outs[0]}
    if case["op"] == "rope":
        H, Hk, D, R, P = (case[k] for k in ("heads", "kv_heads", "D", "R", "page"))
        x = s["qkv"].view(-1, H + 2 * Hk, D).double()
        phase = torch.polar(torch.full((1, R // 2), float(s["factor"]), dtype=torch.float64, device="cuda").expand(case["T"], -1).contiguous(),
                            torch.remainder(s["positions"].double()[:, None] * s["turns"], 1.0) * 2 * math.pi)
        i = torch.arange(R // 2, device="cuda")
        first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
        z = torch.complex(x[:, : H + Hk, first], x[:, : H + Hk, second]) * phase[:, None]
        x[:, : H + Hk, first], x[:, : H + Hk, second] = z.real, z.imag
        out = {"q": x[:, :H].clone()}
        row, pos = s["table_row"].long(), s["positions"].long()
        slot = s["table"][row, pos // P].long() * P + pos % P
        for n, at in (("k", H), ("v", H + Hk)):
            y = x[:, at: at + Hk]
            if case["e4m3"]:
                y = y / s["cache"][n + "_scale"].double()[:, None]
            c = s["cache"][n]
            full = torch.zeros((c.shape[0] * P, Hk, D), dtype=torch.float64, device="cuda")
            full[slot] = y
            out[n] = full.view(c.shape)
        return out
    if case["op"] == "attention":
        H, Hk, D, P = (case[k] for k in ("heads", "kv_heads", "D", "page"))
        out = torch.zeros((case["T"], H, D), dtype=torch.float64, device="cuda")
        lse = torch.full((case["T"], H), -math.inf, dtype=torch.float64, device="cuda")
        for t, n in enumerate(s["lengths"].tolist()):
            if n == 0:
                continue
            lo = max(0, n - case["window"]) if case["window"] else 0
            pos = torch.arange(lo, n, device="cuda")
            page = s["table"][t, pos // P].long()
            for h in range(Hk):
                k, v = (s["cache"][c][:, :, h][page, pos % P] if not case["e4m3"] else
                        s["cache"][c].view(torch.uint8)[:, :, h][page, pos % P].view(E4M3) for c in ("k", "v"))
                k, v = k.double(), v.double()
                if case["e4m3"]:
                    k, v = k * s["cache"]["k_scale"][h].double(), v * s["cache"]["v_scale"][h].double()
                g = slice(h * (H // Hk), (h + 1) * (H // Hk))
                a = s["q"][t, g].double() @ k.t() * s["scale"]
                lse[t, g] = torch.logsumexp(a, 1)
                out[t, g] = torch.softmax(a, 1) @ v
        return {"out": out, "lse": lse}
    M, N, K = case["M"], case["N"], case["K"]
    out = torch.zeros((M, N), dtype=torch.float64, device="cuda")
    w = s["w8"].double()
    for n in range(0, N, 128):
        for b in range(0, K, 128):
            w[n: n + 128, b: b + 128] *= s["w_scale"][n // 128, b // 128].double()
    for m in range(0, M, 2048):
        a = s["x8"][m: m + 2048].double()
        for b in range(0, K, 128):
            a[:, b: b + 128] *= s["x_scale"][b // 128, m: m + 2048].double()[:, None]
        out[m: m + 2048] = a @ w.t()
    return {"out": out}
