"""One decoder layer served from a paged key-value cache: the operators around the MoE layer and the layer itself, as a serving
program calls them.

  norm + residual -> q, k, v in 8 bits -> rotary positions, append -> attention over the pages -> 8 bits -> output projection
  -> norm + residual -> BrownoutMoE layer

A batch of sequences gets its prompts in chunks (all tokens of a chunk in one call each) and is then decoded token by token; the
decode step is captured in a HIP graph and replayed with new positions.  Weights are random, of the shape of a configuration in
`workloads` (its heads are 128 columns wide, eight query heads to a key head where the width allows).

  python examples/decoder_layer.py [--config qwen3_30b_a3b] [--batch 32] [--prompt 500] [--steps 50] [--kv8] [--threshold 0.6]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_17133_amd as P
from paper_2507_17133_amd import workloads as WL


class DecoderLayer:
    """Weights of one layer, its cache and its workspaces.  A batch's tokens come with their position and the sequence they belong to."""

    def __init__(self, cfg: WL.LayerConfig, n_pages: int, page_size: int = 16, kv8: bool = False, seed: int = 0, max_tokens: int = 4096):
        d, dev = cfg.d, "cuda"
        g = torch.Generator(device=dev).manual_seed(seed)
        normal = lambda *shape: (torch.randn(shape, generator=g, device=dev) / shape[-1] ** 0.5).to(torch.bfloat16)
        self.D = 128 if d % 128 == 0 and d >= 512 else 64
        self.H = d // self.D
        self.Hk = max(1, self.H // 8)
        self.qkv_weight, self.o_weight = normal((self.H + 2 * self.Hk) * self.D, d), normal(d, self.H * self.D)
        self.wqkv, self.wo = P.moe_quantize_weight(self.qkv_weight), P.moe_quantize_weight(self.o_weight)     # once per weight
        self.norm1, self.norm2 = (torch.ones(d, dtype=torch.bfloat16, device=dev) for _ in range(2))
        # keys and values of unit size: 448 steps reach to 448 / 64 = 7 of their standard deviations
        scale = torch.full((self.Hk,), 1 / 64, device=dev) if kv8 else None
        self.cache = P.alloc_kv_cache(n_pages, page_size, self.Hk, self.D, scale, scale)
        self.rope = P.make_rope(self.D)
        layer = WL.make_layer(cfg.with_(T=1), seed, dev)
        self.moe_cfg = P.config_of(cfg)
        self.gate, self.gate_b = P.pack_gate(self.moe_cfg, layer.gate_w), layer.gate_b
        self.moe_cfg = P.with_packed_gate(self.moe_cfg)
        self.experts, self.shared = layer.experts, layer.shared
        self.united, _ = P.moe_build_united(self.moe_cfg, self.experts)
        self.moe_ws = P.alloc_workspace(self.moe_cfg, max_tokens)
        self.attn_ws = P.alloc_attention_workspace(self.cache, max_tokens, self.H)

    def __call__(self, x, residual, positions, lengths, block_table, row=None, threshold: float = 1.0):
        """x [T, d] and the residual stream before the layer -> the layer's output and the residual stream behind it."""
        T, D, H, Hk = x.shape[0], self.D, self.H, self.Hk
        n = P.moe_rms_norm(x, self.norm1, residual=residual, want=("y8",))
        qkv = P.moe_linear_e4m3(n.y8, n.scale, *self.wqkv)
        q, k, v = qkv.view(T, H + 2 * Hk, D).split((H, Hk, Hk), 1)
        q = P.moe_rope_append(self.cache, self.rope, q, k, v, positions, block_table, table_row=row)
        o = P.moe_paged_attention(self.cache, q, block_table, lengths, table_row=row, workspace=self.attn_ws)
        a = P.moe_linear_e4m3(*P.moe_quantize_rows(o.view(T, H * D)), *self.wo)
        n = P.moe_rms_norm(a, self.norm2, residual=n.residual)
        y = P.moe_forward(self.moe_cfg, n.y, self.gate, self.gate_b, self.experts, self.united, self.shared, threshold, workspace=self.moe_ws)
        return y, n.residual


def serve(cfg, batch: int, prompt: int, steps: int, kv8: bool = False, threshold: float = 1.0, chunk: int = 1024, page_size: int = 16, seed: int = 0):
    """Prompts of `prompt` tokens in chunks, then `steps` tokens each.  Returns the layer, all inputs and outputs [batch, tokens, d]
    and the seconds that the prompts and the steps took."""
    per_seq = -(-(prompt + steps) // page_size)
    layer = DecoderLayer(cfg, batch * per_seq, page_size, kv8, seed, max(chunk, batch))
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    table = torch.randperm(batch * per_seq, generator=g, device="cuda").to(torch.int32).view(batch, per_seq)
    x = torch.randn((batch, prompt + steps, cfg.d), generator=g, device="cuda").to(torch.bfloat16)
    out, res = torch.empty_like(x), torch.empty_like(x)
    zero = torch.zeros((max(chunk, batch), cfg.d), dtype=torch.bfloat16, device="cuda")

    # prompts: the tokens of all sequences one after the other, cut into chunks
    rows = torch.arange(batch, device="cuda").repeat_interleave(prompt).to(torch.int32)
    pos = torch.arange(prompt, device="cuda").repeat(batch).to(torch.int32)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for t0 in range(0, batch * prompt, chunk):
        r, p = rows[t0:t0 + chunk], pos[t0:t0 + chunk]
        xt = x[r.long(), p.long()]
        out[r.long(), p.long()], res[r.long(), p.long()] = layer(xt, zero[:len(r)], p, p + 1, table, r, threshold)
    torch.cuda.synchronize()
    prompt_s = time.perf_counter() - began

    # decoding: one token per sequence and step, the step captured once
    if steps == 0:
        return layer, table, x, out, res, prompt_s, 0.0
    xt = x[:, prompt].clone()
    p = torch.full((batch,), prompt, dtype=torch.int32, device="cuda")
    n = p + 1
    step = lambda: layer(xt, zero[:batch], p, n, table, threshold=threshold)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                     # workspaces and set-up before the capture; writes what the first replay writes again
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, r = step()
    torch.cuda.synchronize()
    began = time.perf_counter()
    for s in range(steps):
        xt.copy_(x[:, prompt + s])
        p.fill_(prompt + s)
        n.fill_(prompt + s + 1)
        graph.replay()
        out[:, prompt + s], res[:, prompt + s] = y, r
    torch.cuda.synchronize()
    return layer, table, x, out, res, prompt_s, time.perf_counter() - began


def main():
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--config", default="qwen3_30b_a3b", choices=sorted(WL.CONFIGS))
    a.add_argument("--batch", type=int, default=32)
    a.add_argument("--prompt", type=int, default=500)
    a.add_argument("--steps", type=int, default=50)
    a.add_argument("--kv8", action="store_true", help="key-value cache in e4m3")
    a.add_argument("--threshold", type=float, default=1.0, help="share of token-expert assignments that stay on original experts")
    o = a.parse_args()
    layer, _, _, out, _, prompt_s, steps_s = serve(WL.CONFIGS[o.config], o.batch, o.prompt, o.steps, o.kv8, o.threshold)
    assert bool(out.isfinite().all())
    print(f"{o.config}: {layer.H} query over {layer.Hk} key heads of {layer.D}; {o.batch} prompts of {o.prompt} tokens {prompt_s * 1e3:.1f} ms, "
          f"{o.steps} steps {steps_s / max(o.steps, 1) * 1e6:.0f} us each ({o.batch * o.steps / max(steps_s, 1e-9):.0f} tokens/s through one layer)")


if __name__ == "__main__":
    main()
