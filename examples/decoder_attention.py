"""The attention half of a decoder layer on 4-bit weights, 8-bit activations and a 4-bit cache, from prompt to single tokens.

    residual sum + RMS norm + int8  ->  W4A8 projection to q, k, v  ->  k, v into the 4-bit cache
    ->  attention over the cache  ->  W4A8 output projection

Two sequences of unequal lengths share a paged cache; after the prompts every step is one token for each, captured into a graph
once and replayed (lengths are device memory: nothing waits for the host).  A rotary embedding would go between the projection and
the cache.  Run it from the repository's root on a GPU:  python examples/decoder_attention.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2311_05161_amd as w  # noqa: E402


class Attention:
    """Weights quantized once; `step` runs any number of new tokens per sequence over the cache."""

    def __init__(self, width, heads, kv_heads, head_dim, group_size=128, dtype=torch.float16, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.heads, self.kv_heads, self.head_dim, self.group, self.dtype = heads, kv_heads, head_dim, group_size, dtype

        def weights(n, k):
            m = torch.randn((n, k), generator=g, device=device).to(dtype) * k ** -0.5
            s = 0.5 + torch.rand((k,), generator=g, device=device)            # the per-channel scale, from calibration in earnest
            codes, step, zero = w.quantize_weight_dint4(m, s, group_size)
            return w.pack_dint4(codes), step, zero, s

        self.norm = (1.0 + 0.1 * torch.randn((width,), generator=g, device=device)).to(dtype)
        self.qkv = weights((heads + 2 * kv_heads) * head_dim, width)
        self.out = weights(width, heads * head_dim)

    def project(self, x, residual):
        """x, residual [B, S, width] -> q, k, v [B, S, heads, head_dim] and the sum that the next residual is."""
        B, S, width = x.shape
        packed, step, zero, s = self.qkv
        q8, scale, h = w.rms_norm_act_int8(x.reshape(-1, width), self.norm, residual=residual.reshape(-1, width), s=s)
        n = (self.heads + 2 * self.kv_heads) * self.head_dim
        y = w.w4a8_gemm(q8, scale, packed, step, zero, n, width, self.group, out_dtype=self.dtype)
        y = y.view(B, S, -1, self.head_dim)
        return (*y.split([self.heads, self.kv_heads, self.kv_heads], dim=2), h.view(B, S, width))

    def step(self, x, residual, cache, start, count, table, max_len):
        q, k, v, h = self.project(x, residual)
        w.kv_cache_write_dint4(k, v, cache, start, count, table)
        o = w.attention_kv_dint4(q, cache, start, count, table, max_len=max_len)
        packed, step, zero, s = self.out
        y = w.w4a8_linear(o.flatten(0, 1).flatten(1), s, packed, step, zero, x.shape[-1], self.group, out_dtype=self.dtype)
        return y.view_as(x), h


def main(width=1024, heads=8, kv_heads=2, head_dim=128, prompts=(300, 77), new_tokens=20, page=64):
    layer = Attention(width, heads, kv_heads, head_dim)
    B, S, most = len(prompts), max(prompts), max(prompts) + new_tokens
    each = (most + page - 1) // page
    cache = w.KVCacheDint4.empty(B * each, kv_heads, page, head_dim)
    table = torch.randperm(B * each, device="cuda").reshape(B, each).to(torch.int32)
    start, count = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.tensor(prompts, dtype=torch.int32, device="cuda")

    x, r = (torch.randn((B, S, width), device="cuda").to(layer.dtype) for _ in range(2))
    y, h = layer.step(x, r, cache, start, count, table, max_len=S)
    print("prompt", tuple(y.shape), "rms", float(y[0].float().square().mean().sqrt()))

    start.copy_(count)                                   # one token each from here on
    x, r = y[:, -1:].clone(), h[:, -1:].clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(x, r, cache, start, None, table, max_len=most)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        y, h = layer.step(x, r, cache, start, None, table, max_len=most)
    for _ in range(new_tokens):
        graph.replay()
        x.copy_(y), r.copy_(h), start.add_(1)
    torch.cuda.synchronize()
    print("after", new_tokens, "tokens", tuple(y.shape), "rms", float(y.float().square().mean().sqrt()), "lengths", start.tolist())
    return y


if __name__ == "__main__":
    main()
