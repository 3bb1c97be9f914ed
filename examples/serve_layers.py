"""Decoder layers with sparse weights, served: prompts of several requests, then token steps replayed as one HIP graph.

Each layer is  x += o(attention(q, k, v)),  x += down(silu(gate) * up)  on RMS-normalised inputs, its seven linears held in
the packed format, its keys and values in 4 bits.  A step of the batch, whatever mix of prompts and single tokens, is

    plan = block_tables(...)                       pages and slots for the new tokens
    q, k, v = sparse_linear_group(...)             (per layer)
    q = qk_norm_rope_append(q, k, v, ...)          norms, rotation, keys and values into the layer's cache
    a = attention_fp4(q, cache, ...)
    o, gate, up, down                              sparse_linear, sparse_linear_silu_mul

    python examples/serve_layers.py --layers 4 --requests 16 --prompt 500 --steps 64

Weights and inputs are random: this shows the calls and their speed, not a model's text.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2405_03594_amd as spl  # noqa: E402


class Config:
    def __init__(self, hidden=4096, ffn=11008, heads=32, kv_heads=32, head_dim=128, layers=4, sparsity=0.7, page=64,
                 dtype=torch.bfloat16, eps=1e-5):
        self.hidden, self.ffn, self.heads, self.kv_heads, self.head_dim = hidden, ffn, heads, kv_heads, head_dim
        self.layers, self.sparsity, self.page, self.dtype, self.eps = layers, sparsity, page, dtype, eps


def _packed(n, k, cfg, gen):
    w = (torch.randn(n, k, generator=gen, device="cuda") * 0.02).to(cfg.dtype)
    return spl.pack_sparse(w, spl.magnitude_mask(w, int(cfg.sparsity * n * k)))


class Layer:
    def __init__(self, cfg, pages, gen):
        h, f, d = cfg.hidden, cfg.ffn, cfg.head_dim
        self.cfg = cfg
        self.q, self.k, self.v = (_packed(n * d, h, cfg, gen) for n in (cfg.heads, cfg.kv_heads, cfg.kv_heads))
        self.o, self.gate, self.up, self.down = (_packed(*s, cfg, gen) for s in ((h, cfg.heads * d), (f, h), (f, h), (h, f)))
        self.qw, self.kw = (torch.ones(d, dtype=cfg.dtype, device="cuda") for _ in range(2))
        self.cache = spl.KVCache.empty(pages, cfg.kv_heads, d, cfg.page, cfg.dtype)

    def __call__(self, x, plan, table, rope, max_new, max_len):
        cfg, T = self.cfg, x.shape[0]
        y = _rms(x, cfg.eps)
        q, k, v = (t.view(T, -1, cfg.head_dim) for t in spl.sparse_linear_group([y, y, y], [self.q, self.k, self.v]))
        q = spl.qk_norm_rope_append(q, k, v, plan.positions, rope, plan.slots, self.cache, self.qw, self.kw, eps=cfg.eps)
        a = spl.attention_fp4(q, self.cache, table, plan.lens, plan.row_start, max_new=max_new, max_len=max_len)
        x = x + spl.sparse_linear(a.view(T, -1), self.o)
        y = spl.sparse_linear_silu_mul(_rms(x, cfg.eps), self.gate, self.up)
        return x + spl.sparse_linear(y, self.down)


def _rms(x, eps):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + eps)).to(x.dtype)


class Server:
    """A batch of requests over layers that share the page table: one page number is a page of every layer's cache."""

    def __init__(self, cfg, requests, max_len, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.cfg, self.max_len = cfg, max_len
        width = -(-max_len // cfg.page)
        pages = requests * width
        self.layers = [Layer(cfg, pages, gen) for _ in range(cfg.layers)]
        angle = torch.arange(max_len, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(0, cfg.head_dim, 2, device="cuda", dtype=torch.float64) / cfg.head_dim)
        self.rope = torch.stack((angle.cos(), angle.sin()), -1).float().contiguous()
        i32 = dict(dtype=torch.int32, device="cuda")
        self.table = torch.full((requests, width), -1, **i32)
        self.free = torch.randperm(pages, generator=gen, device="cuda").int()
        self.head, self.lens = torch.zeros(1, **i32), torch.zeros(requests, **i32)

    def step(self, x, new, max_new):
        """The hidden states of the batch's new rows x, `new` (int32 [requests], on the GPU) of each request: through all
        layers.  Rows past the requests' are computed as tokens without keys."""
        plan = spl.block_tables(self.lens, new, self.table, self.free, self.head, self.cfg.page, x.shape[0])
        for layer in self.layers:
            x = layer(x, plan, self.table, self.rope, max_new, self.max_len)
        self.lens.copy_(plan.lens)
        self.head.copy_(plan.free_head)
        return x

    def capture(self):
        """One token of every request as a graph: (graph, its input, its output).  Capturing runs no step."""
        requests = self.lens.shape[0]
        x = torch.zeros(requests, self.cfg.hidden, dtype=self.cfg.dtype, device="cuda")
        new = torch.ones(requests, dtype=torch.int32, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = self.step(x, new, 1)
        return graph, x, y


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("requests", 16), ("prompt", 500), ("steps", 64), ("hidden", 4096), ("ffn", 11008),
                        ("heads", 32), ("kv-heads", 32), ("head-dim", 128)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    cfg = Config(hidden=a.hidden, ffn=a.ffn, heads=a.heads, kv_heads=a.kv_heads, head_dim=a.head_dim, layers=a.layers)
    server = Server(cfg, a.requests, a.prompt + a.steps + 1)
    gen = torch.Generator(device="cuda").manual_seed(1)
    # prompts of different lengths, all in one step
    lens = [max(1, int(a.prompt * (0.2 + 0.8 * (i * 0.618 % 1)))) for i in range(a.requests)]
    new = torch.tensor(lens, dtype=torch.int32, device="cuda")
    x = torch.randn(sum(lens), cfg.hidden, generator=gen, device="cuda").to(cfg.dtype)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    y = server.step(x, new, max(lens))
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    last = new.cumsum(0) - 1
    graph, x, out = server.capture()
    x.copy_(y[last])
    torch.cuda.synchronize()
    t2 = time.perf_counter()
    for _ in range(a.steps):
        graph.replay()
        x.copy_(out)                               # a model would sample a token and look up its embedding here
    torch.cuda.synchronize()
    t3 = time.perf_counter()
    if not torch.isfinite(out).all():
        raise RuntimeError("the outputs are not finite")
    per = server.layers[0].cache.data.numel() / (server.layers[0].cache.pages * cfg.page)
    print(f"prompts: {sum(lens)} tokens of {a.requests} requests through {a.layers} layers in {(t1 - t0) * 1e3:.1f} ms "
          "(first call: kernels are loaded)")
    print(f"token steps: {(t3 - t2) / a.steps * 1e6:.0f} us a step of {a.requests} tokens, "
          f"{a.requests * a.steps / (t3 - t2):.0f} tokens/s through {a.layers} layers")
    print(f"cache: {per:.0f} bytes a token and layer ({4 * cfg.kv_heads * cfg.head_dim} in 16 bits)")


if __name__ == "__main__":
    main()
