"""One layer of a transformer, one new token for each request of a batch, in 8 bits: the calls on tokens in the order in which a
serving loop makes them.

    python examples/transformer_step.py [--batch 64] [--context 4096] [--width 4096]

Weights are int8 with a scale per output channel, the cache is int8 with a scale per token and head, activations are quantised
token by token where a product needs them.  Random weights; positions are left out (rotate q and k before they are appended).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2202_05239_amd import binding as f8  # noqa: E402


class Layer:
    """Weights of one layer: norm, q k v projection, output projection, norm, gated MLP."""

    def __init__(self, width=1024, q_heads=16, kv_heads=4, dim=64, hidden=4096, seed=0, device="cuda", dtype=torch.bfloat16):
        g = torch.Generator(device=device).manual_seed(seed)
        self.q_heads, self.kv_heads, self.dim, self.hidden, self.dtype = q_heads, kv_heads, dim, hidden, dtype

        def weight(n, k):
            return f8.f8_quant_tokens(torch.randn(n, k, generator=g, device=device) * k ** -0.5)
        self.qkv = weight((q_heads + 2 * kv_heads) * dim, width)
        self.out = weight(width, q_heads * dim)
        self.gate_up = weight(2 * hidden, width)
        self.down = weight(width, hidden)
        self.norm1, self.norm2 = ((1 + 0.1 * torch.randn(width, generator=g, device=device)).to(dtype) for _ in range(2))

    def step(self, x, delta, cache, table, lens, slots, max_len):
        """x [batch][width]: the residual stream, delta: what the block before adds to it (or None).  lens count the new token,
        slots is where it goes.  Returns the stream and this layer's MLP output, the next layer's delta."""
        B, D, H = x.shape[0], self.dim, self.q_heads * self.dim
        if delta is None:
            x, codes, scale = f8.f8_norm_tokens(x, pre="rms", pre_w=self.norm1, codes=True)
        else:
            x, codes, scale = f8.f8_norm_tokens(delta, res=x, pre="rms", pre_w=self.norm1, codes=True)
        qkv = f8.f8_linear_scaled(codes, scale, *self.qkv, y_dtype=self.dtype)
        q, kv = qkv[:, :H].view(B, self.q_heads, D), qkv[:, H:].view(B, 2, self.kv_heads, D)
        f8.f8_kv_append(kv[:, 0], kv[:, 1], slots, cache["k"], cache["v"], cache["k_scale"], cache["v_scale"])
        a = f8.f8_attend_paged(q, cache["k"], cache["v"], table, lens, cache["k_scale"], cache["v_scale"], max_len=max_len)
        a = f8.f8_linear_tokens(a.view(B, H), *self.out)
        x, codes, scale = f8.f8_norm_tokens(a, res=x, pre="rms", pre_w=self.norm2, codes=True)
        gu = f8.f8_linear_scaled(codes, scale, *self.gate_up, y_dtype=self.dtype)
        codes, scale = f8.f8_quant_tokens(gu[:, self.hidden:], gate=gu[:, :self.hidden], act="silu")
        return x, f8.f8_linear_scaled(codes, scale, *self.down, y_dtype=self.dtype)


def make_cache(pages, page_size, kv_heads, dim, device="cuda"):
    """An 8-bit cache, heads outside the places of a page: a head's tokens then lie one behind the other."""
    def array(*tail, dtype):
        return torch.zeros(pages, kv_heads, page_size, *tail, dtype=dtype, device=device).transpose(1, 2)
    return dict(k=array(dim, dtype=torch.int8), v=array(dim, dtype=torch.int8), k_scale=array(dtype=torch.float32), v_scale=array(dtype=torch.float32))


def make_batch(lens, page_size, width, seed=0, device="cuda", dtype=torch.bfloat16):
    """(x, table, lens, slots of the newest tokens, number of pages) for requests of the given lengths, the new token included."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page_size) for n in lens]
    order = torch.randperm(sum(need), generator=g).int()
    table = torch.zeros(len(lens), max(need), dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    slots = torch.tensor([int(table[b, (n - 1) // page_size]) * page_size + (n - 1) % page_size for b, n in enumerate(lens)])
    x = torch.randn(len(lens), width, generator=g).to(dtype)
    return x.to(device), table.to(device), torch.tensor(lens, dtype=torch.int32, device=device), slots.to(device), sum(need)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--context", type=int, default=4096)
    ap.add_argument("--width", type=int, default=4096)
    a = ap.parse_args()
    layer = Layer(width=a.width, q_heads=a.width // 128, kv_heads=max(1, a.width // 512), dim=128, hidden=4 * a.width)
    lens = [max(1, a.context * (b + 1) // a.batch) for b in range(a.batch)]
    x, table, n, slots, pages = make_batch(lens, 64, a.width)
    cache = make_cache(pages, 64, layer.kv_heads, layer.dim)
    for b in range(0, pages * 64, 4096):               # a context of random tokens
        s = torch.arange(b, min(b + 4096, pages * 64), device="cuda")
        kv = torch.randn(2, len(s), layer.kv_heads, layer.dim, device="cuda")
        f8.f8_kv_append(kv[0], kv[1], s, cache["k"], cache["v"], cache["k_scale"], cache["v_scale"])
    step = lambda: layer.step(x, None, cache, table, n, slots, a.context)  # noqa: E731
    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(50):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    print("batch %d, context up to %d, width %d: %.1f us a layer and step, output norm %.3f"
          % (a.batch, a.context, a.width, begin.elapsed_time(end) * 20, out[1].float().norm().item() / out[1].numel() ** 0.5))


if __name__ == "__main__":
    main()
