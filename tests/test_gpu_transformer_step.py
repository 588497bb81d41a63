"""The calls on tokens together: one layer and step of a transformer in 8 bits (examples/transformer_step.py) against the same layer in
64 bits with the dequantised weights and cache.

Only the activations' 8 bits and the 16-bit tensors between the calls separate the two.  A quantiser's error is uniform in a step of
max / 127; the largest of some thousand normal values is below 5 standard deviations, so it is 5 / 127 / sqrt(12) = 1.1 % of the
row's norm.  Four quantisers lie one behind the other on the longest path (q k v input, attention output, MLP input, MLP middle; the
new token's cache row is a fifth of one token), in quadrature 2.3 %; the bound is twice that.
"""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import transformer_step as ts  # noqa: E402

from paper_2202_05239_amd import binding as f8  # noqa: E402

pytestmark = pytest.mark.gpu


def dense(w):
    return w[0].double() * w[1].double()[:, None]


def reference(layer, x, rows, lens, new_at):
    """rows: per request its cached keys and values [2][n][heads][dim] in 64 bits; the last is replaced by the new token's."""
    rms = lambda v, w: v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w.double()  # noqa: E731
    H, D, G = layer.q_heads * layer.dim, layer.dim, layer.q_heads // layer.kv_heads
    x = x.double()
    qkv = rms(x, layer.norm1) @ dense(layer.qkv).t()
    out = torch.empty(len(lens), layer.q_heads, D, dtype=torch.float64, device=x.device)
    for b, kv in enumerate(rows):
        kv = kv.clone()
        kv[:, -1] = qkv[b, H:].view(2, layer.kv_heads, D)
        for h in range(layer.q_heads):
            k, v = kv[:, :, h // G]
            out[b, h] = (k @ qkv[b, h * D:(h + 1) * D] * D ** -0.5).softmax(0) @ v
    x = x + out.view(len(lens), H) @ dense(layer.out).t()
    gu = rms(x, layer.norm2) @ dense(layer.gate_up).t()
    g, u = gu[:, :layer.hidden], gu[:, layer.hidden:]
    return x, (g * torch.sigmoid(g) * u) @ dense(layer.down).t()


@pytest.mark.parametrize("lens", [[1], [7, 130, 64, 65, 1, 600, 33, 2, 512], [40] * 48])
def test_layer(lens):
    layer = ts.Layer(width=512, q_heads=8, kv_heads=2, dim=64, hidden=1536)
    x, table, n, slots, pages = ts.make_batch(lens, 16, 512)
    cache = ts.make_cache(pages, 16, 2, 64)
    kv = torch.randn(2, pages * 16, 2, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    f8.f8_kv_append(kv[0], kv[1], torch.arange(pages * 16, device="cuda"), cache["k"], cache["v"], cache["k_scale"], cache["v_scale"])
    held = torch.stack([cache[c].double() * cache[c + "_scale"].double()[..., None] for c in "kv"])
    rows = [held[:, table[b, : -(-m // 16)].long()].flatten(1, 2)[:, :m] for b, m in enumerate(lens)]
    stream, delta = layer.step(x, None, cache, table, n, slots, max(lens))
    want_x, want_d = reference(layer, x, rows, lens, slots)
    for got, want in ((stream, want_x), (delta, want_d)):
        assert ((got.double() - want).norm() <= 0.046 * want.norm()).item(), (got.double() - want).norm() / want.norm()
    # the next layer's entry: the stream takes the MLP's output along
    x2, _ = layer.step(stream, delta, cache, table, n, slots, max(lens))
    assert torch.isfinite(x2).all()
    # and the whole step in a graph, replayed with the program's own work in between
    graph = torch.cuda.CUDAGraph()
    layer.step(x, None, cache, table, n, slots, max(lens))
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = layer.step(x, None, cache, table, n, slots, max(lens))
    for _ in range(3):
        out[1].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[1], delta) and torch.equal(out[0], stream)
