"""Decoding in four bits: projections, key/value cache with eviction, and the core-sparse FFN together.

    python examples/decode_4bit.py [--config opt6.7b|relu-llama2-7b] [--layers 4] [--batch 2] [--prompt 512]
                                   [--budget 256] [--tokens 64]

Runs a few layers of the configuration's shape (random weights) through a prompt and then token by token
from a CUDA graph, and compares the first decoded token with the same layers in 16 bits.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2410_18311_b200 as ci  # noqa: E402
from paper_2410_18311_b200.pipeline import Core4Layer  # noqa: E402
from paper_2410_18311_b200.workloads import CONFIGS, layer_weights  # noqa: E402


def build(cfg, args, q_heads, kv_heads, head_dim):
    """The layers, with seeded random weights."""
    layers = []
    for l in range(args.layers):
        g = torch.Generator(device="cuda").manual_seed(1000 * cfg.cid + 900 + l)
        new = lambda *s: (torch.randn(s, generator=g, device="cuda") * 0.02).to(cfg.torch_dtype)
        attn = (new((q_heads + 2 * kv_heads) * head_dim, cfg.d_model), new(cfg.d_model, q_heads * head_dim))
        layers.append(Core4Layer(cfg, args.batch, q_heads, kv_heads, head_dim, args.budget, attn + layer_weights(cfg, l, "cuda"),
                                 max_prompt=args.prompt))
    return layers


def plain_prompt_keys(layer, h):
    """Keys and values of the prompt's tokens at this layer (to be called before the layer's prompt())."""
    _, k, v = layer._split(torch.nn.functional.linear(layer._norm(h), layer.w_qkv), h.shape[1])
    return k.clone(), v.clone()


def plain_step(layer, h, k, v):
    """One token through the layer with its 16-bit weights, every key and value, and the core neurons."""
    F = torch.nn.functional
    q, k1, v1 = layer._split(F.linear(layer._norm(h), layer.w_qkv), 1)
    k, v = torch.cat((k, k1), 1), torch.cat((v, v1), 1)
    ctx = F.scaled_dot_product_attention(q.transpose(1, 2), k.transpose(1, 2), v.transpose(1, 2), enable_gqa=layer.heads[0] != layer.heads[1])
    h = h + F.linear(ctx.transpose(1, 2).reshape(layer.batch, -1), layer.w_o)
    w_up, w_gate, w_down = layer.w_ffn
    core = layer.core_idx.long()
    x = layer._norm(h)
    a = F.linear(x, w_up[core])
    a = F.relu(a) if w_gate is None else a * F.relu(F.linear(x, w_gate[core]))
    return h + F.linear(a, w_down[:, core])


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--config", default="opt6.7b", choices=[n for n, c in CONFIGS.items() if c.dtype == "bf16"])
    for name, value in (("layers", 4), ("batch", 2), ("prompt", 512), ("budget", 256), ("tokens", 64)):
        p.add_argument("--" + name, type=int, default=value)
    args = p.parse_args()
    cfg = CONFIGS[args.config]
    head_dim = 128 if cfg.d_model % 128 == 0 and cfg.d_model >= 1024 else 64
    heads = cfg.d_model // head_dim
    layers = build(cfg, args, heads, heads, head_dim)

    h = torch.randn(args.batch, args.prompt, cfg.d_model, device="cuda", generator=torch.Generator("cuda").manual_seed(7))
    first = torch.randn(args.batch, cfg.d_model, device="cuda", generator=torch.Generator("cuda").manual_seed(8))
    want = first.clone()
    for layer in layers:
        k, v = plain_prompt_keys(layer, h)
        layer.prompt(h)
        want = plain_step(layer, want, k, v)

    x = first.clone()

    def step():
        for layer in layers:
            layer.step(x)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                            # the first token, outside the graph
        step()
    torch.cuda.current_stream().wait_stream(side)
    moved = (want - first).norm()
    print("first token against 16 bits and the whole cache: difference %.3f of what the layers added" % ((x - want).norm() / moved).item())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(args.tokens):
        x.copy_(first)
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    for layer in layers:
        layer.cache.check()
    us = start.elapsed_time(end) * 1e3 / args.tokens
    print("%s, %d layers, %d sequences: %.1f us per token step, %.1f us per layer; slots per head %s of %d tokens"
          % (cfg.name, args.layers, args.batch, us, us / args.layers, layers[0].cache.lengths(), layers[0].cache.state[0, 1].item()))


if __name__ == "__main__":
    main()
