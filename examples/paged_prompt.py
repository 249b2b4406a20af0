"""Prompts in pieces through a paged cache with rotary positions, then decoding over the core neurons from a CUDA graph.

    python examples/paged_prompt.py [--config relu-llama2-7b|opt6.7b] [--layers 4] [--batch 2] [--prompt 1000] [--piece 512]
                                    [--window 0] [--sinks 4] [--tokens 64]

Runs a few layers of the configuration's shape (random weights) and says how long pieces and steps take.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2410_18311_b200.pipeline import CorePagedLayer, Pages, Rotary  # noqa: E402
from paper_2410_18311_b200.workloads import CONFIGS, layer_weights  # noqa: E402


def timed(call):
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    call()
    end.record()
    torch.cuda.synchronize()
    return start.elapsed_time(end) * 1e3


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--config", default="relu-llama2-7b", choices=[n for n, c in CONFIGS.items() if c.dtype == "bf16"])
    for name, value in (("layers", 4), ("batch", 2), ("prompt", 1000), ("piece", 512), ("window", 0), ("sinks", 4), ("tokens", 64)):
        p.add_argument("--" + name, type=int, default=value)
    args = p.parse_args()
    cfg = CONFIGS[args.config]
    D = 128 if cfg.d_model % 128 == 0 and cfg.d_model >= 1024 else 64
    heads, most = cfg.d_model // D, args.prompt + args.tokens + 8
    pages = Pages(args.batch, args.batch * -(-most // 64), 64, most)
    rotary = Rotary(D)
    layers = []
    for l in range(args.layers):
        g = torch.Generator(device="cuda").manual_seed(1000 * cfg.cid + 900 + l)
        new = lambda *s: (torch.randn(s, generator=g, device="cuda") * 0.02).to(cfg.torch_dtype)  # noqa: B023,E731
        layers.append(CorePagedLayer(cfg, pages, heads, heads, D, (new(3 * heads * D, cfg.d_model), new(cfg.d_model, heads * D)) + layer_weights(cfg, l, "cuda"),
                                     rotary, args.window, args.sinks if args.window else 0, args.batch * args.piece))
    g = torch.Generator("cuda").manual_seed(7)
    for at in range(0, args.prompt, args.piece):
        n = min(args.piece, args.prompt - at)
        h = torch.randn(pages.add([n] * args.batch), cfg.d_model, device="cuda", generator=g)
        us = timed(lambda: [layer.piece(h) for layer in layers])  # noqa: B023
        print("piece of %d x %d tokens at %d: %.0f us per layer" % (args.batch, n, at, us / args.layers))
    for layer in layers:
        layer.fix_core()

    x = torch.randn(args.batch, cfg.d_model, device="cuda", generator=g)
    pages.add([1] * args.batch)
    for layer in layers:                                         # the first token, outside the graph
        layer.step(x)
    pages.reserve(args.prompt + 1 + args.tokens)
    pages.decoding()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pages.one_more()
        for layer in layers:
            layer.step(x)
    us = timed(lambda: [graph.replay() for _ in range(args.tokens)]) / args.tokens
    pages.counted(args.tokens)
    for layer in layers:
        layer.cache.check()
    print("%s, %d layers, %d sequences: %.1f us per token step, %.1f us per layer; %s tokens held, output finite: %s"
          % (cfg.name, args.layers, args.batch, us, us / args.layers, pages.tokens, bool(torch.isfinite(x).all())))


if __name__ == "__main__":
    main()
