"""A layer that decodes in four bits, end to end, against the same steps in 64 bits over the stored values."""
import numpy as np
import pytest
import torch

import paper_2410_18311_b200 as ci
from helpers import require_gpu
from paper_2410_18311_b200.pipeline import Core4Layer
from paper_2410_18311_b200.workloads import CONFIGS, layer_weights
from quant4_ref import unpack_cache, values_np, w4_layout

pytestmark = pytest.mark.gpu


def stored(w, group):
    """The 64-bit values that a weight matrix [N, K] is held as."""
    return w4_layout(values_np(w), group)[2]


def norm(h):
    h = h - h.mean(-1, keepdims=True)
    return h / np.sqrt((h * h).mean(-1, keepdims=True) + 1e-5)


class Plain:
    """The decode step of the layer in 64 bits; keys and values as they would be stored, evicted by plain sorting."""

    def __init__(self, layer, group):
        self.layer, cfg = layer, layer.cfg
        core = layer.core_idx.cpu().numpy()
        up, gate, down = layer.w_ffn
        self.qkv, self.o = stored(layer.w_qkv, group), stored(layer.w_o, group)
        self.up, self.down = stored(up[core], group), stored(down[:, core], group)
        self.gate = stored(gate[core], group) if cfg.gated else None

    def step(self, h, keys, values):
        """keys, values [B, slots, H, D] in the cache after this token was appended."""
        l, bf = self.layer, lambda x: values_np(torch.from_numpy(x).to(l.cfg.torch_dtype)).astype(np.float64)
        Hq, H, D = l.heads
        x = bf(norm(h))
        q = bf(x @ self.qkv.T)[:, :Hq * D].reshape(-1, H, Hq // H, D)
        logits = np.einsum("bhgd,bnhd->bhgn", q, keys) * D ** -0.5
        p = np.exp(logits - logits.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        ctx = bf(np.einsum("bhgn,bnhd->bhgd", p, values).reshape(len(h), -1))
        h = h + ctx @ self.o.T
        x = bf(norm(h))
        a = x @ self.up.T
        a = np.maximum(a, 0) if self.gate is None else a * bf(np.maximum(x @ self.gate.T, 0))
        return h + bf(a) @ self.down.T, p.sum(2)


@pytest.mark.parametrize("gated,heads,group", [(False, (4, 4, 64), 128), (True, (4, 2, 64), 64)])
def test_layer(gated, heads, group):
    """Prompt longer than the budget, then tokens; each step is compared from the layer's own state before it.

    Bound: every 16-bit rounding of an intermediate (x, qkv, ctx, a: 2^-9 of it, random) enters through a
    norm-preserving product, and the layer's own rounding may fall on the other side: 4 roundings of each of two sums, so
    the added part differs by at most about 8 * 2^-9 of itself in norm; twice that is asked for."""
    require_gpu()
    cfg = CONFIGS["tiny"].with_(gated=gated, T=40)
    Hq, H, D = heads
    B, T, budget = 3, 40, 24
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s: (torch.randn(s, generator=g, device="cuda") * 0.06).to(cfg.torch_dtype)
    layer = Core4Layer(cfg, B, Hq, H, D, budget, (new((Hq + 2 * H) * D, cfg.d_model), new(cfg.d_model, Hq * D)) + layer_weights(cfg, 0, "cuda"),
                       recent=6, first=2, group=group, cache_group=32)
    h = torch.randn(B, T, cfg.d_model, generator=g, device="cuda")
    layer.prompt(h)
    assert torch.isfinite(h).all() and layer.cache.lengths() == [budget] * B
    position = layer.cache.position[:, :, :budget].cpu().numpy()
    for b in range(B):
        for j in range(H):
            kept = set(position[b, j].tolist())
            assert len(kept) == budget and {0, 1} <= kept and set(range(T - 6, T)) <= kept
    plain = Plain(layer, group)
    for _ in range(5):
        x = torch.randn(B, cfg.d_model, generator=g, device="cuda")
        before = x.cpu().numpy().astype(np.float64)
        weight0 = layer.cache.weight[:, :, :budget].cpu().numpy().astype(np.float64)
        # the step by its parts up to the append, to look at the cache as attention sees it
        c = layer.cache
        buffers = (c.k_codes, c.k_pairs, c.v_codes, c.v_pairs, c.weight, c.position, c.state)
        spare = [t.clone() for t in buffers]
        layer.qkv(layer._norm(x), layer._qkv)
        _, k, v = layer._split(layer._qkv, 1)
        c.append(k, v)
        keys, values = (unpack_cache(codes[:, :, :budget + 1], pairs[:, :, :budget + 1]).transpose(0, 2, 1, 3)
                        for codes, pairs in ((c.k_codes, c.k_pairs), (c.v_codes, c.v_pairs)))
        pos = c.position[:, :, :budget + 1].cpu().numpy()
        for t, was in zip(buffers, spare):
            t.copy_(was)
        layer.step(x)
        want, p = plain.step(before, keys, values)
        added = np.linalg.norm(want - before)
        assert np.linalg.norm(x.cpu().numpy() - want) <= 16 * 2.0 ** -9 * added
        assert layer.cache.lengths() == [budget] * B
        # one slot went: of those that neither the first nor the recent tokens protect, the one with the smallest weight
        total = np.concatenate((weight0, np.zeros((B, H, 1))), 2) + p
        seen = layer.cache.state[0, 1].item()
        now = layer.cache.position[:, :, :budget].cpu().numpy()
        for b in range(B):
            for j in range(H):
                gone = set(pos[b, j].tolist()) - set(now[b, j].tolist())
                assert len(gone) == 1
                n = pos[b, j].tolist().index(gone.pop())
                free = [i for i in range(budget + 1) if 2 <= pos[b, j, i] < seen - 6]
                assert n in free and total[b, j, n] <= total[b, j, free].min() * (1 + 2.0 ** -5)
    layer.cache.check()


def small_layer(max_prompt=40, budget=24, batch=2):
    cfg = CONFIGS["tiny"].with_(gated=True)
    g = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s: (torch.randn(s, generator=g, device="cuda") * 0.06).to(cfg.torch_dtype)  # noqa: E731
    return Core4Layer(cfg, batch, 4, 2, 64, budget, (new(8 * 64, cfg.d_model), new(cfg.d_model, 4 * 64)) + layer_weights(cfg, 0, "cuda"),
                      recent=6, first=2, max_prompt=max_prompt, cache_group=32), cfg


def test_prompt_longer_than_the_cache_is_refused():
    """Nothing is computed and nothing of the cache changes, instead of attention over a cache that refused the tokens."""
    require_gpu()
    layer, cfg = small_layer(max_prompt=40)
    layer.prompt(torch.randn(2, 40, cfg.d_model, device="cuda"))
    state, core = layer.cache.state.clone(), layer.core_idx.clone()
    h = torch.randn(2, 49, cfg.d_model, device="cuda")
    before = h.clone()
    with pytest.raises(ci.CoreInferError):
        layer.prompt(h)
    assert torch.equal(h, before) and torch.equal(layer.cache.state, state) and torch.equal(layer.core_idx, core)
    layer.step(torch.randn(2, cfg.d_model, device="cuda"))
    layer.cache.check()


def test_captured_step_serves_later_prompts():
    """A step captured after one prompt gives, after the next ones, the bits of a step called directly: outputs and cache."""
    require_gpu()
    layer, cfg = small_layer()
    g = torch.Generator(device="cuda").manual_seed(77)
    new = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = new(2, cfg.d_model)
    layer.prompt(new(2, 40, cfg.d_model))
    first_core = layer.core_idx.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x)
    c = layer.cache
    buffers = (c.k_codes, c.k_pairs, c.v_codes, c.v_pairs, c.weight, c.position, c.state)
    for T in (40, 31):
        layer.prompt(new(2, T, cfg.d_model))
        assert not torch.equal(layer.core_idx, first_core)
        start, tokens = [t.clone() for t in buffers], [new(2, cfg.d_model) for _ in range(4)]
        outs = []
        for token in tokens:
            x.copy_(token)
            graph.replay()
            outs.append(x.clone())
        end = [t.clone() for t in buffers]
        for t, was in zip(buffers, start):
            t.copy_(was)
        for token, out in zip(tokens, outs):
            layer.step(token)
            assert torch.equal(token, out)
        used = c.lengths()[0]
        for t, was in zip(buffers, end):
            assert torch.equal(t, was) if t is c.state else torch.equal(t[:, :, :used], was[:, :, :used])
    c.check()
