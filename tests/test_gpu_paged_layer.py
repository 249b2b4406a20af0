"""Rotary positions, paged caches and attention over them as the pipeline uses them: a layer whose prompts come in pieces, captured steps,
streams, and the four-bit layer with rotary positions."""
import numpy as np
import pytest
import torch

import paper_2410_18311_b200 as ci
from helpers import require_gpu
from paged_ref import check, frequencies, turn
from paper_2410_18311_b200.pipeline import Core4Layer, CorePagedLayer, PagedKVCache, Pages, Rotary
from paper_2410_18311_b200.workloads import CONFIGS, layer_weights

pytestmark = pytest.mark.gpu


def build(gated, heads, window, sinks, n_pages=40, batch=2, seed=3):
    cfg = CONFIGS["tiny"].with_(gated=gated)
    Hq, H, D = heads
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: (torch.randn(s, generator=g, device="cuda") * 0.06).to(cfg.torch_dtype)  # noqa: E731
    pages = Pages(batch, n_pages, 16, 200)
    norm = (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(cfg.torch_dtype)
    rotary = Rotary(D, interleaved=gated, q_norm=norm, k_norm=norm)
    layer = CorePagedLayer(cfg, pages, Hq, H, D, (new((Hq + 2 * H) * D, cfg.d_model), new(cfg.d_model, Hq * D)) + layer_weights(cfg, 0, "cuda"),
                           rotary, window, sinks)
    return cfg, pages, layer, norm, g


class Plain:
    """The layer in 64 bits, a sequence at a time, with the 16-bit roundings of its intermediates."""

    def __init__(self, layer, norm, interleaved):
        self.l, self.norm, self.interleaved = layer, norm, interleaved
        self.f, _ = frequencies(layer.heads[2], 10000.0)
        self.keys, self.values = {}, {}

    def rounded(self, x):
        return x.to(self.l.cfg.torch_dtype).double()

    def pre(self, h):
        h = h - h.mean(-1, keepdim=True)
        return self.rounded(h / (h.square().mean(-1, keepdim=True) + 1e-5).sqrt())

    def tokens(self, b, h, core=None):
        l, (Hq, H, D), (window, sinks) = self.l, self.l.heads, self.l.span
        w = lambda t: t.double().cpu()  # noqa: E731
        k0 = self.keys.get(b, torch.zeros(0, H, D, dtype=torch.float64))
        at = torch.arange(len(k0), len(k0) + len(h))
        qkv = self.rounded(self.pre(h) @ w(l.w_qkv).T)
        q, k, v = (x.unflatten(-1, (-1, D)) for x in qkv.split((Hq * D, H * D, H * D), -1))
        q, k = (self.rounded(turn(x, at, self.f, 1.0, self.interleaved, self.norm, 1e-6)[0]) for x in (q, k))
        k = self.keys[b] = torch.cat((k0, k))
        v = self.values[b] = torch.cat((self.values.get(b, v[:0]), v))
        slot = torch.arange(len(k))
        seen = slot <= at[:, None]
        if window:
            seen &= (slot > at[:, None] - window) | (slot < sinks)
        logits = torch.einsum("thgd,nhd->thgn", q.unflatten(1, (H, -1)), k) * D ** -0.5
        p = torch.softmax(logits.masked_fill(~seen[:, None, None], -torch.inf), -1)
        h = h + self.rounded(torch.einsum("thgn,nhd->thgd", p, v).flatten(1)) @ w(l.w_o).T
        up, gate, down = (None if t is None else w(t) for t in l.w_ffn)
        if core is not None:
            up, gate, down = up[core], None if gate is None else gate[core], down[:, core]
        x = self.pre(h)
        a = torch.relu(x @ up.T) if gate is None else torch.relu(x @ gate.T) * (x @ up.T)
        return h + (a if core is not None else self.rounded(a)) @ down.T


@pytest.mark.parametrize("gated,heads,window,sinks", [(False, (4, 4, 64), 0, 0), (True, (8, 2, 128), 24, 3)])
def test_layer(gated, heads, window, sinks):
    """Prompts in ragged pieces, then tokens, each against the layer's own state before it.

    Bound: 16-bit roundings of intermediates (x, qkv, turned q and k, weights, ctx; x, a: 2^-9 of each, random) enter through
    norm-preserving sums, and the layer's own rounding may fall on the other side: eight of them; twice that is asked for."""
    require_gpu()
    cfg, pages, layer, norm, g = build(gated, heads, window, sinks)
    plain = Plain(layer, norm, gated)
    for new in ([40, 45], [30, 0], [1, 17]):
        total = pages.add(new)
        h = torch.randn(total, cfg.d_model, generator=g, device="cuda")
        before = h.double().cpu()
        layer.piece(h)
        at = 0
        for b, n in enumerate(new):
            if n:
                want = plain.tokens(b, before[at:at + n])
                added = (want - before[at:at + n]).norm()
                assert (h[at:at + n].double().cpu() - want).norm() <= 16 * 2.0 ** -9 * added
            at += n
    assert layer.seen == 133 and pages.tokens == [71, 62]
    layer.fix_core()
    core = layer.core_idx.cpu().long()
    assert (core[1:] > core[:-1]).all() and len(core) == layer.K and layer.seen == 0
    for _ in range(4):
        pages.add([1, 1])
        h = torch.randn(2, cfg.d_model, generator=g, device="cuda")
        before = h.double().cpu()
        layer.step(h)
        for b in range(2):
            want = plain.tokens(b, before[b:b + 1], core)
            added = (want - before[b:b + 1]).norm()
            assert (h[b].double().cpu() - want[0]).norm() <= 16 * 2.0 ** -9 * added
    layer.cache.check()
    held = [len(x) for x in pages.held]
    pages.release(0)
    assert len(pages.free) == pages.n_pages - held[1] and pages.length.tolist() == [0, 66]


def test_core_of_pieces_is_the_core_of_the_prompt():
    """Counts add up: two pieces give the set that one call on both gives, by the same activations."""
    require_gpu()
    cfg, pages, layer, _, g = build(False, (4, 4, 64), 0, 0)
    acts = []
    select = ci.binding.coreinfer_select_core

    def keep(act, *args):
        acts.append(act.clone())
        return select(act, *args)

    ci.binding.coreinfer_select_core = keep
    try:
        for new in ([30, 9], [5, 50]):
            layer.piece(torch.randn(pages.add(new), cfg.d_model, generator=g, device="cuda"))
    finally:
        ci.binding.coreinfer_select_core = select
    layer.fix_core()
    act = torch.cat(acts)
    want = torch.empty_like(layer.core_idx)
    ws = torch.empty(ci.coreinfer_select_workspace_bytes(*act.shape), dtype=torch.uint8, device="cuda")
    ci.coreinfer_select_core(act, cfg.alpha, cfg.beta, want, None, ws)
    assert torch.equal(layer.core_idx, want)


def test_captured_step_follows_lengths_and_pages():
    """A step captured once runs on over page borders as the device's lengths grow; attention outputs have the bits of direct calls."""
    require_gpu()
    B, Hq, H, D = 3, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").half()  # noqa: E731
    runs = []
    for captured in (False, True):
        g.manual_seed(1)
        pages = Pages(B, 30, 16, 80)
        cache = PagedKVCache(pages, Hq, H, D, torch.float16)
        rotary = Rotary(D)
        total = pages.add([14, 1, 30])
        cache.append(new(total, H, D), new(total, H, D), rotary, *[new(total, Hq, D)] * 2)
        q, k, v, out = new(B, Hq, D), new(B, H, D), new(B, H, D), torch.zeros(B, Hq, D, dtype=torch.float16, device="cuda")
        x = torch.empty_like(q)

        def step():
            cache.append(k, v, rotary, q, x)
            cache.attend(x, out, window=20, sinks=2)

        outs = []
        if captured:
            pages.reserve(60)
            pages.decoding()
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                pages.one_more()
                step()
        for _ in range(25):
            for t in (q, k, v):
                t.copy_(new(*t.shape))
            if captured:
                graph.replay()
                pages.counted(1)
            else:
                pages.add([1, 1, 1])
                step()
            outs.append(out.clone())
        runs.append(torch.stack(outs))
        assert pages.length.tolist() == pages.tokens == [39, 26, 55]
    assert torch.equal(*runs)


def test_pages_refuse_what_they_do_not_hold():
    require_gpu()
    pages = Pages(2, 5, 16, 64)
    pages.add([33, 16])
    held = [list(x) for x in pages.held]
    for bad in ([1, 17], [32, 0], [0, 49]):
        with pytest.raises(ci.CoreInferError):
            pages.add(bad)
    assert pages.held == held and pages.tokens == [33, 16] and pages.length.tolist() == [33, 16]
    pages.add([15, 16])
    assert not pages.free and sorted(sum(pages.held, [])) == list(range(5))
    pages.release(0)
    pages.add([0, 32])
    assert pages.table[1].unique().numel() == 4 and (pages.table[0] == -1).all()


def test_other_streams():
    """Calls on a stream of the caller's own, behind work on it, while the default stream is idle or busy with other calls."""
    require_gpu()
    pages = Pages(2, 20, 32, 200)
    g = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    caches = [PagedKVCache(pages, 8, 2, 128, max_tokens=200) for _ in range(2)]
    total = pages.add([150, 40])
    k, v, q = new(total, 2, 128), new(total, 2, 128), new(total, 8, 128)
    rotary = Rotary(64)
    want, x = torch.empty_like(q), torch.empty_like(q)
    caches[0].append(k, v, rotary, q, x)
    caches[0].attend(x, want)
    torch.cuda.synchronize()
    for stream in (torch.cuda.Stream(), torch.cuda.Stream()):
        late = [torch.zeros_like(t) for t in (k, v, q)]
        outs = [torch.zeros_like(q) for _ in range(2)]
        x = torch.zeros_like(q)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            torch.cuda._sleep(2000000)
            for t, was in zip(late, (k, v, q)):
                t.copy_(was)
        caches[1].append(late[0], late[1], rotary, late[2], x, stream=stream)
        caches[1].attend(x, outs[1], stream=stream)
        caches[0].attend(want * 0 + new(total, 8, 128), outs[0])     # another call beside it, with its own workspace
        stream.synchronize()
        assert torch.equal(outs[1], want)
        torch.cuda.synchronize()
    turned = torch.empty_like(q)
    with torch.cuda.stream(stream):
        rotary(torch.cat([torch.arange(150), torch.arange(40)]).to(torch.int32).cuda(), q, None, turned)
    stream.synchronize()
    assert torch.equal(turned, x)


@pytest.mark.parametrize("T", [1, 90])
def test_two_graphs_share_a_workspace(T):
    """Two captured calls over caches of their own with one workspace, replayed one behind the other in either order."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(6)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").half()  # noqa: E731
    ws, calls = None, []
    for n in (500, 130):
        pages = Pages(1, 40, 16, 600)
        cache = PagedKVCache(pages, 4, 1, 64, torch.float16, max_tokens=T)
        total = pages.add([n])
        cache.append(new(total, 1, 64), new(total, 1, 64))
        pages.start.copy_(torch.tensor([0, T], dtype=torch.int32))
        q = new(T, 4, 64)
        out, want = torch.zeros_like(q), torch.zeros_like(q)
        cache.attend(q, want)
        ws = cache.ws if ws is None else ws
        cache.ws = ws
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.attend(q, out)
        calls.append((graph, out, want, cache, q, pages))        # a graph holds addresses: all of it stays
    for order in ((0, 1), (1, 0), (0, 1, 1, 0)):
        for i in order:
            calls[i][1].zero_()
            calls[i][0].replay()
        for i in set(order):
            assert torch.equal(calls[i][1], calls[i][2])


def test_four_bit_layer_with_rotary_positions():
    """Keys go into the four-bit cache turned to their positions, in prompts and steps; without a Rotary nothing changes."""
    require_gpu()
    cfg = CONFIGS["tiny"].with_(gated=True)
    g = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s: (torch.randn(s, generator=g, device="cuda") * 0.06).to(cfg.torch_dtype)  # noqa: E731
    weights = (new(8 * 64, cfg.d_model), new(cfg.d_model, 4 * 64)) + layer_weights(cfg, 0, "cuda")
    f, _ = frequencies(64, 10000.0)
    layer = Core4Layer(cfg, 2, 4, 2, 64, 24, weights, recent=6, first=2, max_prompt=40, cache_group=32, rotary=Rotary(64))
    given = []
    append = layer.cache.append
    layer.cache.append = lambda k, v, *a, **kw: (given.append((k.clone(), v.clone())), append(k, v, *a, **kw))
    h = torch.randn(2, 40, cfg.d_model, generator=g, device="cuda")
    _, k, v = layer._split(torch.nn.functional.linear(layer._norm(h), layer.w_qkv), 40)
    want, tol = turn(k.flatten(0, 1), torch.arange(40).repeat(2), f, 1.0, False)
    layer.prompt(h)
    check(given[-1][0].flatten(0, 1), want, tol)
    assert torch.equal(given[-1][1], v)
    for at in (40, 41, 42):
        x = torch.randn(2, cfg.d_model, generator=g, device="cuda")
        layer.qkv(layer._norm(x), layer._qkv)
        k = layer._split(layer._qkv, 1)[1].clone()
        layer.step(x)
        want, tol = turn(k.flatten(0, 1), torch.tensor([at, at]), f, 1.0, False)
        check(given[-1][0].flatten(0, 1), want, tol)
    layer.cache.check()
