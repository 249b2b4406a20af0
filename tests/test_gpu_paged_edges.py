"""Paged attention and its pipeline where they can go wrong beside the ordinary calls: garbage in slots that nobody sees, positions behind
the table, scales at the ends of their range, workspaces that grow, sequences that end while others decode."""
import pytest
import torch

import paper_2410_18311_b200 as ci
from helpers import require_gpu
from paged_ref import Batch
from paper_2410_18311_b200.pipeline import CorePagedLayer, PagedKVCache, Pages, Rotary
from paper_2410_18311_b200.workloads import CONFIGS, layer_weights
from test_gpu_paged import attend, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("garbage", [float("nan"), float("inf")])
@pytest.mark.parametrize("D,window,sinks", [(64, 0, 0), (128, 0, 0), (128, 70, 3), (256, 0, 0)])
def test_garbage_that_nobody_sees_never_reaches_a_product(D, window, sinks, garbage):
    """Chunks whose last tiles hold garbage behind the sequences' ends, and in front of their windows, and none that a row sees: the
    same bits as with zeros there, in each of many launches (the zeros are written beside the product's own reads, so an order
    that is missing would show now and then)."""
    require_gpu()
    new, length = [150, 33, 90], [401, 33, 290]
    b = Batch(new, length, 4, 1, D, 16, "bf16", seed=D + window)
    q = b.rand(4)
    unseen = [~torch.isfinite(p) for p in (b.k, b.v)]             # what no token holds
    if window:
        for s, n in enumerate(new):
            for j in range(sinks, length[s] - n - window + 1):
                unseen[1][b.table[s, j // 16].item(), :, j % 16] = True
    assert all(u.any() for u in unseen)
    outs = []
    for value in (0.0, garbage):
        for pool, u in zip((b.k, b.v), unseen):
            pool[u] = value
        outs.append(attend(b, q, D ** -0.5, window, sinks))
    assert torch.isfinite(outs[0]).all()
    n = ci.coreinfer_paged_attention_workspace_bytes(b.handle(), 4, b.tokens)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    many = torch.empty(50, *q.shape, dtype=q.dtype, device="cuda")
    handle = b.handle()
    for _ in range(20):
        many.fill_(77.0)
        for out in many:
            ci.coreinfer_paged_attention(handle, b.start, q, D ** -0.5, out, ws, window, sinks)
        assert torch.equal(many, outs[0].expand_as(many))
    ci.coreinfer_workspace_status(ws)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,length,share,D", [([3] * 4, [20, 9, 3, 31], 2, 128), ([2, 5], [64, 40], 1, 64), ([4, 3], [50, 7], 4, 128), ([2], [9], 3, 256)])
def test_few_rows_find_infinities_in_their_first_unit(new, length, share, D, dtype):
    """An infinity that the last tokens see and the first do not, in the first unit of every block: in each of many launches it reaches
    those who see it."""
    require_gpu()
    b = Batch(new, length, 2, share, D, 16, dtype, seed=D + share)
    for s, n in enumerate(new):
        j = length[s] - 1
        b.v[b.table[s, j // 16].item(), :, j % 16, 5] = float("inf")
    q = b.rand(2 * share)
    first = attend(b, q, D ** -0.5)
    check_attention(b, q, first, D ** -0.5)
    last = torch.tensor([b.starts[s + 1] - 1 for s in range(len(new))])
    assert (~torch.isfinite(first[last][..., 5])).all() and torch.isfinite(first).sum() == first.numel() - len(new) * 2 * share
    ws = torch.empty(ci.coreinfer_paged_attention_workspace_bytes(b.handle(), 2 * share, b.tokens), dtype=torch.uint8, device="cuda")
    handle, many = b.handle(), torch.empty(500, *q.shape, dtype=q.dtype, device="cuda")
    bits = first.view(torch.int16)
    for _ in range(4):
        many.fill_(77.0)
        for out in many:
            ci.coreinfer_paged_attention(handle, b.start, q, D ** -0.5, out, ws)
        assert torch.equal(many.view(torch.int16), bits.expand_as(many))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,D,window,pages", [(1, 64, 30, 9), (3, 128, 16, 8), (8, 128, 3000, 230), (2, 256, 1, 3), (12, 128, 700, 60), (40, 64, 25, 9),
                                              (300, 128, 1500, 130), (70, 256, 900, 64)])
def test_tokens_a_window_behind_the_table_get_zeros(T, D, window, pages, dtype):
    """Lengths so far behind the table that the last six tokens' windows (or the only one's) hold none of its positions; with first
    tokens they see those."""
    require_gpu()
    b = Batch([T, T], [16 * (pages - 1), 5 + T], 2, 2, D, 16, dtype, seed=T)
    assert b.table.shape[1] == pages or b.table.shape[1] * 16 > 5 + T
    cap = b.table.shape[1] * 16
    b.length_list[0] = cap + window + 5
    b.length[0] = b.length_list[0]
    for pool in (b.k, b.v):
        pool.nan_to_num_(0, 0, 0)
    q = b.rand(4)
    for sinks in (0, 3):
        out = attend(b, q, 0.1, window, sinks)
        check_attention(b, q, out, 0.1, window, sinks)
        if not sinks:
            assert (out[max(0, T - 6):T] == 0).all() and (out[T:] != 0).any()
            # token T - 7 sees the table's last position only, each one before it one more; the last 16 are a page that is none, zeros
            assert T <= 22 or (out[:T - 22] != 0).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,D", [(1, 64), (5, 128), (12, 128), (90, 128), (90, 64), (40, 256)])
def test_a_scale_of_0_times_an_infinite_logit_is_nan(T, D, dtype):
    """In every form alike, whatever the infinity's sign; rows that do not see the key have equal weights."""
    require_gpu()
    b = Batch([T, T], [200, 100 + T], 2, 2, D, 16, dtype, seed=T)
    q = b.rand(4).abs().contiguous()
    at = 200 - (T + 1) // 2                                      # seen by the first sequence's last (T + 1) // 2 tokens
    for value in (float("inf"), float("-inf")):
        b.k[b.table[0, at // 16].item(), 1, at % 16, 3] = value
        for scale in (0.0, -0.0):
            out = attend(b, q, scale)
            bad = torch.isnan(out)
            hit = slice(T - (T + 1) // 2, T)
            assert bad[hit, 2:].all() and bad.sum() == bad[hit, 2:].numel()
            b.k[b.table[0, at // 16].item(), 1, at % 16, 3] = 0.0
            want = attend(b, q, scale)
            b.k[b.table[0, at // 16].item(), 1, at % 16, 3] = value
            assert torch.equal(out[~bad], want[~bad])
    b.k[b.table[0, at // 16].item(), 1, at % 16, 3] = 0.0
    for scale in (0.0, 1e-40, -1e-40, 3e-32):                    # the last two steps below what fp32 holds in full
        check_attention(b, q, attend(b, q, scale), scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_captured_step_outlives_a_longer_call(dtype):
    """A step is captured, then the same cache attends to pieces longer than announced, on the current stream and on another: replays give
    the step's bits and write nobody else's memory."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(2)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    pages = Pages(2, 40, 16, 300)
    one = PagedKVCache(pages, 8, 2, 128, dtype)
    total = pages.add([250, 170])
    one.append(new(total, 2, 128), new(total, 2, 128))
    pages.decoding()
    q, out = new(2, 8, 128), torch.empty(2, 8, 128, dtype=dtype, device="cuda")
    one.attend(q, out)
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        one.attend(q, out)
    size = one.ws.numel()
    for T, stream in ((12, None), (120, torch.cuda.Stream())):
        pages.start.copy_(torch.tensor([0, T, 2 * T], dtype=torch.int32))
        x, y, z = new(2 * T, 8, 128), torch.zeros(2 * T, 8, 128, dtype=dtype, device="cuda"), torch.zeros(2 * T, 8, 128, dtype=dtype, device="cuda")
        torch.cuda.synchronize()
        one.attend(x, y, stream=stream)
        torch.cuda.synchronize()
        other = PagedKVCache(pages, 8, 2, 128, dtype, max_tokens=2 * T)
        other.k.copy_(one.k), other.v.copy_(one.v)
        other.attend(x, z)
        assert torch.equal(y, z)
        assert one.ws.numel() > size
        taken = [torch.full((size,), 85, dtype=torch.uint8, device="cuda") for _ in range(8)]
        pages.decoding()
        for _ in range(5):
            out.zero_()
            graph.replay()
            assert torch.equal(out, want)
        assert all((t == 85).all() for t in taken)
    one.check()


@pytest.mark.parametrize("n", [3, 60])
def test_a_prompt_behind_one_that_ended_while_others_decoded(n):
    """Captured steps with an ended sequence beside one that goes on: the ended one's row comes out 0 and stores nothing, and the next
    prompt in its place gives a fresh cache's bits."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(n)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").half()  # noqa: E731
    rotary = Rotary(64)

    def made():
        pages = Pages(2, 16, 16, 120)
        return pages, PagedKVCache(pages, 4, 2, 64, torch.float16, max_tokens=128)

    def bring(pages, cache, counts, seed):
        g.manual_seed(seed)
        total = pages.add(counts)
        q, k, v = new(total, 4, 64), new(total, 2, 64), new(total, 2, 64)
        out = torch.empty_like(q)
        cache.append(k, v, rotary, q, q)
        cache.attend(q, out)
        return out

    pages, cache = made()
    bring(pages, cache, [30, 20], 1)
    pages.reserve(48)
    pages.decoding()
    q, k, v, out = new(2, 4, 64), new(2, 2, 64), new(2, 2, 64), new(2, 4, 64)
    x = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pages.one_more()
        cache.append(k, v, rotary, q, x)
        cache.attend(x, out)
    graph.replay()
    pages.counted(1)
    assert (out != 0).any(-1).all()
    pages.release(0)
    before = cache.k.clone()
    for _ in range(5):
        graph.replay()
        assert (out[0] == 0).all() and (out[1] != 0).any(-1).all()
    pages.counted(5)
    assert pages.length.tolist() == pages.tokens == [0, 26]
    assert (cache.k != before).any(1).any(-1).sum() == 5             # slots of the one that goes on
    got = bring(pages, cache, [n, 0], 2)
    assert torch.equal(got, bring(*made(), [n, 0], 2))
    pages.decoding()
    graph.replay()
    pages.counted(1)
    assert pages.length.tolist() == pages.tokens == [n + 1, 27] and (out != 0).any(-1).all()
    cache.check()


def layer_of(batch=2, gated=True, pieces=()):
    """A small layer with rotary positions that has been brought pieces of that many tokens a sequence, and its generator."""
    cfg = CONFIGS["tiny"].with_(gated=gated)
    g = torch.Generator(device="cuda").manual_seed(batch)
    new = lambda *s: (torch.randn(s, generator=g, device="cuda") * 0.06).to(cfg.torch_dtype)  # noqa: E731
    pages = Pages(batch, 12 * batch, 16, 200)
    layer = CorePagedLayer(cfg, pages, 8, 2, 64, (new(12 * 64, cfg.d_model), new(cfg.d_model, 8 * 64)) + layer_weights(cfg, 0, "cuda"), Rotary(64))
    for counts in pieces:
        layer.piece(torch.randn(pages.add(counts), cfg.d_model, generator=g, device="cuda"))
    return layer, g


def test_pieces_leave_the_deployed_set_alone():
    """core_idx names the neurons whose weights up, gate and down hold, until the next fix_core()."""
    require_gpu()
    layer, g = layer_of(pieces=([30, 20],))
    layer.fix_core()
    deployed = layer.core_idx.clone()
    w_up, w_gate, w_down = layer.w_ffn
    layer.pages.release(0)
    for counts in ([50, 0], [1, 40]):
        layer.piece(torch.randn(layer.pages.add(counts), layer.cfg.d_model, generator=g, device="cuda") * 3 + 1)
        assert torch.equal(layer.core_idx, deployed)
        assert torch.equal(layer.up, w_up[deployed.long()]) and torch.equal(layer.gate, w_gate[deployed.long()])
    layer.fix_core()
    assert not torch.equal(layer.core_idx, deployed) and torch.equal(layer.up, w_up[layer.core_idx.long()])


def test_a_layer_without_a_core_set_takes_no_step():
    """Before the first fix_core() there are no weights to decode with; fix_core() needs counts."""
    require_gpu()
    layer, g = layer_of()
    with pytest.raises(ci.CoreInferError):
        layer.fix_core()
    layer.piece(torch.randn(layer.pages.add([5, 4]), layer.cfg.d_model, generator=g, device="cuda"))
    h = torch.randn(layer.pages.add([1, 1]), layer.cfg.d_model, generator=g, device="cuda")
    before, k = h.clone(), layer.cache.k.clone()
    with pytest.raises(ci.CoreInferError):
        layer.step(h)
    assert torch.equal(h, before) and torch.equal(layer.cache.k, k)
    layer.fix_core()
    deployed = layer.core_idx.clone()
    layer.step(h)
    assert torch.isfinite(h).all() and not torch.equal(h, before)
    with pytest.raises(ci.CoreInferError):
        layer.fix_core()
    assert torch.equal(layer.core_idx, deployed)


@pytest.mark.parametrize("batch,counts,rows", [(2, [5, 4], 8), (2, [5, 4], 10), (2, [1, 1], 3), (2, [1, 0], 2), (9, [1] * 9, 9)])
def test_a_layer_refuses_rows_that_were_not_announced(batch, counts, rows):
    """Nothing is stored, updated or counted; more than 8 sequences have no step, but pieces."""
    require_gpu()
    layer, g = layer_of(batch, pieces=([3] * batch,))
    layer.fix_core()
    layer.pages.add(counts)
    h = torch.randn(rows, layer.cfg.d_model, generator=g, device="cuda")
    before, k, seen = h.clone(), layer.cache.k.clone(), layer.seen
    for call in (layer.step,) if rows == sum(counts) else (layer.step, layer.piece):
        with pytest.raises(ci.CoreInferError):
            call(h)
        assert torch.equal(h, before) and torch.equal(layer.cache.k, k) and layer.seen == seen and not layer.counts.any()
    h = torch.randn(sum(counts), layer.cfg.d_model, generator=g, device="cuda")
    layer.piece(h)
    assert torch.isfinite(h).all() and layer.seen == sum(counts)


@pytest.mark.parametrize("B,H,share,D,T,L", [(16, 12, 1, 64, 1, 400000), (16, 10, 4, 128, 1, 400000), (40, 8, 1, 256, 1, 150000), (40, 8, 8, 64, 1, 60000),
                                             (38, 8, 1, 128, 12, 60000), (20, 8, 8, 256, 1, 60000), (1, 8, 1, 64, 2400, 60000), (1, 5, 1, 256, 2000, 40000)])
def test_sums_over_many_fp32_positions_are_no_single_chain(B, H, share, D, T, L):
    """Equal weights and equal values, whose sum a chain of additions always rounds to the same side: units that one block sums alone.

    Weights are 1 and their sum a whole number below 2^24, so both are exact.  An addition or fused product is off by half a spacing,
    2^-24 of the sum: at most 1024 of them in a chain, one for every 1024 positions, 300 in the join, and the division."""
    require_gpu()
    pool = torch.empty(1, H, 16, D, device="cuda")
    pool.copy_((torch.arange(D, device="cuda") % 37 + 1) / -97)
    table = torch.zeros(B, -(-L // 16), dtype=torch.int32, device="cuda")
    length = torch.full((B,), L, dtype=torch.int32, device="cuda")
    start = (torch.arange(B + 1, device="cuda") * T).to(torch.int32)
    cache = ci.make_paged_cache(pool, pool, table, length)
    q = torch.zeros(B * T, H * share, D, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(ci.coreinfer_paged_attention_workspace_bytes(cache, H * share, B * T), dtype=torch.uint8, device="cuda")
    ci.coreinfer_paged_attention(cache, start, q, 0.1, out, ws)
    want = pool[0, 0, 0].double()
    assert ((out.double() - want).abs() <= (1024 + L / 1024 + 302) * 2.0 ** -24 * want.abs()).all()


@pytest.mark.parametrize("dtype,T,share", [(torch.float32, 1, 2), (torch.float32, 9, 1), (torch.bfloat16, 1, 4), (torch.bfloat16, 80, 2), (torch.float16, 90, 3)])
def test_pools_and_rows_beyond_32_bits(dtype, T, share):
    """Pages behind 2^32 elements of the pools, and rows of queries and outputs that lie 2^22 elements apart, behind 2^32 of them where many
    are new: the bits of a small cache with rows side by side."""
    require_gpu()
    H, D, page, length = 8, 128, 64, [700, 333]
    g = torch.Generator(device="cuda").manual_seed(T)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    k, v, q = new(1033, H, D), new(1033, H, D), new(2 * T, H * share, D)
    whole = torch.tensor([0, 700, 1033], dtype=torch.int32, device="cuda")
    lengths = torch.tensor(length, dtype=torch.int32, device="cuda")
    pages = torch.randperm(22, generator=torch.Generator().manual_seed(T)).view(2, 11).to(torch.int32)
    outs = []
    for n_pages, step in ((22, H * share * D), (70000, 1 << 22)):
        tokens = 2 * T if n_pages == 22 or T < 10 else 1100
        start = torch.tensor([tokens - 2 * T, tokens - T, tokens], dtype=torch.int32, device="cuda")
        table = (pages + n_pages - 22).cuda()
        pools = [torch.empty(n_pages, H, page, D, dtype=dtype, device="cuda") for _ in range(2)]
        cache = ci.make_paged_cache(*pools, table, lengths)
        x, out = (torch.empty(tokens * step, dtype=dtype, device="cuda").as_strided((tokens, H * share, D), (step, D, 1)) for _ in range(2))
        x[-2 * T:] = q
        ws = torch.empty(ci.coreinfer_paged_attention_workspace_bytes(cache, H * share, tokens), dtype=torch.uint8, device="cuda")
        ci.coreinfer_paged_append(cache, whole, k, v)
        ci.coreinfer_paged_attention(cache, start, x, 0.1, out, ws)
        outs.append(out[-2 * T:].contiguous())
    assert torch.isfinite(outs[0]).all() and (outs[0] != 0).any(-1).all() and torch.equal(*outs)


@pytest.mark.parametrize("dtype,T", [(torch.float32, 1), (torch.float32, 30), (torch.bfloat16, 1), (torch.bfloat16, 6), (torch.float16, 200)])
def test_lengths_that_change_under_a_call(dtype, T):
    """Another stream changes lengths, packing and pages while calls run: what comes out then is nobody's business, but every call ends,
    no wait gives up, no other memory is written, and the next call is as any other."""
    require_gpu()
    B, H, share, D, page = 5, 4, 2, 128, 16
    g = torch.Generator(device="cuda").manual_seed(T)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    k, v = new(300, H, page, D), new(300, H, page, D)
    table = torch.randperm(300, generator=torch.Generator().manual_seed(1))[:B * 60].view(B, 60).to(torch.int32).cuda()
    length = torch.tensor([900, 40 + T, 700, T, 333 + T], dtype=torch.int32, device="cuda")
    start = (torch.arange(B + 1, device="cuda") * T).to(torch.int32)
    cache = ci.make_paged_cache(k, v, table, length)
    held = torch.full((B * T + 2, H * share, D), 77.0, dtype=dtype, device="cuda")
    q, out = new(B * T, H * share, D), held[1:-1]
    n = ci.coreinfer_paged_attention_workspace_bytes(cache, H * share, B * T)
    ws = torch.full((n + 64,), 85, dtype=torch.uint8, device="cuda")
    ci.coreinfer_paged_attention(cache, start, q, 0.1, out, ws[:n])
    want, was = out.clone(), [t.clone() for t in (length, start, table)]
    others = [(length * 0 + x, start * y, table.flip(0) - z) for x, y, z in ((950, 1, 0), (T, 0, 1), (0, 2, 400), (1 << 30, 1, 0), (500, -1, 0))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        for x in others:
            with torch.cuda.stream(side):
                for _ in range(4):
                    for t, y in zip((length, start, table), x):
                        t.copy_(y)
                    for t, y in zip((length, start, table), was):
                        t.copy_(y)
            for window in (0, 100):
                ci.coreinfer_paged_attention(cache, start, q, 0.1, out, ws[:n], window, 3)
    torch.cuda.synchronize()
    ci.coreinfer_workspace_status(ws)
    ci.coreinfer_paged_attention(cache, start, q, 0.1, out, ws[:n])
    assert torch.equal(out, want) and (held[0] == 77).all() and (held[-1] == 77).all() and (ws[n:] == 85).all()


@pytest.mark.parametrize("dtype,T", [(torch.float32, 1), (torch.bfloat16, 2), (torch.float16, 90)])
def test_calls_that_overlap_in_one_workspace_stay_in_their_buffers(dtype, T):
    """Against the rules: calls of other batches, heads and lengths on two streams with one workspace.  Outputs may be anything, rows beside
    them are as they were, and each call alone is right again."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(T)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    calls = []
    for B, H, L in ((1, 2, 3000), (40, 8, 900)):
        pool = new(64, H, 16, 64), new(64, H, 16, 64)
        table = torch.randint(0, 64, (B, 190), generator=torch.Generator().manual_seed(B), dtype=torch.int32).cuda()
        length, start = torch.full((B,), L, dtype=torch.int32, device="cuda"), (torch.arange(B + 1, device="cuda") * T).to(torch.int32)
        held = torch.full((B * T + 2, 2 * H, 64), 77.0, dtype=dtype, device="cuda")
        calls.append((ci.make_paged_cache(*pool, table, length), start, new(B * T, 2 * H, 64), held, pool, table, length))
    ws = torch.empty(max(ci.coreinfer_paged_attention_workspace_bytes(c[0], c[2].shape[1], c[2].shape[0]) for c in calls), dtype=torch.uint8, device="cuda")
    run = lambda c, stream=None: ci.coreinfer_paged_attention(c[0], c[1], c[2], 0.1, c[3][1:-1], ws, stream=stream)  # noqa: E731
    wants = []
    for c in calls:
        run(c)
        wants.append(c[3].clone())
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(200):
        for c, s in zip(calls, streams):
            run(c, s)
    torch.cuda.synchronize()
    for c, want in zip(calls, wants):
        assert (c[3][0] == 77).all() and (c[3][-1] == 77).all()
        run(c)
        assert torch.equal(c[3], want)


@pytest.mark.parametrize("dtype,D,share,most", [("f32", 64, 1, 1), ("f32", 256, 6, 9), ("bf16", 128, 1, 1), ("f16", 128, 16, 1), ("bf16", 256, 6, 9)])
def test_the_largest_batch(dtype, D, share, most):
    """1024 sequences, whose list takes the most of the shared memory, in every form; some of them without new tokens."""
    require_gpu()
    new = [(5 * i) % (most + 1) if i % 3 else most for i in range(1024)]
    b = Batch(new, [n + (7 * i) % 12 for i, n in enumerate(new)], 1, share, D, 16, dtype, seed=share, front=1, pad=1)
    q = b.rand(share)
    check_attention(b, q, attend(b, q, D ** -0.5), D ** -0.5)
