"""Rotary positions, the paged cache and attention over it, against the formulas in 64 bits within bounds that follow from the
arithmetic (paged_ref.py)."""
import math

import pytest
import torch

import paper_2410_18311_b200 as ci
from helpers import require_gpu
from paged_ref import DT, Batch, attention, check, frequencies, turn

pytestmark = pytest.mark.gpu
KIND = {"plain": ci.ROPE_PLAIN, "linear": ci.ROPE_LINEAR, "ntk": ci.ROPE_NTK, "yarn": ci.ROPE_YARN, "bands": ci.ROPE_BANDS}


def rand(*shape, dt, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dt).cuda()


# ---------------------------------------------------------------------------------- rope --

ROPE = [
    # tokens, q heads, kv heads, D, rot, interleaved, norm, dtype, kind
    (1, 12, 12, 64, 64, False, False, "f32", "plain"), (3, 8, 2, 128, 128, False, True, "bf16", "bands"), (5, 4, 4, 128, 64, True, True, "f16", "yarn"),
    (2, 2, 1, 256, 256, False, True, "f32", "ntk"), (7, 1, 0, 256, 48, False, False, "bf16", "linear"), (300, 0, 3, 64, 16, True, True, "f32", "yarn"),
    (1000, 1, 1, 64, 32, False, True, "f16", "plain"), (777, 5, 1, 128, 80, False, True, "bf16", "bands"), (601, 71, 1, 64, 48, True, False, "f16", "ntk"),
    (2500, 2, 1, 64, 64, False, True, "bf16", "plain"), (3001, 1, 0, 64, 64, True, True, "f32", "plain"),
]


@pytest.mark.parametrize("tokens,Hq,H,D,rot,interleaved,norm,dtype,kind", ROPE)
def test_rope(tokens, Hq, H, D, rot, interleaved, norm, dtype, kind):
    """Slices of one projection, positions from negative ones to 2^31 - 1; then the same in place."""
    require_gpu()
    dt, eps = DT[dtype], 1e-5
    args = dict(base=500000.0 if kind == "bands" else 10000.0, kind=kind, factor=8.0, context=4096)
    f, magnitude = frequencies(rot, **args)
    turns, got_magnitude = ci.coreinfer_rope_frequencies(rot, args["base"], KIND[kind], 8.0, 4096, device="cuda")
    assert got_magnitude == pytest.approx(magnitude, rel=1e-6)
    # far positions in the reference are exact products of the 64-bit fractions too, which are cut to steps of 2^-64 of a turn:
    # 2 pi 2^-64 = 3.4e-19 radians, below 2^-61
    fx = [int(t) & (2 ** 64 - 1) for t in turns.tolist()]
    assert all(abs(x / 2 ** 64 * 2 * math.pi - y) <= 1e-14 * y + 2.0 ** -61 for x, y in zip(fx, f.tolist()))
    fused = rand(tokens, (Hq + 2 * H) * D, dt=dt, seed=tokens) * 3
    q = fused[:, :Hq * D].unflatten(-1, (Hq, D)) if Hq else None
    k = fused[:, Hq * D:(Hq + H) * D].unflatten(-1, (H, D)) if H else None
    wq, wk = ((1 + 0.2 * rand(D, dt=torch.float32, seed=s)).to(dt) if norm else None for s in (1, 2))
    positions = torch.randint(0, 1 << 20, (tokens,), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    positions[0] = 2 ** 31 - 1
    positions[-1] = -77 if tokens > 1 else 2 ** 31 - 1
    rope = ci.make_rope(turns, interleaved, got_magnitude, wq, wk, eps)
    outs = [None if t is None else torch.full((tokens, t.shape[1] + 1, D), float("nan"), dtype=dt, device="cuda")[:, :-1] for t in (q, k)]
    ci.coreinfer_rope_apply(rope, positions.cuda(), q, k, *outs)
    # angles modulo a turn, from integers
    small = torch.tensor([[int(p) * x % 2 ** 64 / 2 ** 64 * 2 * math.pi for x in fx] for p in positions.tolist()], dtype=torch.float64)
    for x, out, w in ((q, outs[0], wq), (k, outs[1], wk)):
        if x is None:
            continue
        want, tol = zip(*[turn(x[t:t + 1], torch.ones(1), small[t], magnitude, interleaved, w, eps) for t in range(tokens)])
        check(out, torch.cat(want), torch.cat(tol))
    ci.coreinfer_rope_apply(rope, positions.cuda(), q, k, q, k)
    for x, out in zip((q, k), outs):
        assert x is None or torch.equal(x, out)


def test_rope_norm_of_one_side_and_unusual_values():
    require_gpu()
    D, dt = 128, torch.bfloat16
    turns, _ = ci.coreinfer_rope_frequencies(64, device="cuda")
    q, k = rand(4, 3, D, dt=dt), rand(4, 2, D, dt=dt, seed=1)
    q[0, 0], q[1, 1, 100], q[2, 2, 5] = 0.0, float("nan"), float("inf")
    w = (1 + rand(D, dt=dt, seed=2)).to(dt)
    at = torch.arange(4, dtype=torch.int32).cuda()
    f, m = frequencies(64, 10000.0)
    for wq, wk in ((w, None), (None, w), (w, w)):
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        ci.coreinfer_rope_apply(ci.make_rope(turns, False, 1.0, wq, wk, 1e-6), at, q, k, qo, ko)
        for h in range(2):
            check(ko[:, h], *[t[:, h] for t in turn(k, at, f, m, False, wk, 1e-6)])
        want, tol = turn(q, at, f, m, False, wq, 1e-6)
        assert torch.isfinite(qo[0]).all()
        check(qo[3], want[3], tol[3])
        check(qo[0, 1:], want[0, 1:], tol[0, 1:])
        if wq is None:                                           # what is not finite reaches its own pair, or with a norm its head
            bad = ~torch.isfinite(qo)
            assert bad[1, 1].nonzero().flatten().tolist() == [100] and set(bad[2, 2].nonzero().flatten().tolist()) <= {5, 37} and bad.sum() <= 3
        else:
            assert torch.isnan(qo[1, 1]).all() and torch.isfinite(qo[1, 0]).all() and torch.isfinite(qo[2, :2]).all()


# -------------------------------------------------------------------------------- append --

APPEND = [
    # new, length, H, share, D, page, dtype, order, rot, interleaved, norm
    ([1], [1], 1, 1, 64, 16, "f32", "heads", 0, False, False), ([5, 0, 1], [21, 9, 33], 2, 2, 128, 16, "bf16", "tokens", 128, False, True),
    ([40, 33], [40, 100], 3, 4, 64, 32, "f16", "heads", 32, True, False), ([3, 3], [300, 3], 1, 5, 256, 128, "bf16", "heads", 256, False, True),
    ([1] * 70, list(range(1, 71)), 2, 1, 64, 16, "f16", "tokens", 64, False, False), ([700], [900], 1, 1, 128, 64, "f32", "tokens", 64, True, True),
    ([17, 2], [256, 257], 2, 1, 256, 256, "f16", "heads", 0, False, False),
]


@pytest.mark.parametrize("new,length,H,share,D,page,dtype,order,rot,interleaved,norm", APPEND)
def test_append(new, length, H, share, D, page, dtype, order, rot, interleaved, norm):
    """Rows of nobody before and behind, slices of one projection; every other slot and row keeps its bits."""
    require_gpu()
    b = Batch(new, length, H, share, D, page, dtype, order, seed=page, front=2, pad=3, wide=8 if order == "heads" else 0)
    Hq = H * share
    fused = b.rand(Hq + 2 * H)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:]
    before = [p.clone() for p in (b.k, b.v)]
    q_out = torch.full((b.tokens, Hq, D), float("nan"), dtype=b.dt, device="cuda")
    if rot:
        turns, m = ci.coreinfer_rope_frequencies(rot, device="cuda")
        w = (1 + 0.1 * rand(D, dt=torch.float32, seed=9)).to(b.dt) if norm else None
        f, _ = frequencies(rot, 10000.0)
        ci.coreinfer_paged_append(b.handle(), b.start, k, v, ci.make_rope(turns, interleaved, m, w, w, 1e-6), None, q, q_out)
    else:
        ci.coreinfer_paged_append(b.handle(), b.start, k, v)
    touched = torch.zeros(b.k.shape[0], page, dtype=torch.bool)
    for s, n in enumerate(new):
        at = torch.arange(length[s] - n, length[s])
        rows = slice(b.starts[s], b.starts[s] + n)
        page_of, slot = b.table[s].cpu()[at // page].long(), at % page
        touched[page_of, slot] = True
        got = b.k[page_of.cuda(), :, slot.cuda()]
        assert torch.equal(b.v[page_of.cuda(), :, slot.cuda()], v[rows])
        if rot:
            check(got, *turn(k[rows], at, f, m, interleaved, w, 1e-6))
            check(q_out[rows], *turn(q[rows], at, f, m, interleaved, w, 1e-6))
        else:
            assert torch.equal(got, k[rows])
    bits = {2: torch.int16, 4: torch.int32}[b.k.element_size()]
    for pool, old in ((b.k, before[0]), (b.v, before[1])):
        same = pool.contiguous().view(bits) == old.contiguous().view(bits)
        assert same.all(-1).all(1).cpu()[~touched].all()
    assert torch.isnan(q_out[:2]).all() and torch.isnan(q_out[b.starts[-1]:]).all()
    if not rot:
        assert torch.isnan(q_out).all()


def test_append_given_positions_equals_rope_apply():
    """Positions of the caller's in the slots' place, and in place of q: the same bits as the operator alone."""
    require_gpu()
    b = Batch([6, 1], [30, 2], 2, 3, 128, 16, "bf16")
    q, k, v = b.rand(6), b.rand(2), b.rand(2)
    turns, m = ci.coreinfer_rope_frequencies(128, 500000.0, ci.ROPE_YARN, 4.0, 2048, device="cuda")
    w = (1 + 0.1 * rand(128, dt=torch.float32)).to(b.dt)
    rope = ci.make_rope(turns, True, m, w, w)
    at = torch.tensor([5, 100000, 3, 3, 70, 1, 9], dtype=torch.int32).cuda()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    ci.coreinfer_rope_apply(rope, at, q, k, qo, ko)
    ci.coreinfer_paged_append(b.handle(), b.start, k, v, rope, at, q, q)
    assert torch.equal(q, qo)
    stored = torch.cat([b.slots(0)[0][-6:], b.slots(1)[0][-1:]])
    assert torch.equal(stored, ko.double())


def test_append_outside_the_cache_stores_nothing():
    """Pages that are none, positions below 0 and behind the table, starts that run backwards: no slot changes but those that exist."""
    require_gpu()
    H, D, page = 2, 64, 16
    k, v = torch.zeros(3, H, page, D, device="cuda"), torch.zeros(3, H, page, D, device="cuda")
    table = torch.tensor([[0, 5], [-1, 1], [2, 2]], dtype=torch.int32).cuda()
    length = torch.tensor([20, 18, 1], dtype=torch.int32).cuda()
    start = torch.tensor([0, 8, 12, 15], dtype=torch.int32).cuda()
    x = torch.ones(15, H, D, device="cuda")
    cache = ci.make_paged_cache(k, v, table, length)
    ci.coreinfer_paged_append(cache, start, x, x)
    # sequence 0: positions 12 .. 15 in page 0, 16 .. 19 in a page that is none; 1: 14, 15 in none, 16, 17 in page 1; 2: -2, -1, 0
    for pool in (k, v):
        want = torch.zeros_like(pool)
        want[0, :, 12:16] = want[1, :, 0:2] = want[2, :, 0:1] = 1
        assert torch.equal(pool, want)
    k.zero_()
    v.zero_()
    ci.coreinfer_paged_append(cache, torch.tensor([9, 3, 900, -4], dtype=torch.int32).cuda(), x, x)
    length.copy_(torch.tensor([1 << 30, -5, 2 ** 31 - 1], dtype=torch.int32))
    ci.coreinfer_paged_append(cache, start, x, x)
    torch.cuda.synchronize()
    assert ((k == 0) | (k == 1)).all() and ((v == 0) | (v == 1)).all()


# ----------------------------------------------------------------------------- attention --

def attend(b, q, scale, window=0, sinks=0, out=None, stream=None):
    out = torch.full(q.shape, 77.0, dtype=q.dtype, device="cuda") if out is None else out
    n = ci.coreinfer_paged_attention_workspace_bytes(b.handle(), q.shape[1], q.shape[0])
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    ci.coreinfer_paged_attention(b.handle(), b.start, q, scale, out, ws, window, sinks, stream=stream)
    return out


def check_attention(b, q, out, scale, window=0, sinks=0):
    want, tol = attention(b, q, scale, window, sinks)
    rows = slice(b.starts[0], b.starts[-1])
    check(out[rows], want[rows], tol[rows])
    assert (out[:b.starts[0]] == 77).all() and (out[b.starts[-1]:] == 77).all()


ATTN = [
    # new, length, H, share, D, page, dtype, order, window, sinks
    ([1], [1], 1, 1, 64, 16, "heads", 0, 0), ([1], [77], 12, 1, 64, 16, "tokens", 0, 0), ([2, 1], [2, 300], 2, 4, 128, 16, "heads", 0, 0),
    ([1, 0, 3], [1000, 40, 129], 2, 5, 128, 32, "heads", 0, 0), ([7], [513], 1, 7, 64, 128, "tokens", 100, 4), ([1] * 5, [64, 65, 1, 500, 128], 4, 2, 256, 64, "heads", 0, 0),
    ([16], [16], 2, 1, 128, 16, "heads", 0, 0), ([130], [130], 1, 2, 64, 16, "heads", 0, 0), ([65, 1], [400, 333], 2, 3, 128, 64, "tokens", 64, 3),
    ([300, 20], [300, 290], 2, 1, 256, 256, "heads", 33, 40), ([1], [4000], 2, 8, 128, 64, "heads", 1, 0), ([257], [1025], 1, 4, 128, 128, "heads", 0, 0),
    ([1] * 40, [5 * i + 1 for i in range(40)], 2, 1, 64, 16, "tokens", 0, 0), ([3, 500, 1], [2000, 600, 700], 3, 2, 64, 16, "tokens", 256, 130),
    ([9], [9], 1, 71, 64, 16, "heads", 0, 0), ([384], [384], 2, 1, 128, 128, "heads", 0, 0), ([1], [20000], 1, 1, 128, 16, "heads", 0, 0),
    ([100], [5000], 1, 2, 128, 16, "tokens", 1000, 500), ([33], [4100], 1, 3, 256, 32, "tokens", 0, 0),
    ([2, 1, 0], [5000, 3, 700], 2, 2, 128, 16, "heads", 0, 0), ([1, 1], [6000, 900], 2, 1, 256, 16, "tokens", 700, 20), ([4], [900], 3, 1, 64, 32, "heads", 300, 7),
    ([3, 1], [2000, 1], 1, 1, 256, 64, "heads", 0, 0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("new,length,H,share,D,page,order,window,sinks", ATTN)
def test_attention(new, length, H, share, D, page, order, window, sinks, dtype):
    """Ragged batches in every form, all that no token holds NaN, rows of nobody left as they were, two calls the same bits."""
    require_gpu()
    b = Batch(new, length, H, share, D, page, dtype, order, seed=sum(length) + share, front=1, pad=2, spread=1.5, wide=8 if order == "heads" and D == 128 else 0)
    q = b.rand(H * share, extra=16)
    scale = D ** -0.5
    out = attend(b, q, scale, window, sinks)
    check_attention(b, q, out, scale, window, sinks)
    assert torch.equal(out, attend(b, q, scale, window, sinks))


NINE_TO_SIXTEEN = [([1], [3000], 2, 16, 16, 0, 0), ([3], [2100], 2, 5, 32, 700, 4), ([12, 9], [600, 20], 3, 1, 64, 0, 0), ([2, 30, 0, 1, 1, 1], [900, 31, 50, 1, 128, 700], 2, 2, 16, 0, 0),
                   ([1, 1], [20000, 5], 1, 13, 128, 0, 0), ([11], [11], 1, 1, 16, 3, 1), ([4] * 9, [4 + 77 * i for i in range(9)], 2, 3, 16, 100, 130)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,length,H,share,page,window,sinks", NINE_TO_SIXTEEN)
def test_attention_nine_to_sixteen_rows_of_128(new, length, H, share, page, window, sinks, dtype):
    """Two groups of eight rows a warp, the second of them not full, sequences of more rows beside them; then infinities and NaN in what some rows see."""
    require_gpu()
    b = Batch(new, length, H, share, 128, page, dtype, seed=sum(length) + share, front=1, pad=2, spread=1.5)
    q = b.rand(H * share, extra=16)
    scale = 128 ** -0.5
    out = attend(b, q, scale, window, sinks)
    check_attention(b, q, out, scale, window, sinks)
    assert torch.equal(out, attend(b, q, scale, window, sinks))
    for s, n in enumerate(new):
        for x, j in enumerate({length[s] - 1, max(0, length[s] - n), length[s] // 2} if n else ()):
            b.v[b.table[s, j // page].item(), x % H, j % page, (7 * x) % 128] = (float("nan"), float("inf"), float("-inf"))[x]
    check_attention(b, q, attend(b, q, scale, window, sinks), scale, window, sinks)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("new", [1, 7, 12, 40])
def test_attention_writes_its_status_word(new, dtype):
    """Every form, in a workspace that holds anything, with nothing to do as well."""
    require_gpu()
    b = Batch([new, 0], [200, 30], 2, 1, 128, 16, dtype, seed=new)
    q = b.rand(2)
    out = torch.empty_like(q)
    n = ci.coreinfer_paged_attention_workspace_bytes(b.handle(), 2, b.tokens)
    for start in (b.start, torch.zeros_like(b.start)):
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        ci.coreinfer_paged_attention(b.handle(), start, q, 0.1, out, ws)
        ci.coreinfer_workspace_status(ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attention_many_units_per_block(dtype):
    """Decoding sequences and long pieces of prompts in one call, more tiles than blocks: every block walks several units, most of
    their tiles without a mask, and no wait gives up."""
    require_gpu()
    small = dtype == "f32"
    new = [300 if small else 900, 1, 200 if small else 700, 1, 1]
    b = Batch(new, [1500, 2000, 1000, 40, 1700], 4, 2, 64, 16, dtype, "tokens", seed=4, front=1, pad=2)
    q = b.rand(8)
    out = torch.full(q.shape, 77.0, dtype=q.dtype, device="cuda")
    n = ci.coreinfer_paged_attention_workspace_bytes(b.handle(), 8, b.tokens)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    for window, sinks in ((0, 0), (300, 4)):
        for _ in range(3):
            out.fill_(77.0)
            ci.coreinfer_paged_attention(b.handle(), b.start, q, 0.125, out, ws, window, sinks)
        if not small:
            ci.coreinfer_workspace_status(ws)
        check_attention(b, q, out, 0.125, window, sinks)


ODD = [([1, 1], [300, 40], 2, 64, 16, 0, 0), ([4, 2], [300, 150], 2, 128, 32, 0, 0), ([60, 5], [200, 130], 3, 64, 16, 0, 0), ([150], [400], 1, 128, 64, 0, 0),
       ([50, 1], [600, 290], 2, 128, 16, 100, 5), ([3], [500], 4, 256, 16, 130, 2), ([270], [270], 1, 64, 128, 0, 0), ([9], [1000], 2, 64, 16, 70, 9)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("new,length,share,D,page,window,sinks", ODD)
def test_attention_odd_values_reach_only_who_sees_them(new, length, share, D, page, window, sinks, dtype):
    """Infinities and NaN in keys and values among the new tokens, at a window's edges and far back."""
    require_gpu()
    b = Batch(new, length, 2, share, D, page, dtype, seed=D + sum(new), front=1, pad=2)
    for s, n in enumerate(new):
        L = length[s]
        spots = {L - 1: float("nan"), L - (n + 1) // 2: float("inf"), max(0, L - n): float("-inf"), max(0, L - n - 3): float("inf")}
        if window:
            spots.update({max(0, L - n - window): float("nan"), max(0, L - window - n // 2): float("-inf"), 1: float("inf"), sinks + 3: float("nan")})
        for x, (j, value) in enumerate(spots.items()):
            b.v[b.table[s, j // page].item(), x % 2, j % page, (7 * x) % D] = value
    q = b.rand(2 * share)
    out = attend(b, q, D ** -0.5, window, sinks)
    check_attention(b, q, out, D ** -0.5, window, sinks)
    assert torch.isfinite(out[1:]).any()
    for s, n in enumerate(new):                                  # a key that is not finite makes all of a row that sees it NaN, and no other
        b.k[b.table[s, (length[s] - 1) // page].item(), 1, (length[s] - 1) % page, 3] = float("nan")
    b.v.nan_to_num_(0, 0, 0)
    out = attend(b, q, D ** -0.5, window, sinks)
    rows = torch.arange(q.shape[0])
    last = torch.tensor([b.starts[s + 1] - 1 for s, n in enumerate(new) if n])
    bad = torch.isnan(out).any(-1).any(-1).cpu()
    assert bad[last].all() and bad.sum() == len(last)
    assert torch.isnan(out[last][:, share:]).all() and torch.isfinite(out[:, :share]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,D", [(1, 64), (5, 128), (90, 128), (40, 256)])
def test_attention_scales(T, D, dtype):
    """A scale of 0 (all weights equal), one below 0, logits so large that a single weight is left; logits of -infinity alone give NaN."""
    require_gpu()
    b = Batch([T, T], [200, T], 1, 3, D, 16, dtype, seed=T)
    q = b.rand(3)
    for scale in (0.0, -0.2, 3.0):
        out = attend(b, q, scale)
        check_attention(b, q, out, scale)
    b.k.nan_to_num_(0, 0, 0).abs_()
    b.k[..., 0] = float("inf")
    q = q.abs().contiguous()
    assert torch.isnan(attend(b, q, -1.0)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [1, 6, 100])
def test_attention_outside_the_cache(T, dtype):
    """Pages that are none read as zeros, tokens at positions below 0 see nothing, nobody sees behind the table, starts that run
    backwards or behind the tensors reach nothing."""
    require_gpu()
    b = Batch([T, T, T], [130 + T, T // 2, 160], 2, 2, 128, 16, dtype, seed=T)
    b.table = b.table.clone()
    b.table[0, 2], b.table[0, 5], b.table[1, 0] = -1, b.n_pages, 2 ** 31 - 1
    b.length_list[2] = b.table.shape[1] * 16 + 40                # behind the table
    b.length[2] = b.length_list[2]
    b.k.nan_to_num_(0, 0, 0), b.v.nan_to_num_(0, 0, 0)
    q = b.rand(4)
    for window, sinks in ((0, 0), (50, 3)):
        out = attend(b, q, 0.1, window, sinks)
        want, tol = attention(b, q, 0.1, window, sinks)
        check(out, want, tol)
    assert (out[T:T + T - T // 2] == 0).all()                    # positions below 0
    for start in ([9, 3, 900, -4], [0, 0, 0, 0], [5, 5, 2 ** 31 - 1, 7], [-(2 ** 31), 2, 1, 2]):
        b.start.copy_(torch.tensor(start, dtype=torch.int32))
        b.length.copy_(torch.tensor([2 ** 31 - 1, -9, 50], dtype=torch.int32))
        attend(b, q, 0.1, 10, 3)
    torch.cuda.synchronize()


def test_attention_shared_pages_and_equal_sequences():
    """Two sequences on the same pages come out alike, whatever their place in the batch and the cut of the work."""
    require_gpu()
    for dtype, T in (("bf16", 1), ("f16", 40), ("f32", 3)):
        b = Batch([T, T, T], [700, 333, 700], 2, 4, 64, 16, dtype, seed=2)
        b.table[2] = b.table[0]
        q = b.rand(8)
        q[2 * T:] = q[:T]
        out = attend(b, q, 0.125)
        assert (out[2 * T:].float() - out[:T].float()).abs().max() <= 2.0 ** -7 * out.abs().max().float()
        check_attention(b, q, out, 0.125)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_long_prompts_again_and_again(D):
    """Many launches one behind the other from a graph, keys and values beyond what the L2 holds nearby, so that tiles arrive in any order:
    the same bits each time, and no wait gives up."""
    require_gpu()
    H, T, page, dt = 16, 4096, 128, torch.bfloat16
    pages = 2 * T // page
    states = []
    for seed in range(3):
        k, v = rand(pages, H, page, D, dt=dt, seed=seed), rand(pages, H, page, D, dt=dt, seed=seed + 9)
        table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[None].to(torch.int32).cuda()
        length, start = torch.tensor([T], dtype=torch.int32).cuda(), torch.tensor([0, T], dtype=torch.int32).cuda()
        cache = ci.make_paged_cache(k, v, table, length)
        q = rand(T, H, D, dt=dt, seed=seed + 5)
        ws = torch.empty(ci.coreinfer_paged_attention_workspace_bytes(cache, H, T), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        ci.coreinfer_paged_attention(cache, start, q, D ** -0.5, out, ws)
        states.append((cache, start, q, out, ws, out.clone(), k, v, table, length))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for cache, start, q, out, ws, *_ in states:
            ci.coreinfer_paged_attention(cache, start, q, D ** -0.5, out, ws)
    for _ in range(40):
        for s in states:
            s[3].zero_()
        graph.replay()
        for s in states:
            ci.coreinfer_workspace_status(s[4])
            assert torch.equal(s[3], s[5])


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_attention_of_a_packing_that_is_none(dtype):
    """Hundreds of sequences that all claim the same rows of a long table: more work than any packing holds, which is left undone or
    done in bounds; the next call is as any other."""
    require_gpu()
    B, T, H, D, page = 400, 300, 2, 64, 16
    dt = DT[dtype]
    k, v = rand(4, H, page, D, dt=dt), rand(4, H, page, D, dt=dt, seed=1)
    table = torch.full((B, 1 << 17), -1, dtype=torch.int32, device="cuda")
    length = torch.full((B,), 1 << 21, dtype=torch.int32, device="cuda")
    start = torch.tensor([0, T] * (B // 2) + [0], dtype=torch.int32, device="cuda")
    cache = ci.make_paged_cache(k, v, table, length)
    q = rand(T, 4, D, dt=dt, seed=2)
    out = torch.zeros_like(q)
    ws = torch.empty(ci.coreinfer_paged_attention_workspace_bytes(cache, 4, T), dtype=torch.uint8, device="cuda")
    ci.coreinfer_paged_attention(cache, start, q, 0.125, out, ws, 64, 3)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()
    b = Batch([3, 1], [40, 9], 2, 2, 64, 16, dtype, seed=8)
    q = b.rand(4)
    check_attention(b, q, attend(b, q, 0.125), 0.125)
