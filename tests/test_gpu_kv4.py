"""The 4-bit key/value cache: append and eviction bit-exact against plain loops, attention against the
same sums in 64 bits within bounds that follow from the arithmetic."""
import numpy as np
import pytest
import torch

import paper_2410_18311_b200 as ci
from helpers import require_gpu
from quant4_ref import EPS16, EPS32, OUT_EPS, CacheRef, values_np

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def handle(d):
    return ci.make_kv4_cache(d["k_codes"], d["k_pairs"], d["v_codes"], d["v_pairs"], d["state"], d["weight"], d["position"])


def scratch(n, fill=0xFF):
    return torch.full((n,), fill, dtype=torch.uint8, device="cuda")


# -------------------------------------------------------------------------------- append --

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 128)])
def test_append(D, group, dtype):
    """Ragged sequences, several calls, one sequence that has no room left; k and v slices of one projection."""
    require_gpu()
    B, H, cap = 3, 2, 48
    rng = np.random.default_rng(D + group)
    ref = CacheRef(B, H, cap, D, group, rng)
    ref.set_lengths([0, 17, 40])
    ref.seen = [0, 30, 40]
    d = ref.to_cuda()
    h = handle(d)
    for T in (1, 7, 2):
        fused = torch.from_numpy(rng.standard_normal((B, T, 3 * H * D)).astype(np.float32)).cuda().to(DT[dtype])
        k, v = fused[..., H * D:2 * H * D].unflatten(-1, (H, D)), fused[..., 2 * H * D:].unflatten(-1, (H, D))
        ks, vs = torch.full((B, T, H, D), float("nan"), dtype=DT[dtype], device="cuda"), torch.zeros(B, T, H, D, dtype=DT[dtype], device="cuda")
        ci.coreinfer_kv4_append(h, k, v, ks, vs)
        stored = ref.append(values_np(k), values_np(v))
        for got, want in zip((ks, vs), stored):
            want = torch.from_numpy(want.astype(np.float32)).to(DT[dtype])       # s c is exact in fp32, one rounding each
            assert torch.equal(got.cpu(), want)
    assert ref.refused == [0, 0, 2]
    ref.assert_equal(d)


def test_append_unusual_values_and_without_weights():
    require_gpu()
    B, H, cap, D, group, T = 1, 1, 16, 64, 32, 5
    ref = CacheRef(B, H, cap, D, group, np.random.default_rng(0))
    d = ref.to_cuda()
    bare = ci.make_kv4_cache(d["k_codes"], d["k_pairs"], d["v_codes"], d["v_pairs"], d["state"])
    k = np.random.default_rng(1).standard_normal((B, T, H, D)).astype(np.float32)
    v = k.copy()
    k[0, 0, 0, :32], k[0, 1, 0, 3], k[0, 2, 0, 40], k[0, 3, 0, 0] = 0.5, np.inf, -np.inf, 1e30
    weight, position = ref.weight.copy(), ref.position.copy()
    ci.coreinfer_kv4_append(bare, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda())
    ref.append(k, v)
    ref.weight, ref.position = weight, position                    # a cache without them: nothing is written there
    ref.assert_equal(d)
    k[0, 4, 0, 9] = np.nan
    ks, vs = torch.empty(B, T, H, D, device="cuda"), torch.empty(B, T, H, D, device="cuda")
    ci.coreinfer_kv4_append(bare, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), ks, vs)
    bad = np.isnan(ks.cpu().numpy())
    assert bad[0, 4, 0, :32].all() and bad.sum() == 32 and not torch.isnan(vs).any()


def test_append_full_prompt():
    """A prompt that fills the cache exactly, many thread blocks per sequence."""
    require_gpu()
    B, H, cap, D, group = 2, 8, 304, 128, 64
    rng = np.random.default_rng(2)
    ref = CacheRef(B, H, cap, D, group, rng)
    d = ref.to_cuda()
    k, v = (rng.standard_normal((B, cap, H, D)).astype(np.float32) for _ in "kv")
    ci.coreinfer_kv4_append(handle(d), torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda())
    ref.append(k, v)
    ref.assert_equal(d)
    assert ref.length == [cap, cap]


# ----------------------------------------------------------------------------- attention --

def attend(ref, d, q, accumulate=True, scale=None, out=None, stream=None):
    h = handle(d)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda") if out is None else out
    ws = scratch(ci.coreinfer_kv4_attention_workspace_bytes(h, q.shape[2], q.shape[1]))
    ci.coreinfer_kv4_attention(h, q, ref.D ** -0.5 if scale is None else scale, out, accumulate, ws, stream=stream)
    return out


def check_attention(ref, d, q, out, scale, before, roundings=1):
    """Bounds.  A logit is a sum of D products and their groups in fp32: it is off by at most (D / 8 + 32) spacings of
    its absolute terms (fp32 q enters with 22 bits: 4 spacings more), and by 2^-20 in its exponential.  An error e of a
    logit moves its p and the sum by factors e^(+-e) each.  The weights p s enter the second product with at least
    11 bits for bf16 and 22 for the others; its sums over n slots add n / 8 + 32 spacings at most; then one rounding.
    (More than 8 bf16 rows may share values in fp16: p, the group's offset and the value are rounded, roundings = 3.)"""
    o, add, mass, logit_mass = ref.attention(values_np(q).astype(np.float64), scale)
    n = max(ref.length)
    e = 2 * ((ref.D / 8 + 36) * EPS32 * logit_mass + 2.0 ** -20)[..., None]
    rel = e + (roundings * EPS16 if q.dtype == torch.bfloat16 else 2.0 ** -21) + (n / 8 + 32) * EPS32
    tol = rel * mass + (OUT_EPS[q.dtype] * np.abs(o)) + 1e-30
    err = np.abs(values_np(out) - o)
    assert (err <= tol).all(), "outputs: worst %.3g of the bound" % (err / tol).max()
    if before is not None:
        got = values_np(d["weight"]).astype(np.float64)
        worst = float(e.max()) + (q.shape[1] * q.shape[2] + 4) * EPS32
        tol = worst * add + 2.0 ** -23 * np.abs(before) + 2.0 ** -126
        err = np.abs(got - (before + add))
        live = np.arange(ref.cap) < np.array(ref.length)[:, None, None]
        assert (err <= tol)[np.broadcast_to(live, err.shape)].all(), "weights: worst %.3g of the bound" % (err / tol).max()
        np.testing.assert_array_equal(got[~np.broadcast_to(live, got.shape)], before[~np.broadcast_to(live, before.shape)])


ATTN = [
    # B, H, share, T, D, group, lengths, dtype
    (1, 1, 1, 1, 64, 32, [1], "f32"), (1, 2, 1, 1, 64, 64, [16], "bf16"), (2, 12, 1, 1, 64, 32, [77, 3], "f32"),
    (3, 2, 4, 1, 128, 64, [0, 200, 129], "bf16"), (2, 2, 8, 1, 128, 128, [1000, 17], "f16"), (1, 1, 8, 1, 128, 32, [640], "f32"),
    (2, 3, 5, 3, 128, 32, [300, 2], "bf16"), (2, 1, 12, 2, 64, 64, [65, 128], "f16"), (1, 2, 7, 7, 128, 64, [513], "bf16"),
    (1, 1, 40, 16, 64, 32, [90], "f32"), (2, 2, 1, 16, 128, 128, [15, 100], "f16"), (1, 1, 71, 1, 64, 64, [257], "bf16"),
    (2, 2, 4, 1, 256, 32, [150, 31], "bf16"), (1, 2, 2, 3, 256, 128, [400], "f32"), (1, 1, 16, 5, 256, 64, [97], "f16"),
    (1, 4, 2, 1, 128, 64, [3000], "bf16"), (40, 2, 1, 1, 64, 32, [5 * i for i in range(40)], "bf16"),
    (2, 32, 1, 1, 128, 64, [1100, 700], "bf16"),
]


@pytest.mark.parametrize("B,H,share,T,D,group,lengths,dtype", ATTN)
def test_attention(B, H, share, T, D, group, lengths, dtype):
    require_gpu()
    rng = np.random.default_rng(sum(lengths) + share)
    cap = max(16, -(-max(lengths) // 16) * 16 + 16 * (share % 2))
    ref = CacheRef(B, H, cap, D, group, rng)
    ref.set_lengths(lengths)
    d = ref.to_cuda()
    # what lies beyond the slots in use must not be looked at: all of it NaN
    for b, n in enumerate(lengths):
        d["k_pairs"][b, :, n:] = float("nan")
        d["v_pairs"][b, :, n:] = float("nan")
    before = ref.weight.copy()
    q = torch.from_numpy(rng.standard_normal((B, T, H * share, D)).astype(np.float32)).cuda().to(DT[dtype])
    out = attend(ref, d, q)
    check_attention(ref, d, q, out, D ** -0.5, before)
    # without accumulation: the same outputs, the weights stay
    w = d["weight"].clone()
    again = attend(ref, d, q, accumulate=False)
    assert torch.equal(out, again) and torch.equal(d["weight"], w)


def test_attention_strides_stream_and_bits():
    """q a slice of a fused projection, out a slice of a wider tensor, a side stream; the same call gives the same bits."""
    require_gpu()
    B, H, share, T, D = 2, 4, 2, 2, 128
    rng = np.random.default_rng(4)
    ref = CacheRef(B, H, 256, D, 64, rng)
    ref.set_lengths([200, 91])
    fused = torch.from_numpy(rng.standard_normal((B, T, (share + 2) * H * D)).astype(np.float32)).cuda().bfloat16()
    q = fused[..., : share * H * D].unflatten(-1, (share * H, D))
    wide = torch.zeros(B, T, 3 * share * H * D, dtype=torch.bfloat16, device="cuda")
    out = wide[..., share * H * D:2 * share * H * D].unflatten(-1, (share * H, D))
    runs = []
    for k in range(2):
        d = ref.to_cuda()
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        attend(ref, d, q, out=out, stream=s)
        s.synchronize()
        check_attention(ref, d, q, out, D ** -0.5, ref.weight)
        assert not wide[..., : share * H * D].any() and not wide[..., 2 * share * H * D:].any()
        runs.append((out.clone(), d["weight"].clone()))
    assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attention_sharp_and_scaled(dtype):
    """Logits in the hundreds (one slot takes all, its place differs per head), values from 1e-4 to 1e4 in one cache,
    queries far from 1: nothing overflows on the way."""
    require_gpu()
    B, H, share, T, D, group = 2, 2, 2, 1, 128, 64
    rng = np.random.default_rng(6)
    ref = CacheRef(B, H, 512, D, group, rng)
    ref.set_lengths([500, 333])
    scales = 10.0 ** rng.uniform(-4, 4, size=(B, H, 512, 1))
    ref.s[1], ref.o[1] = (ref.s[1] * scales).astype(np.float16), (ref.o[1] * scales).astype(np.float16)
    for factor in (40.0, 1e-4, 1e4 if dtype == "f16" else 1e8):
        q = torch.from_numpy((factor * rng.standard_normal((B, T, H * share, D))).astype(np.float32)).cuda().to(DT[dtype])
        scale = D ** -0.5 * (1.0 if factor < 1e3 else 100.0 / factor)
        d = ref.to_cuda()
        out = attend(ref, d, q, scale=scale)
        check_attention(ref, d, q, out, scale, ref.weight)


WIDE = [
    # B, H, share, T, D, group, lengths: 9 to 142 bf16 query rows per key head
    (2, 3, 16, 1, 64, 32, [300, 2]), (1, 2, 9, 1, 128, 128, [513]), (1, 2, 5, 4, 128, 64, [77]), (1, 1, 40, 1, 64, 64, [1000]),
    (3, 1, 71, 2, 128, 32, [40, 0, 1]), (2, 2, 16, 1, 256, 32, [150, 31]), (1, 1, 4, 16, 256, 128, [40]), (1, 1, 3, 5, 256, 64, [2000]),
    (1, 8, 4, 3, 128, 32, [3000]), (2, 2, 1, 16, 128, 64, [15, 100]), (7, 16, 11, 1, 128, 128, [16, 129, 1, 500, 300, 128, 64]),
]


@pytest.mark.parametrize("B,H,share,T,D,group,lengths", WIDE)
def test_attention_many_rows(B, H, share, T, D, group, lengths):
    require_gpu()
    rng = np.random.default_rng(1000 + D + len(lengths))
    ref = CacheRef(B, H, 16 * -(-max(lengths) // 16) + 16, D, group, rng)
    ref.set_lengths(lengths)
    d = ref.to_cuda()
    q = torch.from_numpy(rng.standard_normal((B, T, H * share, D)).astype(np.float32)).cuda().bfloat16()
    check_attention(ref, d, q, attend(ref, d, q), D ** -0.5, ref.weight, roundings=3)


@pytest.mark.parametrize("D,group", [(64, 32), (128, 32), (128, 128), (256, 64)])
def test_attention_many_rows_sharp_and_scaled(D, group):
    """Logits in the hundreds and values from 1e-4 to 1e5 (scales and offsets beyond what fp16 holds 16 times)."""
    require_gpu()
    B, H, share, T = 2, 2, 6, 2
    rng = np.random.default_rng(60 + D)
    ref = CacheRef(B, H, 512, D, group, rng)
    ref.set_lengths([500, 333])
    scales = 10.0 ** rng.uniform(-4, 5, size=(B, H, 512, 1))
    with np.errstate(over="ignore"):
        ref.s[1], ref.o[1] = (np.minimum(ref.s[1] * scales, 65504).astype(np.float16), np.clip(ref.o[1] * scales, -65504, 65504).astype(np.float16))
    for factor in (40.0, 1.0, 1e-4, 1e8):
        q = torch.from_numpy((factor * rng.standard_normal((B, T, H * share, D))).astype(np.float32)).cuda().bfloat16()
        scale = D ** -0.5 * (1.0 if factor < 1e3 else 100.0 / factor)
        d = ref.to_cuda()
        check_attention(ref, d, q, attend(ref, d, q, scale=scale), scale, ref.weight, roundings=3)


@pytest.mark.parametrize("share", [1, 5])
def test_attention_nan_in_slots_that_a_token_does_not_see(share):
    """NaN in the newest token's key or value, and beyond the sequence: the tokens before it do not notice."""
    require_gpu()
    T, n = 3, 35
    ref = CacheRef(1, 2, 48, 128, 32, np.random.default_rng(19))
    ref.set_lengths([n])
    q = torch.randn(1, T, 2 * share, 128, device="cuda", dtype=torch.bfloat16)
    clean = ref.to_cuda()
    want = attend(ref, clean, q)
    d = ref.to_cuda()
    d["v_pairs"][0, 1, n - 1, 2] = float("nan")
    for name in ("k_pairs", "v_pairs"):
        d[name][0, :, n:] = float("nan")
    out = attend(ref, d, q)
    assert torch.equal(out[:, :T - 1], want[:, :T - 1]) and torch.equal(out[:, T - 1, :share], want[:, T - 1, :share])
    assert torch.isnan(out[0, T - 1, share:, 64:96]).all()
    assert torch.isfinite(out[0, T - 1, share:, :64]).all() and torch.isfinite(out[0, T - 1, share:, 96:]).all()
    assert torch.equal(d["weight"], clean["weight"])
    d = ref.to_cuda()
    d["k_pairs"][0, 1, n - 1, 0] = float("nan")
    out = attend(ref, d, q)
    assert torch.equal(out[:, :T - 1], want[:, :T - 1]) and torch.isnan(out[0, T - 1, share:]).all()


def test_attention_nan_in_a_value_reaches_its_heads_only():
    require_gpu()
    ref = CacheRef(2, 2, 64, 64, 32, np.random.default_rng(9))
    ref.set_lengths([50, 50])
    d = ref.to_cuda()
    d["v_pairs"][0, 1, 10, 0] = float("nan")
    q = torch.randn(2, 1, 4, 64, device="cuda", dtype=torch.bfloat16)
    out = attend(ref, d, q).float().cpu()
    assert torch.isnan(out[0, 0, 2:, :32]).all()
    assert torch.isfinite(out[0, 0, :2]).all() and torch.isfinite(out[0, 0, 2:, 32:]).all() and torch.isfinite(out[1]).all()


def test_attention_equal_keys_give_the_mean():
    """All keys alike: every p is 1 / n, so the weights are equal and out is the mean of the values."""
    require_gpu()
    ref = CacheRef(1, 1, 112, 64, 64, np.random.default_rng(11))
    ref.set_lengths([100])
    ref.codes[0][:], ref.s[0][:], ref.o[0][:] = 7, 0.5, -2.0
    ref.weight[:] = 0
    d = ref.to_cuda()
    q = torch.ones(1, 1, 1, 64, device="cuda")
    out = attend(ref, d, q)
    np.testing.assert_allclose(out.cpu().numpy()[0, 0, 0], ref.values(1)[0, 0, :100].mean(0), atol=2e-6)
    np.testing.assert_allclose(d["weight"].cpu().numpy()[0, 0, :100], 0.01, rtol=1e-6)


# ------------------------------------------------------------------------------- evict --

def evict(src, dst, budget, recent, first):
    ws = scratch(ci.coreinfer_kv4_evict_workspace_bytes(src), 0xA5)
    ci.coreinfer_kv4_evict(src, dst, budget, recent, first, ws)


EVICT = [
    # B, H, lengths, budget, recent, first, D, group, ties
    (1, 1, [1], 1, 0, 0, 64, 32, False), (2, 2, [40, 10], 20, 4, 2, 64, 64, False), (3, 3, [0, 100, 33], 32, 32, 0, 128, 128, False),
    (2, 4, [300, 257], 256, 10, 4, 128, 64, True), (1, 2, [1500], 100, 0, 0, 256, 32, True), (2, 2, [64, 64], 64, 0, 0, 64, 32, False),
    (1, 3, [2000], 1999, 5, 5, 64, 32, False), (1, 1, [60000], 45000, 1000, 4, 64, 64, True), (2, 1, [33000, 20], 700, 64, 4, 128, 32, False),
    (4, 1, [5000, 4096, 1, 1025], 1024, 256, 4, 64, 64, True), (2, 3, [129, 136], 128, 0, 1, 64, 32, True), (3, 1, [6000, 5996, 5999], 5995, 9, 0, 128, 64, True),
    (1, 2, [140000], 30000, 500, 4, 64, 64, True), (5, 2, [9000, 16000, 0, 8191, 16], 4000, 100, 10, 64, 32, False),
]


@pytest.mark.parametrize("B,H,lengths,budget,recent,first,D,group,ties", EVICT)
@pytest.mark.parametrize("in_place", [True, False])
def test_evict(B, H, lengths, budget, recent, first, D, group, ties, in_place):
    require_gpu()
    rng = np.random.default_rng(budget + len(lengths))
    cap = -(-max(lengths) // 16) * 16
    ref = CacheRef(B, H, cap, D, group, rng)
    if ties:
        ref.weight = np.floor(ref.weight * 3) / 4                  # few distinct values, many zeros
        ref.weight[0, 0, ::11] *= -0.0
    ref.set_lengths(lengths)
    for b in range(B):
        for h in range(H):
            ref.position[b, h, : lengths[b]] = rng.permutation(lengths[b])
    d = ref.to_cuda()
    src = handle(d)
    if in_place:
        evict(src, src, budget, recent, first)
        ref.evict_here(budget, recent, first)
        ref.assert_equal(d)
        evict(src, src, budget, recent, first)                     # nothing is over the budget: nothing changes
        ref.assert_equal(d)
    else:
        small = CacheRef(B, H, max(16, -(-budget // 16) * 16), D, group, rng)
        z = small.to_cuda()
        evict(src, handle(z), budget, recent, first)
        ref.evict_to(small, budget, recent, first)
        small.assert_equal(z)
        ref.assert_equal(d)


def test_evict_odd_weights():
    """NaN weights go first, infinities stay, negative numbers order as numbers."""
    require_gpu()
    ref = CacheRef(1, 1, 64, 64, 32, np.random.default_rng(3))
    ref.set_lengths([60])
    ref.weight[0, 0, 5:25] = np.nan
    ref.weight[0, 0, 40:44] = np.inf
    ref.weight[0, 0, 44:50] = -np.arange(1.0, 7.0)
    for budget in (50, 40, 36, 3):
        d = ref.to_cuda()
        other = CacheRef(1, 1, 64, 64, 32, np.random.default_rng(4))
        z = other.to_cuda()
        evict(handle(d), handle(z), budget, 0, 0)
        ref.evict_to(other, budget, 0, 0)
        other.assert_equal(z)


@pytest.mark.parametrize("budget", [3, 12])
def test_evict_more_certain_slots_than_the_budget(budget):
    """Positions that append did not write: every slot counts as recent; the first ones stay."""
    require_gpu()
    for cap, n in ((16, 15), (48, 40)):
        ref = CacheRef(1, 2, cap, 64, 32, np.random.default_rng(5))
        ref.set_lengths([n])
        ref.position[:] = 10 ** 6
        d = ref.to_cuda()
        evict(handle(d), handle(d), budget, 1, 0)
        ref.evict_here(budget, 1, 0)
        ref.assert_equal(d)


def test_append_attend_evict_loop():
    """A decode loop at a full budget: 40 steps of append, attention with accumulation, and eviction in place.  Positions
    stay distinct, the recent tokens stay, and the attention over what is left matches the plain one."""
    require_gpu()
    B, H, share, D, group, budget, recent, first = 2, 2, 2, 64, 32, 48, 8, 2
    rng = np.random.default_rng(12)
    ref = CacheRef(B, H, 64, D, group, rng)
    d = ref.to_cuda()
    h = handle(d)
    for step in range(40):
        T = 1 + step % 3
        k, v = (torch.from_numpy(rng.standard_normal((B, T, H, D)).astype(np.float32)).cuda() for _ in "kv")
        ci.coreinfer_kv4_append(h, k, v)
        ref.append(values_np(k), values_np(v))
        q = torch.from_numpy(rng.standard_normal((B, T, H * share, D)).astype(np.float32)).cuda()
        out = attend(ref, d, q)
        check_attention(ref, d, q, out, D ** -0.5, ref.weight)
        ref.weight = values_np(d["weight"]).astype(np.float64)     # eviction decides by the weights as accumulated
        evict(h, h, budget, recent, first)
        ref.evict_here(budget, recent, first)
        ref.assert_equal(d)
    pos = d["position"].cpu().numpy()[:, :, :budget]
    seen = ref.seen[0]
    for b in range(B):
        for g in range(H):
            assert len(set(pos[b, g])) == budget and set(range(seen - recent, seen)) <= set(pos[b, g]) and {0, 1} <= set(pos[b, g])


def test_offsets_beyond_32_bits():
    """Three sequences of 64 heads with room for a million slots each: codes end beyond 2^32 bytes.  The same tokens in a
    small cache give the same bits, through append, attention and eviction."""
    require_gpu()
    B, H, D, group = 3, 64, 64, 64
    caches = []
    for cap in (1 << 20, 128):
        new = lambda *s, dtype: torch.empty((B, H, cap) + s, dtype=dtype, device="cuda")  # noqa: E731
        d = {"k_codes": new(D // 2, dtype=torch.uint8), "v_codes": new(D // 2, dtype=torch.uint8), "k_pairs": new(1, 2, dtype=torch.float16),
             "v_pairs": new(1, 2, dtype=torch.float16), "weight": new(dtype=torch.float32), "position": new(dtype=torch.int32),
             "state": torch.zeros(B, 4, dtype=torch.int32, device="cuda")}
        caches.append((d, handle(d)))
    g = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn(B, 100, H, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(B, 1, H, D, generator=g, device="cuda").bfloat16()
    outs = []
    for d, h in caches:
        ci.coreinfer_kv4_append(h, k, v)
        out = torch.empty_like(q)
        ws = torch.empty(ci.coreinfer_kv4_attention_workspace_bytes(h, H, 1), dtype=torch.uint8, device="cuda")
        ci.coreinfer_kv4_attention(h, q, D ** -0.5, out, True, ws)
        ws = torch.empty(ci.coreinfer_kv4_evict_workspace_bytes(h), dtype=torch.uint8, device="cuda")
        ci.coreinfer_kv4_evict(h, h, 40, 10, 2, ws)
        outs.append(out)
    (big, _), (small, _) = caches
    assert torch.equal(outs[0], outs[1]) and big["state"][:, :3].tolist() == [[40, 100, 0]] * B == small["state"][:, :3].tolist()
    for name in big:
        if name != "state":
            assert torch.equal(big[name][:, :, :40], small[name][:, :, :40]), name


@pytest.mark.parametrize("D,group,bad", [(128, 32, (0, 1)), (128, 32, (2, 3)), (128, 32, (0, 1, 3)), (256, 64, (0, 1)), (256, 32, (0, 1, 2, 3)), (256, 32, (4, 5, 6, 7))])
def test_attention_many_rows_nan_groups_of_a_value(D, group, bad):
    """NaN in neighbouring groups of one value that every row sees: its outputs there are NaN, the other groups' are as
    exact as ever (large offsets beside it: a factor chosen from the NaN would take them out of range)."""
    require_gpu()
    n, share = 37, 12
    ref = CacheRef(1, 2, 48, D, group, np.random.default_rng(23))
    ref.set_lengths([n])
    ref.s[1], ref.o[1] = (ref.s[1] * 100).astype(np.float16), (ref.o[1] * 100).astype(np.float16)
    d = ref.to_cuda()
    before = ref.weight.copy()
    q = torch.from_numpy(np.random.default_rng(24).standard_normal((1, 1, 2 * share, D)).astype(np.float32)).cuda().bfloat16()
    want = attend(ref, ref.to_cuda(), q)
    for g in bad:
        d["v_pairs"][0, 1, 5, g] = float("nan")
    out = attend(ref, d, q)
    lost = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    for g in bad:
        lost[0, 0, share:, g * group:(g + 1) * group] = True
    assert torch.isnan(out[lost]).all() and torch.isfinite(out[~lost]).all()
    check_attention(ref, d, q, torch.where(lost, want, out), D ** -0.5, before, roundings=3)


@pytest.mark.parametrize("share", [3, 7])
def test_attention_one_workspace_for_every_number_of_tokens(share):
    """A workspace of the size asked for at 16 tokens serves calls with fewer."""
    require_gpu()
    B, H, D, cap = 8, 4 if share == 7 else 12, 128, 32 if share == 3 else 1024
    ref = CacheRef(B, H, cap, D, 64, np.random.default_rng(share))
    ref.set_lengths([min(cap, 20 + 3 * b) for b in range(B)])
    d = ref.to_cuda()
    h = handle(d)
    ws = scratch(ci.coreinfer_kv4_attention_workspace_bytes(h, H * share, ci.KV4_MAX_QUERIES))
    for T in (1, 6, 8, 10, 12, 15, 16):
        q = torch.from_numpy(np.random.default_rng(T).standard_normal((B, T, H * share, D)).astype(np.float32)).cuda().bfloat16()
        out = torch.full_like(q, float("nan"))
        ci.coreinfer_kv4_attention(h, q, D ** -0.5, out, False, ws)
        check_attention(ref, d, q, out, D ** -0.5, None)


def test_cache_object_with_many_query_heads():
    """200 query heads on one key head: ten tokens a call at most, and a workspace for them."""
    require_gpu()
    from paper_2410_18311_b200.pipeline import KV4Cache
    Hq, D = 200, 64
    cache = KV4Cache(1, Hq, 1, 32, D, 32)
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn(1, 20, 1, D, generator=g, device="cuda") for _ in "kv")
    ks, vs = torch.empty_like(k), torch.empty_like(v)
    cache.append(k, v, ks, vs)
    for T in (1, cache.max_tokens):
        q = torch.randn(1, T, Hq, D, generator=g, device="cuda")
        out = torch.empty_like(q)
        cache.attend(q, out)
        mask = torch.arange(20, device="cuda") > 20 - T + torch.arange(T, device="cuda")[:, None]
        p = torch.einsum("bthd,bnod->bthn", q.double(), ks.double()) * D ** -0.5
        p = torch.softmax(p.masked_fill(mask[None, :, None], float("-inf")), -1)
        # fp32 stored values carry one rounding (2^-24), the kernel about 2^-20 in p: 1e-5 of values of some units is above both
        assert (out - torch.einsum("bthn,bnod->bthd", p, vs.double())).abs().max() < 1e-5 * 8


@pytest.mark.parametrize("D,group,share", [(256, 32, 64), (256, 32, 9), (256, 64, 64), (128, 32, 64)])
def test_attention_many_rows_of_the_largest_batch(D, group, share):
    """1024 sequences (the header's limit) with many bf16 rows: the lists of sequences take shared memory too."""
    require_gpu()
    B = ci.KV4_MAX_BATCH
    rng = np.random.default_rng(D + share)
    ref = CacheRef(B, 1, 16, D, group, rng)
    ref.set_lengths(rng.integers(0, 17, size=B).tolist())
    d = ref.to_cuda()
    before = ref.weight.copy()
    q = torch.from_numpy(rng.standard_normal((B, 1, share, D)).astype(np.float32)).cuda().bfloat16()
    check_attention(ref, d, q, attend(ref, d, q), D ** -0.5, before, roundings=3)


@pytest.mark.parametrize("length,budget", [(100, 40), (30, 40), (5000, 1000), (40000, 700)])
def test_evict_to_another_cache_leaves_the_source_alone(length, budget):
    """Another call may be reading the source, or counting in its scratch word: nothing of it is used or changed."""
    require_gpu()
    H = 3
    ref = CacheRef(1, H, -(-length // 16) * 16, 64, 64, np.random.default_rng(length))
    ref.set_lengths([length])
    d = ref.to_cuda()
    d["state"][:, 3] = 1
    small = CacheRef(1, H, -(-budget // 16) * 16, 64, 64, np.random.default_rng(1))
    z = small.to_cuda()
    evict(handle(d), handle(z), budget, 10, 2)
    ref.evict_to(small, budget, 10, 2)
    small.assert_equal(z)
    assert d["state"].tolist() == [[length, length, 0, 1]]


def test_evict_from_one_source_on_two_streams():
    require_gpu()
    B, H, n, budgets = 2, 16, 4000, (1500, 400)
    ref = CacheRef(B, H, n, 64, 64, np.random.default_rng(31))
    ref.set_lengths([n, n - 123])
    d = ref.to_cuda()
    src = handle(d)
    wants, runs = [], []
    for budget in budgets:
        small = CacheRef(B, H, -(-budget // 16) * 16, 64, 64, np.random.default_rng(budget))
        z = small.to_cuda()
        ref.evict_to(small, budget, 64, 4)
        wants.append(small)
        runs.append((budget, z, handle(z), scratch(ci.coreinfer_kv4_evict_workspace_bytes(src)), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for budget, _, dst, ws, stream in runs:
            ci.coreinfer_kv4_evict(src, dst, budget, 64, 4, ws, stream=stream)
    torch.cuda.synchronize()
    for small, (_, z, _, _, _) in zip(wants, runs):
        small.assert_equal(z)
    ref.assert_equal(d)


def test_tensors_on_the_host_are_refused():
    """Any argument of the four-bit calls that is not beside the others raises before a kernel starts."""
    require_gpu()
    ref = CacheRef(1, 1, 16, 64, 32, np.random.default_rng(1))
    ref.set_lengths([5])
    d = ref.to_cuda()
    h = handle(d)
    with pytest.raises(ci.CoreInferError, match="one CUDA device"):
        handle({**d, "v_pairs": d["v_pairs"].cpu()})
    on_host = handle({n: t.cpu() for n, t in d.items()})
    t = torch.zeros(1, 1, 1, 64, device="cuda")
    ws = scratch(max(ci.coreinfer_kv4_attention_workspace_bytes(h, 1, 1), ci.coreinfer_kv4_evict_workspace_bytes(h)))
    w, codes, pairs = torch.zeros(16, 128, device="cuda"), scratch(ci.coreinfer_w4_codes_bytes(16, 128)), scratch(ci.coreinfer_w4_pairs_bytes(16, 128, 32))
    w4, x, y, b = ci.make_w4_matrix(codes, pairs, 16, 128, 32), torch.zeros(1, 128, device="cuda"), torch.zeros(1, 16, device="cuda"), torch.zeros(16, device="cuda")
    w4_host = ci.make_w4_matrix(codes.cpu(), pairs.cpu(), 16, 128, 32)
    with pytest.raises(ci.CoreInferError, match="one CUDA device"):
        ci.make_w4_matrix(codes, pairs.cpu(), 16, 128, 32)
    for call in (lambda: ci.coreinfer_kv4_append(h, t, t.cpu()), lambda: ci.coreinfer_kv4_append(h, t.cpu(), t.cpu()),
                 lambda: ci.coreinfer_kv4_append(h, t, t, t.clone(), t.cpu()), lambda: ci.coreinfer_kv4_append(h, t, t, t.cpu(), t.clone()),
                 lambda: ci.coreinfer_kv4_append(on_host, t, t),
                 lambda: ci.coreinfer_kv4_attention(h, t, 1.0, t.cpu(), True, ws), lambda: ci.coreinfer_kv4_attention(h, t.cpu(), 1.0, t, True, ws),
                 lambda: ci.coreinfer_kv4_attention(h, t, 1.0, t.clone(), True, ws.cpu()),
                 lambda: ci.coreinfer_kv4_attention(on_host, t, 1.0, t.clone(), True, ws),
                 lambda: ci.coreinfer_kv4_evict(h, h, 4, 0, 0, ws.cpu()), lambda: ci.coreinfer_kv4_evict(h, on_host, 4, 0, 0, ws),
                 lambda: ci.coreinfer_kv4_evict(on_host, h, 4, 0, 0, ws),
                 lambda: ci.coreinfer_w4_quantize(w.cpu(), 32, codes, pairs), lambda: ci.coreinfer_w4_quantize(w, 32, codes.cpu(), pairs.cpu()),
                 lambda: ci.coreinfer_w4_quantize(w, 32, codes, pairs.cpu()),
                 lambda: ci.coreinfer_w4_matvec(w4, x, 0, None, None, y.cpu()), lambda: ci.coreinfer_w4_matvec(w4, x.cpu(), 0, None, None, y),
                 lambda: ci.coreinfer_w4_matvec(w4, x, 0, b.cpu(), None, y), lambda: ci.coreinfer_w4_matvec(w4, x, 0, b, y.cpu(), y),
                 lambda: ci.coreinfer_w4_matvec(w4_host, x, 0, None, None, y)):
        with pytest.raises(ci.CoreInferError):
            call()
    torch.cuda.synchronize()
    ref.assert_equal(d)


@pytest.mark.parametrize("flat", [False, True])
@pytest.mark.parametrize("D,group,dtype", [(64, 32, "f32"), (128, 64, "f32"), (128, 128, "f16"), (256, 64, "f16"), (128, 64, "bf16")])
def test_attention_over_long_caches(D, group, dtype, flat):
    """20000 and 5000 slots: hundreds of MMAs add up in one accumulator, which cuts off below its last place.  flat: keys
    so small that all slots weigh about the same, where the sums hold the most beside their result."""
    require_gpu()
    rng = np.random.default_rng(D + flat)
    ref = CacheRef(2, 1, 20000, D, group, rng)
    ref.set_lengths([20000, 5001])
    if flat:
        ref.s[0], ref.o[0] = (ref.s[0] * 0.01).astype(np.float16), (ref.o[0] * 0.01).astype(np.float16)
    ref.weight[:] = 0
    d = ref.to_cuda()
    q = torch.from_numpy(rng.standard_normal((2, 2, 2, D)).astype(np.float32)).cuda().to(DT[dtype])
    check_attention(ref, d, q, attend(ref, d, q), D ** -0.5, ref.weight.copy())


@pytest.mark.parametrize("D,group,share,dtype", [(64, 32, 1, "f16"), (64, 64, 4, "f16"), (128, 128, 2, "f16"), (256, 64, 1, "f16"), (64, 64, 1, "f32"), (128, 32, 4, "f32")])
def test_attention_values_that_cancel(D, group, share, dtype):
    """Sixteen slots in pairs of one weight and opposite values, whose sum is 0: the output is what the sums lose.  Weights fall
    by 3 to 4 from pair to pair, so that products of many sizes meet in one MMA.  Products of 11-bit weights and codes are
    exact; a sum of 17 terms that keeps 24 bits of the largest loses at most 17 units of 2^-24 of it, the rest of the way a few."""
    require_gpu()
    n = 16
    rng = np.random.default_rng(D + share)
    ref = CacheRef(2, 2, n, D, group, rng)
    ref.set_lengths([n, n - 4])
    ref.codes[1][:, :, 1::2] = 15 - ref.codes[1][:, :, ::2]
    ref.s[1] = (rng.integers(8, 64, size=ref.s[1].shape) / 64).astype(np.float16)          # 7.5 s is an fp16 number
    ref.s[1][:, :, 1::2] = ref.s[1][:, :, ::2]
    ref.o[1] = (-7.5 * ref.s[1].astype(np.float64)).astype(np.float16)
    ref.s[0][:], ref.o[0][:] = 0, -np.floor((1.2 * np.arange(n // 2)[:, None] + rng.uniform(0, 0.2, size=(2, 2, n // 2, 1))).repeat(2, 2) * 64) / 64
    d = ref.to_cuda()
    q = torch.full((2, 1, 2 * share, D), D ** -0.5, device="cuda").to(DT[dtype])
    out = values_np(attend(ref, d, q))
    want, _, mass, _ = ref.attention(values_np(q).astype(np.float64), D ** -0.5)
    assert np.abs(want).max() < 1e-12
    assert (np.abs(out) <= 24 * 2.0 ** -24 * mass + 2.0 ** -25).all(), "worst %.3g of the absolute terms" % (np.abs(out) / mass).max()


@pytest.mark.parametrize("T,D,group,dtype", [(16, 64, 32, "f32"), (4, 128, 64, "f32"), (3, 256, 128, "f32"), (16, 64, 64, "f16"), (2, 128, 128, "f16"),
                                             (16, 64, 32, "bf16"), (8, 128, 128, "bf16"), (4, 128, 64, "bf16"), (2, 256, 32, "bf16"), (16, 128, 32, "bf16")])
@pytest.mark.parametrize("sharp", [False, True])
def test_attention_of_small_values_beside_large_ones(T, D, group, dtype, sharp):
    """Values grow from slot to slot, up to 1e10 times in all.  Every token's largest ones are its newest, and those after it,
    which it does not see, are far larger (sharp: or it sees them and gives them e^-80).  What a row gives weight to keeps its bits."""
    require_gpu()
    lengths = [T, T + 21]
    ref = CacheRef(2, 2, 48, D, group, np.random.default_rng(D + T))
    ref.set_lengths(lengths)
    low, high = (-5.0, 5.0) if dtype != "f16" else (-2.5, 4.5)             # fp16 outputs stay above its subnormal numbers
    scales = np.full((2, 1, 48, 1), 10.0 ** low)
    for b, n in enumerate(lengths):
        scales[b, 0, n - T:n, 0] = 10.0 ** np.linspace(low, high, T)
    with np.errstate(over="ignore"):
        ref.s[1], ref.o[1] = np.minimum(ref.s[1] * scales, 65504).astype(np.float16), np.clip(ref.o[1] * scales, -65504, 65504).astype(np.float16)
    # keys that are one number each, so that logits are theirs: 0, or -80 for the newer half
    ref.s[0][:], ref.o[0][:] = 0, 0
    if sharp:
        for b, n in enumerate(lengths):
            ref.o[0][b, :, n - (T + 1) // 2:] = -80
    d = ref.to_cuda()
    before = ref.weight.copy()
    q = torch.full((2, T, 2, D), D ** -0.5, device="cuda").to(DT[dtype])
    check_attention(ref, d, q, attend(ref, d, q), D ** -0.5, before, roundings=3 if T > 8 and D // group >= 4 else 1)


@pytest.mark.parametrize("D,group,T,dtype", [(128, 32, 1, "f32"), (64, 32, 2, "f32"), (256, 128, 1, "f32"), (128, 64, 3, "f16"), (128, 32, 1, "f16")])
def test_attention_groups_of_different_scales(D, group, T, dtype):
    """Every second group of the values is 1000 times smaller than its neighbours: its outputs are as exact as theirs."""
    require_gpu()
    ref = CacheRef(2, 2, 16, D, group, np.random.default_rng(D + T))
    ref.set_lengths([9, 4])
    ref.s[1][..., ::2], ref.o[1][..., ::2] = ref.s[1][..., ::2] / np.float16(16), ref.o[1][..., ::2] / np.float16(16)
    ref.s[1][..., 1::2], ref.o[1][..., 1::2] = ref.s[1][..., 1::2] * np.float16(64), ref.o[1][..., 1::2] * np.float16(64)
    ref.s[0][:], ref.o[0][:] = 0, (np.random.default_rng(1).integers(-64, 64, size=ref.o[0].shape[:3] + (1,)) / 64).astype(np.float16)
    d = ref.to_cuda()
    before = ref.weight.copy()
    q = torch.full((2, T, 4, D), D ** -0.5, device="cuda").to(DT[dtype])
    check_attention(ref, d, q, attend(ref, d, q), D ** -0.5, before)


@pytest.mark.parametrize("share,T,lengths", [(5, 1, [300, 7]), (8, 1, [129, 0]), (2, 4, [3, 77]), (1, 7, [40, 16])])
def test_attention_eight_rows_of_the_widest_heads(share, T, lengths):
    """bf16 rows 5 to 8 of head_dim 256 in groups of 32, a form of their own; NaN beyond the sequences."""
    require_gpu()
    D, group = 256, 32
    rng = np.random.default_rng(share)
    ref = CacheRef(2, 2, 16 * -(-max(lengths) // 16) + 16, D, group, rng)
    ref.set_lengths(lengths)
    d = ref.to_cuda()
    for b, n in enumerate(lengths):
        d["k_pairs"][b, :, n:] = float("nan")
        d["v_pairs"][b, :, n:] = float("nan")
    q = torch.from_numpy(rng.standard_normal((2, T, 2 * share, D)).astype(np.float32)).cuda().bfloat16()
    check_attention(ref, d, q, attend(ref, d, q), D ** -0.5, ref.weight.copy())
