"""What is measured of the 4-bit operators of a decode step: the projections (matrix-vector products
with 4-bit weights), the 4-bit key/value cache (append), attention over it, and eviction from it.

Each case is a dict of plain values; `prepare` makes its inputs on the GPU from a seed, `run` is one
pass through an operator as a decode loop calls it (`own`: the framework's kernels; otherwise the
plain torch form in 32 bits), `exact` the same from the definition in 64 bits, `work` the bytes and
operations that a pass cannot do without.

Formats (the framework's): a group of G values x along a row is held as codes c = 0..15 and an fp16
pair (s, o), x^ = s c + o, with o = min x and s = (max x - min x) / 15.  A row piece of 32 H values is
stored as 16 H bytes in 2-byte units: unit 8-lane index i (0..7), block h (0..H-1) at 2 (i H + h)
holds values 32 h + 4 i .. + 3, the first in the lowest 4 bits.  A weight matrix [N, K] is padded to
16 rows and 128 columns (codes and pairs zero) and stored [N/16][K/128][16][64 bytes], its pairs
[N/16][K/G][16][2].  A cache holds [batch][heads][capacity][D/2] codes and [..][D/G][2] pairs for
keys and values, per slot a weight (fp32) and a position (int32), and per sequence the words
(length, tokens seen, tokens refused, scratch).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ------------------------------------------------------------------------------------ cases --

def listed():
    return [
        # one attention projection of the one-layer fp32 configuration: the smallest call, latency counts
        {"name": "matvec proj 768 f32", "op": "matvec", "N": 768, "K": 768, "batch": 1, "dtype": "f32", "out": "f32",
         "group": 32, "act": "none", "bias": True, "mul": False},
        # an attention projection of the 4096-wide configurations at batch 1, fp32 result as the FFN's
        {"name": "matvec proj 4096 bf16", "op": "matvec", "N": 4096, "K": 4096, "batch": 1, "dtype": "bf16", "out": "f32",
         "group": 128, "act": "none", "bias": True, "mul": False},
        # down projection over a core set of 0.2 * 16384 neurons (an odd length), five sequences
        {"name": "matvec core down 3277 f16", "op": "matvec", "N": 4096, "K": 3277, "batch": 5, "dtype": "f16", "out": "f16",
         "group": 64, "act": "none", "bias": False, "mul": False},
        # the widest up projection, all neurons, eight sequences
        {"name": "matvec up 36864 bf16", "op": "matvec", "N": 36864, "K": 9216, "batch": 8, "dtype": "bf16", "out": "bf16",
         "group": 128, "act": "relu", "bias": True, "mul": False},
        # a prompt of one sequence enters a cleared cache
        {"name": "append prompt bf16", "op": "append", "B": 1, "heads": 32, "D": 128, "group": 64, "T": 1000, "capacity": 1024,
         "dtype": "bf16"},
        # one decode step at a full budget: eight sequences append a token, and one leaves every head
        {"name": "append and evict one", "op": "step", "B": 8, "heads": 32, "D": 128, "group": 64, "T": 1, "length": 2048,
         "budget": 2048, "recent": 256, "first": 4, "capacity": 2064, "dtype": "bf16"},
        # a piece of a long prompt through a bounded cache: 256 tokens enter and 256 leave
        {"name": "append and evict piece f32", "op": "step", "B": 2, "heads": 12, "D": 64, "group": 32, "T": 256, "length": 1024,
         "budget": 1024, "recent": 256, "first": 0, "capacity": 1280, "dtype": "f32"},
        # the heavy hitters of long prompts move into the small cache that decoding uses
        {"name": "evict after prompt", "op": "evict", "B": 4, "heads": 8, "D": 128, "group": 128, "length": 16384,
         "budget": 2048, "recent": 512, "first": 4, "capacity": 16384, "dtype": "bf16"},
        # a short conversation on the one-layer fp32 configuration's heads: latency counts
        {"name": "attend short f32", "op": "attend", "B": 1, "heads": 12, "q_heads": 12, "D": 64, "group": 32, "T": 1,
         "length": 77, "capacity": 128, "dtype": "f32", "accumulate": True},
        # ordinary decoding, one key head per query head, weights accumulated for the eviction
        {"name": "attend 8 x 4001 bf16", "op": "attend", "B": 8, "heads": 32, "q_heads": 32, "D": 128, "group": 64, "T": 1,
         "length": 4001, "capacity": 4096, "dtype": "bf16", "accumulate": True},
        # three drafted tokens a sequence are checked at once, five query heads per key head
        {"name": "attend draft 3 x 5 bf16", "op": "attend", "B": 6, "heads": 8, "q_heads": 40, "D": 128, "group": 32, "T": 3,
         "length": 9000, "capacity": 9008, "dtype": "bf16", "accumulate": True},
        # two long documents, grouped heads, nothing evicted
        {"name": "attend long 130000 f16", "op": "attend", "B": 2, "heads": 8, "q_heads": 32, "D": 128, "group": 128, "T": 1,
         "length": 130000, "capacity": 131072, "dtype": "f16", "accumulate": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("matvec", "attend", "attend", "append", "step", "evict"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    if op == "matvec":
        K = _log(rng, 100, 16384)
        return {"op": op, "N": _log(rng, 64, min(36864, 36864 * 9216 // K)), "K": K, "batch": rng.randint(1, 8), "dtype": dtype,
                "out": rng.choice((dtype, "f32")), "group": rng.choice((32, 64, 128)),
                "act": rng.choice(("none", "relu", "silu")), "bias": rng.random() < 0.5, "mul": rng.random() < 0.3}
    D = rng.choice((64, 128, 128, 256))
    case = {"op": op, "D": D, "dtype": dtype, "group": rng.choice([g for g in (32, 64, 128) if g <= D])}
    if op == "attend":
        heads, share = rng.choice((1, 2, 4, 8, 12, 32)), rng.choice((1, 2, 4, 5, 8))
        B = rng.randint(1, 16)
        most = min(130000, 2 * 8 * 131072 * 128 // (B * heads * D * 2))
        length = _log(rng, 1, most)
        return {**case, "B": B, "heads": heads, "q_heads": heads * share, "T": rng.choice((1, 1, 1, 2, 4, 7)), "length": length,
                "capacity": 16 * -(-(length + rng.randint(0, 64)) // 16), "accumulate": rng.random() < 0.6}
    B, heads = rng.randint(1, 8), rng.choice((2, 8, 12, 32))
    if op == "append":
        T = _log(rng, 1, 1000)
        return {**case, "B": B, "heads": heads, "T": T, "capacity": 16 * -(-(T + rng.randint(0, 40)) // 16)}
    if op == "step":
        budget = _log(rng, 64, 4096)
        T = _log(rng, 1, max(2, budget // 4))
        return {**case, "B": B, "heads": heads, "T": T, "length": budget, "budget": budget, "first": rng.choice((0, 4)),
                "recent": rng.randint(T, max(T, budget // 2)), "capacity": 16 * -(-(budget + T + rng.randint(0, 40)) // 16)}
    length = _log(rng, 200, min(32768, 2 * 8 * 131072 * 128 // (B * heads * D * 4)))
    budget = max(64, int(length * rng.uniform(0.1, 0.9)))
    return {**case, "B": B, "heads": heads, "length": length, "budget": budget, "recent": budget // 4, "first": rng.choice((0, 4)),
            "capacity": 16 * -(-(length + rng.randint(0, 40)) // 16)}


def _lengths(case):
    """Ragged lengths of the sequences, the first the longest; the same for every seed."""
    n = case["length"]
    return [max(1, n - int(n * 0.5 * ((0.618 * b) % 1.0))) for b in range(case["B"])]


def _row_bytes(case):
    return case["D"] + 8 * (case["D"] // case["group"])          # keys and values of a slot: codes and pairs


def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "matvec":
        N, K, m = case["N"], case["K"], case["batch"]
        b = N * K / 2 + 4 * N * -(-K // case["group"]) + m * K * e + m * N * BYTES[case["out"]] * (2 if case["mul"] else 1)
        return {"bytes": b + (N * e if case["bias"] else 0), "flops": 2 * m * N * K}
    B, H, D = case["B"], case["heads"], case["D"]
    if case["op"] == "attend":
        slots = sum(_lengths(case)) * H
        b = slots * (_row_bytes(case) + (8 if case["accumulate"] else 0)) + 2 * B * case["T"] * case["q_heads"] * D * e
        return {"bytes": b, "flops": 4 * sum(_lengths(case)) * case["q_heads"] * case["T"] * D}
    b, f = 0, 0
    if case["op"] in ("append", "step"):
        new = B * H * case["T"]
        b += new * (4 * D * e + _row_bytes(case) + 8)            # read, stored values written, cache written
        f += new * 2 * D * 4
    if case["op"] in ("step", "evict"):
        slots = B * H * (case["budget"] + case["T"]) if case["op"] == "step" else H * sum(_lengths(case))
        kept = H * sum(min(n, case["budget"]) for n in _lengths(case)) if case["op"] == "evict" else B * H * case["T"]
        b += 8 * slots + 2 * kept * (_row_bytes(case) + 8)
        f += slots
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------------------ plain format --

def _pack(codes):
    """Codes [..., 32 H] (uint8) -> bytes [..., 16 H]."""
    lead, d = codes.shape[:-1], codes.shape[-1]
    c = codes.reshape(*lead, d // 32, 8, 4).transpose(-3, -2).reshape(*lead, d // 2, 2)
    return c[..., 0] | (c[..., 1] << 4)


def _unpack(packed):
    """Bytes [..., 16 H] -> codes [..., 32 H] as fp32."""
    lead, n = packed.shape[:-1], packed.shape[-1]
    c = torch.stack((packed & 15, packed >> 4), -1).reshape(*lead, 8, n // 16, 4).transpose(-3, -2)
    return c.reshape(*lead, 2 * n).float()


def _quantise(x, group):
    """fp32 [..., d] -> (codes uint8 [..., d], pairs fp16 [..., d / group, 2])."""
    g = x.reshape(*x.shape[:-1], -1, group)
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    o = lo.clamp(-65504.0, 65504.0).half()
    s = ((hi - lo) / 15.0).clamp(max=65504.0).half()
    c = torch.round((g - o.float()) / s.float()).clamp(0, 15)
    c = torch.where(s > 0, c, torch.zeros_like(c))
    return c.to(torch.uint8).reshape(x.shape), torch.cat((s, o), -1)


def _values(codes, pairs):
    """(codes fp32 [..., d], pairs [..., d / group, 2]) -> the fp32 values they stand for."""
    group = codes.shape[-1] // pairs.shape[-2]
    c = codes.reshape(*codes.shape[:-1], -1, group)
    return (c * pairs[..., :1].float() + pairs[..., 1:].float()).reshape(codes.shape)


# ---------------------------------------------------------------------------------- prepare --

def _weights(gen, N, K, group):
    """A weight matrix ~ N(0, 0.02), quantised and laid out once."""
    w = torch.randn(N, K, generator=gen, device="cuda") * 0.02
    Np, Kp = 16 * -(-N // 16), 128 * -(-K // 128)
    kg = group * -(-K // group)
    if kg > K:                                # the last group's values end before the group: they alone set its pair
        w = torch.cat((w, w[:, -1:].expand(N, kg - K)), 1)
    codes, pairs = _quantise(w, group)
    codes = torch.cat((codes[:, :K], torch.zeros(N, Kp - K, dtype=torch.uint8, device="cuda")), 1)
    pairs = torch.cat((pairs, torch.zeros(N, (Kp - kg) // group, 2, dtype=torch.float16, device="cuda")), 1)
    codes = torch.cat((codes, torch.zeros(Np - N, Kp, dtype=torch.uint8, device="cuda")))
    pairs = torch.cat((pairs, torch.zeros(Np - N, Kp // group, 2, dtype=torch.float16, device="cuda")))
    codes = _pack(codes.reshape(Np // 16, 16, Kp // 128, 128).transpose(1, 2)).contiguous()
    return codes, pairs.reshape(Np // 16, 16, Kp // group, 2).transpose(1, 2).contiguous()


def _cache(gen, case, lengths, capacity):
    """A cache whose first `lengths` slots hold quantised keys (with channels that stand out, as keys
    have) and values; what lies beyond them is whatever was there before."""
    B, H, D, group = case["B"], case["heads"], case["D"], case["group"]
    c = {}
    for name in ("k", "v"):
        x = torch.randn(B, H, capacity, D, generator=gen, device="cuda")
        if name == "k":
            x += 2.0 * torch.randn(H, 1, D, generator=gen, device="cuda") * (torch.rand(H, 1, D, generator=gen, device="cuda") < 0.1)
        codes, pairs = _quantise(x, group)
        c[name + "_codes"], c[name + "_pairs"] = _pack(codes), pairs
        del x, codes
    c["state"] = torch.tensor([[n, n + 100, 0, 0] for n in lengths], dtype=torch.int32).cuda()
    # weights accumulated over some twenty steps fall off fast, and a part of the slots has none at all
    w = torch.empty(B, H, capacity, device="cuda").exponential_(1.0, generator=gen) ** 3 * (3.0 / capacity)
    c["weight"] = w * (torch.rand(B, H, capacity, generator=gen, device="cuda") < 0.9)
    # slots hold tokens in the order of their positions, from which 100 have left
    at = torch.arange(capacity, dtype=torch.int32, device="cuda")
    c["position"] = torch.where(at < 10, at, at + 100).expand(B, H, capacity).contiguous()
    return c


def _handle(c):
    import paper_2410_18311_b200 as ci
    return ci.make_kv4_cache(c["k_codes"], c["k_pairs"], c["v_codes"], c["v_pairs"], c["state"], c["weight"], c["position"])


def _scratch(n):
    return torch.empty(max(1, n), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if own:
        import paper_2410_18311_b200 as ci
        s["ci"] = ci
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    if case["op"] == "matvec":
        N, K, m, out = case["N"], case["K"], case["batch"], DTYPES[case["out"]]
        s["codes"], s["pairs"] = _weights(gen, N, K, case["group"])
        s["x"] = rand(m, K).to(dt)
        s["bias"] = (0.1 * rand(N)).to(dt) if case["bias"] else None
        s["mul"] = rand(m, N).to(out) if case["mul"] else None
        s["y"] = torch.empty(m, N, dtype=out, device="cuda")
        if own:
            s["w"] = ci.make_w4_matrix(s["codes"], s["pairs"], N, K, case["group"])
            s["act_code"] = {"none": ci.ACT_NONE, "relu": ci.ACT_RELU, "silu": ci.ACT_SILU}[case["act"]]
        return s
    B, H, D = case["B"], case["heads"], case["D"]
    lengths = {"append": lambda: [0] * B, "step": lambda: [case["length"]] * B}.get(case["op"], lambda: _lengths(case))()
    s["cache"] = _cache(gen, case, lengths, case["capacity"])
    if case["op"] == "attend":
        s["q"] = rand(B, case["T"], case["q_heads"], D).to(dt)
        s["out"] = torch.empty_like(s["q"])
    if case["op"] in ("append", "step"):
        s["k"], s["v"] = rand(B, case["T"], H, D).to(dt), rand(B, case["T"], H, D).to(dt)
        s["k_stored"], s["v_stored"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
    if case["op"] == "evict":
        small = 16 * -(-case["budget"] // 16)
        s["small"] = {n: torch.zeros(B, H, small, *t.shape[3:], dtype=t.dtype, device="cuda") for n, t in s["cache"].items() if n != "state"}
        s["small"]["state"] = torch.zeros(B, 4, dtype=torch.int32, device="cuda")
    if own:
        s["h"] = _handle(s["cache"])
        if case["op"] == "attend":
            s["ws"] = _scratch(ci.coreinfer_kv4_attention_workspace_bytes(s["h"], case["q_heads"], case["T"]))
        if case["op"] in ("step", "evict"):
            s["ws"] = _scratch(ci.coreinfer_kv4_evict_workspace_bytes(s["h"]))
        if case["op"] == "evict":
            s["h_small"] = _handle(s["small"])
    return s


# -------------------------------------------------------------------------------------- run --

def _plain_matvec(s):
    c, codes, pairs = s["case"], s["codes"], s["pairs"]
    N, K = c["N"], c["K"]
    w = _values(_unpack(codes).transpose(1, 2).reshape(16 * codes.shape[0], -1), pairs.transpose(1, 2).reshape(16 * pairs.shape[0], -1, 2))
    y = s["x"].float() @ w[:N, :K].t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if c["act"] == "relu":
        y = y.clamp(min=0)
    elif c["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    if s["mul"] is not None:
        y = y * s["mul"].float()
    s["y"].copy_(y)


def _plain_append(s):
    """New tokens at the end of each sequence; their values as the cache holds them."""
    c, cache = s["case"], s["cache"]
    B, H, T, st = c["B"], c["heads"], c["T"], cache["state"]
    b = torch.arange(B, device="cuda")[:, None, None]
    h = torch.arange(H, device="cuda")[None, :, None]
    t = torch.arange(T, dtype=torch.int32, device="cuda")
    at = (st[:, :1] + t)[:, None, :].long()
    stored = (("k", s["k"], s["k_stored"]), ("v", s["v"], s["v_stored"]))
    _ = [_plain_put(cache, name, x, to, (b, h, at), c["group"]) for name, x, to in stored]
    cache["weight"][b, h, at] = 0.0
    cache["position"][b, h, at] = (st[:, 1:2] + t)[:, None, :].expand(B, H, T)
    st[:, :2] += T


def _plain_put(cache, name, x, to, at, group):
    codes, pairs = _quantise(x.float().transpose(1, 2), group)
    cache[name + "_codes"][at] = _pack(codes)
    cache[name + "_pairs"][at] = pairs
    to.copy_(_values(codes.float(), pairs).transpose(1, 2))


def _plain_attend(s):
    c, cache = s["case"], s["cache"]
    B, H, T, D, n = c["B"], c["heads"], c["T"], c["D"], c["capacity"]
    k, v = _values(_unpack(cache["k_codes"]), cache["k_pairs"]), _values(_unpack(cache["v_codes"]), cache["v_pairs"])
    q = s["q"].float().reshape(B, T, H, -1, D)
    logits = torch.einsum("bthgd,bhnd->bhtgn", q, k) / math.sqrt(D)
    # a new token sees the slots up to its own, which is one of the last T
    limit = cache["state"][:, :1] - (T - 1 - torch.arange(T, device="cuda"))
    seen = (torch.arange(n, device="cuda") < limit[:, :, None])[:, None, :, None, :]
    logits = torch.where(seen, logits, torch.full_like(logits, -torch.inf))
    top = logits.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(logits - top), torch.zeros_like(logits))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    s["out"].copy_(torch.einsum("bhtgn,bhnd->bthgd", p, v).reshape(s["out"].shape))
    if c["accumulate"]:
        cache["weight"] += p.sum((2, 3))


def _plain_kept(cache, budget, recent, first):
    """Which slots stay: the first and the recent tokens, then the largest weights, ties to the lower slot."""
    n, seen = cache["state"][:, 0], cache["state"][:, 1]
    slot = torch.arange(cache["weight"].shape[2], device="cuda")
    live = (slot < n[:, None])[:, None, :]
    must = (cache["position"] >= (seen - recent)[:, None, None]) | (cache["position"] < first)
    key = torch.where(must, torch.full_like(cache["weight"], torch.inf), cache["weight"])
    key = torch.where(live, key, torch.full_like(key, -torch.inf))
    rank = torch.argsort(torch.argsort(key, dim=-1, descending=True, stable=True), dim=-1, stable=True)
    keep = n.clamp(max=budget)
    return live & (rank < keep[:, None, None]), keep


def _plain_evict_to(src, dst, c):
    kept, keep = _plain_kept(src, c["budget"], c["recent"], c["first"])
    order = torch.argsort(kept.to(torch.uint8), dim=-1, descending=True, stable=True)[..., : min(c["budget"], kept.shape[2])]
    B, H, m = order.shape
    live = (torch.arange(m, device="cuda") < keep[:, None])[:, None, :].expand(B, H, m)
    _ = [_plain_take(src[name], dst[name], order, live) for name in ("k_codes", "k_pairs", "v_codes", "v_pairs", "weight", "position")]
    dst["state"][:, 0] = keep
    dst["state"][:, 1] = src["state"][:, 1]


def _plain_take(src, dst, order, live):
    at = order.reshape(*order.shape, *[1] * (src.dim() - 3)).expand(*order.shape, *src.shape[3:])
    to = dst[:, :, : order.shape[2]]
    ok = live.reshape(*live.shape, *[1] * (src.dim() - 3))
    to.copy_(torch.where(ok, torch.gather(src, 2, at), to))


def _plain_evict_here(cache, c):
    """In place: the kept slots beyond the budget move, in order, into the free ones below it."""
    kept, keep = _plain_kept(cache, c["budget"], c["recent"], c["first"])
    slot = torch.arange(kept.shape[2], device="cuda")
    low = slot < keep[:, None, None]
    hole, mover = low & ~kept, ~low & kept
    b, h, to = torch.nonzero(hole, as_tuple=True)       # holes and movers of a head are as many, both in ascending order
    src = torch.nonzero(mover, as_tuple=True)[2]
    names = ("k_codes", "k_pairs", "v_codes", "v_pairs", "weight", "position")
    _ = [cache[n].index_put_((b, h, to), cache[n][b, h, src]) for n in names]
    cache["state"][:, 0] = keep


def run(s):
    c = s["case"]
    op = c["op"]
    if op == "matvec":
        if own:
            s["ci"].coreinfer_w4_matvec(s["w"], s["x"], s["act_code"], s["bias"], s["mul"], s["y"])
        else:
            _plain_matvec(s)
        return {"y": s["y"]}
    cache = s["cache"]
    if op == "attend":
        if own:
            s["ci"].coreinfer_kv4_attention(s["h"], s["q"], 1.0 / math.sqrt(c["D"]), s["out"], c["accumulate"], s["ws"])
        else:
            _plain_attend(s)
        return {"out": s["out"], "weight": cache["weight"] if c["accumulate"] else None}
    if op == "evict":
        if own:
            s["ci"].coreinfer_kv4_evict(s["h"], s["h_small"], c["budget"], c["recent"], c["first"], s["ws"])
        else:
            _plain_evict_to(cache, s["small"], c)
        return dict(s["small"])                         # codes are moved, not computed: they come back as they are held
    if op == "append":
        cache["state"].zero_()                          # a new conversation takes the cache
    if own:
        s["ci"].coreinfer_kv4_append(s["h"], s["k"], s["v"], s["k_stored"], s["v_stored"])
    else:
        _plain_append(s)
    r = {"k_stored": s["k_stored"], "v_stored": s["v_stored"], "state": cache["state"], "position": cache["position"],
         "weight": cache["weight"]}
    if op == "step":
        if own:
            s["ci"].coreinfer_kv4_evict(s["h"], s["h"], c["budget"], c["recent"], c["first"], s["ws"])
        else:
            _plain_evict_here(cache, c)
        r.update({name: cache[name] for name in ("k_codes", "k_pairs", "v_codes", "v_pairs")})
    return r


# ------------------------------------------------------------------------------------ exact --

def _exact_values(packed, pairs):
    """The values of rows of packed codes, value by value from the format's rule, in 64 bits."""
    d = 2 * packed.shape[-1]
    i = torch.arange(d, device="cuda")
    h, lane, e = i // 32, (i % 32) // 4, i % 4
    byte = 2 * (lane * (d // 32) + h) + e // 2
    code = (packed[..., byte].to(torch.int64) >> (4 * (e % 2))) & 15
    pair = pairs.double().repeat_interleave(d // pairs.shape[-2], dim=-2)
    return code.double() * pair[..., 0] + pair[..., 1]


def _exact_stored(x, group):
    g = x.double().unflatten(-1, (-1, group))
    o = g.min(-1, keepdim=True).values.to(torch.float16).double()
    s = ((g.max(-1, keepdim=True).values - g.min(-1, keepdim=True).values) / 15).to(torch.float16).double()
    code = torch.where(s > 0, torch.round((g - o) / s), torch.zeros_like(g))
    return (code.clamp(0, 15) * s + o).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "matvec":
        y = torch.empty(case["batch"], case["N"], dtype=torch.float64, device="cuda")
        x = s["x"].double()
        for r in range(s["codes"].shape[0]):            # 16 rows at a time
            n = min(16, case["N"] - 16 * r)
            pairs = s["pairs"][r].transpose(0, 1)       # [16, groups, 2]
            per = 128 // case["group"]
            w = _exact_values(s["codes"][r][:, :n].transpose(0, 1), pairs[:n].unflatten(1, (-1, per))).flatten(1)
            y[:, 16 * r : 16 * r + n] = x @ w[:, : case["K"]].t()
        if s["bias"] is not None:
            y += s["bias"].double()
        y = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t * torch.sigmoid(t)}[case["act"]](y)
        return {"y": y if s["mul"] is None else y * s["mul"].double()}
    cache, B, H = s["cache"], case["B"], case["heads"]
    if op == "attend":
        D, T = case["D"], case["T"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        weight = cache["weight"].double()
        for b, n in enumerate(_lengths(case)):
            for h in range(H):
                k = _exact_values(cache["k_codes"][b, h, :n], cache["k_pairs"][b, h, :n])
                v = _exact_values(cache["v_codes"][b, h, :n], cache["v_pairs"][b, h, :n])
                share = case["q_heads"] // H
                for t in range(T):
                    m = n - (T - 1 - t)
                    if m <= 0:
                        continue
                    p = torch.softmax(s["q"][b, t, h * share : (h + 1) * share].double() @ k[:m].t() * D ** -0.5, -1)
                    out[b, t, h * share : (h + 1) * share] = p @ v[:m]
                    weight[b, h, :m] += p.sum(0)
        return {"out": out, "weight": weight if case["accumulate"] else None}
    weight, position = cache["weight"].double().cpu(), cache["position"].cpu()
    r = {"state": None, "position": None}
    if op != "append":
        r.update(k_codes=None, k_pairs=None, v_codes=None, v_pairs=None)
    if op in ("append", "step"):
        T = case["T"]
        r["k_stored"], r["v_stored"] = _exact_stored(s["k"], case["group"]), _exact_stored(s["v"], case["group"])
        n = 0 if op == "append" else case["length"]
        weight[:, :, n : n + T] = 0
        position[:, :, n : n + T] = (0 if op == "append" else n + 100) + torch.arange(T)
        if op == "append":
            return {**r, "weight": weight}
        lengths = [n + T] * B
    else:
        lengths = _lengths(case)
        new = torch.zeros(s["small"]["weight"].shape, dtype=torch.float64)
    for b, n in enumerate(lengths):
        seen = n + 100
        keep = min(n, case["budget"])
        for h in range(H):
            w, p = weight[b, h, :n].numpy(), position[b, h, :n].numpy()
            safe = (p >= seen - case["recent"]) | (p < case["first"])
            stay = np.sort(np.lexsort((np.arange(n), np.where(safe, 0.0, -w), ~safe))[:keep])
            if op == "evict":
                new[b, h, :keep] = torch.from_numpy(w[stay])
            else:
                w[np.setdiff1d(np.arange(keep), stay)] = w[stay[stay >= keep]]
    return {**r, "weight": new if op == "evict" else weight}
