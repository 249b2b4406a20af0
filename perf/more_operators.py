"""What is measured of the operators around attention in 16 and 32 bits: rotary positions with the norms of
queries and keys (rope), tokens that enter a paged key/value cache with both on the way (append), and attention of
a chunk of new tokens over that cache, from one token to whole prompts, with a sliding window and first tokens
that stay visible (attend).

Each case is a dict of plain values; `prepare` makes its inputs on the GPU from a seed, `run` is one pass
through an operator as a decoder layer calls it (`own`: the framework's kernels; otherwise the plain torch form in
32 bits), `exact` the same from the definition in 64 bits, `work` the bytes and operations that a pass cannot do without.

A batch of B sequences is packed: tokens start[b] .. start[b + 1] - 1 belong to sequence b, rows behind start[B] to
none.  A cache is two pools [pages, kv heads, page size, head dim] (or with tokens before heads, "order"), a table
[B, pages of a sequence] and the lengths, which count the call's own tokens: token t of the n new ones of a sequence
is at position length - n + t, in slot position % page size of page table[b, position // page size].
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5                                                       # of the norms


# ------------------------------------------------------------------------------------ cases --

def listed():
    plain = {"scaling": "plain", "factor": 1.0, "context": 0, "base": 10000.0}
    return [
        # queries and keys of one token of the one-layer fp32 configuration: the smallest call, latency counts
        {"name": "rope token f32", "op": "rope", "tokens": 1, "q_heads": 12, "heads": 12, "D": 64, "rot": 64, "interleaved": False,
         "norm": False, "far": 100, "dtype": "f32", **plain},
        # a long prompt, head norms, neighbouring pairs of half the head turned, contexts stretched 16 times
        {"name": "rope norm 8191 f16", "op": "rope", "tokens": 8191, "q_heads": 32, "heads": 8, "D": 128, "rot": 64, "interleaved": True,
         "norm": True, "far": 120000, "dtype": "f16", "scaling": "yarn", "factor": 16.0, "context": 8192, "base": 500000.0},
        # one decode step of eight sequences, a key head per query head
        {"name": "append step 8 bf16", "op": "append", "B": 8, "T": 1, "length": 4001, "q_heads": 32, "heads": 32, "D": 128, "rot": 128,
         "interleaved": False, "norm": False, "page": 16, "order": "heads", "pad": 0, "mix": False, "dtype": "bf16", **plain},
        # pieces of three prompts enter together, head norms, wavelengths stretched where they are long
        {"name": "append pieces bf16", "op": "append", "B": 3, "T": 2000, "length": 9000, "q_heads": 32, "heads": 8, "D": 128, "rot": 128,
         "interleaved": False, "norm": True, "page": 64, "order": "tokens", "pad": 40, "mix": False, "dtype": "bf16",
         "scaling": "bands", "factor": 8.0, "context": 8192, "base": 500000.0},
        # a short prompt in fp32
        {"name": "append prompt f32", "op": "append", "B": 2, "T": 333, "length": 400, "q_heads": 12, "heads": 12, "D": 64, "rot": 64,
         "interleaved": True, "norm": False, "page": 16, "order": "heads", "pad": 0, "mix": False, "dtype": "f32", **plain},
        # a short conversation on the one-layer fp32 configuration's heads: latency counts
        {"name": "attend short f32", "op": "attend", "B": 1, "T": 1, "length": 77, "q_heads": 12, "heads": 12, "D": 64, "page": 16,
         "order": "heads", "pad": 0, "mix": False, "window": 0, "sinks": 0, "dtype": "f32"},
        # ordinary decoding, a key head per query head
        {"name": "attend 8 x 4001 bf16", "op": "attend", "B": 8, "T": 1, "length": 4001, "q_heads": 32, "heads": 32, "D": 128, "page": 16,
         "order": "tokens", "pad": 0, "mix": False, "window": 0, "sinks": 0, "dtype": "bf16"},
        # two long documents, grouped heads
        {"name": "attend long 130000 f16", "op": "attend", "B": 2, "T": 1, "length": 130000, "q_heads": 32, "heads": 8, "D": 128, "page": 64,
         "order": "heads", "pad": 0, "mix": False, "window": 0, "sinks": 0, "dtype": "f16"},
        # three drafted tokens a sequence are checked at once through a window, five query heads per key head
        {"name": "attend draft window bf16", "op": "attend", "B": 6, "T": 3, "length": 9000, "q_heads": 40, "heads": 8, "D": 128, "page": 32,
         "order": "heads", "pad": 3, "mix": False, "window": 4096, "sinks": 4, "dtype": "bf16"},
        # a piece of a long prompt over what is in the cache already
        {"name": "attend piece 500 f16", "op": "attend", "B": 1, "T": 500, "length": 16001, "q_heads": 40, "heads": 8, "D": 128, "page": 64,
         "order": "heads", "pad": 12, "mix": False, "window": 0, "sinks": 0, "dtype": "f16"},
        # a whole prompt, a key head per query head
        {"name": "attend prompt 8192 bf16", "op": "attend", "B": 1, "T": 8192, "length": 8192, "q_heads": 32, "heads": 32, "D": 128, "page": 128,
         "order": "heads", "pad": 0, "mix": False, "window": 0, "sinks": 0, "dtype": "bf16"},
        # decoding sequences and pieces of prompts in one batch, a window with first tokens, small heads
        {"name": "attend mixed window f16", "op": "attend", "B": 7, "T": 2000, "length": 5000, "q_heads": 32, "heads": 8, "D": 64, "page": 16,
         "order": "tokens", "pad": 0, "mix": True, "window": 1024, "sinks": 4, "dtype": "f16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(("rope", "append", "attend", "attend", "attend"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    D = rng.choice((64, 128, 128, 256))
    heads, share = rng.choice((1, 2, 4, 8, 12, 32)), rng.choice((1, 1, 2, 4, 5, 8))
    case = {"op": op, "dtype": dtype, "D": D, "heads": heads, "q_heads": heads * share}
    if op != "attend":
        case.update(rot=rng.choice((D, D, D // 2, 32)), interleaved=rng.random() < 0.5, norm=rng.random() < 0.5)
        case.update(rng.choice(({"scaling": "plain", "factor": 1.0, "context": 0, "base": 10000.0},
                                {"scaling": "linear", "factor": 4.0, "context": 0, "base": 10000.0},
                                {"scaling": "ntk", "factor": 2.0, "context": 0, "base": 10000.0},
                                {"scaling": "yarn", "factor": 8.0, "context": 4096, "base": 10000.0},
                                {"scaling": "bands", "factor": 8.0, "context": 8192, "base": 500000.0})))
    wide = (heads + 2 * heads * share) * D * BYTES[dtype]
    if op == "rope":
        return {**case, "tokens": _log(rng, 1, min(20000, 160000000 // wide)), "far": _log(rng, 10, 1000000)}
    case.update(page=rng.choice((16, 32, 64, 128)), order=rng.choice(("heads", "tokens")), pad=rng.choice((0, 0, 1, 17)),
                mix=rng.random() < 0.25, B=rng.choice((1, 1, 2, 3, 5, 8, 16)))
    B = case["B"]
    if op == "append":
        T = rng.choice((1, _log(rng, 1, min(4000, 160000000 // (wide * B)))))
        return {**case, "T": T, "length": T + _log(rng, 1, min(20000, 400000000 // (heads * D * BYTES[dtype] * 2 * B)))}
    T = rng.choice((1, 1, rng.randint(2, 9), _log(rng, 10, 4000)))
    # within the largest listed prompt's products (a twentieth of them in fp32), the longest listed cache's bytes and room for the plain form
    most = min((5e11 if dtype != "f32" else 2.5e10) / (4 * T * B * heads * share * D), 1e9 / (B * heads * D * 2 * BYTES[dtype]),
               2e9 / (B * heads * share * T), 130000)
    if most < T:
        T = max(1, int(math.sqrt(T * most)) // 2)
    window = rng.choice((0, 0, 0, 128, 1000, 4096))
    return {**case, "T": T, "length": _log(rng, T, max(T, int(most))), "window": window, "sinks": rng.choice((0, 4, 130)) if window else 0}


def _batch(case):
    """New tokens and lengths (those among them) of the sequences, ragged, the first the longest; the same for every seed."""
    n = [max(1, case["T"] - int(case["T"] * 0.6 * ((0.618 * b) % 1.0))) for b in range(case["B"])]
    if case["mix"]:
        n = [1 if b % 2 else x for b, x in enumerate(n)]
    length = [max(n[b], case["length"] - int(case["length"] * 0.5 * ((0.618 * b) % 1.0))) for b in range(case["B"])]
    return n, length


def _pairs(case):
    """Pairs of a new token and a slot that it sees, and the slots that some token of their sequence sees."""
    w, s = case["window"], case["sinks"]
    pairs, slots = 0, 0
    for n, length in zip(*_batch(case)):
        if not w:
            pairs += n * (2 * length - n + 1) // 2
            slots += length
            continue
        seen = [min(p + 1, w) + max(0, min(s, p + 1 - w)) for p in range(length - n, length)]
        pairs += sum(seen)
        slots += min(length, w + n - 1) + max(0, min(s, length - n + 1 - w))
    return pairs, slots


def work(case):
    e, D, H, Hq = BYTES[case["dtype"]], case["D"], case["heads"], case["q_heads"]
    if case["op"] == "rope":
        n = case["tokens"]
        return {"bytes": n * ((Hq + H) * D * 2 * e + 4), "flops": n * (Hq + H) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    new, length = _batch(case)
    n = sum(new)
    if case["op"] == "append":
        return {"bytes": n * (Hq + 2 * H) * D * 2 * e, "flops": n * (Hq + H) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    pairs, slots = _pairs(case)
    return {"bytes": slots * H * D * 2 * e + 2 * n * Hq * D * e, "flops": 4 * pairs * Hq * D}


# ---------------------------------------------------------------------------------- prepare --

def _frequencies(case):
    """Radians a position for each pair of dimensions (64 bits), and what cosines and sines are multiplied by."""
    rot, base, factor, context = case["rot"], case["base"], case["factor"], case["context"]
    i = torch.arange(rot // 2, dtype=torch.float64)
    if case["scaling"] == "ntk":
        base *= factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "yarn":                                # dimensions that turn 32 times in a context stay, those that turn less than once are stretched
        at = lambda turns: rot * math.log(context / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(0, math.floor(at(32.0))), min(rot - 1, math.ceil(at(1.0)))
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1
    if case["scaling"] == "bands":                               # by wavelength: above a context stretched, below a quarter of it not
        s = ((context * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return (1 - s) * f / factor + s * f, 1.0
    return f, 1.0


def _rope(s, case, gen, dt):
    f, s["magnitude"] = _frequencies(case)
    s["f"] = f.cuda()
    s["q_norm"], s["k_norm"] = ((1 + 0.1 * torch.randn(case["D"], generator=gen, device="cuda")).to(dt) if case["norm"] else None for _ in "qk")
    if own:
        import paper_2410_18311_b200 as ci
        kind = {"plain": ci.ROPE_PLAIN, "linear": ci.ROPE_LINEAR, "ntk": ci.ROPE_NTK, "yarn": ci.ROPE_YARN, "bands": ci.ROPE_BANDS}[case["scaling"]]
        s["turns"], magnitude = ci.coreinfer_rope_frequencies(case["rot"], case["base"], kind, case["factor"], case["context"], device="cuda")
        s["rope"] = ci.make_rope(s["turns"], case["interleaved"], magnitude, s["q_norm"], s["k_norm"], EPS)


def _cache(s, case, gen, dt):
    """Pools whose pages lie in random order, some of them nobody's; lengths, table and the packing of the batch."""
    B, H, D, page = case["B"], case["heads"], case["D"], case["page"]
    new, length = _batch(case)
    need = [-(-n // page) for n in length]
    width = max(need) + 1
    spare = 3
    order = torch.randperm(sum(need) + spare, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros(B, width, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at : at + n]
        at += n
    shape = (sum(need) + spare, page, H, D) if case["order"] == "tokens" else (sum(need) + spare, H, page, D)
    for name in ("k", "v"):
        pool = torch.randn(shape, generator=gen, device="cuda").to(dt)
        if name == "k":                                          # channels that stand out, as keys have
            pool *= torch.where(torch.rand(D, generator=gen, device="cuda") < 0.05, 3.0, 1.0).to(dt)
        s[name + "_pool"] = pool.transpose(1, 2) if case["order"] == "tokens" else pool
    s["table"], s["length"] = table, torch.tensor(length, dtype=torch.int32).cuda()
    s["start"] = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32).cuda()
    if own:
        import paper_2410_18311_b200 as ci
        s["ci"] = ci
        s["h"] = ci.make_paged_cache(s["k_pool"], s["v_pool"], table, s["length"])
    return sum(new) + case["pad"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, H, Hq, D = DTYPES[case["dtype"]], case["heads"], case["q_heads"], case["D"]
    s = {"case": case}
    if own:
        import paper_2410_18311_b200 as ci
        s["ci"] = ci
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(dt)  # noqa: E731
    if case["op"] == "rope":
        n = case["tokens"]
        _rope(s, case, gen, dt)
        s["positions"] = torch.randint(0, case["far"], (n,), generator=gen, device="cuda", dtype=torch.int32)
        s["qkv"] = rand(n, (Hq + 2 * H) * D)                     # a projection's output, of which queries and keys are slices
        s["q_out"], s["k_out"] = (torch.zeros(n, h, D, dtype=dt, device="cuda") for h in (Hq, H))
        return s
    n = _cache(s, case, gen, dt)
    if case["op"] == "append":
        _rope(s, case, gen, dt)
        s["qkv"] = rand(n, (Hq + 2 * H) * D)
        s["q_out"] = torch.zeros(n, Hq, D, dtype=dt, device="cuda")
        return s
    s["q"] = rand(n, Hq, D)
    s["out"] = torch.zeros(n, Hq, D, dtype=dt, device="cuda")
    if own:
        s["ws"] = torch.empty(max(1, ci.coreinfer_paged_attention_workspace_bytes(s["h"], Hq, n)), dtype=torch.uint8, device="cuda")
    return s


def _split(s):
    c, x = s["case"], s["qkv"]
    Hq, H, D = c["q_heads"], c["heads"], c["D"]
    q, k, v = x.split((Hq * D, H * D, H * D), -1)
    return q.unflatten(-1, (Hq, D)), k.unflatten(-1, (H, D)), v.unflatten(-1, (H, D))


# -------------------------------------------------------------------------------------- run --

def _plain_turn(s, x, weight, positions):
    """Norm of each head and rotation by its token's position, in 32 bits (the angles in 64)."""
    c, rot = s["case"], s["case"]["rot"]
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    angle = positions.double()[:, None] * s["f"]
    cos, sin = (s["magnitude"] * torch.cos(angle)).float()[:, None], (s["magnitude"] * torch.sin(angle)).float()[:, None]
    if c["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2 : rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_tokens(s, n):
    """Sequence, number among the new tokens, and position of each of n packed rows; rows that are nobody's last."""
    start, length = s["start"].long(), s["length"].long()
    i = torch.arange(n, device="cuda")
    b = (torch.searchsorted(start, i, right=True) - 1).clamp(max=len(length) - 1)
    return b, i - start[b], length[b] - start[b + 1] + i


def _plain_append(s):
    c = s["case"]
    n = s["qkv"].shape[0] - c["pad"]
    b, _, position = _plain_tokens(s, n)
    q, k, v = _split(s)
    s["q_out"][:n] = _plain_turn(s, q[:n], s["q_norm"], position).to(s["q_out"].dtype)
    page, slot = s["table"][b, position // c["page"]].long(), position % c["page"]
    s["k_pool"][page, :, slot] = _plain_turn(s, k[:n], s["k_norm"], position).to(k.dtype)
    s["v_pool"][page, :, slot] = v[:n]


def _plain_attend(s):
    c = s["case"]
    B, H, D = c["B"], c["heads"], c["D"]
    n = s["q"].shape[0] - c["pad"]
    k, v = (s[p][s["table"].long()].transpose(1, 2).reshape(B, H, -1, D).float() for p in ("k_pool", "v_pool"))
    first, length = s["start"].long(), s["length"].long()
    t = torch.arange(c["T"], device="cuda")
    row = (first[:-1, None] + t).clamp(max=n - 1)
    q = s["q"][row].float().reshape(B, c["T"], H, -1, D)
    logits = torch.einsum("bthgd,bhnd->bhtgn", q, k)
    logits *= 1 / math.sqrt(D)
    position = (length - first[1:] + first[:-1])[:, None, None] + t[:, None]
    slot = torch.arange(k.shape[2], device="cuda")
    seen = slot <= position
    if c["window"]:
        seen &= (slot > position - c["window"]) | (slot < c["sinks"])
    # rows behind a sequence's own are not taken below; as the others they see a slot at least
    logits.masked_fill_(~seen[:, None, :, None, :], -torch.inf)
    logits -= logits.amax(-1, keepdim=True)
    p = logits.exp_()
    p /= p.sum(-1, keepdim=True)
    out = torch.einsum("bhtgn,bhnd->bthgd", p, v).reshape(B, c["T"], -1, D)
    b, t, _ = _plain_tokens(s, n)
    s["out"][:n] = out[b, t].to(s["out"].dtype)


def run(s):
    c = s["case"]
    if c["op"] == "rope":
        q, k, _ = _split(s)
        if own:
            s["ci"].coreinfer_rope_apply(s["rope"], s["positions"], q, k, s["q_out"], s["k_out"])
        else:
            s["q_out"].copy_(_plain_turn(s, q, s["q_norm"], s["positions"]))
            s["k_out"].copy_(_plain_turn(s, k, s["k_norm"], s["positions"]))
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["op"] == "append":
        if own:
            q, k, v = _split(s)
            s["ci"].coreinfer_paged_append(s["h"], s["start"], k, v, s["rope"], None, q, s["q_out"])
        else:
            _plain_append(s)
        return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}
    if own:
        s["ci"].coreinfer_paged_attention(s["h"], s["start"], s["q"], 1 / math.sqrt(c["D"]), s["out"], s["ws"], c["window"], c["sinks"])
    else:
        _plain_attend(s)
    return {"out": s["out"]}


# ------------------------------------------------------------------------------------ exact --

def _exact_turn(case, x, weight, positions):
    """Each pair of dimensions as a complex number times e^(i angle)."""
    x = x.double()
    if weight is not None:
        x = x / (x.square().sum(-1, keepdim=True) / case["D"] + EPS).sqrt() * weight.double()
    f, magnitude = _frequencies(case)
    rot = case["rot"]
    angle = torch.outer(positions.double(), f.cuda())
    turn = torch.polar(torch.full_like(angle, magnitude), angle)[:, None]
    out = x.clone()
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(x[..., one], x[..., two]) * turn
    out[..., one], out[..., two] = z.real, z.imag
    return out


def exact(case, seed):
    s = prepare(case, seed)
    D, Hq, H = case["D"], case["q_heads"], case["heads"]
    if case["op"] == "rope":
        q, k, _ = _split(s)
        return {"q": _exact_turn(case, q, s["q_norm"], s["positions"]), "k": _exact_turn(case, k, s["k_norm"], s["positions"])}
    new, length = _batch(case)
    page, table = case["page"], s["table"].cpu()
    if case["op"] == "append":
        q, k, v = _split(s)
        out, pools = s["q_out"].double(), [s["k_pool"].double(), s["v_pool"].double()]
        at = 0
        for b, n in enumerate(new):
            position = torch.arange(length[b] - n, length[b])
            rows = slice(at, at + n)
            out[rows] = _exact_turn(case, q[rows], s["q_norm"], position.cuda())
            where = (table[b, position // page].long().cuda(), slice(None), (position % page).cuda())
            pools[0][where] = _exact_turn(case, k[rows], s["k_norm"], position.cuda())
            pools[1][where] = v[rows].double()
            at += n
        return {"q": out, "k": pools[0], "v": pools[1]}
    if 4.0 * _pairs(case)[0] * Hq * D > 2e12:
        return None
    out = s["out"].double()
    w, sinks, share, at = case["window"], case["sinks"], Hq // H, 0
    for b, (n, m) in enumerate(zip(new, length)):
        pages = table[b, : -(-m // page)].long().cuda()
        slot = torch.arange(m, device="cuda")
        for h in range(H):
            k, v = (s[p][pages, h].flatten(0, 1)[:m].double() for p in ("k_pool", "v_pool"))
            step = max(1, 40000000 // (share * m))
            for t in range(0, n, step):
                rows = torch.arange(t, min(n, t + step), device="cuda")
                position = (m - n + rows)[:, None, None]
                hidden = slot > position
                if w:
                    hidden = hidden | ((slot <= position - w) & (slot >= sinks))
                logits = s["q"][at + rows, h * share : (h + 1) * share].double() @ k.t() / math.sqrt(D)
                out[at + rows, h * share : (h + 1) * share] = torch.softmax(logits.masked_fill(hidden, -torch.inf), -1) @ v
        at += n
    return {"out": out}
