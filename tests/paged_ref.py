"""Plain 64-bit forms of rotary positions with head norms and of attention over a paged cache, written from the formulas."""
import math

import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS32 = 2.0 ** -24
OUT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # half a step of a rounding


def frequencies(rot, base, kind="plain", factor=1.0, context=0, low=1.0, high=None):
    """Radians a position of each pair, pair by pair from the definitions; and the magnitude."""
    f = []
    if kind == "ntk":
        base = base * factor ** (rot / (rot - 2))
    for i in range(rot // 2):
        x = base ** (-2 * i / rot)
        if kind == "linear":
            x /= factor
        if kind == "yarn":
            pair = lambda turns: rot / 2 * math.log(context / (2 * math.pi * turns), base)
            a, b = max(0, math.floor(pair(32.0 if high is None else high))), min(rot - 1, math.ceil(pair(low)))
            r = min(1.0, max(0.0, (i - a) / max(b - a, 0.001)))
            x = x * (1 - r) + x / factor * r
        if kind == "bands":
            turns = context * x / (2 * math.pi)                  # in the original context
            hi = 4.0 if high is None else high
            s = min(1.0, max(0.0, (turns - low) / (hi - low)))
            x = s * x + (1 - s) * x / factor
        f.append(x)
    return torch.tensor(f, dtype=torch.float64), 0.1 * math.log(factor) + 1 if kind == "yarn" else 1.0


def turn(x, positions, f, magnitude, interleaved, weight=None, eps=0.0):
    """x [tokens, heads, D] -> (64-bit result, bound of the error of its computation in fp32).

    The norm: a sum of D squares (relative error at most D / 8 + 8 spacings, as eight lanes' worth or more are added apart), its
    root halves that; root, products: 4 more.  The rotation: cosine and sine are off by at most 2 spacings of 1 and by the angle's
    2.3e-8 (less than a spacing); their product with the magnitude, the two products and the sum: 4 more of |a| + |b|."""
    x = x.double().cpu()
    D, rot = x.shape[-1], 2 * len(f)
    rel = torch.zeros(())
    if weight is not None:
        x = x / ((x * x).sum(-1, keepdim=True) / D + eps).sqrt() * weight.double().cpu()
        rel = torch.tensor((D / 8 + 8) / 2 + 4)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    angle = positions.cpu().double()[:, None, None] * f
    cos, sin = angle.cos() * magnitude, angle.sin() * magnitude
    y, tol = x.clone(), x.abs() * rel * EPS32
    t = (a.abs() + b.abs()) * magnitude * (8 + rel) * EPS32
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
        tol[..., 0:rot:2] = tol[..., 1:rot:2] = t
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
        tol[..., :rot // 2] = tol[..., rot // 2:rot] = t
    return y, tol


def check(got, want, tol, what=""):
    """|got - want| within tol and one rounding to got's type; NaN or infinite where `want` is, and NaN where that is NaN.  (An
    infinity may come out NaN: a weight, or one of its two parts, may be 0.)"""
    got64, want = got.double().cpu(), want.cpu()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got64), fine), what + ": not finite elsewhere"
    assert torch.isnan(got64[torch.isnan(want)]).all(), what + ": NaN"
    left = ~fine & ~torch.isnan(want) & ~torch.isnan(got64)
    assert torch.equal(got64[left], want[left]), what + ": infinities"
    bound = (tol.cpu() * 1.01 + OUT[got.dtype] * want.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 1e-38))[fine]
    err = (got64 - want).abs()[fine]
    assert (err <= bound).all(), "%s: worst %.3g of the bound" % (what, (err / bound).max().item())


class Batch:
    """Random pools and a packed batch.  new and length per sequence; `order` of the pools' axes; pages in random order with some
    that are nobody's; everything that no token holds is NaN."""

    def __init__(self, new, length, H, share, D, page, dtype, order="heads", seed=0, front=0, pad=0, spread=1.0, wide=0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.length_list, self.H, self.share, self.D, self.page, self.dt = new, length, H, share, D, page, DT[dtype]
        need = [-(-n // page) for n in length]
        self.n_pages = sum(need) + 2
        perm = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        table = torch.full((len(new), max(1, max(need)) + 1), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = perm[at:at + n]
            at += n
        shape = (self.n_pages, H, page, D + wide) if order == "heads" else (self.n_pages, page, H, D + wide)
        self.pools = []
        for _ in "kv":
            pool = torch.full(shape, float("nan"), dtype=self.dt)[..., :D]
            self.pools.append(pool if order == "heads" else pool.transpose(1, 2))
        for b, n in enumerate(length):
            for j in range(n):
                for pool in self.pools:
                    pool[table[b, j // page], :, j % page] = (torch.randn(H, D, generator=g) * spread).to(self.dt)
        # `.cuda()` would make a sliced view dense: the strides are part of what is tested
        self.k, self.v = (torch.empty_strided(p.shape, p.stride(), dtype=p.dtype, device="cuda").copy_(p) for p in self.pools)
        self.table, self.length = table.cuda(), torch.tensor(length, dtype=torch.int32).cuda()
        start = [front]
        for n in new:
            start.append(start[-1] + n)
        self.start, self.tokens = torch.tensor(start, dtype=torch.int32).cuda(), start[-1] + pad
        self.starts = start
        self.g = g

    def handle(self):
        import paper_2410_18311_b200 as ci
        return ci.make_paged_cache(self.k, self.v, self.table, self.length)

    def rand(self, heads, extra=0):
        """[tokens, heads, D], with `extra` values between the rows."""
        t = torch.randn(self.tokens, heads * self.D + extra, generator=self.g).to(self.dt).cuda()
        return t[:, :heads * self.D].unflatten(-1, (heads, self.D))

    def slots(self, b, n=None):
        """Keys and values [n, H, D] of sequence b in 64 bits, zeros for pages that are none."""
        n = self.length_list[b] if n is None else n
        cap = self.table.shape[1] * self.page
        out = []
        for pool in (self.k, self.v):
            x = torch.zeros(min(n, cap), self.H, self.D, dtype=torch.float64, device="cuda")
            table = self.table[b].cpu()
            for g in range(-(-min(n, cap) // self.page)):
                rows = min(self.page, min(n, cap) - g * self.page)
                if 0 <= table[g] < pool.shape[0]:
                    x[g * self.page:g * self.page + rows] = pool[table[g], :, :rows].transpose(0, 1).double()
            out.append(x)
        return out


def attention(batch, q, scale, window=0, sinks=0):
    """(64-bit outputs [tokens, Hq, D] with NaN rows where nobody's, bound of the error).

    A logit is a sum of D products in fp32: off by at most D / 4 + 36 spacings of its absolute terms (products in groups, every order of
    them), and by 2^-20 in its exponential.  An error e of a logit moves its weight and the sum by factors e^(+-e) each.  Weights enter
    the product with the values after at most one rounding to the cache's type (fp16: to steps of 2^-25 of the largest at least);
    the sums over n add n / 8 + 64 spacings at most."""
    D, share = batch.D, batch.share
    out = torch.full(q.shape, float("nan"), dtype=torch.float64, device="cuda")
    tol = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(batch.new):
        if not n:
            continue
        L = batch.length_list[b]
        k, v = batch.slots(b)
        slot = torch.arange(k.shape[0], device="cuda")
        position = torch.arange(L - n, L, device="cuda")[:, None]
        seen = slot <= position
        if window:
            seen &= (slot > position - window) | (slot < sinks)
        some = seen.any(-1)
        rows = slice(batch.starts[b], batch.starts[b] + n)
        for h in range(q.shape[1]):
            x, kh, vh = q[rows, h].double(), k[:, h // share], v[:, h // share]
            if not kh.shape[0]:
                out[rows, h] = 0
                continue
            kept = seen[:, :, None]
            logits = x @ kh.T if torch.isfinite(kh).all() else (x[:, None] * kh).sum(-1)
            logits = logits * scale
            logits = logits.masked_fill(~seen, -math.inf)
            p = torch.exp(logits - logits.amax(-1, keepdim=True))
            p = p / p.sum(-1, keepdim=True)
            if torch.isfinite(vh).all():
                o = p @ vh
            else:                                                # what is not seen is left out, not multiplied by 0; a weight is above 0
                o = (p[:, :, None].clamp(min=1e-300) * vh[None]).where(kept, 0.0).sum(1)
            out[rows, h] = torch.where(some[:, None], o, 0.0)
            av = vh.nan_to_num(0, 0, 0).abs()
            e = 2 * ((D / 4 + 36) * EPS32 * (x.abs() @ kh.nan_to_num(0, 0, 0).abs().T).amax(-1) * abs(scale) + 2.0 ** -20)[:, None]
            rel = e + (0 if batch.dt == torch.float32 else OUT[batch.dt]) + (L / 8 + 64) * EPS32
            tol[rows, h] = rel * (torch.where(seen, p.nan_to_num(1), 0.0) @ av) + (2.0 ** -25 * av.sum(0) if batch.dt == torch.float16 else 0.0)
    return out, tol
