"""Plain implementations of the 4-bit operators for their tests: the format from its rule, everything
else in 64 bits.  numpy and torch on the CPU only; none of the library's code."""
import numpy as np
import torch

EPS32, EPS16, EPSB = 2.0 ** -23, 2.0 ** -11, 2.0 ** -8       # spacing of fp32, half spacing of fp16 and of bf16 (relative)
OUT_EPS = {torch.float32: 2.0 ** -24, torch.float16: EPS16, torch.bfloat16: EPSB}


def values_np(t):
    return t.detach().float().cpu().numpy()


def quantise(x, group):
    """fp32 array [..., d] (d a multiple of group) -> (codes, s, o): codes uint8 [..., d], s and o float16 [..., d / group].
    The format is defined by fp32 operations, so this is exact."""
    g = x.astype(np.float32).reshape(*x.shape[:-1], -1, group)
    with np.errstate(all="ignore"):
        lo, hi = g.min(-1), g.max(-1)
        nan = np.isnan(g).any(-1)
        lo, hi = np.where(nan, np.float32(0), lo), np.where(nan, np.float32(0), hi)
        o = np.clip(lo, np.float32(-65504), np.float32(65504)).astype(np.float16)
        s = np.minimum((hi - lo) * (np.float32(1) / np.float32(15)), np.float32(65504)).astype(np.float16)
        o, s = np.where(nan, np.float16(np.nan), o), np.where(nan, np.float16(np.nan), s)
        c = np.rint((g - o.astype(np.float32)[..., None]) / s.astype(np.float32)[..., None])
        c = np.where(s.astype(np.float32)[..., None] > 0, np.clip(c, 0, 15), 0)
    return c.astype(np.uint8).reshape(x.shape), s, o


def pack(codes):
    """codes [..., 32 H] -> bytes [..., 16 H] (value v of a piece in unit (v % 32) // 4 * H + v // 32)."""
    d = codes.shape[-1]
    out = np.zeros((*codes.shape[:-1], d // 2), np.uint8)
    for v in range(d):
        byte = 2 * (((v % 32) // 4) * (d // 32) + v // 32) + (v % 4) // 2
        out[..., byte] |= (codes[..., v] << (4 * (v % 2))).astype(np.uint8)
    return out


def dequantise(codes, s, o):
    """64-bit values of codes [..., d] with pairs [..., d / group]."""
    rep = codes.shape[-1] // s.shape[-1]
    return codes.astype(np.float64) * np.repeat(s.astype(np.float64), rep, -1) + np.repeat(o.astype(np.float64), rep, -1)


def unpack_cache(codes, pairs):
    """64-bit values of cache buffers: codes bytes [..., d / 2], pairs fp16 [..., d / group, 2] (tensors)."""
    b, p = codes.cpu().numpy(), pairs.cpu().numpy()
    d = 2 * b.shape[-1]
    v = np.arange(d)
    byte = 2 * (((v % 32) // 4) * (d // 32) + v // 32) + (v % 4) // 2
    return dequantise((b[..., byte] >> (4 * (v % 2))) & 15, p[..., 0], p[..., 1])


def pairs_array(s, o):
    return np.stack((s, o), -1)


def w4_layout(w, group):
    """w fp32 [N, K] -> (codes bytes, pairs, the 64-bit values [N, K] they stand for)."""
    N, K = w.shape
    Np, Kp, Kg = -(-N // 16) * 16, -(-K // 128) * 128, -(-K // group) * group
    ext = np.concatenate((w, np.repeat(w[:, -1:], Kg - K, 1)), 1) if Kg > K else w
    codes, s, o = quantise(ext, group)
    vals = dequantise(codes, s, o)[:, :K]
    c = np.zeros((Np, Kp), np.uint8)
    c[:N, :K] = codes[:, :K]
    sp, op = np.zeros((Np, Kp // group), np.float16), np.zeros((Np, Kp // group), np.float16)
    sp[:N, : Kg // group], op[:N, : Kg // group] = s, o
    packed = pack(c.reshape(Np // 16, 16, Kp // 128, 128).transpose(0, 2, 1, 3))
    pr = pairs_array(sp, op).reshape(Np // 16, 16, Kp // group, 2).transpose(0, 2, 1, 3)
    return np.ascontiguousarray(packed), np.ascontiguousarray(pr), vals


class CacheRef:
    """A 4-bit cache on the host: codes as numbers, weights in 64 bits, positions and lengths."""

    def __init__(self, B, H, cap, D, group, rng):
        self.B, self.H, self.cap, self.D, self.group = B, H, cap, D, group
        x = rng.standard_normal((2, B, H, cap, D)).astype(np.float32)
        self.codes, self.s, self.o = quantise(x, group)
        self.weight = rng.exponential(size=(B, H, cap)).astype(np.float32).astype(np.float64)
        self.position = np.broadcast_to(np.arange(cap, dtype=np.int32), (B, H, cap)).copy()
        self.length, self.seen, self.refused = [0] * B, [0] * B, [0] * B

    def set_lengths(self, lengths):
        self.length, self.seen = list(lengths), list(lengths)

    def values(self, which):
        return dequantise(self.codes[which], self.s[which], self.o[which])

    def append(self, k, v):
        """k, v fp32 [B, T, H, D]; returns the stored values, 64-bit."""
        T, stored = k.shape[1], []
        for w, x in enumerate((k, v)):
            codes, s, o = quantise(x.transpose(0, 2, 1, 3), self.group)
            stored.append(dequantise(codes, s, o).transpose(0, 2, 1, 3))
            for b in range(self.B):
                n = self.length[b]
                if n + T <= self.cap:
                    self.codes[w][b, :, n:n + T], self.s[w][b, :, n:n + T], self.o[w][b, :, n:n + T] = codes[b], s[b], o[b]
        for b in range(self.B):
            n = self.length[b]
            if n + T <= self.cap:
                self.weight[b, :, n:n + T] = 0
                self.position[b, :, n:n + T] = self.seen[b] + np.arange(T)
                self.length[b] += T
                self.seen[b] += T
            else:
                self.refused[b] += T
        return stored

    def attention(self, q, scale):
        """q float64 [B, T, Hq, D] -> (out, weight added [B, H, cap], bounds): 64-bit results and, for each output, the
        sums of absolute terms that rounding errors are measured by."""
        B, T, Hq, D = q.shape
        share = Hq // self.H
        out, add = np.zeros(q.shape), np.zeros((self.B, self.H, self.cap))
        mass, logit_mass = np.zeros(q.shape), np.zeros((B, T, Hq))
        k, v = self.values(0), self.values(1)
        ak = self.codes[0] * np.repeat(self.s[0].astype(np.float64), self.group, -1) + np.abs(np.repeat(self.o[0].astype(np.float64), self.group, -1))
        av = self.codes[1] * np.repeat(self.s[1].astype(np.float64), self.group, -1) + np.abs(np.repeat(self.o[1].astype(np.float64), self.group, -1))
        for b in range(B):
            for t in range(T):
                m = self.length[b] - (T - 1 - t)
                if m <= 0:
                    continue
                for g in range(Hq):
                    h = g // share
                    logit = scale * (k[b, h, :m] @ q[b, t, g])
                    p = np.exp(logit - logit.max())
                    p /= p.sum()
                    out[b, t, g] = p @ v[b, h, :m]
                    add[b, h, :m] += p
                    mass[b, t, g] = p @ av[b, h, :m]
                    logit_mass[b, t, g] = (abs(scale) * (ak[b, h, :m] @ np.abs(q[b, t, g]))).max()
        return out, add, mass, logit_mass

    def kept(self, b, h, budget, recent, first):
        n = self.length[b]
        w, p = self.weight[b, h, :n], self.position[b, h, :n]
        safe = (p >= self.seen[b] - recent) | (p < first)
        big = [(0 if safe[i] else (2 if np.isnan(w[i]) else 1), 0.0 if safe[i] or np.isnan(w[i]) else -w[i], i) for i in range(n)]
        return sorted(i for _, _, i in sorted(big)[: min(n, budget)])

    def _rows(self):
        return (self.codes[0], self.codes[1], self.s[0], self.s[1], self.o[0], self.o[1], self.weight, self.position)

    def evict_here(self, budget, recent, first):
        for b in range(self.B):
            keep = min(self.length[b], budget)
            for h in range(self.H):
                stay = self.kept(b, h, budget, recent, first)
                inside = set(stay)
                holes = [i for i in range(keep) if i not in inside]
                movers = [i for i in stay if i >= keep]
                for a in self._rows():
                    a[b, h, holes] = a[b, h, movers].copy()
            self.length[b] = keep

    def evict_to(self, dst, budget, recent, first):
        for b in range(self.B):
            for h in range(self.H):
                stay = self.kept(b, h, budget, recent, first)
                for a, z in zip(self._rows(), dst._rows()):
                    z[b, h, : len(stay)] = a[b, h, stay]
            dst.length[b], dst.seen[b] = min(self.length[b], budget), self.seen[b]

    def to_cuda(self, weighted=True):
        """The library's buffers: dict of CUDA tensors."""
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        d = {}
        for w, name in enumerate("kv"):
            d[name + "_codes"], d[name + "_pairs"] = up(pack(self.codes[w])), up(pairs_array(self.s[w], self.o[w]))
        d["state"] = up(np.array([[n, s, r, 0] for n, s, r in zip(self.length, self.seen, self.refused)], np.int32))
        d["weight"] = up(self.weight.astype(np.float32)) if weighted else None
        d["position"] = up(self.position) if weighted else None
        return d

    def assert_equal(self, d, weight_exact=True):
        for w, name in enumerate("kv"):
            np.testing.assert_array_equal(d[name + "_codes"].cpu().numpy(), pack(self.codes[w]))
            np.testing.assert_array_equal(d[name + "_pairs"].cpu().numpy().view(np.uint16), pairs_array(self.s[w], self.o[w]).view(np.uint16))
        np.testing.assert_array_equal(d["state"].cpu().numpy(), [[n, s, r, 0] for n, s, r in zip(self.length, self.seen, self.refused)])
        np.testing.assert_array_equal(d["position"].cpu().numpy(), self.position)
        if weight_exact:
            np.testing.assert_array_equal(d["weight"].cpu().numpy(), self.weight.astype(np.float32))
