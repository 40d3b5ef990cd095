"""Plain implementations (numpy, float64) of the 4-bit cache format, of attention
over it and of head norms with rotation, and a cache of 4 bits for the tests:
every slot of its pool that no query of the call sees holds codes and scale bytes
that read as NaN."""
import numpy as np

from paged_util import Cache, visible

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """(codes uint8 [..., hd], scale bytes uint8 [..., hd / 32]) of float64 x: by
    trying every scale from the least on and every value."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, 32)
    with np.errstate(invalid="ignore"):
        top = np.abs(g).max(-1)
    fine = np.isfinite(g).all(-1)
    b = np.full(top.shape, 252, dtype=np.int64)
    for byte in range(251, 1, -1):
        b = np.where(top < 7.0 * 2.0 ** (byte - 127), byte, b)
    y = np.abs(np.where(fine[..., None], g, 0.0)) / 2.0 ** (b - 127.0)[..., None]
    c = np.zeros(g.shape, dtype=np.uint8)
    for k in range(7):   # past the middle of two codes, or on it where the upper one is even
        mid = (VALUES[k] + VALUES[k + 1]) / 2
        c += (y > mid) | ((y == mid) & (k % 2 == 1))
    c = np.where(fine[..., None], c + 8 * np.signbit(g).astype(np.uint8), 0).astype(np.uint8)
    return c.reshape(x.shape), np.where(fine, b, 255).astype(np.uint8)


def dequantise(codes, scales):
    v = VALUES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    return v * np.repeat(s, 32, axis=-1)


def pack(codes, scales):
    """Pools uint8 [n_pages][hkv][pt][17 hd / 32] of codes [n_pages][hkv][pt][hd]."""
    n, h, pt, hd = codes.shape
    both = (codes[..., 0::2] | (codes[..., 1::2] << 4)).reshape(n, h, -1)
    return np.concatenate([both, scales.reshape(n, h, -1)], -1).reshape(n, h, pt, 17 * hd // 32)


def unpack(pool):
    n, h, pt, nb = pool.shape
    hd = nb * 32 // 17
    flat = pool.reshape(n, h, -1)
    both = flat[..., :pt * hd // 2].reshape(n, h, pt, hd // 2)
    codes = np.stack([both & 15, both >> 4], -1).reshape(n, h, pt, hd)
    return codes, flat[..., pt * hd // 2:].reshape(n, h, pt, hd // 32)


class Cache4(Cache):
    """paged_util.Cache with keys and values of 4 bits; k and v are what they stand
    for."""

    def __init__(self, rng, lens, pt, hkv, hd, **kw):
        super().__init__(rng, lens, pt, hkv, hd, False, **kw)
        self.raw = [quantise(x.astype(np.float64) * np.exp(rng.normal(size=x.shape[:3] + (1,)))) for x in (self.k, self.v)]
        self.k, self.v = (dequantise(*r) for r in self.raw)

    def poison(self, n_new, window, sinks):
        super().poison(n_new, window, sinks)
        self.packed = []
        for (codes, scales), shown in zip(self.raw, (self.k_dev, self.v_dev)):
            hide = np.isnan(shown[..., 0]) & ~np.isnan(dequantise(codes, scales)[..., 0])
            self.packed.append(pack(np.where(hide[..., None], np.uint8(15), codes), np.where(hide[..., None], np.uint8(255), scales)))

    def device(self, torch):
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        return t(self.packed[0]), t(self.packed[1]), t(self.table), t(self.lens)


def attention(cache, q, n_new, window, sinks, bf16):
    """(out [rows][lr][hq][hd], bound): float64 attention over the values of the
    cache, and how far roundings may move each element.

    Keys and values are exact.  bf16: queries enter the products with a relative
    error of 2^-16 where a row has at most 16 columns (two halves, 2^-8 each).  Where it
    has more they enter as three parts of 6 bits (steps of 1/8 up to 2, 1/4 up to 4, 1/2 up to 7.5), each times a
    power of two s for 32 dimensions, the least with which the largest is at most 7.5 s,
    so above 3.75 s: the first part leaves at most s / 4, which is at most 4 of the
    second's steps of scale s / 16, so that leaves s / 128, and the third s / 4096, below
    2^-13 of the largest of the 32; the products of such a group are cut at some 2^-14
    of the largest of them, another 2^-13 of that sum of magnitudes: 2^-12 together.
    Probabilities enter with 2^-8; the output is rounded, 2^-8.  fp32:
    three parts, 2^-24, and 2^-24 each.  A score adds up hd products (and their
    parts: three times as many, each step 2^-24 of the sum of magnitudes) and a
    factor; so it moves by d and a probability by a factor within e^(2 d); the
    exponentials and the two sums over n keys add 2 (3 n + 8) 2^-24.  What falls below
    2^-126 may be flushed to 0: a weight (of at least one that is 1), its parts, a
    product and a sum, each at most 2^-126 max(1, |v|) a key, 2^-123 in all."""
    rows, lr, hq, hd = q.shape
    g = hq // cache.hkv
    U = 2.0 ** -24
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    step = 2.0 ** -16 if bf16 else U
    grouped = bf16 and lr * g > 16
    last = 2.0 ** -8 if bf16 else U
    for r in range(rows):
        k, v, there = cache.rows_kv(r)
        L = len(k)
        for t in range(n_new[r]):
            see = visible(L - n_new[r] + t, L, window, sinks) & there
            if not see.any():
                continue
            for h in range(cache.hkv):
                ks, vs = k[see][:, h], v[see][:, h]
                qh = q[r, t, h * g:(h + 1) * g].astype(np.float64)
                s = qh @ ks.T / np.sqrt(hd)
                p = np.exp(s - s.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                o = p @ vs
                d = (step + (3 * hd + 4) * U) * (np.abs(qh) @ np.abs(ks).T).max(1) / np.sqrt(hd)
                if grouped:
                    top = np.repeat(np.abs(qh).reshape(g, -1, 32).max(2), 32, axis=1)
                    d += 2.0 ** -12 * (top @ np.abs(ks).T).max(1) / np.sqrt(hd)
                rel = np.expm1(2 * d) + last + 2 * (3 * see.sum() + 8) * U
                low = see.sum() * 2.0 ** -123 * max(1.0, np.abs(vs).max())
                out[r, t, h * g:(h + 1) * g] = o
                bound[r, t, h * g:(h + 1) * g] = rel[:, None] * (p @ np.abs(vs)) + last * np.abs(o) * (1 + rel[:, None]) + low
    return out, bound


def rotate(x, pos, freqs, interleaved):
    """Heads [.., hd] at position pos."""
    y, n = x.copy(), len(freqs)
    i = np.arange(n)
    a, c = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    co, si = np.cos(pos * freqs), np.sin(pos * freqs)
    y[..., a], y[..., c] = x[..., a] * co - x[..., c] * si, x[..., c] * co + x[..., a] * si
    return y


def norm(x, gain, eps):
    x = np.asarray(x, dtype=np.float64)
    return x if gain is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain.astype(np.float64)
