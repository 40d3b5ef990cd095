"""What the roundings of attention over 4 bits leave of its precision, in the 2-norm:
plain models of them (numpy, float64) and the limit that they give."""
import numpy as np

from paged_util import bf16_round, visible

E2M3 = np.concatenate([np.arange(16) / 8, 2 + np.arange(8) / 4, 4 + np.arange(8) / 2])   # (6 bits without the sign)


def six_bit_parts(x, parts):
    """float32 x [..., hd] as `parts` parts of 6 bits, groups of 32 with the least scale 2^k
    that keeps the largest at 7.5 scales or below; what they add up to, and what is left."""
    rest = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, 32)
    total = np.zeros_like(rest)
    mids = (E2M3[:-1] + E2M3[1:]) / 2
    for _ in range(parts):
        top = np.abs(rest).max(-1, keepdims=True)
        scale = 2.0 ** np.ceil(np.log2(np.maximum(top, 1e-300) / 7.5))
        y = E2M3[np.searchsorted(mids, np.abs(rest) / scale)] * np.sign(rest) * scale
        total, rest = total + y, rest - y
    return total.reshape(x.shape), rest.reshape(x.shape)


def limit(cache, q, n_new, window, sinks, columns, p_bits=None):
    """(out, limit): float64 attention, and how far from it the outputs of a bf16 call
    with `columns` query columns a row may lie in the 2-norm.

    A sum of many independent roundings grows as the root of the sum of their squares; a
    rounding that is off by u at most is off by u / sqrt(3) in the mean square.  The
    output's is taken as it falls.  A key's score is off by that of a dimension times |k|
    / sqrt(hd), added over the dimensions: a query keeps 16 bits (2^-16 |q|) for up to 16
    columns; for more it is off by up to 1 / 15360 of the largest of 32 dimensions
    (fp4_util.attention derives it; products of 6 bits with 4-bit keys are exact).  A probability keeps 16 bits (2^-16) for up to 8 columns, 8 bits (2^-8)
    for more, or p_bits.  A weight p that is off by e relative moves an output by e p times
    its value, less the output where the sum of the weights moves with it.  A
    tenth on top: the errors add up over some thousand outputs, not over all there could
    be."""
    rows, lr, hq, hd = q.shape
    g = hq // cache.hkv
    out, var = np.zeros(q.shape), 0.0
    up = 2.0 ** -(p_bits or (16 if columns <= 8 else 8))
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
                per = 2.0 ** -16 * np.abs(qh)
                if columns > 16:
                    per = np.repeat(np.abs(qh).reshape(g, -1, 32).max(2), 32, axis=1) / 15360
                e2 = (per ** 2 @ (ks ** 2).T / hd + up ** 2) / 3          # of a weight, squared
                w2 = p ** 2 * e2
                moved = np.maximum(w2 @ vs ** 2, w2 @ vs ** 2 - 2 * o * (w2 @ vs) + o ** 2 * w2.sum(1, keepdims=True))
                var += moved.sum()
                out[r, t, h * g:(h + 1) * g] = o
    rounded = bf16_round(out.astype(np.float32)).astype(np.float64)
    return out, 1.1 * np.sqrt(var + np.square(rounded - out).sum())


def with_8_bits(cache, q, n_new, window, sinks):
    """Attention whose probabilities (their sum is not) and outputs are rounded to 8 bits."""
    rows, lr, hq, hd = q.shape
    g = hq // cache.hkv
    out = np.zeros(q.shape)
    for r in range(rows):
        k, v, there = cache.rows_kv(r)
        L = len(k)
        for t in range(n_new[r]):
            see = visible(L - n_new[r] + t, L, window, sinks) & there
            for h in range(cache.hkv) if see.any() else ():
                s = q[r, t, h * g:(h + 1) * g].astype(np.float64) @ k[see][:, h].T / np.sqrt(hd)
                p = np.exp(s - s.max(1, keepdims=True))
                out[r, t, h * g:(h + 1) * g] = bf16_round(p).astype(np.float64) @ v[see][:, h] / p.sum(1, keepdims=True)
    return bf16_round(out).astype(np.float64)
