"""Long rows for the matrix-core attention kernels: inputs on which every part of
a row matters, and a bound on the 2-norm of an output's error that is small
against what any lost part would take away.

Inputs.  A query is c + N(0, 0.7^2), c a fixed N(0, 1) vector per KV head, and
values are N(0, 1).
  flat    keys are N(0, 1): an output over n keys has size about
          1.7 sqrt(hd / n), and a share of them lost changes it by the share's
          square root;
  marked  some keys are gamma c, so that each holds a few per cent of the weight:
          the keys at the edges of what is seen (first, last, last sink, window
          start) and one in every sixteenth of the row.

Bound.  Roundings to bf16 have half a step of at most 2^-8 of the value and are
taken as independent and uniform: a standard deviation of at most s = 2^-8 /
sqrt(3) of it.  To first order they move an output o = sum p_j v_j by
  queries        sum_i e_i q_i J_i,  J_i = sum_j p_j k_ji (v_j - o) / sqrt(hd)
  probabilities  sum_j e_j p_j v_j, less o sum_j e_j p_j where their sum is of the
                 rounded ones
  the output     e_d o_d
so the mean square of the error's 2-norm is at most
  s^2 (sum_i q_i^2 |J_i|^2 + sum_j p_j^2 (|v_j|^2 + |o|^2) + |o|^2).
What is left in 32 bits (scores, exponentials, sums: 2^-24 each, n of them adding
up like sqrt(n)) is at most 2^-24 (hd + 64 + sqrt(n)) sum p_j |v_j|.  The bound is
five times the root mean square of the former plus the latter.  A queries' error of
exactly five deviations in one direction has a chance below 1e-6, and the three
parts, of many components each, come nowhere near theirs together."""
import numpy as np

from paged_util import Cache, bf16_round, new_tokens, visible

S = 2.0 ** -8 / np.sqrt(3.0)


class Long:
    """One call.  pick: the (row, token) pairs that are compared (None: all)."""

    def __init__(self, hd, hq, hkv, lens, lr, pt, window=0, sinks=0, n_new=None, shared=0, max_len=None, marked=True,
                 pick=None, seed=1):
        self.hd, self.hq, self.hkv, self.lr, self.pt, self.window, self.sinks = hd, hq, hkv, lr, pt, window, sinks
        self.shared, self.max_len, self.asked = shared, max_len, n_new
        rng = np.random.default_rng(seed)
        self.cache = Cache(rng, lens, pt, hkv, hd, True, shared // pt)
        self.new = new_tokens(lens, [lr] * len(lens) if n_new is None else n_new, lr)
        self.g = hq // hkv
        c = rng.normal(size=(hkv, hd)).astype(np.float32)
        self.q = (np.repeat(c, self.g, 0) + 0.7 * rng.normal(size=(len(lens), lr, hq, hd))).astype(np.float32)
        self.pick = [(r, t) for r, n in enumerate(self.new) for t in range(n)] if pick is None else pick
        if marked:
            for r in sorted({r for r, _ in self.pick}):
                self.mark(rng, r, c)

    def mark(self, rng, r, c):
        L, n = int(self.cache.lens[r]), self.new[r]
        if n == 0:
            return
        lo = max(0, L - n - self.window + 1) if self.window else 0
        end = max(0, L - self.window) if self.window else 0      # the window start of the last token
        keys = {0, lo, end, L - n, L - 1, max(0, min(self.sinks, lo) - 1)}
        keys |= {int(lo + (L - lo) * (i + rng.random()) / 16) for i in range(16)}
        if self.shared:
            keys |= {self.shared - 1, min(self.shared, L - 1)}
        # exp(gamma |c|^2 / sqrt(hd)) = 4 % of what the other keys weigh, exp(1.49 / 2) each
        gamma = np.log(0.04 * 2.1 * max(30, L - lo)) * np.sqrt(self.hd) / (c ** 2).sum(1, keepdims=True)
        for k in keys:
            pg = self.cache.table[r, k // self.pt]
            self.cache.k[pg, :, k % self.pt] = bf16_round(gamma * c)

    def kv(self, r):
        k, v, _ = self.cache.rows_kv(r)
        return k, v

    def sees(self, r, t):
        L = int(self.cache.lens[r])
        return visible(L - self.new[r] + t, L, self.window, self.sinks)

    def oracle(self, see=None, rounded=False, bound=True):
        """{(row, token): (out [hq][hd], limit [hq])} in 64 bits.  see(row, token,
        mask) may change what is seen (a planted mistake); rounded: queries,
        probabilities and outputs rounded to bf16 (what a right kernel may do)."""
        got, last = {}, None
        for r, t in self.pick:
            if last is None or last[0] != r:
                last = (r, *self.kv(r))
            k, v = last[1:]
            mask = self.sees(r, t)
            if see is not None:
                mask = see(self, r, t, mask.copy())
            if not mask.any():
                got[r, t] = np.zeros((self.hq, self.hd)), np.zeros(self.hq)
                continue
            out, lim = np.zeros((self.hq, self.hd)), np.zeros(self.hq)
            for h in range(self.hkv):
                ks, vs = k[mask][:, h], v[mask][:, h]
                qh = self.q[r, t, h * self.g:(h + 1) * self.g].astype(np.float64)
                if rounded:
                    qh = bf16_round(qh).astype(np.float64)
                z = qh @ ks.T / np.sqrt(self.hd)
                e = np.exp(z - z.max(1, keepdims=True))
                total = e.sum(1, keepdims=True)
                if rounded:
                    e = bf16_round(e).astype(np.float64)
                p = e / total
                o = p @ vs
                for i in range(self.g):
                    x = h * self.g + i
                    out[x] = bf16_round(o[i]).astype(np.float64) if rounded else o[i]
                    if bound:
                        J = (ks * p[i][:, None]).T @ vs - np.outer(p[i] @ ks, o[i])
                        v2, o2 = (vs ** 2).sum(1), (o[i] ** 2).sum()
                        ms = (qh[i] ** 2 * (J ** 2).sum(1)).sum() / self.hd + (p[i] ** 2 * (v2 + o2)).sum() + o2
                        lim[x] = 5 * S * np.sqrt(ms) + 2.0 ** -24 * (self.hd + 64 + np.sqrt(len(ks))) * (p[i] @ np.sqrt(v2))
            got[r, t] = out, lim
        return got

    def worst(self, out, ref):
        """The largest error of out[row][token][head] in units of its limit."""
        w = 0.0
        for (r, t), (want, lim) in ref.items():
            err = np.sqrt(((out[r][t] - want) ** 2).sum(1))
            if np.isnan(err).any():
                return np.inf
            w = max(w, float((err / np.maximum(lim, 1e-30)).max()))
        return w


def some_tokens(row, n, cols):
    """Tokens of a row of n whose columns lie at the edges of work-groups of `cols`
    tokens, and a few between."""
    return [(row, t) for t in sorted({0, 1, cols - 1, cols, n // 2, n - cols, n - 2, n - 1}) if 0 <= t < n]


TAILS = [3001, 7, 1, 2500, 640, 33, 900, 64, 1]
_rows = np.random.default_rng(700)
SHARE = {k: (1024 + _rows.integers(1, 40, n)).tolist() for k, n in ((128, 700), (64, 1300))}
SHARE_PICK = [(r, 0) for r in (0, 1, 31, 32, 63, 350, 698, 699)]

# name: arguments of Long
CASES = {
    "splits_hd64": dict(hd=64, hq=1, hkv=1, lens=[17001], lr=1, pt=64),
    "splits_hd128": dict(hd=128, hq=4, hkv=1, lens=[17001], lr=1, pt=64),
    "splits_hd32": dict(hd=32, hq=2, hkv=1, lens=[17001], lr=1, pt=64),
    "splits_ragged": dict(hd=128, hq=4, hkv=1, lens=[17400, 9000], lr=1, pt=128, n_new=[1, 0]),
    "rows_hd128": dict(hd=128, hq=8, hkv=2, lens=[5003], lr=1, pt=64),
    "rows_hd64": dict(hd=64, hq=4, hkv=1, lens=[5003], lr=1, pt=64),
    "unplanned": dict(hd=64, hq=4, hkv=1, lens=[2777, 901], lr=1, pt=32, max_len=10),
    "window": dict(hd=128, hq=8, hkv=2, lens=[3001, 12, 4096], lr=1, pt=16, window=2500, sinks=3),
    "window_hd64": dict(hd=64, hq=4, hkv=1, lens=[3001, 12, 4096], lr=1, pt=16, window=2500, sinks=3),
    "drafts": dict(hd=128, hq=8, hkv=2, lens=[4001, 700], lr=3, pt=64),
    "drafts_window": dict(hd=64, hq=8, hkv=2, lens=[4001, 700], lr=4, pt=32, window=600, sinks=5),
    "chunk": dict(hd=128, hq=8, hkv=2, lens=[2100], lr=40, pt=64, pick=some_tokens(0, 40, 32)),
    "chunk_hd64": dict(hd=64, hq=4, hkv=1, lens=[2100], lr=40, pt=64, pick=some_tokens(0, 40, 32)),
    "chunks": dict(hd=128, hq=8, hkv=2, lens=[2100, 333], lr=33, pt=64, n_new=[33, 20], max_len=4000,
                   pick=some_tokens(0, 33, 32) + some_tokens(1, 20, 8)),
    "prompt": dict(hd=128, hq=4, hkv=1, lens=[1500], lr=1500, pt=32, window=700, sinks=5,
                   pick=some_tokens(0, 1500, 32) + [(0, 698), (0, 699), (0, 700), (0, 705), (0, 1033)]),
    "prompt_hd64": dict(hd=64, hq=8, hkv=2, lens=[1500, 800], lr=1500, pt=64, n_new=[1500, 700],
                        pick=some_tokens(0, 1500, 32) + some_tokens(1, 700, 32)),
    "shared_hd128": dict(hd=128, hq=4, hkv=1, lens=SHARE[128], lr=1, pt=64, shared=1024, pick=SHARE_PICK),
    "shared_hd64": dict(hd=64, hq=2, hkv=1, lens=SHARE[64], lr=1, pt=16, shared=1024, pick=SHARE_PICK),
    "shared_tails_hd128": dict(hd=128, hq=8, hkv=8, lens=[16384 + n for n in TAILS[:5]], lr=1, pt=128, shared=16384,
                               pick=[(0, 0), (2, 0)]),
    "shared_tails_hd64": dict(hd=64, hq=16, hkv=8, lens=[17408 + n for n in TAILS], lr=2, pt=256, shared=17408,
                              n_new=[2, 1, 0, 2, 2, 2, 1, 2, 1], pick=[(0, 1), (5, 0)]),
}


def make(name, marked):
    return Long(marked=marked, seed=sorted(CASES).index(name) + 100 * marked, **CASES[name])
