"""Plain implementations of the paged-cache operators (integers and float64)
and the inputs of their tests.  Every slot of a test's pool that no query of
its call sees holds NaN."""
import numpy as np


def bf16_round(a):
    u = np.asarray(a, dtype=np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).view(np.float32)


def visible(p, n, window, sinks):
    """Mask over n keys of a query at position p."""
    j = np.arange(n)
    see = j <= p
    if window > 0:
        see &= (j > p - window) | (j < sinks)
    return see


class Cache:
    """A pool of one layer, a table and lengths.  lens: tokens per row; shared:
    leading pages that every row has in common with row 0; holes: {(row,
    column): entry} of entries that name no page."""

    def __init__(self, rng, lens, pt, hkv, hd, bf16, shared=0, holes=None, extra_cols=2, spare=3, cols=None):
        self.pt, self.hkv, self.hd, self.bf16 = pt, hkv, hd, bf16
        self.lens = np.asarray(lens, dtype=np.int32)
        rows, used = len(lens), -(-self.lens // pt)
        self.n_pages = int(shared + np.maximum(used - shared, 0).sum()) + spare
        pages = rng.permutation(self.n_pages).astype(np.int32)
        mp = (int(used.max()) if rows else 0) + extra_cols if cols is None else cols
        self.table = np.full((rows, mp), 1 << 30, dtype=np.int32)   # past the length: never read
        at = shared
        for r in range(rows):
            for c in range(used[r]):
                if c < shared:
                    self.table[r, c] = pages[c]
                else:
                    self.table[r, c] = pages[at]
                    at += 1
        for (r, c), v in (holes or {}).items():
            self.table[r, c] = v
        rnd = bf16_round if bf16 else (lambda a: a.astype(np.float32))
        self.k = rnd(rng.normal(size=(self.n_pages, hkv, pt, hd)).astype(np.float32))
        self.v = rnd(rng.normal(size=(self.n_pages, hkv, pt, hd)).astype(np.float32))

    def is_page(self, pg):
        return 0 <= pg < self.n_pages

    def rows_kv(self, r):
        """(keys, values, there) of row r's tokens; zeros where no page is named."""
        n = int(self.lens[r])
        k, v = np.zeros((n, self.hkv, self.hd)), np.zeros((n, self.hkv, self.hd))
        there = np.zeros(n, dtype=bool)
        for c in range(-(-n // self.pt)):
            pg = self.table[r, c]
            if not self.is_page(pg):
                continue
            a, b = c * self.pt, min(n, (c + 1) * self.pt)
            k[a:b] = self.k[pg, :, :b - a].transpose(1, 0, 2)
            v[a:b] = self.v[pg, :, :b - a].transpose(1, 0, 2)
            there[a:b] = True
        return k, v, there

    def poison(self, n_new, window, sinks):
        """NaN in every slot that no query of the call sees."""
        seen = np.zeros((self.n_pages, self.pt), dtype=bool)
        for r, L in enumerate(self.lens.tolist()):
            any_ = np.zeros(L, dtype=bool)
            for t in range(n_new[r]):
                any_ |= visible(L - n_new[r] + t, L, window, sinks)
            for j in np.nonzero(any_)[0]:
                pg = self.table[r, j // self.pt]
                if self.is_page(pg):
                    seen[pg, j % self.pt] = True
        hide = ~seen[:, None, :, None]
        self.k_dev = np.where(hide, np.float32(np.nan), self.k)
        self.v_dev = np.where(hide, np.float32(np.nan), self.v)

    def device(self, torch):
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        typ = torch.bfloat16 if self.bf16 else torch.float32
        return t(self.k_dev).to(typ), t(self.v_dev).to(typ), t(self.table), t(self.lens)


def new_tokens(lens, n_new, lr):
    return [max(0, min(int(n), lr, int(L))) for n, L in zip(n_new, lens)]


def attention(cache, q, n_new, window, sinks, bf16):
    """(out [rows][lr][hq][hd], bound): float64 attention of the bf16 / fp32
    inputs, and how far roundings may move each element.

    bf16: queries are rounded (half a step, 2^-8 of each), so a score moves by at
    most d = 2^-8 sum |q_i k_i| / sqrt(hd) and a probability by a factor within
    e^(2 d); probabilities are rounded on their way into the product (2^-8) and
    so is the output (2^-8).  fp32: each of the hd products and sums of a score
    rounds (2^-24 each, with the factor log2 e / sqrt(hd) two more).  Sums over n
    keys and the exponentials add (n + 8) 2^-24 (two sums: twice)."""
    rows, lr, hq, hd = q.shape
    g = hq // cache.hkv
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
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
                step = 2.0 ** -8 if bf16 else (hd + 4) * 2.0 ** -24
                d = step * (np.abs(qh) @ np.abs(ks).T).max(1) / np.sqrt(hd) + (hd + 4) * 2.0 ** -24
                n = see.sum()
                rel = np.expm1(2 * d) + (2.0 ** -8 if bf16 else 0.0) + 2 * (n + 8) * 2.0 ** -24
                out[r, t, h * g:(h + 1) * g] = o
                bound[r, t, h * g:(h + 1) * g] = rel[:, None] * (p @ np.abs(vs)) + \
                    (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(o) * (1 + rel[:, None])
    return out, bound


# ------------------------------------------------------------------ integers
def is_page(pg, n_pages):
    return 0 <= pg < n_pages


def fork(table, lens, parent, pt, n_pages, window=0, sinks=0):
    rows, mp = table.shape
    to, lo = np.full((len(parent), mp), -1, np.int32), np.zeros(len(parent), np.int32)
    refs = np.zeros(n_pages, np.int32)
    for j, par in enumerate(parent):
        if not 0 <= par < rows:
            continue
        L = max(0, min(int(lens[par]), mp * pt))
        lo[j] = L
        for c in range(-(-L // pt)):
            pg = table[par, c]
            # seen by the token at position L or a later one?
            seen = window == 0 or any(t > L - window or t < sinks for t in range(c * pt, (c + 1) * pt))
            if is_page(pg, n_pages) and seen:
                to[j, c] = pg
                refs[pg] += 1
    return to, lo, refs


def reserve(table, lens, refs, n_add, pt, n_pages):
    """(table, lens, refs, granted, info, copies [(src, dst, filled slots)])"""
    rows, mp = table.shape
    lens = np.clip(lens, 0, mp * pt).astype(np.int32)
    clean = np.full_like(table, -1)
    for r in range(rows):
        for c in range(-(-int(lens[r]) // pt)):
            if is_page(table[r, c], n_pages):
                clean[r, c] = table[r, c]
    add = [max(0, int(n)) for n in n_add]
    wide = sum(int(L) + n > mp * pt for L, n in zip(lens, add))
    add = [min(n, mp * pt - int(L)) for L, n in zip(lens, add)]
    last = [clean[r, (int(L) - 1) // pt] if add[r] and L % pt else None for r, L in enumerate(lens)]
    out, new_refs, copies, taken = clean.copy(), refs.copy(), [], 0
    free = [p for p in range(n_pages) if refs[p] == 0]
    wanted = 0
    for r in range(rows):
        L, used = int(lens[r]), -(-int(lens[r]) // pt)
        fresh = list(range(used, -(-(L + add[r]) // pt)))
        if last[r] is not None:
            sharers = [i for i in range(rows) if last[i] is not None and last[i] == last[r]]
            if last[r] == -1:
                fresh.insert(0, used - 1)
            elif refs[last[r]] > 1 and not (len(sharers) == refs[last[r]] and sharers[0] == r):
                fresh.insert(0, used - 1)
                if wanted < len(free):
                    copies.append((int(last[r]), free[wanted], L % pt))
                    new_refs[last[r]] -= 1
        for c in fresh:
            if wanted < len(free):
                out[r, c] = free[wanted]
                new_refs[free[wanted]] = 1
            wanted += 1
        taken += len(fresh)
    missing = max(0, taken - len(free))
    if missing or wide:
        return clean, lens, refs.copy(), np.zeros(rows, np.int32), [missing, wide, 0, 0], []
    return out, lens + np.array(add, np.int32), new_refs, np.array(add, np.int32), [0, 0, taken, len(copies)], copies


def compact(table, lens, refs, pt):
    n_pages, (rows, mp) = len(refs), table.shape
    live = int((refs > 0).sum())
    tail = [p for p in range(live, n_pages) if refs[p] > 0]
    hole = [p for p in range(live) if refs[p] <= 0]
    to = {a: b for a, b in zip(tail, hole)}
    out = np.full_like(table, -1)
    for r in range(rows):
        for c in range(-(-max(0, min(int(lens[r]), mp * pt)) // pt)):
            if is_page(table[r, c], n_pages):
                out[r, c] = to.get(int(table[r, c]), table[r, c])
    new = refs.copy()
    new[live:] = 0
    for a, b in to.items():
        new[b] = refs[a]
    return out, new, [live, len(tail), 0, 0], sorted(to.items())
