"""Attention over the paged cache where a query, a visible key or a visible value
is no number: the outputs that depend on it are NaN, in every kernel and with
every split of the work, and all others are as without it."""
import numpy as np
import pytest

from gpu_util import need_gpu, say
from paged_util import Cache, attention, new_tokens
from test_gpu_paged_attention import run

pytestmark = pytest.mark.gpu

# what runs: (bf16, hd, hq, hkv, lens, lr, pt, window, sinks, shared, n_new)
CASES = {
    "vector": (False, 64, 8, 2, [70, 33, 5], 1, 16, 0, 0, 0, None),
    "vector_window": (False, 32, 4, 4, [70, 133, 5], 1, 16, 30, 3, 0, None),
    "vector_split": (False, 64, 8, 2, [3001, 40], 1, 64, 0, 0, 0, None),
    "vector_prompt": (False, 64, 4, 2, [90, 40], 30, 16, 0, 0, 0, None),
    "vector_bf16_split": (True, 32, 4, 4, [2500, 40], 1, 64, 0, 0, 0, None),
    "wave": (True, 128, 8, 2, [70] * 600, 1, 16, 0, 0, 0, None),
    "wave_window": (True, 64, 8, 2, [700, 95, 33], 1, 16, 50, 5, 0, None),
    "wave_split": (True, 64, 8, 2, [3001, 40, 20], 1, 64, 0, 0, 0, None),
    "wave_columns": (True, 128, 8, 2, [200, 90], 3, 32, 0, 0, 0, None),
    "wave_columns_split": (True, 64, 12, 1, [3001, 40], 1, 64, 0, 0, 0, None),
    "tile": (True, 128, 8, 2, [150, 70], 40, 32, 0, 0, 0, None),
    "tile_window": (True, 64, 8, 2, [400, 300], 40, 16, 100, 5, 0, None),
    "tile_split": (True, 64, 8, 2, [2100, 333], 40, 64, 0, 0, 0, [40, 20]),
    "shared": (True, 128, 4, 1, [1024 + 1 + i % 40 for i in range(700)], 1, 64, 0, 0, 1024, None),
    "shared_split": (True, 64, 16, 8, [17408 + n for n in (3001, 7, 1, 2500, 640, 33, 900, 64, 1)], 1, 128, 0, 0, 17408, None),
}


class Made:
    """A case's cache and queries; oracle() attends the rows in `of`."""

    def __init__(self, name):
        self.bf16, self.hd, hq, self.hkv, lens, self.lr, self.pt, self.window, self.sinks, self.shared, n_new = CASES[name]
        rng = np.random.default_rng(len(lens) + self.hd)
        self.cache = Cache(rng, lens, self.pt, self.hkv, self.hd, self.bf16, self.shared // self.pt)
        self.ragged = n_new is not None
        self.asked = n_new or [self.lr] * len(lens)
        self.new = new_tokens(lens, self.asked, self.lr)
        self.q = rng.normal(size=(len(lens), self.lr, hq, self.hd)).astype(np.float32)
        self.g = hq // self.hkv

    def at(self, row, key):
        return self.cache.table[row, key // self.pt], key % self.pt

    def gpu(self, torch, sr):
        self.cache.poison(self.new, self.window, self.sinks)
        out, _ = run(torch, sr, self.cache, self.q, self.asked, self.lr, self.window, self.sinks, self.shared,
                     ragged=self.ragged)
        return out

    def oracle(self, of):
        """(out, bound) of the rows `of`: rows alone see what they see together."""
        new = [n if r in of else 0 for r, n in enumerate(self.new)]
        return attention(self.cache, self.q, new, self.window, self.sinks, self.bf16)

    def check(self, out, of, none):
        """Elements where `none` holds are NaN, the others within their bounds of
        the row's attention without what was planted."""
        ref, bound = self.oracle(of)
        for r in of:
            n = self.new[r]
            nan = np.isnan(out[r, :n])
            assert np.array_equal(nan, none[r, :n]), (r, int(nan.sum()), int(none[r, :n].sum()))
            err = np.where(nan, 0.0, np.abs(out[r, :n] - ref[r, :n]))
            assert (err <= np.where(nan, 0.0, bound[r, :n])).all(), (r, np.nanmax(err))


def some(made):
    """A few rows: the first, one in the middle, the last."""
    n = len(made.new)
    return sorted({0, n // 2, n - 1})


@pytest.mark.parametrize("name", list(CASES))
def test_a_query_that_is_no_number(name):
    """One element of one head's query: that head's outputs of that token."""
    torch, sr = need_gpu()
    say(f"NaN query {name}")
    m = Made(name)
    rows = some(m)
    none = np.zeros(m.q.shape, dtype=bool)
    clean = m.q.copy()
    for i, r in enumerate(rows):
        t, h = m.new[r] - 1 - i % m.new[r], (3 * i + 1) % m.q.shape[2]
        m.q[r, t, h, (7 * i) % m.hd] = np.nan
        none[r, t, h] = True
    out = m.gpu(torch, sr)
    m.q = clean
    m.check(out, rows, none)


def visible_to_all(m, r):
    """Positions that every query of row r sees: one at the end of them, one in
    the middle, the first; and the last sink."""
    p0, last = int(m.cache.lens[r]) - m.new[r], int(m.cache.lens[r]) - 1
    lo = 0 if m.window == 0 else max(0, last - m.window + 1)
    keys = {lo, (lo + p0) // 2, p0}
    if lo > 0 and m.sinks:
        keys.add(min(m.sinks, lo) - 1)
    return sorted(keys)


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("value", [False, True])
def test_a_key_or_value_that_is_no_number(name, value):
    """One element of a key: every output of the rows that see it, in the heads
    of its KV head; of a value: that dimension of them."""
    torch, sr = need_gpu()
    say(f"NaN {'value' if value else 'key'} {name}")
    m = Made(name)
    hurt = len(m.new) // 2 if len(m.new) > 2 else 0
    for i, key in enumerate(visible_to_all(m, hurt)):
        pg, slot = m.at(hurt, key)
        h, d = i % m.hkv, (13 * i + 5) % m.hd
        store = m.cache.v if value else m.cache.k
        kept = store[pg, h, slot, d]
        store[pg, h, slot, d] = np.nan
        out = m.gpu(torch, sr)
        store[pg, h, slot, d] = kept
        none = np.zeros(m.q.shape, dtype=bool)
        rows = sorted({hurt} | set(some(m)))
        for r in rows:
            if r == hurt or key < m.shared:
                none[r, :, h * m.g:(h + 1) * m.g, d if value else slice(None)] = True
        m.check(out, rows, none)


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_an_infinite_value(name, sign):
    """An infinity in a value that every query of the call sees, beside slots that
    none sees: that dimension of the outputs is infinite, all else is as it was
    (a slot that nobody sees takes no part, whatever is read in its place)."""
    torch, sr = need_gpu()
    say(f"infinite value {name}")
    m = Made(name)
    hurt = len(m.new) // 2 if len(m.new) > 2 else 0
    keys = visible_to_all(m, hurt)
    if m.lr == 1:
        keys.append(int(m.cache.lens[hurt]) - 1)            # the last: free slots beside it
    for i, key in enumerate(keys):
        pg, slot = m.at(hurt, key)
        h, d = i % m.hkv, (13 * i + 5) % m.hd
        kept = m.cache.v[pg, h, slot, d]
        m.cache.v[pg, h, slot, d] = sign * np.inf
        out = m.gpu(torch, sr)
        m.cache.v[pg, h, slot, d] = kept
        rows = sorted({hurt} | set(some(m)))
        hit = np.zeros(m.q.shape, dtype=bool)
        for r in rows:
            if r == hurt or key < m.shared:
                hit[r, :m.new[r], h * m.g:(h + 1) * m.g, d] = True
        assert (out[hit] == sign * np.inf).all(), (key, out[hit])
        m.check(np.where(hit, np.nan, out), rows, hit)
