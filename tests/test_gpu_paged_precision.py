"""Attention of few query columns a row keeps the queries' precision whichever way
the call is split: single tokens, drafts, and leading keys that rows share.

With queries that lose nothing to bf16, what moves an output o = sum p_j v_j is the
rounding of the probabilities and its own: a rounding to bf16 with a mantissa
spread evenly over its logarithm has a mean square of 0.54 (2^-8)^2 / 3 of the
value's, so the mean square of an output's error over heads is
  0.54 (2^-8)^2 / 3 (sum_j p_j^2 |v_j|^2 + |o|^2),
on flat rows the same again for each of the two, and half as much again where
queries are rounded to bf16.  The mean over more than 20000 elements is within a
few per cent of it; 1.25 is asked for."""
import numpy as np
import pytest

from gpu_util import need_gpu, say
from paged_long import Long
from test_gpu_paged_attention import run

pytestmark = pytest.mark.gpu

LENS = (1024 + np.random.default_rng(7).integers(30, 200, 700)).tolist()
CASES = {
    "single": dict(hd=128, hq=8, hkv=2, lens=[900 + 7 * i for i in range(24)], lr=1, pt=64),
    "single_hd64": dict(hd=64, hq=8, hkv=2, lens=[900 + 7 * i for i in range(48)], lr=1, pt=64),
    "columns": dict(hd=128, hq=8, hkv=2, lens=[900 + 7 * i for i in range(8)], lr=3, pt=64),
    "columns_hd64": dict(hd=64, hq=16, hkv=1, lens=[900 + 7 * i for i in range(24)], lr=1, pt=64),
    "columns_split": dict(hd=128, hq=8, hkv=2, lens=[5003, 4001, 3500, 2900, 4444, 5000], lr=4, pt=64, window=3000, sinks=3),
    "shared": dict(hd=128, hq=4, hkv=1, lens=LENS, lr=1, pt=64, shared=1024, pick=[(r, 0) for r in range(0, 700, 14)]),
    "shared_hd64": dict(hd=64, hq=4, hkv=2, lens=LENS, lr=1, pt=16, shared=1024, pick=[(r, 0) for r in range(0, 700, 7)]),
    "shared_columns": dict(hd=128, hq=4, hkv=1, lens=LENS, lr=3, pt=64, shared=1024, pick=[(r, r % 3) for r in range(0, 700, 14)]),
}


def expected(c):
    """Mean squares of the error, summed over the compared heads."""
    ms, n = 0.0, 0
    ref = c.oracle(bound=False)
    for r, t in c.pick:
        k, v = c.kv(r)
        m = c.sees(r, t)
        for h in range(c.hkv):
            z = c.q[r, t, h * c.g:(h + 1) * c.g].astype(np.float64) @ k[m][:, h].T / np.sqrt(c.hd)
            p = np.exp(z - z.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o = ref[r, t][0][h * c.g:(h + 1) * c.g]
            ms += ((p ** 2) @ (v[m][:, h] ** 2).sum(1)).sum() + (o ** 2).sum()
            n += c.g * c.hd
    return 0.54 * 2.0 ** -16 / 3 * ms, n, ref


@pytest.mark.parametrize("name", list(CASES))
def test_queries_keep_their_precision(name):
    torch, sr = need_gpu()
    c = Long(marked=False, seed=3, **CASES[name])
    c.cache.poison(c.new, c.window, c.sinks)
    out, _ = run(torch, sr, c.cache, c.q, [c.lr] * len(c.new), c.lr, c.window, c.sinks, c.shared, ragged=False)
    want, n, ref = expected(c)
    got = sum(((out[r, t] - ref[r, t][0]) ** 2).sum() for r, t in c.pick)
    size = sum((ref[r, t][0] ** 2).sum() for r, t in c.pick)
    say(f"precision {name}: {np.sqrt(got / size):.5f} in the 2-norm, mean square {got / want:.3f} of the expected, {n} elements")
    assert n > 20000 and got <= 1.25 * want
