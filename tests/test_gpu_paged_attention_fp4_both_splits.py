"""Attention over 4 bits where the shared keys have a pass of their own and the rows'
own keys are split over work-groups too, so that partials of both meet in one join:
rows that share less than the others, an empty one, one whose shared pages have a hole,
tokens of a draft past some rows' ends."""
import numpy as np
import pytest

from fp4_precision import limit
from fp4_util import Cache4, attention, pack
from gpu_util import need_gpu, say
from paged_util import new_tokens
from test_gpu_paged_attention_fp4 import SENTINEL, run

pytestmark = pytest.mark.gpu

ROWS, HQ, HKV, PT = 64, 32, 8, 64
CHECKED = [0, 3, 4, 5, 6, 7, 20, 40, 63]


class Rows(Cache4):
    """Of which the plain implementation sees the CHECKED rows only."""

    def rows_kv(self, r):
        if r in CHECKED:
            return super().rows_kv(r)
        return np.zeros((0, HKV, self.hd)), np.zeros((0, HKV, self.hd)), np.zeros(0, bool)


def slots(sr, dtype, hd, lr, cols, shared, max_len):
    """(partial slots of a call, whether the shared keys have a pass), by its scratch."""
    n = sr.lib().sr_paged_attention_fp4_scratch(dtype, hd, HQ, HKV, ROWS, lr, PT, cols, 0, 0, shared, max_len)
    return divmod(n, ROWS * lr * HQ * (hd + 2))


@pytest.mark.parametrize("bf16,lr", [(True, 1), (True, 2), (False, 1)])
@pytest.mark.parametrize("hd,shared", [(128, 4096), (64, 6144)])
def test_shared_pass_and_split_rows(bf16, lr, hd, shared):
    torch, sr = need_gpu()
    rng = np.random.default_rng(hd + lr)
    lens = [shared + int(n) for n in rng.integers(1, 60, ROWS)]
    for r in (0, 20, 40, 63):
        lens[r] = shared + int(rng.integers(1000, 2000))
    lens[3], lens[4], lens[5], lens[6] = 700, 5, 0, shared
    max_len, cols = shared + 2048, (shared + 2048) // PT + 3
    dtype = sr.SR_BF16 if bf16 else sr.SR_F32
    both, alone = slots(sr, dtype, hd, lr, cols, shared, max_len), slots(sr, dtype, hd, lr, cols, shared, shared + 32)
    assert both[1] == alone[1] == ROWS and both[0] > alone[0] > 1, (both, alone)     # the plan that is meant
    say(f"attention over 4 bits, shared pass and splits bf16={bf16} hd={hd} lr={lr}")
    cache = Rows(rng, lens, PT, HKV, hd, shared=shared // PT, holes={(7, 40): -1, (40, shared // PT + 5): -1}, cols=cols)
    asked = [int(n) for n in rng.integers(0, lr + 1, ROWS)] if lr > 1 else [1] * ROWS
    for r in CHECKED:
        asked[r] = lr
    new = new_tokens(lens, asked, lr)
    cache.packed = [pack(*raw) for raw in cache.raw]
    q = rng.normal(size=(ROWS, lr, HQ, hd)).astype(np.float32)
    out, _ = run(torch, sr, cache, q, asked, bf16, 0, 0, shared=shared, max_len=max_len)
    checked = [n if r in CHECKED else 0 for r, n in enumerate(new)]
    ref, bound = attention(cache, q, checked, 0, 0, bf16)
    got, want = ([a[r, :n] for r, n in enumerate(checked)] for a in (out, ref))
    for r, n in enumerate(new):
        assert (out[r, n:] == SENTINEL).all() and np.isfinite(out[r, :n]).all(), r
        if checked[r]:
            assert (np.abs(got[r] - want[r]) <= bound[r, :n]).all(), (r, np.abs(got[r] - want[r]).max())
    err = np.sqrt(sum(np.square(a - b).sum() for a, b in zip(got, want)))
    size = np.sqrt(sum(np.square(b).sum() for b in want))
    # fp32: scores of up to 100 are some 2^-23 of that off (2^-17); bf16: as the roundings add up
    most = limit(cache, q, checked, 0, 0, 4 * lr, p_bits=8)[1] if bf16 else 2.0 ** -17 * size
    assert err <= most, (err / size, most / size)

