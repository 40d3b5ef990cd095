"""How precise bf16 calls of attention over 4 bits are as a whole: the 2-norm of the
error of all outputs stays within what the stated roundings add up to
(fp4_precision.limit).  The elements' own bounds (test_gpu_paged_attention_fp4) allow
for roundings that all lie the same way and would hide a lost part of a query or of a
probability."""
import numpy as np
import pytest

from fp4_precision import limit, with_8_bits
from fp4_util import Cache4
from gpu_util import need_gpu, say
from paged_util import new_tokens
from test_gpu_paged_attention_fp4 import run

pytestmark = pytest.mark.gpu


def error(out, ref, new):
    return np.linalg.norm(np.concatenate([(out - ref)[r, :n].ravel() for r, n in enumerate(new)]))


@pytest.mark.parametrize("hd,hq,hkv,lr", [(32, 4, 4, 1), (32, 16, 2, 1), (64, 8, 2, 1), (64, 4, 2, 4), (128, 8, 1, 1), (128, 8, 2, 2), (128, 6, 2, 1)])
def test_up_to_8_columns_are_off_by_the_outputs_rounding(hd, hq, hkv, lr):
    """Queries and probabilities keep 16 bits: what is left is the outputs' own rounding."""
    torch, sr = need_gpu()
    say(f"attention over 4 bits, precision of probabilities hd={hd} {hq}/{hkv} lr={lr}")
    lens = [257, 100, 164, 133, 700, 140, 2000, 90, 120]
    for window, sinks in ((0, 0), (70, 3)):
        rng = np.random.default_rng(hd + lr)
        cache = Cache4(rng, lens, 32, hkv, hd)
        new = new_tokens(lens, [lr] * len(lens), lr)
        cache.poison(new, window, sinks)
        q = (0.05 * rng.normal(size=(len(lens), lr, hq, hd))).astype(np.float32)     # (many keys weigh)
        ref, most = limit(cache, q, new, window, sinks, lr * hq // hkv)
        assert error(with_8_bits(cache, q, new, window, sinks), ref, new) > most    # (or there is nothing to see)
        out, _ = run(torch, sr, cache, q, [lr] * len(lens), True, window, sinks)
        assert error(out, ref, new) <= most, (error(out, ref, new) / np.linalg.norm(ref), most / np.linalg.norm(ref))
