"""How precise bf16 calls of attention over 4 bits are as a whole: the 2-norm of the
error of all outputs stays within what the stated roundings add up to
(fp4_precision.limit).  The elements' own bounds (test_gpu_paged_attention_fp4) allow
for roundings that all lie the same way and would hide a lost part of a query or of a
probability."""
import numpy as np
import pytest

from fp4_precision import limit, six_bit_parts, with_8_bits
from fp4_util import Cache4, dequantise
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


def in_parts(q, parts):
    """Queries as the prompts' products see them: parts of 6 bits."""
    scale = np.float32(1.4426950408889634 / np.sqrt(q.shape[-1]))
    return six_bit_parts(q * scale, parts)[0] / scale


def check_prompt(cache, q, lens, window, sinks, needed, what):
    """Its 2-norm; that queries of fewer than `needed` parts would exceed the limit is seen
    first."""
    rows, lr, hq, hd = q.shape
    new = new_tokens(lens, [lr] * rows, lr)
    cache.poison(new, window, sinks)
    ref, most = limit(cache, q, new, window, sinks, lr * hq // cache.hkv)
    whole, short = (limit(cache, in_parts(q, n), new, window, sinks, 99)[0] for n in (3, needed - 1))
    assert error(whole, ref, new) < most / 4 and error(short, ref, new) > most
    torch, sr = need_gpu()
    say(f"attention over 4 bits, precision of prompts {what} hd={hd} {hq}/{cache.hkv} lr={lr} window={window}")
    out, _ = run(torch, sr, cache, q, [lr] * rows, True, window, sinks)
    assert error(out, ref, new) <= most, (error(out, ref, new) / np.linalg.norm(ref), most / np.linalg.norm(ref))


def positive_keys(cache):
    cache.raw[0] = (cache.raw[0][0] & 7, np.full_like(cache.raw[0][1], 126))      # of one scale
    cache.k = dequantise(*cache.raw[0])


@pytest.mark.parametrize("hd,hq,hkv", [(32, 4, 2), (64, 8, 2), (128, 8, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
def test_prompts(hd, hq, hkv, window, sinks):
    rng = np.random.default_rng(hd)
    lens = [300, 150, 45]
    cache = Cache4(rng, lens, 32, hkv, hd)
    check_prompt(cache, rng.normal(size=(3, 40, hq, hd)).astype(np.float32), lens, window, sinks, 2, "moderate")


@pytest.mark.parametrize("hd,hq,hkv", [(32, 4, 2), (64, 8, 2), (128, 8, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
@pytest.mark.parametrize("sign", [-1, 1])
def test_prompts_with_scores_far_from_zero(hd, hq, hkv, window, sinks, sign):
    """All scores of a row some hundreds below or above 0, where the running maximum comes
    off in the products."""
    rng = np.random.default_rng(hd + sign)
    lens = [700, 75, 41]
    cache = Cache4(rng, lens, 32, hkv, hd)
    positive_keys(cache)
    check_prompt(cache, (sign * 60 * (1 + 0.05 * rng.normal(size=(3, 40, hq, hd)))).astype(np.float32), lens, window, sinks, 2, f"far {sign}")


@pytest.mark.parametrize("hd,hq,hkv", [(32, 4, 2), (64, 8, 2), (128, 8, 2)])
@pytest.mark.parametrize("sign", [-1, 1])
def test_prompts_whose_far_scores_almost_tie(hd, hq, hkv, sign):
    """Every token sees two keys whose scores, some hundreds from 0, differ by about 1:
    every part of a query moves the output."""
    rng = np.random.default_rng(hd + sign)
    lens, lr = [200, 131], 70
    cache = Cache4(rng, lens, 16, hkv, hd)
    positive_keys(cache)
    q = sign * 60 * (1 + 0.5 * rng.normal(size=(2, lr, hq, hd)))
    for r in range(2):
        k = cache.rows_kv(r)[0]
        for t in range(lr):
            pos = lens[r] - lr + t
            diff = np.repeat(k[pos] - k[pos - 1], hq // hkv, axis=0)
            q[r, t] += ((rng.normal(size=hq) * np.sqrt(hd) - (q[r, t] * diff).sum(1)) / (diff * diff).sum(1))[:, None] * diff
    check_prompt(cache, q.astype(np.float32), lens, 2, 0, 3, f"far, close {sign}")
