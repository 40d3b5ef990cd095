"""Attention over long rows in bf16, every part of which matters, against 64 bits
within a bound on each head's 2-norm (paged_long): many splits, joins, the shared
pass beside tails, windows and sinks, drafts, chunks and prompts."""
import numpy as np
import pytest

from gpu_util import need_gpu, say
from paged_long import CASES, make
from test_gpu_paged_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("marked", [True, False])
def test_long_rows(name, marked):
    torch, sr = need_gpu()
    c = make(name, marked)
    say(f"long rows {name} marked={marked} rows={len(c.new)}")
    c.cache.poison(c.new, c.window, c.sinks)
    asked = c.asked or [c.lr] * len(c.new)
    out, _ = run(torch, sr, c.cache, c.q, asked, c.lr, c.window, c.sinks, c.shared, c.max_len, ragged=c.asked is not None)
    worst = c.worst(out, c.oracle())
    say(f"  {worst:.3f} of the bound")
    assert worst <= 1.0
    if c.shared:                                    # the hint changes nothing beyond rounding
        alone, _ = run(torch, sr, c.cache, c.q, asked, c.lr, c.window, c.sinks, 0, c.max_len, ragged=c.asked is not None)
        assert c.worst(alone, c.oracle()) <= 1.0
