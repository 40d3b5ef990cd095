"""What lies in the padded queries of a ragged call changes nothing, not even a
rounding: outputs are the same bit for bit whatever is there."""
import numpy as np
import pytest

from gpu_util import need_gpu, say
from paged_util import Cache, new_tokens
from test_gpu_paged_attention import SENTINEL, run

pytestmark = pytest.mark.gpu

# (bf16, hd, hq, hkv, lens, lr, pt, window, sinks, shared, n_new)
CASES = {
    "vector": (False, 64, 8, 2, [90, 40], 30, 16, 0, 0, 0, [17, 3]),
    "wave": (True, 128, 8, 2, [200, 90], 3, 32, 0, 0, 0, [2, 1]),
    "tile": (True, 128, 8, 2, [150, 370, 70, 1], 70, 32, 0, 0, 0, [33, 41, 70, 1]),
    "tile_window": (True, 64, 8, 2, [400, 300], 90, 16, 100, 5, 0, [21, 75]),
    "tile_split": (True, 64, 8, 2, [2100, 333], 40, 64, 0, 0, 0, [13, 20]),
    "shared": (True, 128, 4, 1, [1024 + 1 + i % 40 for i in range(700)], 2, 64, 0, 0, 1024, [i % 3 for i in range(700)]),
}


@pytest.mark.parametrize("name", list(CASES))
def test_padded_queries_change_nothing(name):
    torch, sr = need_gpu()
    say(f"padded queries {name}")
    bf16, hd, hq, hkv, lens, lr, pt, window, sinks, shared, n_new = CASES[name]
    rng = np.random.default_rng(41)
    cache = Cache(rng, lens, pt, hkv, hd, bf16, shared // pt)
    new = new_tokens(lens, n_new, lr)
    cache.poison(new, window, sinks)
    q = rng.normal(size=(len(lens), lr, hq, hd)).astype(np.float32)
    pad = np.arange(lr)[None, :] >= np.array(new)[:, None]
    assert pad.any()
    outs = []
    for fill in (0.0, 1.0, 300.0, np.nan, np.inf):
        x = q.copy()
        x[pad] = fill if fill in (0.0,) or not np.isfinite(fill) else fill * rng.normal(size=x[pad].shape)
        out, _ = run(torch, sr, cache, x, n_new, lr, window, sinks, shared)
        assert (out[pad] == SENTINEL).all()
        assert np.isfinite(out[~pad]).all()
        outs.append(out)
    for out in outs[1:]:
        assert np.array_equal(out, outs[0])
