"""The filtered draw of rows whose logits depend on the token's index, so many rows
that a row's list of its best entries comes from one reading: logits that fall or rise
with the index, the best entries in one tile, whole tiles masked by -inf, by the types'
lowest values or by some large negative number, few entries left.  Results against whole
numbers; and such rows take no more than twice the time of rows without an order."""
import numpy as np
import pytest

from gpu_util import need_gpu, say
from test_gpu_sample_filtered import check

pytestmark = pytest.mark.gpu

KINDS = ["falls", "falls fast", "rises", "one tile", "first tile", "masked -inf", "masked lowest", "masked finite", "all but one masked",
         "few left", "falls in steps", "lowest everywhere", "lowest but 60"]


def ordered(rng, vocab, kind):
    x, i = rng.normal(0, 2, vocab), np.arange(vocab)
    low = np.finfo(np.float32).min
    if kind == "falls":
        x -= 0.6 * np.log1p(i)
    elif kind == "falls fast":
        x = 5 - i * 1e-3
    elif kind == "rises":
        x = i * 1e-4
    elif kind == "one tile":
        x[20 * 1024:21 * 1024] += 8
    elif kind == "first tile":
        x[3 * 1024:4 * 1024] += 8
    elif kind == "masked -inf":
        x[5 * 1024:6 * 1024], x[:1030] = -np.inf, -np.inf
    elif kind == "masked lowest":
        x[:9 * 1024] = low
    elif kind == "masked finite":
        x[1024:2048] = -1e9
    elif kind == "all but one masked":
        x[:], x[vocab - 7] = low, 1.0
    elif kind == "few left":
        x[3000:] = -np.inf
    elif kind.startswith("lowest"):
        x[:] = low
        if kind == "lowest but 60":
            x[rng.integers(0, vocab, 60)] = rng.normal(0, 2, 60)
    elif kind == "falls in steps":
        x = np.floor(8 - np.log2(1 + i))
    return x.astype(np.float32)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("vocab", [33000, 40001, 131072])
def test_logits_that_depend_on_the_index(vocab, bf16):
    torch, sr = need_gpu()
    rng = np.random.default_rng(vocab)
    rows = 132
    x = np.full((rows, vocab), -np.inf, np.float32)
    for r in range(rows if vocab < 100000 else 39):    # (the others: nothing allowed)
        x[r] = ordered(rng, vocab, KINDS[r % len(KINDS)])
    t = torch.from_numpy(x).cuda()
    if bf16:
        t = t.clamp(min=torch.finfo(torch.bfloat16).min).to(torch.bfloat16).masked_fill(torch.from_numpy(np.isneginf(x)).cuda(), float("-inf"))
    for s in (dict(k=1), dict(k=50), dict(k=1000, T=0.7), dict(k=1024, p=0.9), dict(k=50, p=0.9, min_p=0.02)):
        check(torch, sr, t, what="by index", **s)


def test_order_costs_no_passes_of_whole_rows():
    """Under a top-k the rows are read once, and in part once more at most, whatever the
    order of their entries: twice the time of rows in no order would be another two readings."""
    torch, sr = need_gpu()
    say("draw, time of rows that fall with the index")
    rows, vocab = 512, 128256
    plain = torch.randn((rows, vocab), device="cuda") * 2
    falls = plain - 0.6 * torch.log1p(torch.arange(vocab, device="cuda", dtype=torch.float32))
    masked = plain.clone()
    masked[:, :1024] = float("-inf")
    words = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows,), dtype=torch.int32, device="cuda")
    token = torch.zeros(rows, dtype=torch.int32, device="cuda")
    best = {}
    for _ in range(12):   # (in turn; the least of each)
        for name, x in (("plain", plain), ("falls", falls), ("masked", masked)):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            sr.sample_filtered(x, words, token, top_k=50, top_p=0.9)
            end.record()
            end.synchronize()
            best[name] = min(best.get(name, 1e9), start.elapsed_time(end))
    say(str(best))
    assert best["falls"] <= 2 * best["plain"] and best["masked"] <= 2 * best["plain"], best
