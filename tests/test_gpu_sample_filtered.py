"""The filtered draw against its definition in whole numbers: every type and size,
settings for all rows and for each, masks, infinities, NaN, ties, flat rows whose
kept part is large, rows whose entries lie in a hair's breadth, strided and
unaligned rows, graphs and streams.  Tokens and counts are equal; the
log-probability of the drawn token is a double's logarithm rounded to fp32, so it
is off by at most 2^-24 of itself and a few 2^-52."""
import numpy as np
import pytest

from gpu_util import need_gpu, say
from oracle.sampler import exp_sr

pytestmark = pytest.mark.gpu

ONE = 1 << 32


def weights(x, T):
    """Integer weights of one row (float32, NaN as -inf), or None for a greedy T."""
    T = np.float32(T)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        inv = np.float32(1.0 / float(T)) if float(T) != 0 else np.float32(np.inf)
    if not T > 0 or not np.isfinite(inv):
        return None
    m = x.max()
    if m == np.inf:
        return np.where(x == m, ONE, 0).astype(np.uint64)
    with np.errstate(invalid="ignore", over="ignore"):
        z = ((x - m).astype(np.float32) * inv).astype(np.float32)
    return (exp_sr(z) * np.float32(ONE)).astype(np.float32).astype(np.uint64)


def plain(x, T, k, p, min_p, word):
    """(token, log-probability, kept) of one row."""
    x = np.where(np.isnan(x), np.float32(-np.inf), x.astype(np.float32))
    if x.max() == -np.inf:
        return 0, -np.inf, 0
    w = weights(x, T)
    if w is None:
        return int(np.argmax(x)), 0.0, 1
    order = np.lexsort((np.arange(len(x)), -x))
    if 1 <= k < len(x):
        order = order[:k]
    run = np.cumsum(w[order], dtype=np.uint64)
    p = np.float32(p)
    if p < 1:
        part = int(max(float(p), 0.0) * ONE)
        need = max(1, -(-part * int(run[-1]) // ONE))
        order = order[:int((run < np.uint64(need)).sum()) + 1]
    min_p = np.float32(min_p)
    least = int(min(float(min_p), 1.0) * ONE) if min_p > 0 else 0
    order = order[w[order] >= np.uint64(least)]
    order = np.sort(order[w[order] > 0])
    run = np.cumsum(w[order], dtype=np.uint64)
    total = int(run[-1])
    i = order[int((run <= np.uint64(word * total >> 32)).sum())]
    return int(i), float(np.log(int(w[i]) / total)), len(order)


def check(torch, sr, logits, T=1.0, k=0, p=1.0, min_p=0.0, words=None, what="", stream=None):
    rows, vocab = logits.shape
    rng = np.random.default_rng(rows * 7 + vocab)
    if words is None:
        words = rng.integers(0, ONE, rows)
        words[0] = ONE - 1
        words[-1] = 0
    say(f"draw {what} {tuple(logits.shape)} strides={logits.stride()} {logits.dtype} T={T} k={k} p={p} min_p={min_p}"[:300])
    arg = lambda v, t: torch.tensor(v, dtype=t, device="cuda") if isinstance(v, (list, np.ndarray)) else v  # noqa: E731
    token, kept = (torch.full((rows,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    lp = torch.full((rows,), 7.0, device="cuda")
    word = torch.from_numpy(words.astype(np.uint32).view(np.int32)).cuda()
    torch.cuda.synchronize()
    sr.sample_filtered(logits, word, token, temperature=arg(T, torch.float32), top_k=arg(k, torch.int32),
                       top_p=arg(p, torch.float32), min_p=arg(min_p, torch.float32), logprob=lp, kept=kept, stream=stream)
    torch.cuda.synchronize()
    x = logits.float().cpu().numpy()
    token, kept, lp = token.cpu().numpy(), kept.cpu().numpy(), lp.cpu().numpy().astype(np.float64)
    at = lambda v, r: v[r] if isinstance(v, (list, np.ndarray)) else v  # noqa: E731
    for r in range(rows):
        want = plain(x[r], at(T, r), at(k, r), at(p, r), at(min_p, r), int(words[r]))
        assert (token[r], kept[r]) == (want[0], want[2]), (r, token[r], kept[r], want)
        if np.isinf(want[1]):
            assert lp[r] == want[1]
        else:
            assert abs(lp[r] - want[1]) <= 2.0 ** -24 * abs(want[1]) + 2.0 ** -50, (r, lp[r], want[1])


SIZES = [(3, 1), (3, 2), (2, 63), (5, 64), (4, 1000), (3, 1024), (3, 1025), (2, 4099), (4, 8192), (3, 32000), (2, 50257),
         (2, 128256), (1, 262144), (70, 513), (300, 1999)]
SETTINGS = [dict(), dict(k=1), dict(k=50), dict(p=0.9), dict(k=40, p=0.8, T=0.7), dict(min_p=0.05), dict(k=200, p=0.95, min_p=0.01),
            dict(k=5000, T=1.5), dict(p=0.999, T=2.0), dict(T=0.0), dict(p=0.5, min_p=0.2, T=0.3)]


def spread(rng, rows, vocab, kind):
    if kind == "flat":
        return rng.normal(0, 2, (rows, vocab))
    return rng.exponential(1.4, (rows, vocab)) + rng.normal(0, 0.3, (rows, vocab))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_against_whole_numbers(rows, vocab, bf16):
    torch, sr = need_gpu()
    rng = np.random.default_rng(vocab)
    for kind in ("flat", "peaked"):
        x = torch.from_numpy(spread(rng, rows, vocab, kind).astype(np.float32)).cuda()
        x = x.to(torch.bfloat16) if bf16 else x
        for s in SETTINGS if vocab < 100000 else SETTINGS[1:7:2] + SETTINGS[6:9]:
            check(torch, sr, x, what=kind, **s)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("vocab", [70, 4100, 33000])
def test_masks_infinities_nan_and_ties(vocab, bf16):
    torch, sr = need_gpu()
    rng = np.random.default_rng(vocab)
    x = rng.normal(0, 2, (13, vocab)).astype(np.float32)
    x[0] = -np.inf                                               # nothing allowed
    x[1, rng.random(vocab) < 0.99] = -np.inf                     # almost nothing
    x[2, :] = -np.inf
    x[2, vocab - 1] = 3.0                                        # one token
    x[3, ::3] = np.nan
    x[4] = np.nan
    x[5, [1, vocab // 2, vocab - 2]] = np.inf                    # three share it
    x[6] = 1.25                                                  # all tie
    x[7] = np.finfo(np.float32).min                              # a mask of the type's lowest value
    x[7, 5] = 0.0
    x[8] = np.round(x[8] * 2) / 2                                # many ties
    x[9] = np.where(rng.random(vocab) < 0.5, 0.0, -0.0)
    x[10] = np.finfo(np.float32).min                             # the lowest value everywhere
    x[11] = 3.0 + rng.integers(0, 9000, vocab) * 2.0 ** -22      # within a hair's breadth
    x[12, ::2] = -np.inf
    t = torch.from_numpy(x).cuda()
    if bf16:
        t = t.clamp(min=-3.3e38).to(torch.bfloat16).masked_fill(torch.from_numpy(np.isneginf(x)).cuda(), float("-inf"))
    for s in SETTINGS + [dict(k=vocab - 1), dict(k=vocab), dict(k=2, p=0.5), dict(k=vocab // 2, p=0.4), dict(p=0.3), dict(p=0.7, T=50.0)]:
        check(torch, sr, t, what="masks", **s)


@pytest.mark.parametrize("vocab", [9000, 131072])
def test_borders_among_many_equals(vocab):
    """More equal entries at the border than a list holds, and more in a bin."""
    torch, sr = need_gpu()
    rng = np.random.default_rng(vocab)
    x = np.zeros((6, vocab), np.float32)
    x[0, ::7] = 1.0
    x[1] = rng.integers(0, 2, vocab)
    x[2] = 5.0 - rng.integers(0, 3, vocab) * np.float32(2.0 ** -20)
    x[3] = 1.0 + rng.random(vocab).astype(np.float32) * np.float32(1e-3)
    x[4] = rng.random(vocab).astype(np.float32) * np.float32(1e-4)
    x[5] = np.where(rng.random(vocab) < 0.9, 2.0, rng.normal(0, 1, vocab))
    t = torch.from_numpy(x).cuda()
    for s in (dict(k=5000), dict(k=vocab // 2 + 1), dict(p=0.5), dict(p=0.77, k=vocab - 3), dict(k=6001, p=0.9), dict(p=1e-9),
              dict(p=0.999999), dict(min_p=1.0), dict(min_p=0.4, p=0.9)):
        check(torch, sr, t, what="equals", **s)


@pytest.mark.parametrize("rows", [2, 140])
def test_entries_down_to_weight_zero(rows):
    """A top-k whose border lies where weights have run out: entries of weight 0 are
    not counted as kept."""
    torch, sr = need_gpu()
    vocab = 40001
    x = np.stack([-np.linspace(0, (22.1, 22.24, 22.3, 23.0, 30.0)[r % 5], vocab)[np.random.default_rng(r).permutation(vocab)]
                  for r in range(rows)]).astype(np.float32)
    for s in (dict(k=vocab - 1), dict(k=39900), dict(k=39900, p=1 - 2.0 ** -24), dict(k=20000), dict(p=1 - 2.0 ** -24), dict(k=39990, min_p=2.0 ** -31)):
        check(torch, sr, torch.from_numpy(x).cuda(), what="ramp", **s)


@pytest.mark.parametrize("bf16", [False, True])
def test_many_long_rows(bf16):
    """More rows than have their readings shared out, each with settings of its own."""
    torch, sr = need_gpu()
    rng = np.random.default_rng(5)
    rows, vocab = 150, 40000
    x = np.concatenate([spread(rng, rows // 2, vocab, kind) for kind in ("flat", "peaked")]).astype(np.float32)
    x[::9] = np.round(x[::9])
    x[4::11, ::2] = -np.inf
    x[5::13, rng.integers(0, vocab, 3)] = np.inf
    x[6::17, rng.integers(0, vocab, 900)] = np.nan
    x[[7, 70]] = -np.inf
    x[[8, 80], 1:] = -np.inf
    x = torch.from_numpy(x).cuda().to(torch.bfloat16 if bf16 else torch.float32)
    f = lambda *v: rng.choice(np.array(v, np.float32), rows)  # noqa: E731
    for _ in range(3):
        check(torch, sr, x, f(0, 0.5, 1, 1.7), rng.choice(np.array([0, 1, 7, 300, 1024, 1025, 6000], np.int32), rows),
              f(1, 0.3, 0.9, 0.99), f(0, 0, 0.02, 0.3), what="long")


def test_odd_settings():
    """What is outside the usual ranges has its documented meaning."""
    torch, sr = need_gpu()
    x = torch.randn((4, 3000), device="cuda") * 2
    nan, inf = float("nan"), float("inf")
    for s in (dict(T=-1.0), dict(T=nan), dict(T=1e-39), dict(T=inf), dict(T=3e38), dict(T=1e-37), dict(k=-5), dict(k=3000), dict(k=2 ** 31 - 1),
              dict(p=0.0), dict(p=-1.0), dict(p=nan), dict(p=2.0), dict(p=inf), dict(p=1 - 2.0 ** -24), dict(min_p=nan), dict(min_p=-1.0),
              dict(min_p=7.0), dict(min_p=inf), dict(p=1e-30), dict(min_p=1e-30)):
        check(torch, sr, x, what="odd", **s)


@pytest.mark.parametrize("bf16", [False, True])
def test_settings_of_every_row(bf16):
    torch, sr = need_gpu()
    rng = np.random.default_rng(11)
    rows, vocab = 64, 5003
    x = np.concatenate([spread(rng, rows // 2, vocab, kind) for kind in ("flat", "peaked")]).astype(np.float32)
    x = torch.from_numpy(x).cuda().to(torch.bfloat16 if bf16 else torch.float32)
    f = lambda *v: rng.choice(np.array(v, np.float32), rows)  # noqa: E731
    check(torch, sr, x, f(0, 0.5, 1, 1.7), rng.choice(np.array([0, 1, 7, 300, 6000], np.int32), rows), f(1, 0.3, 0.9, 0.99),
          f(0, 0.02, 0.3), what="each")
    check(torch, sr, x, 0.8, rng.integers(0, 90, rows).astype(np.int32), 0.9, f(0, 0.1), what="some")


@pytest.mark.parametrize("bf16", [False, True])
def test_strided_and_unaligned_rows(bf16):
    torch, sr = need_gpu()
    big = torch.randn((6, 9001), device="cuda").to(torch.bfloat16 if bf16 else torch.float32)
    for a, b in ((0, 9000), (1, 9001), (3, 700), (2, 5000)):
        for s in (dict(), dict(k=9, p=0.9), dict(p=0.95)):
            check(torch, sr, big[:, a:b], what="strided", **s)
            check(torch, sr, big[::2, a:b], what="every other row", **s)


def test_unfiltered_draws_are_sr_samples():
    torch, sr = need_gpu()
    for rows, vocab, T in ((64, 8191, 1.0), (33, 512, 0.7), (5, 128256, 1.3), (7, 100, 0.0)):
        x = torch.randn((rows, vocab), device="cuda") * 3
        cand = torch.arange(rows, dtype=torch.int32, device="cuda") * 5 + 1
        want, got = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
        for step in range(4):
            sr.sample(x, cand, step, T, 1234567890123, want)
            ctr = torch.zeros((rows, 4), dtype=torch.int32, device="cuda")
            ctr[:, 0], ctr[:, 1] = step, cand
            words = torch.zeros((rows, 4), dtype=torch.int32, device="cuda")
            sr.philox_fill(1234567890123, ctr, words)
            sr.sample_filtered(x, words[:, 0], got, temperature=T)     # (a strided column)
            assert torch.equal(got, want), (rows, vocab, T)


def test_logprob_is_that_of_token_logprobs_when_nothing_is_filtered():
    torch, sr = need_gpu()
    x = torch.randn((40, 3001), device="cuda") * 2
    words = torch.randint(-2 ** 31, 2 ** 31 - 1, (40,), dtype=torch.int32, device="cuda")
    token, lp, want = torch.zeros(40, dtype=torch.int32, device="cuda"), torch.zeros(40, device="cuda"), torch.zeros(40, device="cuda")
    sr.sample_filtered(x, words, token, temperature=0.9, logprob=lp)
    sr.token_logprobs(x, token, want, temperature=0.9)
    # weights are cut to 2^-32 of the largest: 3001 of them, and fp32 sums
    assert float((lp - want).abs().max()) <= 3001 * 2.0 ** -32 + 2.0 ** -24 * 3200


def test_outputs_are_optional():
    torch, sr = need_gpu()
    x = torch.randn((3, 5000), device="cuda")
    words = torch.tensor([5, -5, 2 ** 30], dtype=torch.int32, device="cuda")
    full = dict(tokens=torch.zeros(3, dtype=torch.int32, device="cuda"), logprob=torch.zeros(3, device="cuda"),
                kept=torch.zeros(3, dtype=torch.int32, device="cuda"))
    for s in (dict(), dict(top_k=30), dict(top_p=0.9), dict(temperature=0.0)):
        sr.sample_filtered(x, words, **full, **s)
        for name, t in full.items():
            part = {n: torch.zeros_like(t) if n == name else None for n in full}
            sr.sample_filtered(x, words, **part, **s)
            assert torch.equal(part[name], t)


def test_graph_replays_and_streams():
    torch, sr = need_gpu()
    for rows, vocab, s in ((1, 100003, dict(top_k=40, top_p=0.9)), (300, 3001, dict(top_p=0.95)), (7, 50000, dict()),
                           (2, 60000, dict(top_k=9000, temperature=2.0))):
        x = torch.randn((rows, vocab), device="cuda") * 2
        words = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows,), dtype=torch.int32, device="cuda")
        outs = lambda: [torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, device="cuda"),  # noqa: E731
                        torch.zeros(rows, dtype=torch.int32, device="cuda")]
        call = lambda y, o, st=None: sr.sample_filtered(y, words, o[0], logprob=o[1], kept=o[2], stream=st, **s)  # noqa: E731
        want, got = outs(), outs()
        call(x, want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        call(x, got, side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(x, got)
        for _ in range(3):
            for t in got:
                t.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            call(x * 2, outs())
