"""Log-probabilities of given tokens, entropy and top alternatives against
float64, with masked and infinite logits, NaN, ties, strided and unaligned rows.

Bounds: z = (x - max) / T has three roundings (the difference, 1 / T, the
product): |dz| <= 3 2^-24 |z|.  e^z adds two half steps and moves by a factor
1 + dz; the sum of n terms in fixed tree order at most n 2^-24 (loose), so ln S
moves by at most 3 2^-24 E|z| + (n + 2) 2^-24, plus one step of the logarithm.
n here counts the additions an entry goes through: at most 2048 per lane and
12 across lanes and work-groups; 2^-24 (2100 + ...) is used for all sizes."""
import numpy as np
import pytest

from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ADDS = 2100.0


def plain(x, T):
    """(lp [rows][vocab], entropy) in float64 with the operator's limits."""
    x = x.astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    m = x.max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        z = np.where(x == m, 0.0, (x - m) / T)
    z = np.where(np.isneginf(m), -np.inf, z)
    e = np.exp(z)
    s = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        lp = np.where(s > 0, z - np.log(s), -np.inf)
        lp = np.where(lp < -float(np.finfo(np.float32).max), -np.inf, lp)      # no float is that low
        p = np.where(s > 0, e / s, 0.0)
        h = -np.where(p > 0, p * lp, 0.0).sum(1)
        mean = np.where(p > 0, p * np.abs(z), 0.0).sum(1)
        mean2 = np.where(p > 0, p * z * z, 0.0).sum(1)
    return x, z, lp, h, mean, mean2


def check(torch, sr, logits, tokens, T, top, what):
    say(f"logprobs {what} shape={tuple(logits.shape)} strides={logits.stride()} {logits.dtype} T={T} top={top}")
    rows, vocab = logits.shape
    f = lambda *s: torch.full(s, 77.0, device="cuda")  # noqa: E731
    lp, h, tl = f(rows), f(rows), f(rows, top)
    ti = torch.full((rows, top), 77, dtype=torch.int32, device="cuda")
    tok = torch.tensor(tokens, dtype=torch.int32, device="cuda")
    sr.token_logprobs(logits, tok, lp, h, ti if top else None, tl if top else None, temperature=T)
    x, z, ref, rh, mean, mean2 = plain(logits.float().cpu().numpy(), T)
    base = U * (3 * mean + ADDS + 4)                                # of ln S
    lp, h, tl, ti = (a.cpu().numpy().astype(np.float64) for a in (lp, h, tl, ti))
    for r, t in enumerate(tokens):
        if t == -1:
            assert lp[r] == 0.0
        elif not 0 <= t < vocab:
            assert np.isnan(lp[r])
        elif np.isneginf(ref[r, t]):
            assert np.isneginf(lp[r])
        else:
            assert abs(lp[r] - ref[r, t]) <= base[r] + U * (4 * abs(z[r, t]) + 2 * abs(ref[r, t])), (r, lp[r], ref[r, t])
    # H = ln S + E|z|: the mean's terms move by 3 |z| (once in z, once in e^z) and the sums
    hb = base + U * (3 * mean + 3 * mean2 + mean * (2 * ADDS + 8) + 3 * mean * mean + 2 * np.abs(rh))
    assert (np.abs(h - rh) <= hb).all(), (np.abs(h - rh) - hb).max()
    if top:
        order = np.argsort(-x, axis=1, kind="stable")[:, :top]
        assert np.array_equal(ti, order)
        want = np.take_along_axis(ref, order, 1)
        zt = np.take_along_axis(z, order, 1)
        inf = np.isneginf(want)
        assert np.array_equal(np.isneginf(tl), inf)
        ok = np.abs(np.where(inf, 0, tl) - np.where(inf, 0, want)) <= \
            base[:, None] + U * (4 * np.abs(np.where(inf, 0, zt)) + 2 * np.abs(np.where(inf, 0, want)))
        assert ok.all()


SIZES = [(1, 1, 1), (1, 2, 2), (3, 63, 5), (2, 64, 32), (5, 257, 1), (4, 1000, 32), (2, 4099, 7), (3, 8192, 20),
         (2, 32000, 5), (1, 50257, 32), (1, 128256, 20), (2, 262144, 0), (300, 5000, 4), (700, 1023, 0), (1100, 129, 3)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,vocab,top", SIZES)
def test_against_float64(rows, vocab, top, bf16):
    torch, sr = need_gpu()
    rng = np.random.default_rng(vocab + rows)
    x = torch.from_numpy(rng.normal(0, 2.5, (rows, vocab)).astype(np.float32)).cuda()
    x = x.to(torch.bfloat16) if bf16 else x
    tokens = rng.integers(0, vocab, rows).tolist()
    if rows > 2:
        tokens[0], tokens[1], tokens[2] = -1, vocab, -7
    for T in (1.0, 0.7, 3.0):
        check(torch, sr, x, tokens, T, top, "normal")


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("vocab", [70, 4100, 33000, 128256])
def test_masks_infinities_nan_and_ties(vocab, bf16):
    torch, sr = need_gpu()
    rng = np.random.default_rng(vocab)
    x = rng.normal(0, 2, (11, vocab)).astype(np.float32)
    x[0] = -np.inf                                               # nothing allowed
    x[1, rng.random(vocab) < 0.99] = -np.inf                     # almost nothing (maybe fewer than top)
    x[2, :] = -np.inf
    x[2, vocab - 1] = 3.0                                        # one token
    x[3, ::3] = np.nan
    x[4] = np.nan
    x[5, [1, vocab - 2]] = np.inf                                # two share it
    x[6] = 1.25                                                  # all tie
    x[7] = np.finfo(np.float32).min                              # a mask of the type's lowest value
    x[7, 5] = 0.0
    x[8] = np.round(x[8] * 2) / 2                                # many ties
    x[9] = np.where(rng.random(vocab) < 0.5, 0.0, -0.0)
    x[10] = np.finfo(np.float32).min                             # the lowest value everywhere
    t = torch.from_numpy(x).cuda()
    if bf16:
        t = t.clamp(min=-3.3e38).to(torch.bfloat16).masked_fill(torch.from_numpy(np.isneginf(x)).cuda(), float("-inf"))
    for tok in (0, 1, vocab - 1):
        check(torch, sr, t, [tok] * 11, 1.0, 20, "masks")
    check(torch, sr, t, [5] * 11, 0.5, 32, "masks")


@pytest.mark.parametrize("bf16", [False, True])
def test_strided_and_unaligned_rows(bf16):
    torch, sr = need_gpu()
    big = torch.randn((6, 9001), device="cuda").to(torch.bfloat16 if bf16 else torch.float32)
    for a, b in ((0, 9000), (1, 9001), (3, 700), (2, 5000)):
        check(torch, sr, big[:, a:b], [0, 5, 6, 100, -1, 3], 1.0, 6, "strided")
        check(torch, sr, big[::2, a:b], [0, 5, 6], 1.0, 6, "every other row")


def test_outputs_are_optional():
    torch, sr = need_gpu()
    x = torch.randn((3, 5000), device="cuda")
    tok = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    full = [torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda"), torch.zeros((3, 4), dtype=torch.int32, device="cuda"),
            torch.zeros((3, 4), device="cuda")]
    sr.token_logprobs(x, tok, *full)
    for i in range(4):
        part = [torch.zeros_like(t) if j == i else None for j, t in enumerate(full)]
        sr.token_logprobs(x, tok if i == 0 else None, *part)
        assert torch.equal(part[i], full[i])


def test_agrees_with_the_log_probability_reward():
    """The sum over a response equals what sr_generate accumulates, to rounding."""
    torch, sr = need_gpu()
    x = torch.randn((64, 4097), device="cuda") * 3
    tok = torch.randint(0, 4097, (64,), dtype=torch.int32, device="cuda")
    lp = torch.zeros(64, device="cuda")
    sr.token_logprobs(x, tok, lp)
    want = torch.log_softmax(x.double(), 1).gather(1, tok.long()[:, None])[:, 0]
    assert float((lp.double() - want).abs().max()) < 2e-4   # U * (ADDS + 3 * 30 + ...) with |lp| < 30


def test_graph_replays_and_streams():
    torch, sr = need_gpu()
    for rows, vocab in ((1, 100003), (400, 3001)):
        x = torch.randn((rows, vocab), device="cuda")
        tok = torch.randint(0, vocab, (rows,), dtype=torch.int32, device="cuda")
        outs = lambda: [torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"),  # noqa: E731
                        torch.zeros((rows, 9), dtype=torch.int32, device="cuda"), torch.zeros((rows, 9), device="cuda")]
        want, got = outs(), outs()
        sr.token_logprobs(x, tok, *want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        sr.token_logprobs(x, tok, *got, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sr.token_logprobs(x, tok, *got)
        for _ in range(3):
            for t in got:
                t.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            sr.token_logprobs(x * 2, tok, *outs())
