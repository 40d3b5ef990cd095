"""token_logprobs against the framework's own log-probability reward and sampler:
the sum over a response is what sr_generate scores it by, and the distribution is
the one that sr_sample draws from, at any temperature and with NaN logits."""
import numpy as np
import pytest

from gpu_util import device_models, need_gpu, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,temperature", [("tiny_fp32", 1.0), ("tiny_fp32", 0.6), ("small_bf16", 1.3)])
def test_sum_is_the_score_of_a_run(name, temperature):
    """sr_generate with the log-probability reward: mean ln p of the answer's and
    other candidates' tokens under the logits the run drew them from (softmax at
    temperature 1, whatever it drew at)."""
    torch, sr = need_gpu()
    say(f"log-probability reward {name} T={temperature}")
    c, gen, _, prompt = device_models(name)
    c = c.with_(temperature=temperature)
    p = sr.make_params(c.n, c.alpha, c.tau, c.max_new_tokens, temperature, c.sample_seed, c.eos_id, c.max_rounds,
                       reward_kind=sr.SR_REWARD_LOGPROB)
    out = sr.generate(gen, None, prompt, p, trace=True)
    final = out["trace"]["final_scores"]
    watch = [int(k) for k in np.nonzero(~np.isnan(final))[0][:3]]
    assert out["best_index"] in np.nonzero(~np.isnan(final))[0] and len(watch) > 0
    out = sr.generate(gen, None, prompt, p, watch=watch)
    t = out["trace"]
    for i, k in enumerate(watch):
        n = int(t["all_len"][k])
        logits = torch.from_numpy(t["watch_logits"][i, :n].copy()).cuda()
        tokens = torch.from_numpy(t["all_tokens"][k, :n].copy()).cuda()
        lp = torch.zeros(n, device="cuda")
        sr.token_logprobs(logits, tokens, lp)
        # each ln p: 2^-24 (2100 + 3 E|z| + 4 |z| + 2 |ln p|) on either side with |z| < 40;
        # the run adds them up one by one in fp32: n steps of 2^-24 of the sum
        each = lp.double().cpu().numpy()
        bound = 2 * 2.0 ** -24 * (2100 + 9 * 40) + n * 2.0 ** -24 * np.abs(each).mean()
        assert abs(each.mean() - t["final_scores"][k]) <= bound, (k, each.mean(), t["final_scores"][k])


@pytest.mark.parametrize("temperature", [0.5, 1.0, 2.0])
def test_distribution_is_the_samplers(temperature):
    """200000 draws of one row: every token's share is its probability within six
    standard deviations; a NaN logit is never drawn."""
    torch, sr = need_gpu()
    say(f"sampler's distribution T={temperature}")
    vocab, rows, seen = 24, 4096, np.zeros(24, dtype=np.int64)
    g = torch.Generator(device="cuda").manual_seed(11)
    x = torch.randn(vocab, device="cuda", generator=g) * 1.5
    x[3], x[17] = float("nan"), float("-inf")
    logits = x.expand(rows, vocab).contiguous()
    cand = torch.arange(rows, dtype=torch.int32, device="cuda")
    steps = 49
    for step in range(steps):
        tok = torch.zeros(rows, dtype=torch.int32, device="cuda")
        sr.sample(logits, cand, step, temperature, 77, tok)
        seen += np.bincount(tok.cpu().numpy(), minlength=vocab)
    lp = torch.zeros(vocab, device="cuda")
    sr.token_logprobs(x.expand(vocab, vocab).contiguous(), torch.arange(vocab, dtype=torch.int32, device="cuda"), lp,
                      temperature=temperature)
    p = np.exp(lp.double().cpu().numpy())
    assert p[3] == 0 and p[17] == 0 and abs(p.sum() - 1) < 1e-4
    n = rows * steps
    assert (np.abs(seen - n * p) <= 6 * np.sqrt(n * p * (1 - p))).all(), (seen / n - p)
