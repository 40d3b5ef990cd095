"""The paged operators together, as a run uses them: a prompt goes into pages,
is forked into candidates that grow token by token (projection, rotary append,
attention with a window and sinks, sampling, log-probabilities of the sampled
tokens), the better half by mean log-probability is kept at every cut and forked
into the freed rows, pages behind the window are let go, and the pool is
compacted.  Every surviving candidate's logits at every step are then those of a
dense float64 forward pass over its tokens, within the bounds the model tests
use (1e-4 of the largest for fp32, 2e-2 for bf16); its summed log-probability
differs by at most twice that per token."""
import numpy as np
import pytest

from gpu_util import need_gpu, say
from paged_util import bf16_round, visible

pytestmark = pytest.mark.gpu

LAYERS, HQ, HKV, VOCAB = 2, 4, 2, 320


def dense_logits(w, toks, hd, rot, window, sinks, freqs):
    """Logits at every position of one sequence, float64."""
    n, hs = len(toks), hd
    h = w["embed"][toks].astype(np.float64)
    pos = np.arange(n)
    ang = pos[:, None] * freqs
    see = np.stack([visible(p, n, window, sinks) for p in pos])
    for wqkv, wo in zip(w["wqkv"], w["wo"]):
        x = (h @ wqkv.T.astype(np.float64)).reshape(n, HQ + 2 * HKV, hs)
        qk = x[:, :HQ + HKV].copy()
        a, b = qk[..., 0:rot:2].copy(), qk[..., 1:rot:2].copy()
        qk[..., 0:rot:2] = a * np.cos(ang)[:, None] - b * np.sin(ang)[:, None]
        qk[..., 1:rot:2] = b * np.cos(ang)[:, None] + a * np.sin(ang)[:, None]
        o = np.zeros((n, HQ, hs))
        for i in range(HQ):
            j = i * HKV // HQ
            s = qk[:, i] @ qk[:, HQ + j].T / np.sqrt(hs)
            s = np.where(see, s, -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            o[:, i] = p / p.sum(1, keepdims=True) @ x[:, HQ + HKV + j]
        h = h + o.reshape(n, -1) @ wo.T.astype(np.float64)
    return h @ w["head"].T.astype(np.float64)


@pytest.mark.parametrize("bf16,hd,window,sinks", [(False, 32, 0, 0), (False, 32, 24, 3), (True, 64, 0, 0), (True, 64, 40, 2),
                                                  (True, 128, 33, 5)])
def test_speculative_rejection_over_pages(bf16, hd, window, sinks):
    torch, sr = need_gpu()
    say(f"run over pages bf16={bf16} hd={hd} window={window} sinks={sinks}")
    rng = np.random.default_rng(hd + window)
    d, pt, P, N, steps, cut_every = HQ * hd, 16, 37, 12, 30, 10
    rnd = bf16_round if bf16 else (lambda a: a.astype(np.float32))
    mat = lambda *s: rnd((rng.normal(size=s) / np.sqrt(s[-1])).astype(np.float32))  # noqa: E731
    w = {"embed": rnd(rng.normal(size=(VOCAB, d)).astype(np.float32)), "head": mat(VOCAB, d) * 2,
         "wqkv": [mat((HQ + 2 * HKV) * hd, d) for _ in range(LAYERS)], "wo": [mat(d, HQ * hd) for _ in range(LAYERS)]}
    w["head"] = rnd(w["head"])
    typ = torch.bfloat16 if bf16 else torch.float32
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    W = {"embed": dev(w["embed"]), "head": dev(w["head"]).to(typ), "wqkv": [dev(x).to(typ) for x in w["wqkv"]],
         "wo": [dev(x).to(typ) for x in w["wo"]]}
    rot = hd // 2
    freqs = sr.rope_frequencies(rot, 1e4, sr.SR_ROPE_LINEAR, 2.0)
    F = dev(freqs)
    n_pages, mp = 90, (P + steps + pt) // pt + 1
    pool = torch.full((LAYERS, 2, n_pages, HKV, pt, hd), float("nan"), device="cuda").to(typ)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731

    def forward(tokens, table, lens, granted, shared):
        """tokens int32 [rows][lr] -> logits float [rows][vocab] of the last."""
        rows, lr = tokens.shape
        h = W["embed"][tokens.long()].view(rows * lr, d).float()
        for layer in range(LAYERS):
            qkv = torch.empty((rows * lr, (HQ + 2 * HKV) * hd), device="cuda")
            sr.projection(h.to(typ).contiguous(), W["wqkv"][layer], 0, qkv)
            q = torch.empty((rows, lr, HQ, hd), device="cuda")
            k, v = pool[layer, 0], pool[layer, 1]
            sr.page_append(qkv.view(rows, lr, -1), F, table, lens, k, v, q, n_new=granted, interleaved=True)
            o = torch.empty((rows, lr, HQ * hd), dtype=typ, device="cuda")
            sr.paged_attention(q, k, v, table, lens, o, n_new=granted, window=window, sinks=sinks, shared=shared,
                               max_len=P + steps)
            sr.projection(o.view(rows * lr, HQ * hd), W["wo"][layer], 1, h)
        logits = torch.empty((rows, VOCAB), device="cuda")
        sr.projection(h.view(rows, lr, d)[:, -1].to(typ).contiguous(), W["head"], 0, logits)
        return logits

    # the prompt, then one row per candidate
    prompt = rng.integers(0, VOCAB, P).astype(np.int32)
    table, lens, refs, granted, info = i32(1, mp) - 1, i32(1), i32(n_pages), i32(1), i32(4)
    sr.page_reserve(pool, table, lens, refs, P, table, lens, refs, granted, info)
    logits = forward(dev(prompt[None]), table, lens, granted, 0)
    toks, cand = [list(prompt) for _ in range(N)], np.arange(N)
    seen_logits = [[] for _ in range(N)]
    lp_sum = torch.zeros(N, device="cuda")
    ft, fl, fr = i32(N, mp), i32(N), i32(n_pages)
    sr.page_fork(table, lens, i32(N), pt, ft, fl, fr, window, sinks)
    table, lens, refs, granted = ft, fl, fr, i32(N)
    logits = logits.expand(N, VOCAB).contiguous()
    for step in range(steps):
        tok, lp = i32(N), torch.zeros(N, device="cuda")
        sr.sample(logits, dev(cand.astype(np.int32)), step, 1.0, 99, tok)
        sr.token_logprobs(logits, tok, lp)
        lp_sum += lp
        host, lg = tok.cpu().numpy(), logits.cpu().numpy().astype(np.float64)
        for r in range(N):
            seen_logits[r].append(lg[r])
            toks[r].append(int(host[r]))
        if step == steps - 1:
            break
        if step % cut_every == cut_every - 1:
            # the better half stays; each survivor takes a freed row too
            score, accept = lp_sum / (step + 1), i32(N)
            sr.select(score, dev(np.arange(N, dtype=np.int32)), N // 2, accept)
            keep = np.nonzero(accept.cpu().numpy())[0]
            assert len(keep) == N // 2
            parent = np.sort(np.concatenate([keep, keep])).astype(np.int32)
            ft, fl, fr = i32(N, mp), i32(N), i32(n_pages)
            sr.page_fork(table, lens, dev(parent), pt, ft, fl, fr, window, sinks)
            before = int((refs > 0).sum())
            table, lens, refs = ft, fl, fr
            assert int((refs > 0).sum()) < before                              # the rejected rows' pages are free
            sr.page_compact(pool, table, lens, refs, table, refs, info)
            live, moved, _, _ = info.tolist()
            assert bool((refs[:live] > 0).all()) and not bool(refs[live:].any())
            toks = [list(toks[p]) for p in parent]
            seen_logits = [list(seen_logits[p]) for p in parent]
            lp_sum = lp_sum[dev(parent.astype(np.int64))].contiguous()
            cand = 1000 * (step + 1) + np.arange(N)                            # forked rows draw for themselves
            tok = dev(np.array([t[-1] for t in toks], dtype=np.int32))
        sr.page_reserve(pool, table, lens, refs, 1, table, lens, refs, granted, info)
        assert info.tolist()[:2] == [0, 0] and granted.tolist() == [1] * N
        counts = np.bincount(table[table >= 0].cpu().numpy(), minlength=n_pages)
        assert np.array_equal(refs.cpu().numpy(), counts)
        logits = forward(tok.view(N, 1), table, lens, granted, (P // pt) * pt)
    tol = 2e-2 if bf16 else 1e-4
    assert len({tuple(t) for t in toks}) > 1
    for r in range(N):
        ref = dense_logits(w, np.array(toks[r][:-1]), hd, rot, window, sinks, freqs)[P - 1:]
        got = np.stack(seen_logits[r])
        bound = tol * np.abs(ref).max()
        assert np.abs(got - ref).max() <= bound, (r, np.abs(got - ref).max(), bound)
        z = ref - ref.max(1, keepdims=True)
        lp = (z - np.log(np.exp(z).sum(1, keepdims=True)))[np.arange(steps), toks[r][P:]].sum()
        assert abs(float(lp_sum[r]) - lp) <= steps * 2 * bound
