"""The operators of specrej_serving.h together, as a decoding loop uses them: a
prompt goes into pages of 4 bits, is forked into candidates that grow token by
token (projection, head norms, rotation and append, attention with a window and
sinks, a filtered draw with settings of every row), the better half by the mean
log-probability of the draws is kept and forked into the freed rows, and the pool is
compacted.  At every step and layer the appended keys and values are the nearest
4-bit values of a float64 norm and rotation of that step's projections, attention
lies within its bound of float64 attention over everything that the row has
appended so far, and the drawn tokens, counts and log-probabilities are those of
the definition in whole numbers; after every fork and compaction the pages still
hold every row's history, bit for bit."""
import numpy as np
import pytest

from fp4_util import attention, dequantise, norm, quantise, rotate
from gpu_util import need_gpu, say
from test_gpu_sample_filtered import ONE, plain

pytestmark = pytest.mark.gpu

LAYERS, HQ, HKV, VOCAB = 2, 4, 2, 700


class History:
    """What the rows of one layer hold, for fp4_util.attention."""

    def __init__(self, hd, rows):
        self.hkv, self.k, self.v = HKV, [np.zeros((0, HKV, hd)) for _ in range(rows)], [np.zeros((0, HKV, hd)) for _ in range(rows)]

    def append(self, r, k, v):
        self.k[r], self.v[r] = np.concatenate([self.k[r], k]), np.concatenate([self.v[r], v])

    def fork(self, parent):
        self.k, self.v = [self.k[p] for p in parent], [self.v[p] for p in parent]

    def rows_kv(self, r):
        return self.k[r], self.v[r], np.ones(len(self.k[r]), dtype=bool)


@pytest.mark.parametrize("bf16,hd,window,sinks,pt", [(False, 32, 0, 0, 16), (True, 64, 40, 2, 16), (True, 128, 0, 0, 32), (False, 128, 24, 3, 16)])
def test_candidates_in_four_bits(bf16, hd, window, sinks, pt):
    torch, sr = need_gpu()
    say(f"run over pages of 4 bits bf16={bf16} hd={hd} window={window} sinks={sinks}")
    rng = np.random.default_rng(hd + window)
    d, P, N, steps, cut_every = HQ * hd, 37, 10, 21, 7
    typ = torch.bfloat16 if bf16 else torch.float32
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    mat = lambda *s: dev((rng.normal(size=s) / np.sqrt(s[-1])).astype(np.float32)).to(typ)  # noqa: E731
    embed, head = dev(rng.normal(size=(VOCAB, d)).astype(np.float32)), mat(VOCAB, d) * 2
    wqkv, wo = [mat((HQ + 2 * HKV) * hd, d) for _ in range(LAYERS)], [mat(d, HQ * hd) for _ in range(LAYERS)]
    gains = [[(1 + 0.2 * rng.normal(size=hd)).astype(np.float32) for _ in range(2)] for _ in range(LAYERS)]
    rot, eps = hd // 2, 1e-6
    freqs = sr.rope_frequencies(rot, 1e4)
    F = dev(freqs)
    n_pages, mp = 80, (P + steps + pt) // pt + 1
    pool = torch.full((LAYERS, 2, n_pages, HKV, pt, sr.fp4_token_bytes(hd)), 0xFF, dtype=torch.uint8, device="cuda")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    held = [History(hd, 1) for _ in range(LAYERS)]

    def forward(tokens, table, lens, granted, shared):
        """tokens int32 [rows][lr] -> logits float [rows][vocab] of the last."""
        rows, lr = tokens.shape
        h = embed[tokens.long()].view(rows * lr, d).clone()
        at = lens.cpu().numpy()
        for layer in range(LAYERS):
            qkv = torch.empty((rows * lr, (HQ + 2 * HKV) * hd), device="cuda")
            sr.projection(h.to(typ).contiguous(), wqkv[layer], 0, qkv)
            q = torch.empty((rows, lr, HQ, hd), device="cuda")
            k, v = pool[layer, 0], pool[layer, 1]
            gq, gk = gains[layer]
            sr.page_append_norm(qkv.view(rows, lr, -1), F, table, lens, k, v, q, q_norm=dev(gq), k_norm=dev(gk), eps=eps, n_new=granted)
            o = torch.empty((rows, lr, HQ * hd), dtype=typ, device="cuda")
            sr.paged_attention_fp4(q, k, v, table, lens, o, n_new=granted, window=window, sinks=sinks, shared=shared, max_len=P + steps)
            x = qkv.cpu().numpy().astype(np.float64).reshape(rows, lr, HQ + 2 * HKV, hd)
            ko, vo = (torch.empty((rows, lr, HKV, hd), device="cuda") for _ in range(2))
            sr.page_read(k, v, table, lens, ko, vo, n_new=granted)
            for r in range(rows):
                for t in range(lr):
                    key = rotate(norm(x[r, t, HQ:HQ + HKV], gk, eps), at[r] - lr + t, freqs, False)
                    want = [dequantise(*quantise(a)) for a in (key, x[r, t, HQ + HKV:])]
                    assert np.array_equal(ko[r, t].cpu().numpy(), want[0]) and np.array_equal(vo[r, t].cpu().numpy(), want[1])
                    held[layer].append(r, want[0][None], want[1][None])
            ref, bound = attention(held[layer], q.cpu().numpy(), [lr] * rows, window, sinks, bf16)
            err = np.abs(o.float().cpu().numpy().reshape(ref.shape) - ref)
            assert (err <= bound).all(), (layer, (err - bound).max())
            sr.projection(o.view(rows * lr, HQ * hd), wo[layer], 1, h)
        logits = torch.empty((rows, VOCAB), device="cuda")
        sr.projection(h.view(rows, lr, d)[:, -1].to(typ).contiguous(), head, 0, logits)
        return logits

    table, lens, refs, granted, info = i32(1, mp) - 1, i32(1), i32(n_pages), i32(1), i32(4)
    sr.page_reserve(pool, table, lens, refs, P, table, lens, refs, granted, info)
    logits = forward(dev(rng.integers(0, VOCAB, (1, P)).astype(np.int32)), table, lens, granted, 0)
    ft, fl, fr = i32(N, mp), i32(N), i32(n_pages)
    sr.page_fork(table, lens, i32(N), pt, ft, fl, fr, window, sinks)
    table, lens, refs, granted = ft, fl, fr, i32(N)
    for x in held:
        x.fork([0] * N)
    logits = logits.expand(N, VOCAB).contiguous()
    T, top_k = rng.choice([0.7, 1.0, 1.3], N).astype(np.float32), rng.choice([0, 40, 90], N).astype(np.int32)
    top_p, score = rng.choice([1.0, 0.95, 0.8], N).astype(np.float32), torch.zeros(N, device="cuda")
    for step in range(steps):
        ctr, words = i32(N, 4), i32(N, 4)
        ctr[:, 0], ctr[:, 1] = step, torch.arange(N, dtype=torch.int32, device="cuda")
        sr.philox_fill(77, ctr, words)
        tok, kept, lp = i32(N), i32(N), torch.zeros(N, device="cuda")
        sr.sample_filtered(logits, words[:, 0], tok, temperature=dev(T), top_k=dev(top_k), top_p=dev(top_p), min_p=0.01,
                           logprob=lp, kept=kept)
        score += lp
        word, lg = words[:, 0].cpu().numpy().astype(np.int64) % ONE, logits.cpu().numpy()
        for r in range(N):
            want = plain(lg[r], T[r], top_k[r], top_p[r], 0.01, int(word[r]))
            assert (int(tok[r]), int(kept[r])) == (want[0], want[2])
            assert abs(float(lp[r]) - want[1]) <= 2.0 ** -24 * abs(want[1]) + 2.0 ** -50
        if step == steps - 1:
            break
        if step % cut_every == cut_every - 1:
            keep = torch.argsort(score, descending=True)[:N // 2].cpu().numpy()
            parent = np.sort(np.concatenate([keep, keep])).astype(np.int32)
            ft, fl, fr = i32(N, mp), i32(N), i32(n_pages)
            sr.page_fork(table, lens, dev(parent), pt, ft, fl, fr, window, sinks)
            table, lens, refs = ft, fl, fr
            sr.page_compact(pool, table, lens, refs, table, refs, info)
            live = int(info[0])
            assert bool((refs[:live] > 0).all()) and not bool(refs[live:].any())
            pool[:, :, live:] = 0xFF                                      # (nothing is left there)
            tok, score = tok[dev(parent.astype(np.int64))].contiguous(), score[dev(parent.astype(np.int64))].contiguous()
            for x in held:
                x.fork(parent)
            L = int(lens.max())
            for layer in range(LAYERS):
                ko, vo = (torch.full((N, L, HKV, hd), 9.0, device="cuda") for _ in range(2))
                sr.page_read(pool[layer, 0], pool[layer, 1], table, lens, ko, vo)
                for r in range(N):
                    n = int(lens[r])
                    there = np.arange(n) >= (max(0, n - window) // pt * pt if window else 0)
                    there |= np.arange(n) // pt * pt < sinks                # (a page behind the window is let go)
                    for got, want in ((ko, held[layer].k[r]), (vo, held[layer].v[r])):
                        assert np.array_equal(got[r, :n].cpu().numpy()[there], want[there])
                        assert (got[r, n:] == 9.0).all()
        sr.page_reserve(pool, table, lens, refs, 1, table, lens, refs, granted, info)
        assert info.tolist()[:2] == [0, 0] and granted.tolist() == [1] * N
        logits = forward(tok.view(N, 1), table, lens, granted, P // pt * pt)


def test_two_graphs_over_one_memory_pool():
    """Two captured steps whose workspaces share memory, replayed in turn with eager
    calls between them: the results of the eager calls, bit for bit."""
    torch, sr = need_gpu()
    say("two graphs over one memory pool")
    hd, hq, hkv, pt, vocab = 64, 8, 2, 64, 50001
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    steps = []
    for rows, length in ((3, 5000), (7, 900)):
        mp = -(-length // pt)
        table = torch.randperm(rows * mp, device="cuda", generator=gen).to(torch.int32).view(rows, mp)
        lens = torch.full((rows,), length, dtype=torch.int32, device="cuda") - torch.arange(rows, dtype=torch.int32, device="cuda")
        k, v = (torch.zeros((rows * mp, hkv, pt, sr.fp4_token_bytes(hd)), dtype=torch.uint8, device="cuda") for _ in range(2))
        fill = torch.zeros((rows, length, hq, hd), device="cuda")
        sr.page_append_norm(rnd(rows, length, (hq + 2 * hkv) * hd), None, table, lens, k, v, fill, n_new=lens)
        qkv, head, words = rnd(rows, 1, (hq + 2 * hkv) * hd), rnd(vocab, hq * hd) / 10, torch.arange(rows, dtype=torch.int32, device="cuda") * 98765431
        q = torch.zeros((rows, 1, hq, hd), device="cuda")
        o, logits = torch.zeros((rows, 1, hq * hd), device="cuda"), torch.zeros((rows, vocab), device="cuda")
        tok, lp, kept = torch.zeros_like(lens), torch.zeros(rows, device="cuda"), torch.zeros_like(lens)

        def step(a=(qkv, table, lens, k, v, q, o, logits, head, words, tok, lp, kept)):
            qkv, table, lens, k, v, q, o, logits, head, words, tok, lp, kept = a
            sr.page_append_norm(qkv, None, table, lens, k, v, q)          # (the last token again)
            sr.paged_attention_fp4(q, k, v, table, lens, o)
            sr.projection(o.view(len(lens), -1), head, 0, logits)
            sr.sample_filtered(logits, words, tok, top_k=50, top_p=0.9, logprob=lp, kept=kept)
            return o, tok, lp, kept
        steps.append(step)
    want = [[t.clone() for t in s()] for s in steps]
    torch.cuda.synchronize()
    pool, graphs = torch.cuda.graph_pool_handle(), []
    for s in steps:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], pool=pool):
            outs = s()
        steps[len(graphs) - 1] = (s, outs)
    for i in (0, 1, 0, 0, 1, 1, 0):
        for _, outs in steps:
            for t in outs:
                t.zero_()
        torch.cuda.synchronize()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(steps[i][1], want[i])), i
        steps[1 - i][0]()                                               # (eager, with a workspace of its own)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(steps[1 - i][1], want[1 - i])), i
