"""Performance cases of the paged candidate cache and of token log-probabilities.

A generator step over a paged cache goes through these operators of
paper_2410_20290_amd, each one kind of case here:

  append    page_append: rotary positions on the queries and keys of a QKV
            projection, keys and values written into the rows' pages
  attn      paged_attention: causal attention over the rows' pages, for single
            tokens and for prompts, with a sliding window and sink tokens
  logprobs  token_logprobs: log-probabilities of given tokens, the entropy of
            their distribution and its most likely alternatives
  fork      page_fork + page_reserve: the survivors of a cut are forked into
            the freed rows and every row gets room for its next token
  compact   page_compact: the live pages move to the front of the pool

Where `own` is false, run() computes the same in elementary torch operations.
The shapes are the repository's own configurations; a row's length is spread
evenly over a range and dealt out by the seed.
"""
import math

import numpy as np
import torch

import synth

own = False

BASE = {
    "tiny": synth.CONFIGS["tiny_fp32"].model,
    "small": synth.CONFIGS["small_bf16"].model,
    "1b": synth.CONFIGS["1b_bf16"].model,
    "8b": synth.CONFIGS["8b_bf16"].model,
}


def listed():
    return [
        # a decode step of the tiny fp32 pair: launches are all there is
        {"name": "attn_tiny_decode", "kind": "attn", "shape": "tiny", "rows": 16, "lr": 1, "shared": 32, "past": 0, "past_max": 31,
         "pt": 16, "window": 0, "sinks": 0, "ragged": False},
        # the whole first-round batch over one long shared prompt, the responses
        # of different lengths
        {"name": "attn_8b_decode_512", "kind": "attn", "shape": "8b", "rows": 512, "lr": 1, "shared": 2048,
         "past": 63, "past_max": 380, "pt": 32, "window": 0, "sinks": 0, "ragged": False},
        # a few long contexts of odd lengths, nothing shared
        {"name": "attn_8b_decode_long", "kind": "attn", "shape": "8b", "rows": 3, "lr": 1, "shared": 0,
         "past": 20011, "past_max": 40007, "pt": 64, "window": 0, "sinks": 0, "ragged": False},
        # windowed decode with sinks, head_dim 64: most pages are out of sight
        {"name": "attn_1b_decode_window", "kind": "attn", "shape": "1b", "rows": 64, "lr": 1, "shared": 0,
         "past": 3001, "past_max": 9001, "pt": 16, "window": 1024, "sinks": 4, "ragged": False},
        # one long prompt of odd length through a window of 4096
        {"name": "attn_8b_prompt_window", "kind": "attn", "shape": "8b", "rows": 1, "lr": 7777, "shared": 0,
         "past": 0, "past_max": 0, "pt": 64, "window": 4096, "sinks": 4, "ragged": False},
        # ragged chunks of new tokens after cached ones (a scoring round)
        {"name": "attn_8b_chunks_ragged", "kind": "attn", "shape": "8b", "rows": 61, "lr": 381, "shared": 256,
         "past": 17, "past_max": 131, "pt": 32, "window": 0, "sinks": 0, "ragged": True},
        # one decode step's queries, keys and values of the first-round batch
        {"name": "append_8b_512", "kind": "append", "shape": "8b", "rows": 512, "lr": 1, "past": 300, "past_max": 383, "pt": 32,
         "rot": 128, "interleaved": False, "ragged": False},
        # ragged prompts, half of the head rotated, neighbouring pairs
        {"name": "append_1b_prompts", "kind": "append", "shape": "1b", "rows": 24, "lr": 2011, "past": 0, "past_max": 90, "pt": 64,
         "rot": 32, "interleaved": True, "ragged": True},
        # one row's token with the most likely alternatives
        {"name": "logprobs_1x128256", "kind": "logprobs", "rows": 1, "vocab": 128256, "dtype": "f32", "top": 20,
         "temperature": 1.0, "masked": False},
        # the whole batch's sampled tokens
        {"name": "logprobs_512x128256", "kind": "logprobs", "rows": 512, "vocab": 128256, "dtype": "f32", "top": 5,
         "temperature": 0.7, "masked": False},
        # a cut of 512 rows: 103 survivors forked into all 512 rows, each with
        # its own copy of the part-filled page, four layers
        {"name": "fork_8b_103_512", "kind": "fork", "shape": "8b", "layers": 4, "rows": 512, "keep": 103, "children": 512,
         "P": 256, "len": 403, "pt": 32},
        # a pool of which a third is live moves to its front, four layers
        {"name": "compact_8b", "kind": "compact", "shape": "8b", "layers": 4, "rows": 103, "P": 256, "len": 641, "pt": 32,
         "live": 0.3},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "attn", "append", "logprobs", "logprobs", "fork", "compact"])
    shape = rng.choice(["tiny", "small", "1b", "8b", "8b"])
    pt = rng.choice([16, 32, 64, 128])
    if kind == "attn":
        c = {"kind": kind, "shape": shape, "pt": pt, "window": 0, "sinks": 0, "ragged": False, "shared": 0}
        if rng.random() < 0.4:
            c["window"], c["sinks"] = _log(rng, 30, 4096), rng.choice([0, 1, 4, 37])
        if rng.random() < 0.6:
            rows = _log(rng, 1, 512)
            hi = min(40000, _log(rng, 40, max(60, 120000 // rows)))
            c.update(rows=rows, lr=1 if rng.random() < 0.8 else rng.randint(2, 5), past=rng.randint(0, hi), past_max=hi)
        else:
            rows = _log(rng, 1, 60)
            lr = _log(rng, 6, max(12, min(4000, 12000 // rows)))
            hi = rng.choice([0, rng.randint(1, 300)])
            c.update(rows=rows, lr=lr, past=hi // 2, past_max=hi, ragged=rng.random() < 0.5)
        if rows > 1 and rng.random() < 0.5:
            c["shared"] = pt * rng.randint(1, max(1, 1024 // pt))
        return c
    if kind == "append":
        m = BASE[shape]
        rows = _log(rng, 1, 512)
        return {"kind": kind, "shape": shape, "rows": rows, "lr": 1 if rng.random() < 0.5 else _log(rng, 2, max(3, 20000 // rows)),
                "past": 0, "past_max": _log(rng, 1, min(9000, 200000 // rows)), "pt": pt, "rot": rng.choice([m.head_dim, m.head_dim // 2]),
                "interleaved": rng.random() < 0.5, "ragged": rng.random() < 0.5}
    if kind == "logprobs":
        return {"kind": kind, "rows": _log(rng, 1, 512), "vocab": rng.choice([512, 8192, 32000, 50257, 128256]),
                "dtype": rng.choice(["f32", "f32", "bf16"]), "top": rng.choice([0, 1, 5, 20, 32]),
                "temperature": rng.choice([0.7, 1.0, 1.0]), "masked": rng.random() < 0.3}
    if kind == "fork":
        rows = _log(rng, 2, 512)
        return {"kind": kind, "shape": shape, "layers": 2, "rows": rows, "keep": max(1, int(rows * rng.uniform(0.1, 0.7))),
                "children": rows, "P": rng.randint(1, 400), "len": 400 + rng.randint(1, 250), "pt": pt}
    return {"kind": kind, "shape": shape, "layers": 2, "rows": _log(rng, 1, 128), "P": rng.randint(1, 400),
            "len": 400 + rng.randint(1, 400), "pt": pt, "live": rng.uniform(0.2, 0.9)}


# ---------------------------------------------------------------- inputs
def _dtype(m):
    return torch.bfloat16 if m.dtype == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 29)
    return g


def _randn(g, shape, std, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _int(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _spread(lo, hi, n):
    return lo + (hi - lo) * np.arange(n) // max(1, n - 1)


def _lengths(case):
    """(cached tokens before the new ones, new tokens) of every row, undealt."""
    past = case.get("shared", 0) + _spread(case["past"], case["past_max"], case["rows"])
    new = _spread(max(1, case["lr"] // 3), case["lr"], case["rows"]) if case["ragged"] else np.full(case["rows"], case["lr"])
    return past, new


def _table(rng, lens, shared_pages, pt, spare=3, cols=2):
    """Page table of rows of `lens` tokens whose first shared_pages pages are
    the same, the pages in random order; and the number of pages."""
    used = -(-lens // pt)
    own_pages = np.maximum(used - shared_pages, 0)
    n_pages = int(shared_pages + own_pages.sum() + spare)
    pages = rng.permutation(n_pages)
    table = np.full((len(lens), int(used.max()) + cols), -1)
    c = np.arange(table.shape[1])[None, :]
    at = shared_pages + (np.cumsum(own_pages) - own_pages)[:, None] + c - shared_pages
    table = np.where(c < used[:, None], pages[np.where(c < shared_pages, c, np.minimum(at, n_pages - 1))], -1)
    return table, n_pages


def prepare(case, seed):
    kind, g = case["kind"], _gen(seed)
    rng = np.random.default_rng(1000003 * int(seed) + 31)
    if kind == "logprobs":
        R, V, K = case["rows"], case["vocab"], case["top"]
        logits = _randn(g, (R, V), 2.0, torch.float32).to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        ruled_out = torch.rand((V,), generator=g, device="cuda") < (0.8 if case["masked"] else 0.0)  # by a grammar
        logits.masked_fill_(ruled_out, float("-inf"))
        tokens = torch.rand((R, V), generator=g, device="cuda").masked_fill_(ruled_out, -1.0).argmax(1).to(torch.int32)
        f32 = lambda *s: torch.empty(s, dtype=torch.float32, device="cuda")  # noqa: E731
        return {"case": case, "logits": logits, "tokens": tokens,
                "logprob": f32(R), "entropy": f32(R), "top_ids": torch.empty((R, K), dtype=torch.int32, device="cuda"),
                "top_logprobs": f32(R, K)}
    m = BASE[case["shape"]]
    dt, hq, hk, hd, pt, R = _dtype(m), m.n_heads, m.n_kv_heads, m.head_dim, case["pt"], case["rows"]
    if kind in ("attn", "append"):
        past, new = (a[deal] for deal in [rng.permutation(R)] for a in _lengths(case))
        lens = past + new
        table, n_pages = _table(rng, lens, case.get("shared", 0) // pt, pt)
        pool = _randn(g, (1, 2, n_pages, hk, pt, hd), 1.2, dt)
        st = {"case": case, "m": m, "pool": pool, "k": pool[0, 0], "v": pool[0, 1], "table": _int(table), "lens": _int(lens), "new": _int(new),
              "max_len": int(lens.max())}
        if kind == "attn":
            st["q"] = _randn(g, (R, case["lr"], hq, hd), 1.2, torch.float32)
            st["out"] = torch.zeros((R, case["lr"], hq * hd), dtype=dt, device="cuda")
            return st
        st["qkv"] = _randn(g, (R, case["lr"], m.qkv_dim), 1.0, torch.float32)
        st["q"] = torch.zeros((R, case["lr"], hq, hd), dtype=torch.float32, device="cuda")
        rot = case["rot"]
        st["freqs"] = torch.from_numpy(float(m.rope_theta) ** (-2.0 * np.arange(rot // 2) / rot)).cuda()
        return st
    sp = case["P"] // pt  # whole pages of the prompt, shared by every row
    lens = np.full(R, case["len"])
    if kind == "fork":
        keep, kids = case["keep"], case["children"]
        table, n_pages = _table(rng, lens, sp, pt, spare=kids + 5)
        parent = np.sort(np.sort(rng.choice(R, keep, replace=False))[np.arange(kids) % keep])
        st = {"parent": _int(parent), "lens_out": _int(np.zeros(kids)), "granted": _int(np.zeros(kids)),
              "n_add": _int(np.ones(kids)), "forked": _int(np.zeros((kids, table.shape[1]))),
              "fork_lens": _int(np.zeros(kids)), "fork_refs": _int(np.zeros(n_pages))}
    else:
        live = sp + R * (-(-case["len"] // pt) - sp)
        table, n_pages = _table(rng, lens, sp, pt, spare=int(live * (1.0 / case["live"] - 1.0)))
        kids, st = R, {}
    refs = np.bincount(table[table >= 0], minlength=n_pages)
    st.update({"case": case, "m": m, "table": _int(table), "lens": _int(lens), "refs": _int(refs),
               "pool": _randn(g, (case["layers"], 2, n_pages, hk, pt, hd), 1.0, dt),
               "table_out": _int(np.zeros((kids, table.shape[1]))), "refs_out": _int(np.zeros(n_pages)),
               "info": _int(np.zeros(4))})
    return st


# ------------------------------------------------------- the operators, plain
def _plain_attention(q, pool, table, lens, new, window, sinks):
    R, lr, hq, hd = q.shape
    n_pages, hk, pt = pool.shape[2:5]
    S = table.shape[1] * pt
    kv = pool[0][:, table.clamp(min=0).long()].float()                    # [2, R, pages, hk, pt, hd]
    kv = kv.permute(0, 1, 3, 2, 4, 5).reshape(2, R, hk, S, hd)
    lens, new = lens.long(), new.long()
    t = torch.arange(lr, device=q.device)
    pos = (lens - new)[:, None] + t                                       # [R, lr]
    key = torch.arange(S, device=q.device)
    see = (key <= pos[..., None]) & (t < new[:, None])[..., None]
    see &= ((table >= 0) & (table < n_pages)).repeat_interleave(pt, 1)[:, None, :]
    if window > 0:
        see &= (key > pos[..., None] - window) | (key < sinks)
    qg = q.view(R, lr, hk, hq // hk, hd).permute(0, 2, 3, 1, 4).reshape(R, hk, -1, hd)
    z = torch.matmul(qg, kv[0].transpose(2, 3).contiguous()) / math.sqrt(hd)
    z = z.view(R, hk, hq // hk, lr, S).masked_fill_(~see[:, None, None], float("-inf"))
    p = (z - z.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(R, hk, -1, S), kv[1]).view(R, hk, hq // hk, lr, hd)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.permute(0, 3, 1, 2, 4).reshape(R, lr, hq * hd)


def _plain_append(st):
    case, m, table, pool = st["case"], st["m"], st["table"], st["pool"]
    R, lr, hq, hk, hd, pt, rot = case["rows"], case["lr"], m.n_heads, m.n_kv_heads, m.head_dim, case["pt"], case["rot"]
    t = torch.arange(lr, device="cuda")
    new = st["new"].long()
    pos = (st["lens"].long() - new)[:, None] + t
    there = t < new[:, None]
    x = st["qkv"].view(R, lr, hq + 2 * hk, hd)
    angle = pos.double()[..., None] * st["freqs"]
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
    r = x[:, :, :hq + hk].clone()
    xa, xb = x[:, :, :hq + hk, a], x[:, :, :hq + hk, b]
    r[..., a] = xa * cos - xb * sin
    r[..., b] = xb * cos + xa * sin
    st["q"][there] = r[there][:, :hq]
    page = table.long().gather(1, (pos // pt).clamp(max=table.shape[1] - 1))[there]
    slot = (pos % pt)[there]
    pool[0, 0][page, :, slot] = r[there][:, hq:].to(pool.dtype)
    pool[0, 1][page, :, slot] = x[there][:, hq + hk:].to(pool.dtype)


def _plain_logprobs(st):
    case = st["case"]
    x = st["logits"].float()
    x = torch.where(x.isnan(), torch.full_like(x, float("-inf")), x)
    z = (x - x.amax(1, keepdim=True)) / case["temperature"]
    z = torch.where(x == x.amax(1, keepdim=True), torch.zeros_like(z), z)
    e = z.exp()
    total = e.sum(1)
    lse = total.log()
    st["logprob"].copy_(z.gather(1, st["tokens"].long()[:, None])[:, 0] - lse)
    st["entropy"].copy_(lse - torch.where(e > 0, e * z, torch.zeros_like(e)).sum(1) / total)
    if case["top"] > 0:
        ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]  # ties: the lowest id
        st["top_ids"].copy_(ids)
        st["top_logprobs"].copy_(z.gather(1, ids) - lse[:, None])


def _plain_fork(st):
    case = st["case"]
    pt, par = case["pt"], st["parent"].long()
    lens = st["lens"][par]
    c = torch.arange(st["table"].shape[1], device="cuda")
    n_pages = st["fork_refs"].numel()
    table = torch.where(c < -(-lens[:, None] // pt), st["table"][par], -1)
    st["forked"].copy_(table)
    st["fork_lens"].copy_(lens)
    st["fork_refs"].copy_(torch.bincount(table[table >= 0].long(), minlength=n_pages))
    # room for the next tokens
    refs, add, R = st["fork_refs"], st["n_add"], len(lens)
    used, part = -(-lens // pt), lens % pt
    last = table.gather(1, (used - 1).clamp(min=0)[:, None].long())[:, 0]
    cand = (add > 0) & (part > 0) & (refs[last.long()] > 1)
    same = (last[:, None] == last) & cand[:, None] & cand
    row = torch.arange(R, device="cuda")
    first = ~(same & (row[None, :] < row[:, None])).any(1)
    copy = cand & ~(first & (same.sum(1) == refs[last.long()]))
    need = -(-(lens + add) // pt) - used + copy
    free = torch.argsort((refs != 0).to(torch.int8), stable=True)
    at = torch.cumsum(need, 0) - need
    n_free = (refs == 0).sum()
    short = (need.sum() - n_free).clamp(min=0)
    wide = (-(-(lens + add) // pt) > table.shape[1]).sum()
    ok = (short == 0) & (wide == 0)
    start = (used - copy.int())[:, None]
    fresh = (c >= start) & (c < start + need[:, None]) & ok
    page = free[(at[:, None] + c - start).clamp(0, n_pages - 1).long()].to(torch.int32)
    st["table_out"].copy_(torch.where(fresh, page, table))
    st["granted"].copy_(torch.where(ok, add, torch.zeros_like(add)))
    st["lens_out"].copy_(lens + st["granted"])
    moved = copy & ok
    src, dst = last[moved].long(), free[at[moved].long().clamp(max=n_pages - 1)]
    filled = (torch.arange(pt, device="cuda") < part[moved][:, None])[None, None, :, None, :, None]
    pool = st["pool"]
    pool[:, :, dst] = torch.where(filled, pool[:, :, src], pool[:, :, dst])
    new_refs = refs.clone()
    new_refs.index_add_(0, src, torch.full_like(src, -1, dtype=torch.int32))
    new_refs.index_fill_(0, st["table_out"][fresh].long(), 1)
    st["refs_out"].copy_(new_refs)
    st["info"].copy_(torch.stack([short, wide, torch.where(ok, need.sum(), 0), moved.sum()]))


def _plain_compact(st):
    refs, table, pool, pt = st["refs"], st["table"], st["pool"], st["case"]["pt"]
    page = torch.arange(refs.numel(), device="cuda")
    live = (refs > 0).sum()
    src = ((refs > 0) & (page >= live)).nonzero()[:, 0]
    dst = ((refs == 0) & (page < live)).nonzero()[:, 0]
    to = page.clone()
    to[src] = dst
    used = torch.arange(table.shape[1], device="cuda") < -(-st["lens"][:, None] // pt)
    st["table_out"].copy_(torch.where(used & (table >= 0), to[table.clamp(min=0).long()].int(), -1))
    pool[:, :, dst] = pool[:, :, src]
    out = refs.clone()
    out[dst] = refs[src]
    out[src] = 0
    st["refs_out"].copy_(out)
    st["info"].copy_(torch.stack([live, torch.tensor(len(src), device="cuda"), live * 0, live * 0]))


def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        import paper_2410_20290_amd as sr
    if kind == "attn":
        if own:
            sr.paged_attention(st["q"], st["k"], st["v"], st["table"], st["lens"], st["out"],
                               n_new=st["new"] if case["ragged"] else None, window=case["window"], sinks=case["sinks"],
                               shared=case["shared"], max_len=st["max_len"])
        else:
            st["out"].copy_(_plain_attention(st["q"], st["pool"], st["table"], st["lens"], st["new"], case["window"],
                                             case["sinks"]))
        return st["out"]
    if kind == "append":
        if own:
            sr.page_append(st["qkv"], st["freqs"], st["table"], st["lens"], st["k"], st["v"], st["q"],
                           n_new=st["new"] if case["ragged"] else None, interleaved=case["interleaved"])
        else:
            _plain_append(st)
        return {"q": st["q"], "pool": st["pool"]}
    if kind == "logprobs":
        if own:
            sr.token_logprobs(st["logits"], st["tokens"], st["logprob"], st["entropy"], st["top_ids"], st["top_logprobs"],
                              temperature=case["temperature"])
        else:
            _plain_logprobs(st)
        out = {"logprob": st["logprob"], "entropy": st["entropy"]}
        if case["top"] > 0:
            out.update(top_ids=st["top_ids"], top_logprobs=st["top_logprobs"])
        return out
    if kind == "fork":
        if own:
            sr.page_fork(st["table"], st["lens"], st["parent"], case["pt"], st["forked"], st["fork_lens"], st["fork_refs"])
            sr.page_reserve(st["pool"], st["forked"], st["fork_lens"], st["fork_refs"], st["n_add"], st["table_out"],
                            st["lens_out"], st["refs_out"], st["granted"], st["info"])
        else:
            _plain_fork(st)
        return {k: st[k] for k in ("forked", "fork_lens", "fork_refs", "table_out", "lens_out", "refs_out", "granted", "info",
                                   "pool")}
    if own:
        sr.page_compact(st["pool"], st["table"], st["lens"], st["refs"], st["table_out"], st["refs_out"], st["info"])
    else:
        _plain_compact(st)
    return {k: st[k] for k in ("table_out", "refs_out", "info", "pool")}


# ------------------------------------------------------------ what a pass needs
def work(case):
    kind = case["kind"]
    if kind == "logprobs":
        n = case["rows"] * case["vocab"]
        return {"bytes": float(n * (2 if case["dtype"] == "bf16" else 4) + case["rows"] * (12 + 8 * case["top"])), "flops": 4.0 * n}
    m = BASE[case["shape"]]
    es, hq, hk, hd, pt = 2 if m.dtype == "bf16" else 4, m.n_heads, m.n_kv_heads, m.head_dim, case["pt"]
    row = hk * hd * es  # bytes of one token's keys (or values) in one layer
    if kind == "attn":
        past, new = _lengths(case)
        w, s, sh = case["window"], case["sinks"], case["shared"]
        pairs = keys = 0
        common = np.zeros(sh, dtype=bool)
        for a, n in zip(past.tolist(), new.tolist()):
            pos = np.arange(a, a + n)
            lo = np.maximum(0, pos - w + 1) if w else np.zeros_like(pos)
            pairs += int((pos + 1 - lo + np.minimum(lo, s)).sum())
            first = int(lo.min())  # the row's keys that some query sees: [0, s) and [first, a + n)
            keys += a + n - max(first, sh) + max(0, min(s, first) - sh)
            common[min(first, sh):] = True
            common[:min(s, sh)] = True
        q = int(new.sum()) * hq * hd
        return {"bytes": float(2 * row * (keys + int(common.sum())) + q * (4 + es)), "flops": 4.0 * hq * hd * pairs}
    if kind == "append":
        T = int(_lengths(case)[1].sum())
        return {"bytes": float(T * (m.qkv_dim * 4 + hq * hd * 4 + 2 * row)), "flops": 4.0 * T * (hq + hk) * case["rot"]}
    nl, used = case["layers"], -(-case["len"] // pt)
    if kind == "fork":
        kids, shared_by = case["children"], np.bincount(np.arange(case["children"]) % case["keep"])
        part = case["len"] % pt
        tail = part if case["P"] // pt < used else 0
        copies = int((shared_by - 1).clip(min=0).sum()) * tail
        pages = case["P"] // pt + case["rows"] * (used - case["P"] // pt) + kids + 5
        return {"bytes": float(2 * copies * 2 * nl * row + 4 * (3 * kids * (used + 3) + 3 * pages)), "flops": 0.0}
    sp = case["P"] // pt
    live = sp + case["rows"] * (used - sp)
    moved = live * (1.0 - case["live"])  # of the live pages, those past the first `live` of the pool
    return {"bytes": float(2 * moved * 2 * nl * row * pt + 4 * (2 * case["rows"] * used + 2 * live / case["live"])), "flops": 0.0}


# --------------------------------------------------------- in 64 bits, apart
def exact(case, seed):
    kind = case["kind"]
    if kind in ("fork", "compact"):
        return None
    st = prepare(case, seed)
    if kind == "logprobs":
        x = st["logits"].double() / case["temperature"]
        lp = torch.log_softmax(x, 1)
        p = lp.exp()
        out = {"logprob": lp.gather(1, st["tokens"].long()[:, None])[:, 0],
               "entropy": -(p * torch.where(p > 0, lp, torch.zeros_like(lp))).sum(1)}
        if case["top"] > 0:
            out.update(top_ids=None, top_logprobs=torch.topk(lp, case["top"], dim=1).values)
        return out
    m, pt = st["m"], case["pt"]
    hq, hk, hd = m.n_heads, m.n_kv_heads, m.head_dim
    table, lens, new = (st[k].cpu().tolist() for k in ("table", "lens", "new"))
    if kind == "append":
        rot, pool = case["rot"], st["pool"].double()
        q = st["q"].double()
        for r in range(case["rows"]):
            n = new[r]
            pos = torch.arange(lens[r] - n, lens[r], device="cuda")
            x = st["qkv"][r, :n].double().view(n, hq + 2 * hk, hd)
            turn = torch.polar(torch.ones((n, rot // 2), dtype=torch.float64, device="cuda"), pos[:, None] * st["freqs"])[:, None]
            y = x[:, :hq + hk].clone()
            if case["interleaved"]:
                pair = torch.view_as_complex(y[..., :rot].reshape(n, hq + hk, rot // 2, 2).contiguous())
                y[..., :rot] = torch.view_as_real(pair * turn).flatten(2)
            else:
                pair = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * turn
                y[..., :rot] = torch.cat([pair.real, pair.imag], -1)
            q[r, :n] = y[:, :hq]
            page = torch.tensor(table[r], device="cuda")[pos // pt]
            pool[0, 0, page, :, pos % pt] = y[:, hq:]
            pool[0, 1, page, :, pos % pt] = x[:, hq + hk:]
        return {"q": q, "pool": pool}
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    for r in range(case["rows"]):
        L, n = lens[r], new[r]
        pages = torch.tensor(table[r][:-(-L // pt)], device="cuda")
        k, v = (st["pool"][0, i][pages].transpose(0, 1).reshape(hk, -1, hd)[:, :L].double() for i in (0, 1))
        i = torch.arange(L - n, L, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None, :]
        seen = j <= i
        if case["window"]:
            seen = seen & ((i - j < case["window"]) | (j < case["sinks"]))
        for h in range(hq):
            z = st["q"][r, :n, h].double() @ k[h * hk // hq].t() * hd ** -0.5
            p = torch.softmax(z.masked_fill(~seen, float("-inf")), 1)
            out[r, :n, h * hd:(h + 1) * hd] = p @ v[h * hk // hq]
    return out
