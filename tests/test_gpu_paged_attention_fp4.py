"""Attention over a cache of 4 bits against float64 attention on the values that
it stands for: head sizes and groupings, both output types, rows of their own
lengths (empty ones too), windows and sinks, entries that name no page, padded new
tokens, shared prompts, long rows split over work-groups, graphs and other
streams.  The bound of every element follows from the roundings (fp4_util.
attention); whatever no query sees reads as NaN."""
import numpy as np
import pytest

from fp4_util import Cache4, attention, dequantise
from gpu_util import need_gpu, say
from paged_util import new_tokens

pytestmark = pytest.mark.gpu

SENTINEL = 7.0


def run(torch, sr, cache, q, n_new, bf16, window, sinks, shared=0, max_len=None, stream=None, ragged=True):
    rows, lr, hq, hd = q.shape
    k, v, table, lens = cache.device(torch)
    out = torch.full((rows, lr, hq * hd), SENTINEL, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    new = torch.tensor(n_new, dtype=torch.int32, device="cuda") if ragged else None
    qd = torch.from_numpy(q).cuda()
    torch.cuda.synchronize()
    sr.paged_attention_fp4(qd, k, v, table, lens, out, n_new=new, window=window, sinks=sinks, shared=shared, max_len=max_len,
                           stream=stream)
    torch.cuda.synchronize()
    return out.float().cpu().numpy().reshape(q.shape).astype(np.float64), (qd, k, v, table, lens, new, out)


def check(out, ref, bound, new, norm=None):
    """Every element within its bound; and all of them within `norm` in the 2-norm:
    the elements' bounds have to allow for roundings that add up, and would hide a
    lost part of a probability."""
    got, want = (np.concatenate([a[r, :n].ravel() for r, n in enumerate(new)]) for a in (out, ref))
    assert norm is None or np.linalg.norm(got - want) <= norm * np.linalg.norm(want), np.linalg.norm(got - want) / np.linalg.norm(want)
    for r, n in enumerate(new):
        assert (out[r, n:] == SENTINEL).all(), r            # rows past n_new: as they were
        err = np.abs(out[r, :n] - ref[r, :n])
        assert not np.isnan(err).any(), r
        worst = (err - bound[r, :n]).max() if n else 0.0
        assert worst <= 0.0, (r, worst, err.max())


def case(seed, bf16, hd, hq, hkv, lens, lr, pt, window=0, sinks=0, n_new=None, shared=0, shared_arg=None, holes=None,
         max_len=None, cols=None):
    torch, sr = need_gpu()
    say(f"attention over 4 bits bf16={bf16} hd={hd} {hq}/{hkv} lens={lens if len(lens) < 9 else len(lens)} lr={lr} pt={pt} "
        f"window={window} sinks={sinks} n_new={n_new} shared={shared} holes={holes} max_len={max_len}")
    rng = np.random.default_rng(seed)
    cache = Cache4(rng, lens, pt, hkv, hd, shared=shared // pt, holes=holes, cols=cols)
    asked = [lr] * len(lens) if n_new is None else n_new
    new = new_tokens(lens, asked, lr)
    cache.poison(new, window, sinks)
    q = rng.normal(size=(len(lens), lr, hq, hd)).astype(np.float32)
    out, _ = run(torch, sr, cache, q, asked, bf16, window, sinks, shared if shared_arg is None else shared_arg, max_len,
                 ragged=n_new is not None)
    ref, bound = attention(cache, q, new, window, sinks, bf16)
    # fp32: a score of magnitude s = sum |q k| / sqrt(hd), up to 100 here, is some 2^-23
    # s off, and a probability by that, 2^-17; bf16: the output's and the
    # probabilities' roundings, 2^-9 each in the mean square at most; with more than 16
    # columns scores are off by some 2^-13 of s too, as their queries are
    check(out, ref, bound, new, 2.0 ** -17 if not bf16 else 2.0 ** -8 if lr * hq // hkv <= 16 else 2.0 ** -6)


SHAPES = [(32, 4, 4), (32, 16, 1), (64, 8, 2), (64, 4, 4), (64, 16, 1), (128, 8, 2), (128, 8, 1), (128, 6, 2), (128, 5, 1)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd,hq,hkv", SHAPES)
@pytest.mark.parametrize("pt", [16, 64])
def test_single_tokens(bf16, hd, hq, hkv, pt):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 0, 63, 64, 65, 100, 257]
    case(1, bf16, hd, hq, hkv, lens, 1, pt)
    case(2, bf16, hd, hq, hkv, lens, 1, pt, window=1)
    case(3, bf16, hd, hq, hkv, lens, 1, pt, window=20, sinks=3)
    case(4, bf16, hd, hq, hkv, lens, 1, pt, window=33, sinks=40)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd,hq,hkv", SHAPES)
def test_a_few_tokens(bf16, hd, hq, hkv):
    """Drafts: lr * heads per KV head below and above the 16 columns."""
    lens = [3, 5, 40, 1, 0, 130]
    for lr in (2, 3, 5):
        case(5, bf16, hd, hq, hkv, lens, lr, 32)
        case(6, bf16, hd, hq, hkv, lens, lr, 16, window=9, sinks=2)
        case(7, bf16, hd, hq, hkv, lens, lr, 32, n_new=[2, 0, 1, 9, 3, -4])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd,hq,hkv", [(32, 4, 4), (64, 8, 2), (64, 16, 1), (128, 8, 2), (128, 3, 1)])
def test_prompts(bf16, hd, hq, hkv):
    """Whole prompts and chunks after cached tokens, ragged, with padded rows."""
    case(8, bf16, hd, hq, hkv, [70, 33], 33, 16)
    case(9, bf16, hd, hq, hkv, [150, 129, 7, 64], 129, 64, n_new=[129, 40, 99, -3])
    case(10, bf16, hd, hq, hkv, [300, 131], 100, 128, window=37, sinks=5)
    case(11, bf16, hd, hq, hkv, [257], 257, 256, window=64)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd,hq,hkv", [(32, 4, 2), (64, 8, 2), (128, 8, 2)])
def test_entries_that_name_no_page(bf16, hd, hq, hkv):
    holes = {(0, 0): -1, (1, 1): 1 << 30, (2, 0): -7, (2, 1): -1, (2, 2): -1, (3, 4): -1}
    for lr in (1, 3, 20):
        case(12, bf16, hd, hq, hkv, [40, 33, 45, 80], lr, 16, holes=holes)
        case(13, bf16, hd, hq, hkv, [40, 33, 45, 80], lr, 16, holes=holes, window=18, sinks=2)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd,hq,hkv", [(32, 4, 4), (64, 8, 2), (128, 8, 2)])
def test_long_rows_in_splits(bf16, hd, hq, hkv):
    case(14, bf16, hd, hq, hkv, [3000, 1, 1777], 1, 64)
    case(15, bf16, hd, hq, hkv, [2500, 2047], 3, 256, window=1500, sinks=3)
    case(16, bf16, hd, hq, hkv, [4100], 1, 16, max_len=50)      # longer than the caller said
    case(17, bf16, hd, hq, hkv, [1300], 24, 32, max_len=1300)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd,hq,hkv,rows,shared", [(128, 8, 2, 40, 128), (64, 8, 2, 33, 64), (32, 4, 4, 21, 64)])
def test_shared_pages(bf16, hd, hq, hkv, rows, shared):
    """Rows over common leading pages; some are shorter than these, one names others."""
    rng = np.random.default_rng(5)
    lens = [shared + int(n) for n in rng.integers(1, 60, rows)]
    lens[3], lens[4] = shared // 2 + 1, 5
    case(18, bf16, hd, hq, hkv, lens, 1, 32, shared=shared)
    case(19, bf16, hd, hq, hkv, lens, 1, 32, shared=shared, holes={(7, 1): -1})
    case(20, bf16, hd, hq, hkv, lens, 2, 32, shared=shared, window=40, sinks=3)
    case(21, bf16, hd, hq, hkv, lens, 1, 32, shared=0, shared_arg=shared)   # nothing in common


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd,hq,hkv", [(32, 16, 8), (64, 8, 4), (128, 6, 2)])
def test_shared_pages_of_many_rows(bf16, hd, hq, hkv):
    """So many that the shared keys are read once for all rows; some rows share less
    than the others, or nothing."""
    rng = np.random.default_rng(6)
    rows, shared, pt = 512, 2048, 64
    lens = [shared + int(n) for n in rng.integers(1, 90, rows)]
    lens[3], lens[4], lens[5], lens[6] = 700, 5, 0, shared
    new = [int(n) for n in rng.integers(0, 3, rows)]
    holes = {(7, 0): -1, (8, 3): -1, (9, 31): -1}
    case(30, bf16, hd, hq, hkv, lens, 1, pt, shared=shared, holes=holes)
    case(31, bf16, hd, hq, hkv, lens, 2, pt, shared=shared, n_new=new)


@pytest.mark.parametrize("hd,hq,hkv", [(32, 4, 2), (64, 8, 2), (128, 8, 2)])
@pytest.mark.parametrize("lr", [2, 70])
def test_what_queries_keep_beyond_a_bf16(hd, hq, hkv, lr):
    """Every token sees two keys, and its queries, 30 times as large as the keys, lie
    almost across their difference: rounding the queries to bf16 moves the output more
    than all other roundings.  What the kernel keeps beyond that (another 8 bits, or
    parts of 6 bits in groups, some 2^-14 of a group's largest) has to take at least three
    quarters of it away, beside the probabilities' and the output's 2^-9 each in the mean square."""
    rng = np.random.default_rng(hd)
    lens = [200, 131]
    cache = Cache4(rng, lens, 16, hkv, hd)
    q = 30 * rng.normal(size=(2, lr, hq, hd))
    for r in range(2):
        k = cache.rows_kv(r)[0]
        for t in range(lr):
            pos = lens[r] - lr + t
            diff = np.repeat(k[pos] - k[pos - 1], hq // hkv, axis=0)
            q[r, t] += ((rng.normal(size=hq) * np.sqrt(hd) - (q[r, t] * diff).sum(1)) / (diff * diff).sum(1))[:, None] * diff
    q = q.astype(np.float32)
    ref, _ = attention(cache, q, [lr, lr], 2, 0, True)
    half = ((q.view(np.uint32) + 0x7FFF + ((q.view(np.uint32) >> 16) & 1)) & 0xFFFF0000).view(np.float32)
    short, _ = attention(cache, half, [lr, lr], 2, 0, True)
    size = np.linalg.norm(ref)
    lost = np.linalg.norm(short - ref) / size
    assert lost > 2.0 ** -6                                     # (or there is nothing to see)
    torch, sr = need_gpu()
    say(f"attention over 4 bits, precision of queries hd={hd} lr={lr}")
    cache.poison([lr, lr], 2, 0)
    out, _ = run(torch, sr, cache, q, [lr, lr], True, 2, 0)
    assert np.linalg.norm(out - ref) / size <= np.hypot(lost / 4, np.sqrt(2) * 2.0 ** -9)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd,hq,hkv", [(32, 4, 2), (64, 8, 2), (128, 8, 2)])
@pytest.mark.parametrize("sign", [-1, 1])
def test_scores_far_from_zero(bf16, hd, hq, hkv, sign):
    """All scores of a row some hundreds below or above 0; a window leaves whole splits
    and blocks unseen."""
    torch, sr = need_gpu()
    say(f"attention over 4 bits, far scores bf16={bf16} hd={hd} sign={sign}")
    rng = np.random.default_rng(hd + sign)
    lens = [700, 75, 1]
    for lr, window, sinks in ((1, 0, 0), (40, 0, 0), (40, 70, 3), (1, 5, 1)):
        cache = Cache4(rng, lens, 32, hkv, hd)
        cache.raw[0] = (cache.raw[0][0] & 7, np.full_like(cache.raw[0][1], 126))      # all positive, of one scale
        cache.k = dequantise(*cache.raw[0])
        new = new_tokens(lens, [lr] * 3, lr)
        cache.poison(new, window, sinks)
        q = (sign * 40 * (1 + 0.02 * rng.normal(size=(3, lr, hq, hd)))).astype(np.float32)
        out, _ = run(torch, sr, cache, q, [lr] * 3, bf16, window, sinks)
        ref, bound = attention(cache, q, new, window, sinks, bf16)
        check(out, ref, bound, new)


def test_pools_past_32_bits():
    """Pages that lie past 2^32 bytes of a pool hold what is put there, and are read
    from there: as a small pool of the same tokens, bit for bit."""
    torch, sr = need_gpu()
    say("pools past 2^32 bytes")
    rng = np.random.default_rng(9)
    hd, hq, hkv, pt, rows, lr, mp = 128, 8, 8, 256, 3, 300, 3
    n_pages = (1 << 32) // (hkv * pt * sr.fp4_token_bytes(hd)) + 40
    far = n_pages - 1 - np.arange(rows * mp, dtype=np.int32).reshape(rows, mp)
    near = far - far.min()
    lens = torch.tensor([700, 301, 300], dtype=torch.int32, device="cuda")
    qkv = torch.from_numpy(rng.normal(size=(rows, 700, (hq + 2 * hkv) * hd)).astype(np.float32)).cuda()
    got = []
    for table, n in ((near, rows * mp), (far, n_pages)):
        k, v = (torch.empty((n, hkv, pt, sr.fp4_token_bytes(hd)), dtype=torch.uint8, device="cuda") for _ in range(2))
        t = torch.from_numpy(table.astype(np.int32)).cuda()
        q = torch.zeros((rows, 700, hq, hd), device="cuda")
        sr.page_append_norm(qkv, None, t, lens, k, v, q, n_new=lens)
        ko, vo = (torch.zeros((rows, 700, hkv, hd), device="cuda") for _ in range(2))
        sr.page_read(k, v, t, lens, ko, vo, n_new=lens)
        outs = [ko, vo]
        for m in (1, lr):
            for typ in (torch.bfloat16, torch.float32):
                o = torch.zeros((rows, m, hq * hd), dtype=typ, device="cuda")
                sr.paged_attention_fp4(q[:, :m].contiguous(), k, v, t, lens, o)
                outs.append(o)
        torch.cuda.synchronize()
        got.append([x.cpu() for x in outs])
        del k, v
    assert float(got[0][0].abs().max()) > 1 and all(float(x.float().abs().max()) > 0 for x in got[0])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_nan_and_infinities():
    """A group with byte 255 gives NaN in the outputs that depend on it and in no
    others, in a key and in a value; a NaN query too."""
    torch, sr = need_gpu()
    for bf16 in (False, True):
        for hd, lr in ((32, 1), (64, 1), (128, 1), (64, 20), (128, 20)):
            rng = np.random.default_rng(hd)
            lens, hq, hkv = [90, 70, 33], 8, 2
            cache = Cache4(rng, lens, 16, hkv, hd)
            cache.poison([lr] * 3, 0, 0)
            q = rng.normal(size=(3, lr, hq, hd)).astype(np.float32)
            clean, _ = run(torch, sr, cache, q, [lr] * 3, bf16, 0, 0)
            assert np.isfinite(clean).all()
            codes, scales = (a.copy() for a in cache.raw[0])
            scales[cache.table[0, 1], 0, 3, hd // 32 - 1] = 255       # token 19 of row 0, KV head 0
            packed = cache.packed
            cache.packed = [pack_like(packed[0], codes, scales, cache), packed[1]]
            out, _ = run(torch, sr, cache, q, [lr] * 3, bf16, 0, 0)
            assert np.isnan(out[0, :, :4]).all() and np.array_equal(out[0, :, 4:], clean[0, :, 4:])
            assert np.array_equal(out[1:], clean[1:])
            codes, scales = (a.copy() for a in cache.raw[1])
            scales[cache.table[1, 0], 1, 5, 0] = 255                  # a value: the group's dimensions
            cache.packed = [packed[0], pack_like(packed[1], codes, scales, cache)]
            out, _ = run(torch, sr, cache, q, [lr] * 3, bf16, 0, 0)
            assert np.isnan(out[1, :, 4:, :32]).all() and np.array_equal(out[1, :, 4:, 32:], clean[1, :, 4:, 32:])
            assert np.array_equal(out[[0, 2]], clean[[0, 2]]) and np.array_equal(out[1, :, :4], clean[1, :, :4])
            cache.packed = packed
            q[2, lr - 1, 6, 5] = np.nan
            out, _ = run(torch, sr, cache, q, [lr] * 3, bf16, 0, 0)
            assert np.isnan(out[2, lr - 1, 6]).all()
            same = np.ones(out.shape[:3], bool)
            same[2, lr - 1, 6] = False
            assert np.array_equal(out[same], clean[same])


def pack_like(packed, codes, scales, cache):
    """The packed pool with these scale bytes where the slot is seen."""
    from fp4_util import pack, unpack
    c0, s0 = unpack(packed)
    shown = s0[..., 0] != 255
    return pack(c0, np.where(shown[..., None], scales, s0))


def test_scales_over_the_whole_range():
    """Every scale byte that the operators write, from 2^-125 to 2^125, in values; and
    in keys where scores stay finite."""
    torch, sr = need_gpu()
    for bf16 in (False, True):
        for hd in (32, 64, 128):
            rng = np.random.default_rng(3)
            lens = [1] * 251
            cache = Cache4(rng, lens, 16, 1, hd)
            codes, scales = cache.raw[1]
            for r in range(251):
                scales[cache.table[r, 0]] = r + 2
            cache.v = dequantise(codes, scales)
            cache.poison([1] * 251, 0, 0)
            q = rng.normal(size=(251, 1, 2, hd)).astype(np.float32)
            out, _ = run(torch, sr, cache, q, [1] * 251, bf16, 0, 0)
            for r in range(251):   # one key: the value itself (exact in bf16)
                want = cache.v[cache.table[r, 0], 0, 0]
                assert np.array_equal(out[r, 0, 0], want) and np.array_equal(out[r, 0, 1], want), (r, out[r, 0, 0], want)
            codes, scales = cache.raw[0]
            cache = Cache4(rng, [64], 16, 1, hd)
            cache.raw[0][1][:] = rng.integers(100, 128, cache.raw[0][1].shape)
            cache.k = dequantise(*cache.raw[0])
            cache.poison([1], 0, 0)
            q = rng.normal(size=(1, 1, 2, hd)).astype(np.float32)
            out, _ = run(torch, sr, cache, q, [1], bf16, 0, 0)
            ref, bound = attention(cache, q, [1], 0, 0, bf16)
            check(out, ref, bound, [1])


@pytest.mark.parametrize("bf16", [False, True])
def test_graph_replays_and_streams(bf16):
    torch, sr = need_gpu()
    for lens, lr, hd in (([700, 90, 1500], 1, 128), ([200, 130], 40, 64), ([300, 20], 1, 32)):
        rng = np.random.default_rng(lr)
        cache = Cache4(rng, lens, 32, 2, hd)
        cache.poison(new_tokens(lens, [lr] * len(lens), lr), 0, 0)
        q = rng.normal(size=(len(lens), lr, 8, hd)).astype(np.float32)
        want, (qd, k, v, table, ln, _, out) = run(torch, sr, cache, q, [lr] * len(lens), bf16, 0, 0, ragged=False)
        side = torch.cuda.Stream()
        got, _ = run(torch, sr, cache, q, [lr] * len(lens), bf16, 0, 0, stream=side, ragged=False)
        assert np.array_equal(got, want)
        first = out.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sr.paged_attention_fp4(qd, k, v, table, ln, out)
        other = torch.empty_like(out)
        for i in range(3):
            out.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            err = (out.float() - first.float()).abs().max()   # (max_len differs: other splits)
            assert float(err) <= (2.0 ** -6 if bf16 else 2.0 ** -18) * float(first.float().abs().max())
            sr.paged_attention_fp4(qd * 2, k, v, table, ln, other)
