"""Attention over the paged cache against float64 attention on the same inputs:
every type, head size and head grouping, rows of their own lengths (empty ones
too), windows and sinks, entries that name no page, padded new tokens, shared
prompts, long rows split over work-groups, graphs and other streams.  The error
bound of every element follows from the roundings (paged_util.attention);
whatever no query sees is NaN."""
import numpy as np
import pytest

from gpu_util import need_gpu, say
from paged_util import Cache, attention, new_tokens

pytestmark = pytest.mark.gpu

SENTINEL = 7.0


def run(torch, sr, cache, q, n_new, lr, window, sinks, shared=0, max_len=None, stream=None, ragged=True):
    rows, _, hq, hd = q.shape
    k, v, table, lens = cache.device(torch)
    out = torch.full((rows, lr, hq * hd), SENTINEL, dtype=k.dtype, device="cuda")
    new = torch.tensor(n_new, dtype=torch.int32, device="cuda") if ragged else None
    qd = torch.from_numpy(q).cuda()
    torch.cuda.synchronize()
    sr.paged_attention(qd, k, v, table, lens, out, n_new=new, window=window, sinks=sinks, shared=shared,
                       max_len=max_len, stream=stream)
    torch.cuda.synchronize()
    return out.float().cpu().numpy().reshape(q.shape).astype(np.float64), (qd, k, v, table, lens, new, out)


def check(out, ref, bound, new):
    for r, n in enumerate(new):
        assert (out[r, n:] == SENTINEL).all(), r            # rows past n_new: as they were
        err = np.abs(out[r, :n] - ref[r, :n])
        assert not np.isnan(err).any(), r
        worst = (err - bound[r, :n]).max() if n else 0.0
        assert worst <= 0.0, (r, worst, err.max())


def case(seed, bf16, hd, hq, hkv, lens, lr, pt, window=0, sinks=0, n_new=None, shared=0, shared_arg=None, holes=None,
         max_len=None, cols=None):
    torch, sr = need_gpu()
    say(f"paged attention bf16={bf16} hd={hd} {hq}/{hkv} lens={lens if len(lens) < 9 else len(lens)} lr={lr} pt={pt} "
        f"window={window} sinks={sinks} n_new={n_new} shared={shared} holes={holes} max_len={max_len}")
    rng = np.random.default_rng(seed)
    cache = Cache(rng, lens, pt, hkv, hd, bf16, shared // pt, holes, cols=cols)
    asked = [lr] * len(lens) if n_new is None else n_new
    new = new_tokens(lens, asked, lr)
    cache.poison(new, window, sinks)
    q = rng.normal(size=(len(lens), lr, hq, hd)).astype(np.float32)
    out, _ = run(torch, sr, cache, q, asked, lr, window, sinks, shared if shared_arg is None else shared_arg, max_len,
                 ragged=n_new is not None)
    ref, bound = attention(cache, q, new, window, sinks, bf16)
    check(out, ref, bound, new)


SHAPES = [(False, 32, 4, 4), (False, 64, 8, 2), (False, 128, 8, 1), (True, 32, 4, 4), (True, 64, 8, 2),
          (True, 64, 4, 4), (True, 128, 8, 2), (True, 128, 8, 1), (True, 128, 6, 2), (True, 64, 16, 1), (True, 128, 5, 1)]


@pytest.mark.parametrize("bf16,hd,hq,hkv", SHAPES)
@pytest.mark.parametrize("pt", [16, 64])
def test_single_tokens(bf16, hd, hq, hkv, pt):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 0, 63, 64, 65, 100, 257]
    case(1, bf16, hd, hq, hkv, lens, 1, pt)
    case(2, bf16, hd, hq, hkv, lens, 1, pt, window=1)
    case(3, bf16, hd, hq, hkv, lens, 1, pt, window=20, sinks=3)
    case(4, bf16, hd, hq, hkv, lens, 1, pt, window=33, sinks=40)


@pytest.mark.parametrize("bf16,hd,hq,hkv", SHAPES)
def test_a_few_tokens(bf16, hd, hq, hkv):
    """Drafts: lr * heads per KV head below and above the 16 columns."""
    lens = [3, 5, 40, 1, 0, 130]
    for lr in (2, 3, 5):
        case(5, bf16, hd, hq, hkv, lens, lr, 32)
        case(6, bf16, hd, hq, hkv, lens, lr, 16, window=9, sinks=2)
        case(7, bf16, hd, hq, hkv, lens, lr, 32, n_new=[2, 0, 1, 9, 3, -4])


@pytest.mark.parametrize("bf16,hd,hq,hkv", SHAPES)
def test_prompts(bf16, hd, hq, hkv):
    case(8, bf16, hd, hq, hkv, [37, 70], 37, 16)
    case(9, bf16, hd, hq, hkv, [70, 200, 20], 70, 32, window=25, sinks=5)
    case(10, bf16, hd, hq, hkv, [133, 90, 64, 0], 64, 64, n_new=[64, 17, 64, 3])
    case(11, bf16, hd, hq, hkv, [150], 150, 128, window=64)


@pytest.mark.parametrize("pt", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("bf16", [False, True])
def test_page_sizes(bf16, pt):
    case(12, bf16, 64, 8, 2, [300, 511, 512, 513], 1, pt)
    case(13, bf16, 64, 8, 2, [300, 513], 40, pt, window=100, sinks=17)


@pytest.mark.parametrize("bf16,hd", [(False, 64), (True, 64), (True, 128), (True, 32)])
@pytest.mark.parametrize("pt", [16, 32])
def test_entries_that_name_no_page(bf16, hd, pt):
    bad = {(0, 0): -1, (0, 2): 1 << 30, (1, 1): -(1 << 31), (2, 0): -1, (2, 1): -1, (2, 2): -1, (2, 3): -1}
    lens = [3 * pt + 5, 2 * pt + 1, 3 * pt + 9, 2 * pt]
    for lr, window, sinks in ((1, 0, 0), (1, pt + 3, 4), (3, 0, 0), (20, 0, 0), (20, 30, 2)):
        case(14, bf16, hd, 8, 2, lens, lr, pt, window, sinks, holes=bad)   # row 2 has nothing to see


@pytest.mark.parametrize("bf16,hd", [(False, 64), (True, 64), (True, 128)])
def test_pages_behind_the_window_are_gone(bf16, hd):
    """Entries behind the window and past the sinks name no page any more."""
    pt, window, sinks = 16, 40, 18
    lens = [300, 211, 64]
    holes = {(r, c): -1 for r, L in enumerate(lens) for c in range(L // pt)
             if c * pt >= sinks and (c + 1) * pt <= L - window}
    assert len(holes) > 15
    case(15, bf16, hd, 8, 2, lens, 1, pt, window, sinks, holes=holes)


@pytest.mark.parametrize("bf16,hd,hq,hkv", [(True, 128, 8, 2), (True, 64, 8, 2), (True, 128, 4, 4), (True, 64, 16, 1),
                                            (False, 64, 8, 2)])
@pytest.mark.parametrize("rows", [3, 17, 70])
def test_shared_prompt(bf16, hd, hq, hkv, rows):
    """A prompt whose pages all rows have in common: the hint changes nothing,
    where it is right, too long, or wrong for some rows."""
    rng = np.random.default_rng(rows)
    lens = (160 + rng.integers(1, 70, rows)).tolist()
    for window, sinks in ((0, 0), (50, 4), (150, 40)):
        case(16, bf16, hd, hq, hkv, lens, 1, 32, window, sinks, shared=160)
    case(17, bf16, hd, hq, hkv, lens, 1, 16, shared=144)                        # an odd number of 16-token pages
    case(18, bf16, hd, hq, hkv, lens, 1, 32, shared=96, shared_arg=5000)        # too long a hint
    case(19, bf16, hd, hq, hkv, lens, 2, 32, shared=96, shared_arg=101)
    short = list(lens)
    short[rows // 2], short[-1] = 40, 0                                          # rows shorter than the prompt
    case(20, bf16, hd, hq, hkv, short, 1, 32, shared=160)
    case(21, bf16, hd, hq, hkv, lens, 1, 32, shared=160, holes={(1, 2): -1, (rows - 1, 0): -1})
    case(22, bf16, hd, hq, hkv, [0] + lens[1:], 1, 32, shared=0, shared_arg=160)  # row 0 has nothing


SHARE = [(128, 4, 1, 700), (64, 2, 1, 1300), (128, 2, 2, 350), (64, 16, 1, 1250)]


@pytest.mark.parametrize("hd,hq,hkv,rows", SHARE)
def test_shared_prompt_in_a_pass_of_its_own(hd, hq, hkv, rows):
    """Enough rows that the shared keys are attended once for all of them
    (300 MB of reads saved): right, too long and partly wrong hints, rows that
    leave the prompt early or lack it, windows that have left key 0, drafts."""
    rng = np.random.default_rng(rows)
    S = 1024
    assert rows * S * hkv * hd * 4 >= 300 << 20
    lens = (S + rng.integers(1, 40, rows)).tolist()
    case(40, True, hd, hq, hkv, lens, 1, 64, shared=S)
    case(41, True, hd, hq, hkv, lens, 1, 16, shared=S - 16, shared_arg=S + 777)      # an odd number of 16-token pages
    mixed = list(lens)
    for r in range(0, rows, 7):
        mixed[r] = int(rng.integers(0, S))                                          # row 0 among them
    mixed[0] = S - 70
    case(42, True, hd, hq, hkv, mixed, 1, 32, shared=S)
    holes = {(r, int(rng.integers(0, 32))): -1 for r in range(5, rows, 11)}
    case(43, True, hd, hq, hkv, lens, 1, 32, shared=S, holes=holes)
    case(44, True, hd, hq, hkv, lens, 1, 32, shared=S, holes={(0, 3): -1, (0, 9): 1 << 30})   # row 0's own pages are missing
    case(45, True, hd, hq, hkv, [0] + lens[1:], 1, 32, shared=0, shared_arg=S)       # nothing in common with row 0
    case(46, True, hd, hq, hkv, lens, 1, 32, window=S + 20, sinks=5, shared=S, max_len=S)   # some windows have left key 0
    if 2 * hq // hkv <= 16:
        case(47, True, hd, hq, hkv, lens, 2, 32, shared=S, n_new=[int(n) for n in rng.integers(0, 3, rows)])


@pytest.mark.parametrize("bf16,hd,hq,hkv", [(True, 128, 8, 2), (True, 64, 4, 1), (False, 32, 4, 4)])
def test_long_rows_split_over_work_groups(bf16, hd, hq, hkv):
    case(23, bf16, hd, hq, hkv, [5003], 1, 64)
    case(24, bf16, hd, hq, hkv, [3001, 12, 4096], 1, 16, window=2500, sinks=3)
    case(25, bf16, hd, hq, hkv, [2777, 901], 1, 32, max_len=10)        # rows longer than planned for
    case(26, bf16, hd, hq, hkv, [2100], 40, 64)
    case(27, bf16, hd, hq, hkv, [2100, 333], 33, 64, n_new=[33, 20], max_len=4000)


@pytest.mark.parametrize("bf16,hd,hq,hkv", [(False, 32, 1, 1), (True, 32, 2, 1), (False, 64, 1, 1), (False, 128, 2, 1),
                                            (True, 64, 1, 1), (True, 128, 4, 1)])
def test_rows_in_more_than_32_splits(bf16, hd, hq, hkv):
    case(53, bf16, hd, hq, hkv, [17001], 1, 64)
    case(54, bf16, hd, hq, hkv, [17400, 9000], 1, 128, n_new=[1, 0])


@pytest.mark.parametrize("hd,hq,hkv,rows,S", [(128, 8, 8, 5, 16384), (64, 16, 8, 9, 17408)])
def test_shared_pass_beside_split_tails(hd, hq, hkv, rows, S):
    """Few rows on a long shared prompt: both passes are split, more than 64
    partials in all."""
    lens = [S + 3001, S + 7, S + 1, S + 2500, S + 640, S + 33, S + 900, S + 64, S + 1][:rows]
    case(55, True, hd, hq, hkv, lens, 1, 128, shared=S)
    case(56, True, hd, hq, hkv, lens, 2, 256, shared=S, n_new=[2, 1, 0, 2, 2, 2, 1, 2, 1][:rows])


def test_lengths_past_the_table_are_clamped():
    torch, sr = need_gpu()
    rng = np.random.default_rng(28)
    cache = Cache(rng, [64, 40], 32, 2, 64, True, cols=2)
    cache.poison([1, 1], 0, 0)
    q = rng.normal(size=(2, 1, 8, 64)).astype(np.float32)
    ref, bound = attention(cache, q, [1, 1], 0, 0, True)
    cache.lens = np.array([1 << 30, 40], np.int32)
    out, _ = run(torch, sr, cache, q, [1, 1], 1, 0, 0)
    check(out, ref, bound, [1, 1])


def test_graph_replays_and_streams():
    """A captured call replays with the eager result, with other work between
    the replays, after its inputs changed in place, and on another stream."""
    torch, sr = need_gpu()
    rng = np.random.default_rng(29)
    lens = [1500, 33, 700]
    cache = Cache(rng, lens, 32, 2, 128, True)
    cache.poison([1, 1, 1], 0, 0)
    q = rng.normal(size=(3, 1, 8, 128)).astype(np.float32)
    eager, (qd, k, v, table, ln, _, out) = run(torch, sr, cache, q, [1, 1, 1], 1, 0, 0, ragged=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = torch.zeros_like(out)
    sr.paged_attention(qd, k, v, table, ln, got, stream=side)
    side.synchronize()
    assert torch.equal(got, out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sr.paged_attention(qd, k, v, table, ln, got)
    for i in range(4):
        got.zero_()
        if i == 2:
            qd.mul_(0.5)
            sr.paged_attention(qd, k, v, table, ln, out)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, out), i
        sr.paged_attention(qd * 2, k, v, table, ln, torch.empty_like(out))


@pytest.mark.parametrize("rows,shared", [(80, 192), (700, 1024)])
def test_results_repeat_bit_for_bit(rows, shared):
    torch, sr = need_gpu()
    rng = np.random.default_rng(30)
    lens = (shared + rng.integers(1, 100, rows)).tolist()
    cache = Cache(rng, lens, 32, 2, 128, True, shared=shared // 32)
    cache.poison([1] * rows, 0, 0)
    q = rng.normal(size=(rows, 1, 8, 128)).astype(np.float32)
    first, _ = run(torch, sr, cache, q, [1] * rows, 1, 0, 0, shared=shared)
    for _ in range(3):
        again, _ = run(torch, sr, cache, q, [1] * rows, 1, 0, 0, shared=shared)
        assert np.array_equal(first, again)
