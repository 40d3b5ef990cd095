"""Forking, reserving and compacting pages against plain integer code: tables,
lengths and counts are equal; the pool's pages are where they should be, bit for
bit, and nothing else in it changed."""
import numpy as np
import pytest

from gpu_util import need_gpu, say
from paged_util import compact, fork, reserve

pytestmark = pytest.mark.gpu


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def random_state(rng, rows, mp, pt, n_pages, bad=0.05, shared=2):
    """A table of random lengths over distinct pages with a common beginning;
    some entries name no page."""
    lens = rng.integers(0, mp * pt + 1, rows).astype(np.int32)
    pages = rng.permutation(n_pages)
    table = rng.integers(-5, n_pages + 9, (rows, mp)).astype(np.int32)     # past the lengths: anything
    at = shared
    for r in range(rows):
        for c in range(-(-int(lens[r]) // pt)):
            if c < shared:
                table[r, c] = pages[c]
            elif at < n_pages and rng.random() > bad:
                table[r, c] = pages[at]
                at += 1
            else:
                table[r, c] = rng.choice([-1, n_pages, 1 << 30, -(1 << 31)])
    return table, lens


def counts(table, lens, pt, n_pages):
    return fork(table, lens, np.arange(len(lens)), pt, n_pages)[2]


@pytest.mark.parametrize("rows,mp,pt,n_pages,new", [(1, 1, 16, 1, 1), (5, 3, 16, 40, 9), (17, 8, 32, 300, 40),
                                                    (64, 21, 64, 1500, 33), (3, 5, 256, 20, 0), (300, 11, 128, 4000, 600),
                                                    (200, 300, 16, 50000, 130), (900, 40, 16, 16384, 1000), (7, 3, 32, 16385, 0)])
def test_fork(rows, mp, pt, n_pages, new):
    torch, sr = need_gpu()
    rng = np.random.default_rng(rows)
    table, lens = random_state(rng, rows, mp, pt, n_pages)
    lens[rng.integers(0, rows)] = -3                                          # clamped
    if rows > 4:
        lens[0] = mp * pt + 1000
        table[0] = np.where(np.arange(mp) < 2, table[0], -1)
    parent = rng.integers(-2, rows + 2, new).astype(np.int32)
    for window, sinks in ((0, 0), (1, 0), (pt + 3, 2), (3 * pt, pt + 1), (10 ** 6, 0)):
        say(f"fork rows={rows} mp={mp} pt={pt} new={new} window={window} sinks={sinks}")
        to, lo = (torch.full(s, 99, dtype=torch.int32, device="cuda") for s in ((new, mp), (new,)))
        refs = torch.full((n_pages,), 99, dtype=torch.int32, device="cuda")
        sr.page_fork(dev(torch, table), dev(torch, lens), dev(torch, parent), pt, to, lo, refs, window, sinks)
        rt, rl, rr = fork(table, lens, parent, pt, n_pages, window, sinks)
        assert np.array_equal(to.cpu(), rt) and np.array_equal(lo.cpu(), rl) and np.array_equal(refs.cpu(), rr)


def run_reserve(torch, sr, pool, table, lens, refs, n_add, in_place=False):
    t, ln, rf = dev(torch, table), dev(torch, lens), dev(torch, refs)
    to, lo, ro = (t, ln, rf) if in_place else (torch.full_like(x, 99) for x in (t, ln, rf))
    granted, info = torch.full_like(ln, 99), torch.full((4,), 99, dtype=torch.int32, device="cuda")
    sr.page_reserve(pool, t, ln, rf, dev(torch, n_add) if not np.isscalar(n_add) else n_add, to, lo, ro, granted, info)
    torch.cuda.synchronize()
    return tuple(x.cpu().numpy() for x in (to, lo, ro, granted, info))


def check_reserve(torch, sr, rng, table, lens, refs, n_add, pt, n_pages, nl=2, hkv=2, hd=32, bf16=True):
    adds = np.full(len(lens), n_add) if np.isscalar(n_add) else n_add
    ref = reserve(table, lens, refs, adds, pt, n_pages)
    for in_place in (False, True):
        shape = (nl, 2, n_pages, hkv, pt, hd)
        host = rng.integers(-30000, 30000, shape).astype(np.int16 if bf16 else np.float32)
        pool = torch.from_numpy(host.copy()).cuda()
        got = run_reserve(torch, sr, pool, table, lens, refs, n_add, in_place)
        for g, r, name in zip(got, ref, ("table", "lens", "refs", "granted", "info")):
            assert np.array_equal(g, np.asarray(r)), (name, in_place)
        for src, dst, part in ref[5]:
            host[:, :, dst, :, :part] = host[:, :, src, :, :part]
        assert np.array_equal(pool.cpu().numpy(), host)
    return ref


@pytest.mark.parametrize("rows,mp,pt,n_pages", [(1, 2, 16, 3), (6, 4, 16, 60), (33, 6, 32, 500), (129, 5, 64, 1100),
                                                (700, 3, 16, 2900), (40, 4, 256, 300)])
def test_reserve_after_fork(rows, mp, pt, n_pages):
    torch, sr = need_gpu()
    rng = np.random.default_rng(rows + 7)
    table, lens = random_state(rng, rows, mp, pt, n_pages, bad=0.02)
    lens = np.minimum(lens, (mp - 1) * pt).astype(np.int32)
    parent = np.sort(rng.integers(0, rows, rows)).astype(np.int32)            # some twice and more, some never
    table, lens, refs = fork(table, lens, parent, pt, n_pages)
    seen_copies = 0
    for n_add in (1, 0, pt, rng.integers(-1, 3, rows)):
        say(f"reserve rows={rows} pt={pt} n_add={n_add if np.isscalar(n_add) else 'each'}")
        ref = check_reserve(torch, sr, rng, table, lens, refs, n_add, pt, n_pages, bf16=rows % 2 == 1)
        seen_copies += ref[4][3]
    assert seen_copies > 0 or rows < 6


def test_reserve_all_or_nothing():
    torch, sr = need_gpu()
    rng = np.random.default_rng(3)
    table, lens = random_state(rng, 8, 6, 16, 30, bad=0.0)
    refs = counts(table, lens, 16, 30)
    ref = check_reserve(torch, sr, rng, table, np.minimum(lens, 70).astype(np.int32),
                        counts(table, np.minimum(lens, 70), 16, 30), 2 ** 30, 16, 30)
    assert ref[4][0] > 0 and ref[4][1] == 8
    lens = np.array([0, 16, 5, 96, 90, 33, 1, 95], np.int32)
    table[:] = -1
    refs[:] = 0
    refs[4:28] = 1                                                            # four free pages and two behind
    ref = check_reserve(torch, sr, rng, table, lens, refs, np.array([17, 1, 0, 0, 0, 63, 0, 0]), 16, 30)
    assert ref[4] == [1, 0, 0, 0]                                              # 2 + 1 + (1 lost page + 3) of 6
    ref = check_reserve(torch, sr, rng, table, lens, refs, np.array([17, 0, 0, 0, 0, 40, 0, 0]), 16, 30)
    assert ref[4] == [0, 0, 5, 0]
    ref = check_reserve(torch, sr, rng, table, lens, refs, np.array([0, 0, 0, 1, 0, 0, 0, 0]), 16, 30)
    assert ref[4] == [0, 1, 0, 0]                                              # past the table


def test_reserve_keeps_a_page_for_one_sharer():
    """Three rows forked from one parent: the lowest keeps the part-filled page
    if all add tokens, none does if one does not."""
    torch, sr = need_gpu()
    rng = np.random.default_rng(4)
    table, lens = np.array([[3, 5, -1]], np.int32), np.array([20], np.int32)
    table, lens, refs = fork(table, lens, [0, 0, 0], 16, 9)
    ref = check_reserve(torch, sr, rng, table, lens, refs, 1, 16, 9)
    assert ref[0].tolist() == [[3, 5, -1], [3, 0, -1], [3, 1, -1]] and ref[4] == [0, 0, 2, 2]
    ref = check_reserve(torch, sr, rng, table, lens, refs, np.array([1, 0, 1]), 16, 9)
    assert ref[0].tolist() == [[3, 0, -1], [3, 5, -1], [3, 1, -1]] and ref[2][5] == 1


def test_reserve_many_rows_and_pages():
    """The most rows, all forked from one, and a free list of many rounds."""
    torch, sr = need_gpu()
    rng = np.random.default_rng(5)
    n_pages = 40000
    table, lens = np.array([[35000, 17, -1]], np.int32), np.array([18], np.int32)
    table, lens, refs = fork(table, lens, [0] * 4096, 16, n_pages)
    refs[rng.permutation(n_pages)[:34000]] += 1
    ref = reserve(table, lens, refs, np.full(4096, 14), 16, n_pages)
    assert ref[4][:2] == [0, 0] and ref[4][3] >= 4095
    host = rng.integers(-30000, 30000, (1, 2, n_pages, 1, 16, 8)).astype(np.int16)
    pool = torch.from_numpy(host.copy()).cuda()
    got = run_reserve(torch, sr, pool, table, lens, refs, 14)
    for g, r, name in zip(got, ref, ("table", "lens", "refs", "granted", "info")):
        assert np.array_equal(g, np.asarray(r)), name
    for src, dst, part in ref[5]:
        host[:, :, dst, :, :part] = host[:, :, src, :, :part]
    assert np.array_equal(pool.cpu().numpy(), host)


@pytest.mark.parametrize("rows,mp,pt,n_pages,nl,hkv,hd,bf16",
                         [(1, 1, 16, 1, 1, 1, 8, True), (4, 5, 16, 90, 2, 2, 32, True), (31, 7, 32, 700, 1, 3, 64, False),
                          (12, 4, 128, 60, 3, 8, 128, True), (200, 9, 16, 20000, 1, 1, 8, True)])
def test_compact(rows, mp, pt, n_pages, nl, hkv, hd, bf16):
    torch, sr = need_gpu()
    rng = np.random.default_rng(rows + 11)
    table, lens = random_state(rng, rows, mp, pt, n_pages)
    table, lens, refs = fork(table, lens, rng.integers(-1, rows, rows), pt, n_pages)
    rt, rr, info_ref, moves = compact(table, lens, refs, pt)
    for in_place in (False, True):
        say(f"compact rows={rows} n_pages={n_pages} in_place={in_place} moved={len(moves)}")
        host = rng.integers(-30000, 30000, (nl, 2, n_pages, hkv, pt, hd)).astype(np.int16 if bf16 else np.float32)
        pool = torch.from_numpy(host.copy()).cuda()
        t, ln, rf = dev(torch, table), dev(torch, lens), dev(torch, refs)
        to, ro = (t, rf) if in_place else (torch.full_like(t, 99), torch.full_like(rf, 99))
        info = torch.full((4,), 99, dtype=torch.int32, device="cuda")
        sr.page_compact(pool, t, ln, rf, to, ro, info)
        assert np.array_equal(to.cpu(), rt) and np.array_equal(ro.cpu(), rr) and info.tolist() == info_ref
        for src, dst in moves:
            host[:, :, dst] = host[:, :, src]
        assert np.array_equal(pool.cpu().numpy(), host)


def test_no_rows():
    torch, sr = need_gpu()
    rng = np.random.default_rng(8)
    table, lens = np.zeros((0, 4), np.int32), np.zeros(0, np.int32)
    refs = rng.integers(0, 2, 20).astype(np.int32)
    check_reserve(torch, sr, rng, table, lens, refs, 5, 16, 20)
    pool, info = torch.zeros((1, 2, 20, 1, 16, 8), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    t, rf = dev(torch, table), dev(torch, refs)
    sr.page_compact(pool, t, dev(torch, lens), rf, t, rf, info)
    assert np.array_equal(rf.cpu(), compact(table, lens, refs, 16)[1]) and info[0].item() == refs.sum()


def test_compact_edges():
    """No live page, all live, and live pages only at the end."""
    torch, sr = need_gpu()
    for refs in (np.zeros(50), np.ones(50), np.arange(50) >= 40, np.arange(50) < 10):
        refs = refs.astype(np.int32) * 3
        table = np.nonzero(refs)[0].astype(np.int32)[None, :] if refs.any() else np.full((1, 2), -1, np.int32)
        lens = np.array([16 * int((refs > 0).sum())], np.int32)
        rt, rr, info_ref, moves = compact(table, lens, refs, 16)
        host = np.arange(2 * 50 * 16 * 8).reshape(1, 2, 50, 1, 16, 8).astype(np.float32)
        pool, info = torch.from_numpy(host.copy()).cuda(), torch.zeros(4, dtype=torch.int32, device="cuda")
        t, rf = dev(torch, table), dev(torch, refs)
        sr.page_compact(pool, t, dev(torch, lens), rf, t, rf, info)
        for src, dst in moves:
            host[:, :, dst] = host[:, :, src]
        assert np.array_equal(t.cpu(), rt) and np.array_equal(rf.cpu(), rr) and info.tolist() == info_ref
        assert np.array_equal(pool.cpu().numpy(), host)


def test_graph_replays():
    """fork, reserve and compact captured together replay with the same result."""
    torch, sr = need_gpu()
    rng = np.random.default_rng(6)
    table, lens = random_state(rng, 20, 5, 16, 300, bad=0.0)
    lens = np.minimum(lens, 60).astype(np.int32)
    parent = rng.integers(0, 20, 24).astype(np.int32)
    host = rng.integers(-30000, 30000, (2, 2, 300, 2, 16, 32)).astype(np.int16)
    start, pool = torch.from_numpy(host).cuda(), torch.from_numpy(host).cuda()
    t, ln, par = dev(torch, table), dev(torch, lens), dev(torch, parent)
    e = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    bufs = [e(24, 5), e(24), e(300), e(24), e(4), e(4)]

    def step():
        ft, fl, fr, granted, i1, i2 = bufs
        sr.page_fork(t, ln, par, 16, ft, fl, fr)
        sr.page_reserve(pool, ft, fl, fr, 2, ft, fl, fr, granted, i1)
        sr.page_compact(pool, ft, fl, fr, ft, fr, i2)

    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in bufs + [pool]]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(4):
        for x in bufs:
            x.fill_(77)
        pool.copy_(start)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bufs + [pool], want))
        step()                                                                # eager work between the replays
