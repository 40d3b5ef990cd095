"""Head norms, rotation and append to caches of fp32, bf16 and 4 bits, and the
tokens read back, against float64: both pair layouts, parts of the head, norms on
either side, far positions, padded new tokens, pages that are not there, groups of
zeros, the largest and smallest magnitudes and no numbers.

Bounds: everything is computed in 64 bits and rounded once, so a query is off by
half a step of fp32, 2^-24 of it (and 2^-149 where it is subnormal), an fp32 key
alike, a bf16 key by 2^-8; the 64-bit arithmetic of both sides differs by some
2^-50, of the larger of the pair's magnitudes.  A cache of 4 bits holds exactly
the nearest values: the inputs' draws lie further than that from a border."""
import numpy as np
import pytest

from fp4_util import dequantise, norm, pack, quantise, rotate, unpack
from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu

CACHES = ["f32", "bf16", "fp4"]


def new_pool(torch, cache, n_pages, hkv, pt, hd):
    if cache == "fp4":
        return torch.full((n_pages, hkv, pt, 17 * hd // 32), 0x5A, dtype=torch.uint8, device="cuda")
    return torch.full((n_pages, hkv, pt, hd), 5.0, dtype=torch.bfloat16 if cache == "bf16" else torch.float32, device="cuda")


def table_of(rng, lens, pt):
    rows, used = len(lens), [-(-L // pt) for L in lens]
    mp, n_pages = max(used) + 1, sum(used) + 2
    pages, table, at = rng.permutation(n_pages), np.full((rows, mp), 1 << 30, np.int32), 0
    for r in range(rows):
        for c in range(used[r]):
            table[r, c] = pages[at]
            at += 1
    return table, n_pages


def case(seed, cache, hd, hq, hkv, rot, interleaved, lens, lr, pt, gains=(True, True), n_new=None, holes=(), theta=1e4,
         qkv=None, eps=1e-5):
    torch, sr = need_gpu()
    say(f"append norm {cache} hd={hd} {hq}/{hkv} rot={rot} interleaved={interleaved} lens={lens} lr={lr} pt={pt} gains={gains}")
    rng = np.random.default_rng(seed)
    rows = len(lens)
    table, n_pages = table_of(rng, lens, pt)
    for r, c, v in holes:
        table[r, c] = v
    if qkv is None:
        qkv = (rng.normal(size=(rows, lr, hq + 2 * hkv, hd)) * np.exp(rng.normal(size=(rows, lr, hq + 2 * hkv, 1)))).astype(np.float32)
    qkv = qkv.reshape(rows, lr, -1)
    gq, gk = ((1 + 0.3 * rng.normal(size=hd)).astype(np.float32) if on else None for on in gains)
    freqs = sr.rope_frequencies(rot, theta) if rot else np.zeros(0)
    k, v = (new_pool(torch, cache, n_pages, hkv, pt, hd) for _ in range(2))
    q = torch.full((rows, lr, hq, hd), 5.0, device="cuda")
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    new = None if n_new is None else dev(np.array(n_new, np.int32))
    t, ln = dev(table), dev(np.array(lens, np.int32))
    sr.page_append_norm(dev(qkv), dev(freqs) if rot else None, t, ln, k, v, q, q_norm=dev(gq), k_norm=dev(gk), eps=eps,
                        n_new=new, interleaved=interleaved)
    held = []
    for typ in (torch.float32, torch.bfloat16):
        ko, vo = (torch.full((rows, lr, hkv, hd), 5.0, dtype=typ, device="cuda") for _ in range(2))
        sr.page_read(k, v, t, ln, ko, vo, n_new=new)
        held.append([x.float().cpu().numpy() for x in (ko, vo)])
        alone = torch.full_like(vo, 5.0)
        sr.page_read(None, v, t, ln, None, alone, n_new=new)
        assert torch.equal(alone.view(torch.int16 if typ is torch.bfloat16 else torch.int32),
                           vo.view(torch.int16 if typ is torch.bfloat16 else torch.int32))
    q = q.cpu().numpy().astype(np.float64)
    pools = [x.cpu().numpy() if cache == "fp4" else x.float().cpu().numpy().astype(np.float64) for x in (k, v)]
    want_q, tol_q = np.full(q.shape, 5.0), np.zeros(q.shape)
    if cache == "fp4":
        raw = [unpack(np.full(p.shape, 0x5A, np.uint8)) for p in pools]
        want = [[c.copy(), s.copy()] for c, s in raw]
    else:
        want, tol = [np.full(p.shape, 5.0) for p in pools], [np.zeros(p.shape) for p in pools]
    half, tiny = (2.0 ** -8 if cache == "bf16" else 2.0 ** -24), 2.0 ** -133
    for r, L in enumerate(lens):
        n = max(0, min(lr if n_new is None else n_new[r], lr, L))
        for t_ in range(lr):
            if t_ >= n:
                for a, b in held:
                    assert (a[r, t_] == 5.0).all() and (b[r, t_] == 5.0).all()
                continue
            pos = L - n + t_
            x = qkv[r, t_].reshape(hq + 2 * hkv, hd)
            y = [norm(x[:hq], gq, eps), norm(x[hq:hq + hkv], gk, eps), x[hq + hkv:].astype(np.float64)]
            size = [np.abs(a).max(-1, keepdims=True) for a in y]
            y[0], y[1] = rotate(y[0], pos, freqs, interleaved), rotate(y[1], pos, freqs, interleaved)
            want_q[r, t_], tol_q[r, t_] = y[0], 2.0 ** -24 * np.abs(y[0]) + 2.0 ** -48 * size[0] + tiny
            pg = table[r, pos // pt]
            for i, z in ((0, y[1]), (1, y[2])):
                if not 0 <= pg < n_pages:
                    for a in held:
                        assert (a[i][r, t_] == 0.0).all()
                    continue
                if cache == "fp4":
                    want[i][0][pg, :, pos % pt], want[i][1][pg, :, pos % pt] = quantise(z)
                    there = dequantise(*quantise(z))
                    for a in held:
                        assert np.array_equal(a[i][r, t_], there, equal_nan=True)
                else:
                    want[i][pg, :, pos % pt] = z
                    tol[i][pg, :, pos % pt] = half * np.abs(z) + 2.0 ** -48 * size[1 + i] + tiny
                    assert np.array_equal(held[0][i][r, t_], pools[i][pg, :, pos % pt], equal_nan=True)
    finite = np.isfinite(want_q)
    assert (np.abs(q - want_q)[finite] <= tol_q[finite]).all(), (np.abs(q - want_q)[finite] - tol_q[finite]).max()
    for i, name in ((0, "k"), (1, "v")):
        if cache == "fp4":
            assert np.array_equal(pools[i], pack(*want[i])), name
        else:
            if cache == "bf16":   # from the middle of the largest bf16, 2^128 - 2^120, and 2^128 on: infinity
                far = np.abs(want[i]) >= 2.0 ** 128 - 2.0 ** 119
                want[i] = np.where(far, np.copysign(np.inf, want[i]), want[i])
            ok = np.isfinite(want[i])
            assert np.array_equal(pools[i][~ok], want[i][~ok], equal_nan=True), name
            assert (np.abs(pools[i][ok] - want[i][ok]) <= tol[i][ok]).all(), name


SHAPES = [(32, 4, 4), (64, 8, 2), (128, 8, 2), (128, 5, 1), (32, 2, 1)]


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("hd,hq,hkv", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_layouts(cache, hd, hq, hkv, interleaved):
    for rot in (hd, hd // 2, 8, 24, 0):
        case(1, cache, hd, hq, hkv, rot, interleaved, [1, 16, 17, 40], 1, 16)
        case(2, cache, hd, hq, hkv, rot, interleaved, [9, 20, 3, 0], 9, 32)


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("gains", [(False, False), (True, False), (False, True)])
def test_norms_are_optional(cache, gains):
    case(3, cache, 64, 8, 2, 64, False, [30, 50], 5, 16, gains=gains)
    case(4, cache, 128, 4, 4, 64, True, [30, 50], 5, 256, gains=gains)


@pytest.mark.parametrize("cache", CACHES)
def test_padded_rows_and_missing_pages(cache):
    case(5, cache, 64, 8, 2, 64, False, [30, 50, 7, 12], 11, 16, n_new=[11, 4, 99, -1], holes=[(0, 1, -1), (1, 3, 1 << 30)])


@pytest.mark.parametrize("cache", CACHES)
def test_far_positions(cache):
    case(6, cache, 64, 2, 1, 64, False, [1_000_003, 131_071], 2, 256, theta=5e5)
    case(7, cache, 128, 2, 1, 128, True, [700_001], 3, 256)


@pytest.mark.parametrize("cache", CACHES)
def test_extreme_magnitudes(cache):
    """Zeros, subnormals, the largest numbers, and values on the borders between
    codes (no norm, no rotation: they arrive exactly)."""
    rng = np.random.default_rng(8)
    hd, hq, hkv, rows = 64, 2, 2, 12
    x = rng.normal(size=(rows, 1, hq + 2 * hkv, hd)).astype(np.float32)
    for r, s in enumerate([0.0, 1e-45, 1e-40, 2.0 ** -126, 2.0 ** -120, 1.0, 1e30, 1e38 / 5]):
        x[r] *= np.float32(s)
    x[8] = np.tile(np.float32([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.9]), hd // 8)
    x[9] = -x[8]
    x[10] = np.nextafter(x[8], np.float32(0))
    x[11] = np.nextafter(x[8], np.float32(100))
    x[7, 0, :, 5] = np.finfo(np.float32).max
    x[0, 0, :, 3] = -0.0
    case(8, cache, hd, hq, hkv, 0, False, [1] * rows, 1, 16, gains=(False, False), qkv=x)


def test_no_numbers():
    """A group that holds one is NaN, its neighbours are not; queries carry it."""
    torch, sr = need_gpu()
    for bad in (np.nan, np.inf, -np.inf):
        x = np.random.default_rng(9).normal(size=(1, 1, 6, 64)).astype(np.float32)
        x[0, 0, 5, 40] = bad                                   # a value
        x[0, 0, 2, 3] = bad                                    # a key, unrotated and without a norm
        k, v = (new_pool(torch, "fp4", 1, 2, 16, 64) for _ in range(2))
        q = torch.zeros((1, 1, 2, 64), device="cuda")
        i = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        table, lens = i(0).view(1, 1), i(1)
        ko, vo = (torch.zeros((1, 1, 2, 64), device="cuda") for _ in range(2))
        sr.page_append_norm(torch.from_numpy(x.reshape(1, 1, -1)).cuda(), None, table, lens, k, v, q)
        sr.page_read(k, v, table, lens, ko, vo)
        nan_k, nan_v = torch.isnan(ko[0, 0]).cpu().numpy(), torch.isnan(vo[0, 0]).cpu().numpy()
        assert nan_k[0, :32].all() and not nan_k[0, 32:].any() and not nan_k[1].any()
        assert nan_v[1, 32:].all() and not nan_v[1, :32].any() and not nan_v[0].any()


def test_equals_page_append_without_norms():
    """To rounding: the same queries and keys as page_append's fp32 arithmetic gives."""
    torch, sr = need_gpu()
    qkv = torch.randn((3, 4, 12 * 64), device="cuda")
    f = torch.from_numpy(sr.rope_frequencies(64, 1e4)).cuda()
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    lens = torch.tensor([5, 20, 32], dtype=torch.int32, device="cuda")
    got = []
    for call in (sr.page_append, sr.page_append_norm):
        k, v = (torch.zeros((6, 2, 16, 64), device="cuda") for _ in range(2))
        q = torch.zeros((3, 4, 8, 64), device="cuda")
        call(qkv, f, table, lens, k, v, q)
        got.append((q, k, v))
    for a, b in zip(*got):
        assert float((a - b).abs().max()) <= 2.0 ** -24 * 9 * float(qkv.abs().max())   # 4 (|x| + |y|), and one rounding


@pytest.mark.parametrize("cache", CACHES)
def test_graph_replays_and_streams(cache):
    torch, sr = need_gpu()
    qkv = torch.randn((3, 2, 6 * 64), device="cuda")
    gain = torch.rand(64, device="cuda")
    f = torch.from_numpy(sr.rope_frequencies(64, 1e4)).cuda()
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    lens = torch.tensor([5, 20, 32], dtype=torch.int32, device="cuda")
    k, v = (new_pool(torch, cache, 6, 1, 16, 64) for _ in range(2))
    q = torch.zeros((3, 2, 4, 64), device="cuda")
    ko, vo = (torch.zeros((3, 2, 1, 64), device="cuda") for _ in range(2))

    def both(stream=None):
        sr.page_append_norm(qkv, f, table, lens, k, v, q, q_norm=gain, k_norm=gain, stream=stream)
        sr.page_read(k, v, table, lens, ko, vo, stream=stream)
    both()
    want = [x.clone() for x in (q, k, v, ko, vo)]

    def clear():
        for x in (q, ko, vo):
            x.zero_()
        for x in (k, v):
            x.fill_(0x5A if cache == "fp4" else 5.0)
        torch.cuda.synchronize()
    clear()
    side = torch.cuda.Stream()
    both(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((q, k, v, ko, vo), want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for _ in range(3):
        clear()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((q, k, v, ko, vo), want))
