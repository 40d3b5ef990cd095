"""Rotary positions and cache append against float64: both pair layouts, parts
of the head, far positions, padded new tokens, pages that are not there.

Bounds: the angle is formed in double and its sine and cosine are rounded to
float once after at most a few 2^-24, so a rotated element x c - y s is off by at
most 2^-24 (4 |x| + 4 |y|) (sine and cosine 2 half steps each, two products, one
sum); bf16 keys add half a step, 2^-8."""
import numpy as np
import pytest

from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu


def plain(x, pos, freqs, interleaved):
    """Rotated heads [.., hd] at position pos, and the error bound."""
    y, b = x.astype(np.float64).copy(), np.zeros(x.shape)
    n = len(freqs)
    i = np.arange(n)
    a, c = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    co, si = np.cos(pos * freqs), np.sin(pos * freqs)
    xa, xc = x[..., a].astype(np.float64), x[..., c].astype(np.float64)
    y[..., a], y[..., c] = xa * co - xc * si, xc * co + xa * si
    b[..., a] = b[..., c] = 2.0 ** -24 * 4 * (np.abs(xa) + np.abs(xc))
    return y, b


def case(seed, bf16, hd, hq, hkv, rot, interleaved, lens, lr, pt, n_new=None, holes=(), theta=1e4):
    torch, sr = need_gpu()
    say(f"append bf16={bf16} hd={hd} {hq}/{hkv} rot={rot} interleaved={interleaved} lens={lens} lr={lr} pt={pt}")
    rng = np.random.default_rng(seed)
    rows, used = len(lens), [-(-L // pt) for L in lens]
    mp, n_pages = max(used) + 1, sum(used) + 2
    pages, table, at = rng.permutation(n_pages), np.full((rows, mp), 1 << 30, np.int32), 0
    for r in range(rows):
        for c in range(used[r]):
            table[r, c] = pages[at]
            at += 1
    for r, c, v in holes:
        table[r, c] = v
    qkv = rng.normal(size=(rows, lr, (hq + 2 * hkv) * hd)).astype(np.float32)
    freqs = sr.rope_frequencies(rot, theta) if rot else np.zeros(0)
    typ = torch.bfloat16 if bf16 else torch.float32
    k, v = (torch.full((n_pages, hkv, pt, hd), 5.0, dtype=typ, device="cuda") for _ in range(2))
    q = torch.full((rows, lr, hq, hd), 5.0, device="cuda")
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    sr.page_append(dev(qkv), dev(freqs) if rot else None, dev(table), dev(np.array(lens, np.int32)), k, v, q,
                   n_new=None if n_new is None else dev(np.array(n_new, np.int32)), interleaved=interleaved)
    q, k, v = q.cpu().numpy().astype(np.float64), k.float().cpu().numpy().astype(np.float64), v.float().cpu().numpy()
    want = [np.full(a.shape, 5.0) for a in (q, k, v)]
    tol = [np.zeros(a.shape) for a in (q, k, v)]
    half = 2.0 ** -8 if bf16 else 0.0
    for r, L in enumerate(lens):
        n = max(0, min(lr if n_new is None else n_new[r], lr, L))
        for t in range(n):
            pos = L - n + t
            x = qkv[r, t].reshape(hq + 2 * hkv, hd)
            y, b = plain(x[:hq + hkv], pos, freqs, interleaved)
            want[0][r, t], tol[0][r, t] = y[:hq], b[:hq]
            pg = table[r, pos // pt]
            if 0 <= pg < n_pages:
                want[1][pg, :, pos % pt], tol[1][pg, :, pos % pt] = y[hq:], b[hq:] + half * (np.abs(y[hq:]) + b[hq:])
                z = x[hq + hkv:].astype(np.float64)
                want[2][pg, :, pos % pt], tol[2][pg, :, pos % pt] = z, half * np.abs(z)
    for got, w, e, name in zip((q, k, v), want, tol, "qkv"):
        assert (np.abs(got - w) <= e).all(), (name, (np.abs(got - w) - e).max())


SHAPES = [(False, 32, 4, 4), (True, 64, 8, 2), (True, 128, 8, 2), (True, 128, 5, 1), (False, 128, 3, 3), (True, 32, 2, 1)]


@pytest.mark.parametrize("bf16,hd,hq,hkv", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_layouts(bf16, hd, hq, hkv, interleaved):
    for rot in (hd, hd // 2, 8, 24, 0):
        case(1, bf16, hd, hq, hkv, rot, interleaved, [1, 16, 17, 40], 1, 16)
        case(2, bf16, hd, hq, hkv, rot, interleaved, [9, 20, 3, 0], 9, 32)


@pytest.mark.parametrize("bf16", [False, True])
def test_padded_rows_and_missing_pages(bf16):
    case(3, bf16, 64, 8, 2, 64, False, [30, 50, 7, 12], 11, 16, n_new=[11, 4, 99, -1], holes=[(0, 1, -1), (1, 3, 1 << 30)])


def test_far_positions():
    """Angles of 10^5 and more turns: formed in double."""
    case(4, False, 64, 2, 1, 64, False, [1_000_003, 131_071], 2, 256, theta=5e5)
    case(5, False, 128, 2, 1, 128, True, [700_001], 3, 256)


def test_graph_replays():
    torch, sr = need_gpu()
    qkv = torch.randn((3, 2, 6 * 64), device="cuda")
    f = torch.from_numpy(sr.rope_frequencies(64, 1e4)).cuda()
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    lens = torch.tensor([5, 20, 32], dtype=torch.int32, device="cuda")
    k, v = (torch.zeros((6, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((3, 2, 4, 64), device="cuda")
    sr.page_append(qkv, f, table, lens, k, v, q)
    want = [x.clone() for x in (q, k, v)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sr.page_append(qkv, f, table, lens, k, v, q)
    for _ in range(3):
        for x in (q, k, v):
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((q, k, v), want))
