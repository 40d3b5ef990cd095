"""Reserving room in a row whose part-filled last page is lost."""
import numpy as np
import pytest

from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def test_lost_page_is_the_callers_to_fill():
    """A part-filled last page whose entry names no page is replaced by one that
    holds whatever it held (here NaN): nothing of it is read once the caller has
    written the row's tokens of that page again, together with the new ones."""
    torch, sr = need_gpu()
    rng = np.random.default_rng(12)
    pt, hkv, hq, hd, n_pages, n_add = 16, 2, 4, 64, 12, 5
    for length in (37, 5):
        say(f"lost page, {length} tokens")
        filled = length % pt
        used = -(-length // pt)
        table = np.full((1, 5), -1, np.int32)
        table[0, :used - 1] = rng.permutation(6)[:used - 1]
        lens, refs = np.array([length], np.int32), np.zeros(n_pages, np.int32)
        refs[table[0, :used - 1]] = 1
        pool = torch.full((1, 2, n_pages, hkv, pt, hd), float("nan"), device="cuda")
        t, ln, rf = dev(torch, table), dev(torch, lens), dev(torch, refs)
        granted, info = dev(torch, np.zeros(1)), dev(torch, np.zeros(4))
        qkv = torch.from_numpy(rng.normal(size=(1, length + n_add, (hq + 2 * hkv) * hd)).astype(np.float32)).cuda()
        # the tokens of the whole pages, then the lost ones again with the new ones
        whole = length - filled
        q = torch.zeros((1, length + n_add, hq, hd), device="cuda")
        k, v = pool[0, 0], pool[0, 1]
        if whole:
            first = torch.zeros((1, whole, hq, hd), device="cuda")
            sr.page_append(qkv[:, :whole].contiguous(), None, t, dev(torch, [whole]), k, v, first)
        sr.page_reserve(pool, t, ln, rf, n_add, t, ln, rf, granted, info)
        assert granted.tolist() == [n_add] and ln.tolist() == [length + n_add]
        again = torch.zeros((1, filled + n_add, hq, hd), device="cuda")
        sr.page_append(qkv[:, whole:].contiguous(), None, t, ln, k, v, again)
        out = torch.zeros((1, filled + n_add, hq * hd), device="cuda")
        sr.paged_attention(again, k, v, t, ln, out)
        x = qkv[0].double().cpu().numpy().reshape(length + n_add, hq + 2 * hkv, hd)
        for i in range(filled + n_add):
            p = whole + i
            for h in range(hq):
                z = x[:p + 1, hq + h // 2] @ x[p, h] / np.sqrt(hd)
                w = np.exp(z - z.max())
                want = w / w.sum() @ x[:p + 1, hq + hkv + h // 2]
                got = out[0, i, h * hd:(h + 1) * hd].double().cpu().numpy()
                # scores of up to hd + 2 roundings of 2^-24 of sum |q k| / sqrt(hd) < 100, sums of p + 9 terms
                assert np.abs(got - want).max() <= 2.0 ** -24 * (2 * (hd + 4) * 100 + 2 * (p + 9)) * 5
