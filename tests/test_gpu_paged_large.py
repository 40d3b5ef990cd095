"""Pools whose pages lie beyond 2^32 bytes: appending, attending, copying and
moving there gives bit for bit what it gives in a pool of a few pages."""
import numpy as np
import pytest

from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu

N_PAGES = 9000   # of 512 KB and 1 MB: 4.7 and 9.4 GB of keys, and of values


@pytest.mark.parametrize("bf16", [True, False])
def test_far_pages(bf16):
    torch, sr = need_gpu()
    hq, hkv, hd, pt = 16, 8, 128, 256
    typ = torch.bfloat16 if bf16 else torch.float32
    assert N_PAGES * hkv * pt * hd * (2 if bf16 else 4) > 1 << 32
    far = torch.empty((1, 2, N_PAGES, hkv, pt, hd), dtype=typ, device="cuda")
    near = torch.zeros((1, 2, 8, hkv, pt, hd), dtype=typ, device="cuda")
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    where = {0: 8999, 1: 8500, 2: 17, 3: 8998, 4: 8333}                # near page -> far page
    table = [[0, 1, -1], [2, 3, 4]]
    lens = i32([400, 700])
    tabs = {"near": i32(table), "far": i32([[where.get(p, -1) for p in row] for row in table])}
    freqs = torch.from_numpy(sr.rope_frequencies(hd, 5e5)).cuda()
    got = {}
    for name, pool in (("near", near), ("far", far)):
        say(f"pages {name} bf16={bf16} bytes={pool.numel() * pool.element_size()}")
        g = torch.Generator(device="cuda").manual_seed(7)
        k, v = pool[0, 0], pool[0, 1]
        qkv = torch.randn((2, 700, (hq + 2 * hkv) * hd), device="cuda", generator=g)
        q = torch.zeros((2, 700, hq, hd), device="cuda")
        sr.page_append(qkv, freqs, tabs[name], lens, k, v, q, n_new=lens)
        outs = [q]
        for lr in (1, 20, 300):      # the last tokens alone, a draft's worth, a chunk
            o = torch.zeros((2, lr, hq * hd), dtype=typ, device="cuda")
            last = torch.stack([q[0, 400 - lr:400], q[1, 700 - lr:700]]).contiguous()
            sr.paged_attention(last, k, v, tabs[name], lens, o, window=350, sinks=3)
            outs.append(o)
        got[name] = outs
    for a, b in zip(got["near"], got["far"]):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all()) and bool(a.any())

    # a forked row's part-filled page is copied to the highest page, then the
    # live pages come down to the front
    forked, fl, refs = i32([[0] * 3] * 3), i32([0] * 3), torch.zeros(N_PAGES, dtype=torch.int32, device="cuda")
    sr.page_fork(tabs["far"], lens, i32([0, 0, 1]), pt, forked, fl, refs)
    refs[:8990].clamp_(min=1)                                            # only high pages are free
    granted, info = i32([0] * 3), i32([0] * 4)
    sr.page_reserve(far, forked, fl, refs, i32([1, 1, 0]), forked, fl, refs, granted, info)
    assert info.tolist() == [0, 0, 1, 1] and granted.tolist() == [1, 1, 0]
    assert forked.tolist() == [[8999, 8500, -1], [8999, 8990, -1], [17, 8998, 8333]]
    part = 400 - pt
    assert torch.equal(far[0, :, 8990, :, :part], near[0, :, 1, :, :part])
    live = torch.zeros_like(refs)
    for p in forked.flatten().tolist():
        if p >= 0:
            live[p] += 1
    sr.page_compact(far, forked, fl, live, forked, live, info)
    assert info.tolist() == [6, 6, 0, 0]
    # free 0..5 take 8333, 8500, 8990, 8998, 8999 (17 is past the front too)
    back = {p: i for i, p in enumerate((17, 8333, 8500, 8990, 8998, 8999))}
    assert forked.tolist() == [[back[8999], back[8500], -1], [back[8999], back[8990], -1],
                               [back[17], back[8998], back[8333]]]
    for n, p in where.items():
        slots = part if n == 1 else pt if n != 4 else 700 - 2 * pt
        assert torch.equal(far[0, :, back[p], :, :slots], near[0, :, n, :, :slots])
    del far
    torch.cuda.empty_cache()
