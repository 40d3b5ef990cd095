"""The operators of specrej_ops.h on the CPU: every declared symbol is exported,
bad arguments are refused with the documented status before any device work, the
host-only functions are right, and every index the paged kernels form is in
range."""
import os
import re
import subprocess

import numpy as np
import pytest

import paper_2410_20290_amd as sr
import paged_util

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SMALL, UNSUPPORTED = sr.SR_ERR_INVALID_ARG, sr.SR_ERR_WORKSPACE_TOO_SMALL, sr.SR_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(sr.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return sr.lib()


def test_header_symbols_exported(L):
    text = open(os.path.join(ROOT, "include", "specrej_ops.h")).read()
    names = sorted(set(re.findall(r"^(?:sr_status|size_t)\s+(sr_\w+)\(", text, re.M)))
    assert len(names) == 11, names
    for n in names:
        assert hasattr(L, n), n


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "specrej_ops.h"\nint main(void) { return SR_ROPE_PLAIN; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)],
                   check=True)


def test_indices_of_the_paged_kernels(tmp_path):
    exe = str(tmp_path / "check")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2410_20290_amd", "csrc"), "-o", exe,
                    os.path.join(ROOT, "tests", "paged_index_check.cpp")], check=True)
    assert subprocess.run([exe], capture_output=True, text=True, check=True).stdout == "ok\n"


def args(defaults, order, kw):
    d = dict(defaults)
    d.update(kw)
    return [d[k] for k in order]


FORK = dict(table=0x10000, lens=0x20000, rows=4, mp=8, parent=0x30000, new=4, pt=16, n_pages=64, window=0, sinks=0,
            to=0x40000, lo=0x50000, ro=0x60000, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), INVALID), (dict(mp=0), INVALID), (dict(n_pages=0), INVALID), (dict(new=-1), INVALID),
    (dict(pt=8), UNSUPPORTED), (dict(pt=48), UNSUPPORTED), (dict(pt=512), UNSUPPORTED), (dict(rows=4097), UNSUPPORTED),
    (dict(new=4097), UNSUPPORTED), (dict(mp=65537), UNSUPPORTED), (dict(n_pages=(1 << 20) + 1), UNSUPPORTED),
    (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(table=None), INVALID), (dict(parent=None), INVALID),
    (dict(ro=None), INVALID), (dict(lo=None), INVALID), (dict(to=0x10000), INVALID), (dict(to=0x10000 + 4 * 31), INVALID),
    (dict(lo=0x20000), INVALID), (dict(ro=0x40000), INVALID), (dict(lo=0x30004), INVALID)])
def test_fork_refuses(L, kw, status):
    assert L.sr_page_fork(*args(FORK, FORK, kw)) == status and sr.last_error()


RESERVE = dict(pool=0x1000000, block=64 * 2 * 16 * 64, nl=2, hkv=2, hd=64, eb=2, pt=16, n_pages=64, table=0x10000,
               lens=0x20000, refs=0x30000, rows=4, mp=8, add=None, add_all=1, to=0x40000, lo=0x50000, ro=0x60000,
               granted=0x70000, info=0x80000, scratch=0x90000, n=1 << 20, stream=None)
POOL_BAD = [
    (dict(pool=None), INVALID), (dict(pool=0x1000008), INVALID), (dict(nl=0), INVALID), (dict(hkv=0), INVALID),
    (dict(hd=0), INVALID), (dict(eb=3), INVALID), (dict(hd=4), UNSUPPORTED), (dict(block=64 * 2 * 16 * 64 - 8), INVALID),
    (dict(block=64 * 2 * 16 * 64 + 4), UNSUPPORTED), (dict(pt=24), UNSUPPORTED), (dict(rows=5000), UNSUPPORTED),
    (dict(table=None), INVALID), (dict(refs=None), INVALID), (dict(info=None), INVALID), (dict(to=None), INVALID),
    (dict(scratch=None), SMALL), (dict(n=10), SMALL), (dict(to=0x10004), INVALID), (dict(ro=0x30010), INVALID),
    (dict(info=0x30000), INVALID), (dict(ro=0x10000), INVALID), (dict(scratch=0x60000), INVALID),
    (dict(info=0x1000000), INVALID), (dict(n_pages=0), INVALID)]


@pytest.mark.parametrize("kw,status", POOL_BAD + [
    (dict(lens=None), INVALID), (dict(lo=0x20004), INVALID), (dict(granted=0x50000), INVALID), (dict(granted=None), INVALID),
    (dict(add=0x40000), INVALID), (dict(lo=0x10000), INVALID), (dict(granted=0x20000), INVALID)])
def test_reserve_refuses(L, kw, status):
    assert L.sr_page_reserve(*args(RESERVE, RESERVE, kw)) == status and sr.last_error()


COMPACT = {k: v for k, v in RESERVE.items() if k not in ("add", "add_all", "lo", "granted")}


@pytest.mark.parametrize("kw,status", POOL_BAD + [(dict(lens=0x40000), INVALID)])
def test_compact_refuses(L, kw, status):
    assert L.sr_page_compact(*args(COMPACT, COMPACT, kw)) == status and sr.last_error()


APPEND = dict(dtype=sr.SR_BF16, hd=64, hq=8, hkv=2, rows=2, lr=3, qkv=0x100000, freqs=0x200000, rot=64, inter=0,
              k=0x300000, v=0x400000, pt=16, n_pages=8, table=0x500000, mp=4, lens=0x600000, new=None, q=0x700000,
              stream=None)
LAYER_BAD = [
    (dict(dtype=2), INVALID), (dict(hd=48), UNSUPPORTED), (dict(hd=256), UNSUPPORTED), (dict(hq=7), INVALID),
    (dict(hkv=0), INVALID), (dict(rows=-1), INVALID), (dict(lr=-1), INVALID), (dict(pt=20), UNSUPPORTED),
    (dict(mp=0), INVALID), (dict(n_pages=0), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(q=None), INVALID), (dict(q=0x700004), INVALID),
    (dict(k=0x300008), INVALID), (dict(v=0x400002), INVALID)]


@pytest.mark.parametrize("kw,status", LAYER_BAD + [
    (dict(qkv=None), INVALID), (dict(qkv=0x100008), INVALID), (dict(rot=65), INVALID), (dict(rot=72), INVALID),
    (dict(rot=12), INVALID), (dict(rot=-8), INVALID), (dict(freqs=None), INVALID), (dict(v=0x300000), INVALID),
    (dict(q=0x100000), INVALID), (dict(q=0x300000), INVALID), (dict(rows=4096, lr=1 << 17), UNSUPPORTED),
    (dict(rows=4096, lr=4096), UNSUPPORTED)])   # (2^24 work-groups: a launch holds fewer)
def test_append_refuses(L, kw, status):
    assert L.sr_page_append(*args(APPEND, APPEND, kw)) == status and sr.last_error()


def test_nothing_to_append(L):
    for kw in (dict(rows=0), dict(lr=0)):
        assert L.sr_page_append(*args(APPEND, APPEND, kw)) == sr.SR_OK and sr.last_error() == ""


ATTN = dict(dtype=sr.SR_BF16, hd=64, hq=8, hkv=2, rows=2, lr=3, q=0x700000, k=0x300000, v=0x400000, pt=16, n_pages=8,
            table=0x500000, mp=4, lens=0x600000, new=None, window=0, sinks=0, shared=0, max_len=64, out=0x800000,
            scratch=0x10000000, n=1 << 22, stream=None)


@pytest.mark.parametrize("kw,status", LAYER_BAD + [
    (dict(hq=34), UNSUPPORTED), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(shared=-1), INVALID),
    (dict(max_len=0), INVALID), (dict(out=None), INVALID), (dict(out=0x800002), INVALID), (dict(out=0x700000), INVALID),
    (dict(out=0x300000), INVALID), (dict(rows=4096, lr=1 << 16), UNSUPPORTED),
    (dict(dtype=sr.SR_F32, hd=32, hq=1, hkv=1, rows=16, lr=1 << 24, q=1 << 40, out=1 << 41, mp=65536, pt=256),
     UNSUPPORTED),   # (2^25 work-groups)
    (dict(rows=1, lr=1, mp=4096, max_len=60000, n=8), SMALL),
    (dict(rows=1, lr=1, mp=4096, max_len=60000, scratch=None), SMALL),
    (dict(rows=1, lr=1, mp=4096, max_len=60000, scratch=0x10000004), INVALID),
    (dict(rows=1, lr=1, mp=4096, max_len=60000, scratch=0x800000), INVALID)])
def test_attention_refuses(L, kw, status):
    assert L.sr_paged_attention(*args(ATTN, ATTN, kw)) == status and sr.last_error()


def test_nothing_to_attend(L):
    for kw in (dict(rows=0), dict(lr=0)):
        assert L.sr_paged_attention(*args(ATTN, ATTN, kw)) == sr.SR_OK
    assert L.sr_paged_attention_scratch(9, 64, 8, 2, 1, 1, 16, 4, 0, 0, 0, 64) == 0


LOGP = dict(dtype=sr.SR_F32, logits=0x100000, stride=1000, rows=2, vocab=1000, T=1.0, tokens=0x200000, top=4, lp=0x300000,
            h=0x400000, ti=0x500000, tl=0x600000, scratch=0x10000000, n=1 << 22, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=5), INVALID), (dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(stride=999), INVALID),
    (dict(T=0.0), INVALID), (dict(T=-1.0), INVALID), (dict(T=float("nan")), INVALID), (dict(T=float("inf")), INVALID),
    (dict(T=1e-39), INVALID), (dict(top=-1), INVALID), (dict(top=33), UNSUPPORTED), (dict(vocab=3, top=4), INVALID),
    (dict(vocab=262145, stride=262145), UNSUPPORTED), (dict(logits=None), INVALID), (dict(tokens=None), INVALID),
    (dict(logits=0x100002), INVALID), (dict(lp=0x100000), INVALID), (dict(h=0x300004), INVALID),
    (dict(tl=0x500000), INVALID), (dict(rows=1, vocab=128256, stride=128256, n=3), SMALL),
    (dict(rows=1, vocab=128256, stride=128256, scratch=None), SMALL), (dict(rows=(1 << 20) + 1), UNSUPPORTED)])
def test_logprobs_refuse(L, kw, status):
    assert L.sr_token_logprobs(*args(LOGP, LOGP, kw)) == status and sr.last_error()


def test_scratch_sizes_of_bad_shapes(L):
    assert L.sr_page_reserve_scratch(-1, 4, 4) == 0 and L.sr_page_compact_scratch(0) == 0
    assert L.sr_token_logprobs_scratch(2, 0, 0) == 0 and L.sr_token_logprobs_scratch(2, 10, 40) == 0


def test_rope_frequencies():
    i = np.arange(32)
    f = 10000.0 ** (-2.0 * i / 64)
    assert np.allclose(sr.rope_frequencies(64, 1e4), f, rtol=1e-14)
    assert np.allclose(sr.rope_frequencies(64, 1e4, sr.SR_ROPE_LINEAR, 4.0), f / 4, rtol=1e-14)
    got = sr.rope_frequencies(64, 5e5, sr.SR_ROPE_BANDS, 8.0, 1.0, 4.0, 8192.0)
    g = 5e5 ** (-2.0 * i / 64)
    for a, b in zip(got, g):
        w = 2 * np.pi / b
        if w < 8192 / 4.0:
            want = b
        elif w > 8192 / 1.0:
            want = b / 8
        else:
            s = (8192 / w - 1.0) / 3.0
            want = (1 - s) * b / 8 + s * b
        assert abs(a - want) <= 1e-13 * want
    assert any(a == b for a, b in zip(got, g)) and any(abs(a - b / 8) <= 1e-13 * b for a, b in zip(got, g))
    for bad in (dict(rot_dim=12), dict(rot_dim=0), dict(theta=0.0), dict(theta=float("inf")), dict(scaling=3),
                dict(scaling=1, factor=0.5), dict(scaling=2, low=4.0, high=4.0), dict(scaling=2, n=0.0),
                dict(scaling=2, factor=float("nan"))):
        with pytest.raises(sr.SpecRejError) as e:
            sr.rope_frequencies(**{**dict(rot_dim=64, theta=1e4), **bad})
        assert e.value.status == INVALID


def test_binding_checks_tensors():
    """Wrong types, shapes, layouts and devices raise before the library is called."""
    import torch
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    f = lambda *s: torch.zeros(s)  # noqa: E731
    pool = torch.zeros((2, 2, 8, 2, 16, 64), dtype=torch.bfloat16)
    good = dict(pool=pool, table=i(3, 4), lens=i(3), refs=i(8), n_add=1, table_out=i(3, 4), lens_out=i(3), refs_out=i(8),
                granted=i(3), info=i(4))
    for bad in (dict(table=f(3, 4)), dict(table=i(4, 3).t()), dict(lens=i(4)), dict(refs=i(9)), dict(info=i(3)),
                dict(n_add=f(3)), dict(pool=pool[:, :, :, :, ::2]), dict(pool=pool[0])):
        with pytest.raises(ValueError):
            sr.page_reserve(**{**good, **bad})
    with pytest.raises(ValueError, match="GPU"):
        sr.page_reserve(**good)
    k = torch.zeros((8, 2, 16, 64), dtype=torch.bfloat16)
    good = dict(q=f(3, 2, 8, 64), kpool=k, vpool=k.clone(), table=i(3, 4), lens=i(3), out=torch.zeros((3, 2, 512), dtype=k.dtype))
    for bad in (dict(q=f(3, 2, 8, 32)), dict(q=f(4, 2, 8, 64)), dict(vpool=k.float()), dict(out=f(3, 2, 512)),
                dict(out=torch.zeros((3, 2, 256), dtype=k.dtype)), dict(n_new=i(2)), dict(kpool=k[:, :1])):
        with pytest.raises(ValueError):
            sr.paged_attention(**{**good, **bad})
    with pytest.raises(ValueError, match="GPU"):
        sr.paged_attention(**good)
    good = dict(logits=f(3, 9), tokens=i(3), logprob=f(3), entropy=f(3), top_ids=i(3, 2), top_logprobs=f(3, 2))
    for bad in (dict(logits=f(9, 3).t()), dict(logits=f(3, 9).double()), dict(tokens=i(2)), dict(top_ids=i(3, 3)),
                dict(logprob=f(4)), dict(tokens=torch.zeros(3, dtype=torch.int64))):
        with pytest.raises(ValueError):
            sr.token_logprobs(**{**good, **bad})
    with pytest.raises(ValueError, match="GPU"):
        sr.token_logprobs(**good)
    with pytest.raises(ValueError):
        sr.page_fork(i(3, 4), i(3), i(5), 16, i(5, 3), i(5), i(8))
    with pytest.raises(ValueError):
        sr.page_append(f(3, 1, 768), f(32), i(3, 4), i(3), k, k.clone(), f(3, 1, 8, 64))


def test_the_plain_integer_code():
    """The tests' own plain forms on a case worked by hand: three pages of 16,
    two children of a row of 20 tokens."""
    table, lens = np.array([[2, 4, 7]], np.int32), np.array([20], np.int32)
    t, ln, refs = paged_util.fork(table, lens, [0, 0, 9], 16, 6)
    assert t.tolist() == [[2, 4, -1], [2, 4, -1], [-1, -1, -1]] and ln.tolist() == [20, 20, 0]
    assert refs.tolist() == [0, 0, 2, 0, 2, 0]
    t, ln, refs, granted, info, copies = paged_util.reserve(t, ln, refs, [13, 1, 0], 16, 6)
    assert t.tolist() == [[2, 4, 0], [2, 1, -1], [-1, -1, -1]] and ln.tolist() == [33, 21, 0]
    assert refs.tolist() == [1, 1, 2, 0, 1, 0] and copies == [(4, 1, 4)] and info == [0, 0, 2, 1]
    t, refs, info, moves = paged_util.compact(t, ln, refs, 16)
    assert info == [4, 1, 0, 0] and moves == [(4, 3)] and refs.tolist() == [1, 1, 2, 1, 0, 0]
    assert t.tolist() == [[2, 3, 0], [2, 1, -1], [-1, -1, -1]]
    # a window of 3 at length 40 sees tokens 38 on next; one sink
    t, _, refs = paged_util.fork(np.array([[0, 1, 2]], np.int32), np.array([40], np.int32), [0], 16, 3, 3, 1)
    assert t.tolist() == [[0, -1, 2]] and refs.tolist() == [1, 0, 1]
