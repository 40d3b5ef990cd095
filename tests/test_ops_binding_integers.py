"""Numbers that do not fit the library's 32-bit arguments are refused by the
binding of the paged operators; ctypes would pass their lower half."""
import pytest

import paper_2410_20290_amd as sr

FAR = 2 ** 32 + 5


def tensors():
    import torch
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    pool = torch.zeros((2, 2, 8, 2, 16, 64), dtype=torch.bfloat16)
    return i, pool, torch.zeros((3, 2, 8, 64)), torch.zeros((3, 2, 512), dtype=torch.bfloat16)


@pytest.mark.parametrize("kw", [dict(window=FAR), dict(sinks=FAR), dict(shared=FAR), dict(max_len=FAR),
                                dict(window=-2 ** 32 + 5), dict(window=2 ** 31)])
def test_paged_attention(kw):
    i, pool, q, out = tensors()
    with pytest.raises(ValueError, match="32 bits"):
        sr.paged_attention(q, pool[0, 0], pool[0, 1], i(3, 4), i(3), out, **kw)


@pytest.mark.parametrize("kw", [dict(page_tokens=2 ** 32 + 16), dict(window=FAR), dict(sinks=FAR)])
def test_page_fork(kw):
    i, _, _, _ = tensors()
    with pytest.raises(ValueError, match="32 bits"):
        sr.page_fork(**{**dict(table=i(3, 4), lens=i(3), parent=i(5), page_tokens=16, table_out=i(5, 4), lens_out=i(5),
                               refs_out=i(8)), **kw})


@pytest.mark.parametrize("n_add,match", [(FAR, "32 bits"), (-FAR, "32 bits"), (1.5, "whole number")])
def test_page_reserve(n_add, match):
    i, pool, _, _ = tensors()
    with pytest.raises(ValueError, match=match):
        sr.page_reserve(pool, i(3, 4), i(3), i(8), n_add, i(3, 4), i(3), i(8), i(3), i(4))


def test_rope_frequencies():
    for kw in (dict(rot_dim=2 ** 32 + 64), dict(scaling=2 ** 32)):
        with pytest.raises(ValueError, match="32 bits"):
            sr.rope_frequencies(**{**dict(rot_dim=64, theta=1e4), **kw})


def test_numbers_that_fit_pass_on():
    """The largest ones reach the check after it (the tensors are on no GPU)."""
    i, pool, q, out = tensors()
    top = 2 ** 31 - 1
    with pytest.raises(ValueError, match="GPU"):
        sr.paged_attention(q, pool[0, 0], pool[0, 1], i(3, 4), i(3), out, window=top, sinks=top, shared=top, max_len=top)
    for n_add in (top, 3.0, -2 ** 31):
        with pytest.raises(ValueError, match="GPU"):
            sr.page_reserve(pool, i(3, 4), i(3), i(8), n_add, i(3, 4), i(3), i(8), i(3), i(4))
