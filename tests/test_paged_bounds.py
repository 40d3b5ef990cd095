"""The bound that the long rows of the paged attention are held to, on the CPU:
what a right kernel rounds passes it, and mistakes planted in the oracle do not."""
import numpy as np
import pytest

from paged_long import CASES, make

# Mistakes: what a query sees, changed.  Each returns the mask, or None where it
# changes nothing in this case.


def nothing(c, r, t, m):
    m[:] = False
    return m


def last_quarter(c, r, t, m):
    m[3 * len(m) // 4:] = False
    return m


def one_slot(c, r, t, m):
    """One of sixteen splits of the row's blocks."""
    n = len(m)
    m[n * 5 // 16:n * 6 // 16] = False
    return m


def one_block(c, r, t, m):
    """32 keys in the middle of what is seen."""
    j = np.nonzero(m)[0]
    a = j[len(j) // 2] // 32 * 32
    m[a:a + 32] = False
    return m


def tail(c, r, t, m):
    m[c.shared:] = False
    return m


def prefix(c, r, t, m):
    m[:c.shared] = False
    return m


def no_sinks(c, r, t, m):
    m[:c.sinks] &= np.arange(c.sinks) > len(m) - c.new[r] + t - c.window
    return m


def late_window(c, r, t, m):
    p = len(m) - c.new[r] + t
    if p - c.window + 1 > 0:
        m[p - c.window + 1] = p - c.window + 1 < c.sinks
    return m


def own_key(c, r, t, m):
    m[len(m) - c.new[r] + t] = False
    return m


def first_key(c, r, t, m):
    m[0] = False
    return m


def plants(c, marked):
    yield nothing
    yield last_quarter
    yield one_slot
    if not marked and not c.window:
        yield one_block
    if c.shared:
        yield tail
        yield prefix
    if marked:
        yield own_key
        if not c.window or c.sinks:
            yield first_key
        if c.window:
            yield late_window
            if c.sinks:
                yield no_sinks


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("marked", [True, False])
def test_bound_tells_right_from_wrong(name, marked):
    c = make(name, marked)
    ref = c.oracle()
    arr = lambda got: {r: {t: got[r, t][0] for rr, t in got if rr == r} for r, _ in got}  # noqa: E731
    right = c.worst(arr(c.oracle(rounded=True, bound=False)), ref)
    assert 0.02 < right < 0.8, right            # the roundings show, and stay clear of the bound
    for wrong in plants(c, marked):
        # a mistake may spare some rows and heads, not all of them
        got = c.worst(arr(c.oracle(see=wrong, bound=False)), ref)
        assert got > 1.5, (wrong.__name__, got)
