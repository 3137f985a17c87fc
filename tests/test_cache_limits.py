"""What the entry points of include/rsr_cache.h answer at the limits of their arguments, before anything is launched."""
import ctypes

import paper_2411_06360_amd as R

INVALID = -1
AT = 1 << 20  # an aligned address that nobody reads


def slots(**changes):
    a = dict(held=AT, add=2 * AT, requests=2, table=3 * AT, max_pages=4, page=16, free=4 * AT, most_free=8, count=5 * AT, left=6 * AT, slots=7 * AT, most=9,
             start=8 * AT, now=9 * AT)
    a.update(changes)
    return R.load().rsr_cache_slots_bounded(*a.values(), None)


def test_lists_of_free_pages_that_are_refused():
    assert slots(most_free=-1) == INVALID and "max_free" in R.rsr_last_error()
    assert slots(free=0) == INVALID and slots(count=0) == INVALID
    assert slots(page=12) == INVALID and slots(now=AT) == INVALID
