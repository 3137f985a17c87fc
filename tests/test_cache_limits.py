"""What the entry points of include/rsr_cache.h answer at the limits of their arguments, before anything is launched."""
import ctypes

import pytest
import torch

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


# ---- workspace ----
def workspace(dim, kv_heads, heads, requests, new, pages, page=32):
    c = R.RsrCache(AT, AT, kv_heads * page * dim, page * dim, dim, R.RSR_BF16, 10, page, kv_heads, dim, 0)
    s = R.RsrStep(AT, AT, AT, None, requests, requests * new, new, pages)
    return R.rsr_tree_attention_workspace(c, s, heads)


@pytest.mark.parametrize("dim", [40, 64, 128, 256])
@pytest.mark.parametrize("kv_heads", [1, 5, 20, 127, 128])
def test_a_workspace_for_more_work_is_not_smaller(dim, kv_heads):
    """A program asks once, for its longest table, most requests and tokens: shorter steps must not need more."""
    least = {}
    for requests in (1, 2, 7, 64, 1000):
        for new in (1, 3, 16, 17, 64, 65, 300):
            for pages in (1, 50, 250, 500, 4000, 20000):
                for group in (1, 2, 4, 64):
                    here = (requests, new, pages, group)
                    least[here] = workspace(dim, kv_heads, group * kv_heads, requests, new, pages)
    for (r, n, p, g), bytes_ in least.items():
        for (r1, n1, p1, g1), more in least.items():
            if r <= r1 and n <= n1 and p <= p1 and g <= g1:
                assert bytes_ <= more, ((r, n, p, g), (r1, n1, p1, g1))


def test_the_workspace_of_one_sequence_with_a_table_of_any_length():
    """20 heads of 128, one request, one token: a table of 500 pages of 32 asks for what one of 250 asks for."""
    sizes = [workspace(128, 20, 20, 1, 1, pages) for pages in (1, 250, 500, 8192)]
    assert sizes == sorted(sizes)


# ---- strides ----
def test_the_stride_of_a_single_row_means_nothing():
    """One token's rows come out of tensors of any width, keys and values out of different ones.  (Here the call ends at the workspace,
    which is the last thing that is looked at.)"""
    k = torch.zeros((3, 2, 16, 8), dtype=torch.bfloat16)
    ints = torch.zeros(4, dtype=torch.int32)
    cache, step = R.make_cache(k, k), R.make_step(torch.zeros((1, 2), dtype=torch.int32), ints[:1], ints[:2], 1, 1)
    row = lambda width, stride: torch.zeros(stride)[:width].as_strided((1, width), (stride, 1))  # noqa: E731
    for strides in ((32, 16, 16, 32), (37, 16, 16, 33), (32, 16, 51, 32), (32, 96, 21, 41)):
        q, key, value, out = (row(w, s) for w, s in zip((32, 16, 16, 32), strides))
        with pytest.raises(R.RsrError, match="workspace"):
            R.rsr_tree_attention(cache, step, q, key, value, out, 4, 1.0, torch.zeros(16, dtype=torch.uint8))


# ---- append ----
def test_more_tokens_than_an_append_can_number_are_refused():
    c = R.RsrCache(AT, AT, 1024 * 8 * 256, 8 * 256, 256, R.RSR_BF16, 10, 8, 1024, 256, 0)
    append = lambda count: R.load().rsr_cache_append(ctypes.addressof(c), AT, AT, 1024 * 256, 4, R.RSR_BF16, None, AT, count, None)  # noqa: E731
    for count in (2**41, 2**62, 2**63 - 1):
        assert append(count) == INVALID and "count" in R.rsr_last_error()
