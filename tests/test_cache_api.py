"""The operators around the paged cache without a GPU: their definitions on cases worked out by hand, and what the entry points
answer before anything is launched (include/rsr_cache.h)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2411_06360_amd as R
from oracle import cache as oracle

INVALID, UNSUPPORTED = -1, -2
AT = 1 << 20  # an aligned address that nobody reads: all of these calls end before a launch


def cache(**changes):
    c = R.RsrCache(AT, AT, 4 * 32 * 64, 32 * 64, 64, R.RSR_BF16, 10, 32, 4, 64, 0)
    for name, value in changes.items():
        setattr(c, name, value)
    return c


def step(**changes):
    s = R.RsrStep(AT, AT, AT, None, 2, 6, 3, 5)
    for name, value in changes.items():
        setattr(s, name, value)
    return s


def attention(c=None, s=None, **changes):
    c, s = c or cache(), s or step()
    a = dict(q=AT, q_stride=512, k=AT, v=AT, kv_stride=256, out=2 * AT, out_stride=512, dtype=R.RSR_F32, heads=8, scale=0.125, workspace=AT, bytes=1 << 40)
    a.update(changes)
    return R.load().rsr_tree_attention(ctypes.addressof(c), ctypes.addressof(s), a["q"], a["q_stride"], a["k"], a["v"], a["kv_stride"], a["out"],
                                       a["out_stride"], a["dtype"], a["heads"], a["scale"], a["workspace"], a["bytes"], None)


@pytest.mark.parametrize("changes", [
    dict(k=0), dict(v=0), dict(k=AT + 8), dict(dtype=R.RSR_F32), dict(dtype=7), dict(pages=0), dict(pages=1 << 26), dict(page_size=24), dict(page_size=4),
    dict(page_size=2048), dict(kv_heads=0), dict(kv_heads=1025), dict(head_dim=0), dict(head_dim=60), dict(head_dim=264), dict(token_stride=60),
    dict(token_stride=1 << 24), dict(page_stride=1 << 31), dict(head_stride=-8)])
def test_caches_that_are_refused(changes):
    c = cache(**changes)
    assert attention(c) == INVALID and R.rsr_last_error()
    assert R.load().rsr_tree_attention_workspace(ctypes.addressof(c), ctypes.addressof(step()), 8) == INVALID
    assert R.load().rsr_cache_append(ctypes.addressof(c), AT, AT, 1 << 20, 4, R.RSR_BF16, None, AT, 4, None) == INVALID


@pytest.mark.parametrize("changes", [dict(table=0), dict(held=0), dict(start=0), dict(requests=-1), dict(requests=65536), dict(tokens=-1), dict(max_new=0),
                                     dict(max_new=65536), dict(max_new=65, mask=AT), dict(max_pages=0)])
def test_steps_that_are_refused(changes):
    assert attention(s=step(**changes)) == INVALID
    assert R.load().rsr_tree_attention_workspace(ctypes.addressof(cache()), ctypes.addressof(step(**changes)), 8) == INVALID


@pytest.mark.parametrize("changes", [
    dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(q=AT + 4), dict(out=AT + 8), dict(q_stride=511), dict(q_stride=514), dict(kv_stride=252),
    dict(out_stride=500), dict(q_stride=1 << 31), dict(dtype=R.RSR_F16), dict(dtype=3), dict(heads=0), dict(heads=6), dict(heads=4 * 65),
    dict(scale=math.inf), dict(scale=math.nan), dict(workspace=0), dict(workspace=AT + 128), dict(bytes=1024)])
def test_attention_that_is_refused(changes):
    assert attention(**changes) == INVALID and R.rsr_last_error()


def test_work_that_cannot_be_counted_is_refused():
    c, s = cache(page_size=1024, kv_heads=1024, pages=1000), step(requests=65535, max_pages=1 << 30)
    assert attention(c, s, heads=1024, q_stride=1 << 16, out_stride=1 << 16, kv_stride=1 << 16) == UNSUPPORTED
    assert R.load().rsr_tree_attention_workspace(ctypes.addressof(c), ctypes.addressof(s), 1024) == UNSUPPORTED


def test_nothing_to_do_is_done_without_a_launch():
    null = dict(table=0, held=0, start=0)
    assert attention(s=step(requests=0, **null)) == 0
    assert attention(s=step(tokens=0), q=0, k=0, v=0, out=0) == 0
    lib = R.load()
    assert lib.rsr_cache_append(ctypes.addressof(cache()), 0, 0, 256, 0, R.RSR_F32, None, 0, 4, None) == 0
    assert lib.rsr_cache_append(ctypes.addressof(cache()), 0, 0, 256, 4, R.RSR_F32, None, 0, 0, None) == 0
    assert lib.rsr_tree_masks(0, 0, 0, 5, 0, 0, None) == 0 and lib.rsr_tree_masks(0, 0, 3, 0, 0, 0, None) == 0


@pytest.mark.parametrize("dim,heads", [(64, 8), (128, 4), (256, 256), (40, 4)])
def test_the_workspace_does_not_grow_with_the_batch_beyond_the_chip(dim, heads):
    c = cache(head_dim=dim, page_stride=4 * 32 * dim, head_stride=32 * dim, token_stride=dim)
    sizes = [R.rsr_tree_attention_workspace(c, step(requests=r, tokens=64 * r, max_new=64, max_pages=p), heads) for r, p in ((1, 1), (64, 100), (60000, 4000))]
    assert 0 < sizes[0] <= sizes[1] <= sizes[2] <= 1 << 27


def test_slots_that_are_refused():
    def call(**changes):
        a = dict(held=AT, add=2 * AT, requests=2, table=3 * AT, max_pages=4, page=16, free=4 * AT, count=5 * AT, left=6 * AT, slots=7 * AT, most=9, start=8 * AT,
                 now=9 * AT)
        a.update(changes)
        return R.load().rsr_cache_slots(*a.values(), None)

    for changes in (dict(requests=-1), dict(requests=65536), dict(max_pages=0), dict(page=12), dict(page=0), dict(most=-1), dict(held=0), dict(add=0),
                    dict(table=0), dict(free=0), dict(count=0), dict(left=0), dict(slots=0), dict(start=0), dict(now=0), dict(left=5 * AT), dict(now=AT),
                    dict(now=2 * AT), dict(start=AT)):
        assert call(**changes) == INVALID, changes


def test_masks_and_appends_that_are_refused():
    lib = R.load()
    for a in ((0, AT, 1, 1, AT, AT), (AT, 0, 1, 1, AT, AT), (AT, AT, 1, 1, 0, AT), (AT, AT, 1, 1, AT, 0), (AT, AT, -1, 1, AT, AT), (AT, AT, 1, -1, AT, AT),
              (AT, AT, 65536, 1, AT, AT)):
        assert lib.rsr_tree_masks(*a, None) == INVALID, a
    for a in ((0, AT, 256, 4, 0, None, AT, 4), (AT, 0, 256, 4, 0, None, AT, 4), (AT, AT, 255, 4, 0, None, AT, 4), (AT, AT, 256, -1, 0, None, AT, 4),
              (AT, AT, 256, 4, 1, None, AT, 4), (AT, AT, 256, 4, 0, None, 0, 4), (AT, AT, 256, 4, 0, None, AT, -1), (AT + 4, AT, 256, 4, 0, None, AT, 4)):
        assert lib.rsr_cache_append(ctypes.addressof(cache()), *a, None) == INVALID, a


def test_what_the_binding_refuses():
    k = torch.zeros((3, 2, 16, 8), dtype=torch.bfloat16)
    ints = torch.zeros(4, dtype=torch.int32)
    table = torch.zeros((3, 2), dtype=torch.int32)
    for bad in ((k, k[:2]), (k, k.half()), (k[0], k[0]), (k, k.transpose(0, 1).contiguous().transpose(0, 1)), (k[..., ::2], k[..., ::2])):
        with pytest.raises(ValueError):
            R.make_cache(*bad)
    with pytest.raises(TypeError):
        R.make_cache(k.double(), k.double())
    for bad in ((table, ints, ints), (table, ints[:3], ints[:3]), (table.long(), ints[:3], ints), (table, ints[:3], ints, 4, 2, torch.zeros(3, dtype=torch.int64)),
                (table, ints[:3], ints, 4, 2, ints), (table[:, ::2], ints[:3], ints)):
        with pytest.raises(ValueError):
            R.make_step(*bad, *((4, 2) if len(bad) == 3 else ()))
    c, s, x = R.make_cache(k, k), R.make_step(table, ints[:3], ints, 4, 2), torch.zeros((4, 32))
    space = torch.zeros(16, dtype=torch.uint8)
    for q, key, value, out in ((x[:3], x[:, :16], x[:, 16:], x), (x, x[:, :8], x[:, 16:], x), (x, x[:, :16], x[:, 16:].contiguous(), x),
                               (x, x[:, :16], x[:, 16:], x.half()), (x, x[:, :16], x.half()[:, 16:], x), (x[:, ::2], x[:, :16], x[:, 16:], x)):
        with pytest.raises(ValueError):
            R.rsr_tree_attention(c, s, q, key, value, out, 4, 1.0, space)
    with pytest.raises(ValueError):
        R.rsr_cache_append(c, x[:, :16], x[:, :8], ints)
    with pytest.raises(ValueError):
        R.rsr_tree_masks(ints, ints, ints, ints)


# ---- the definitions ----
def test_masks_by_hand():
    #  0 - 1 - 3      4 hangs on the cache, as does what names itself or a later token
    #    \ 2       ; the second request's parents are counted from its own first token
    mask, depth = oracle.masks([-1, 0, 0, 1, 7, -1, 0], [0, 5, 7], 8)
    assert mask == [0b1, 0b11, 0b101, 0b1011, 0b10000, 0b1, 0b11, None]
    assert depth == [0, 1, 1, 2, 0, 0, 1, None]


def test_slots_by_hand():
    # pages of 4: request 0 holds 3 and adds 2 (a place on page 5, then page 9), request 1 holds nothing and adds 5 (pages 8, 7)
    slots, table, start, now, left = oracle.slots([3, 0], [2, 5], [[5, 0, 0], [0, 0, 0]], 4, [6, 7, 8, 9], 4, 8)
    assert slots == [23, 36, 32, 33, 34, 35, 28, -1] and start == [0, 2, 7] and now == [5, 5] and left == 1
    assert table.tolist() == [[5, 9, 0], [8, 7, 0]]
    # one page for two: the second request gets none of it, and the list is short of one
    slots, table, start, now, left = oracle.slots([4, 0], [1, 2], [[5, 0], [0, 0]], 4, [6], 1, 3)
    assert slots == [24, -1, -1] and now == [5, 0] and left == -1 and table.tolist() == [[5, 6], [-1, 0]]


def test_attention_by_hand():
    # one head of two dimensions; scores log 1 and log 3, then a page that is not there, then a new token
    cache_k = np.array([[[[0.0, 1.0], [math.log(3), 1.0]]]])
    cache_v = np.array([[[[8.0, 0.0], [4.0, 4.0]]]])
    q, k, v = np.array([[1.0, 0.0]]), np.array([[math.log(4), 5.0]]), np.array([[2.0, 1.0]])
    table, held, start = np.array([[0, -1]]), [4], [0, 1]
    out, *_, seen = oracle.attention(q, k, v, cache_k, cache_v, table, held, start, [0], 1, 1.0, 1)
    assert np.allclose(out, [[5.0, 3.0]], rtol=1e-15) and seen == 2
    out, *_ = oracle.attention(q, k, v, cache_k, cache_v, table, held, start, [1], 1, 1.0, 1)
    assert np.allclose(out, [[(8 + 12 + 8) / 8, (12 + 4) / 8]], rtol=1e-15)
    out, *_ = oracle.attention(q, k, v, cache_k, cache_v, np.array([[-1, -1]]), held, start, [0], 1, 1.0, 1)
    assert np.array_equal(out, [[0.0, 0.0]])


def test_append_by_hand():
    x = np.arange(8.0).reshape(2, 4)  # two rows of two heads
    got = oracle.append(np.full((2, 2, 2, 2), -1.0), x, [1, 0, 5, 0], [2, 1, 0, 9], lambda y: y)
    assert got[1, :, 0].tolist() == [[4, 5], [6, 7]] and got[0, :, 1].tolist() == [[0, 1], [2, 3]]
    assert (got == -1).sum() == 8
