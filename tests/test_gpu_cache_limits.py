"""rsr_cache_slots and rsr_cache_append at the limits of what they are given (include/rsr_cache.h)."""
import numpy as np
import pytest
import torch

import paper_2411_06360_amd as R
from oracle import cache as oracle

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("have", [0, 1, 5, 12])
@pytest.mark.parametrize("beyond", [1, 40, 2**31 - 1])
def test_a_count_beyond_the_list_of_free_pages_is_taken_as_its_length(have, beyond):
    """The list is the beginning of a larger tensor, whose other entries are not free."""
    print("free list", have, beyond, flush=True)
    held, add, old, page = [10, 0, 40], [30, 100, 3], np.full((3, 9), 500, np.int32), 16
    all_pages = ints(100 + np.arange(60))
    table, slots, start, now, left = ints(old), ints([-7] * 140), ints([-7] * 4), ints([-7] * 3), ints([-7])
    R.rsr_cache_slots(ints(held), ints(add), table, page, all_pages[:have], ints([min(have + beyond, 2**31 - 1)]), slots, start, now, left, stream())
    torch.cuda.synchronize()
    want = oracle.slots(held, add, old, page, list(range(100, 100 + have)), have, 140)
    assert slots.tolist() == want[0] and np.array_equal(table.cpu().numpy(), want[1])
    assert start.tolist() == want[2] and now.tolist() == want[3] and left.item() == want[4]


def test_slots_beyond_31_bits_do_not_wrap():
    """More added tokens than an int32 counts, with room for their slots: `start` stays at the largest that it can say."""
    print("2^31 slots", flush=True)
    most = 2**31 - 1
    table = ints([[7], [-1], [9], [3]])
    slots, start, now, left = torch.full((most + 300,), -7, dtype=torch.int32, device="cuda"), ints([0] * 5), ints([0] * 4), ints([0])
    R.rsr_cache_slots(ints([2, 0, 3, 1]), ints([most - 1, 100, 7, 50]), table, 8, ints([4]), ints([1]), slots, start, now, left, stream())
    torch.cuda.synchronize()
    assert start.tolist() == [0, most - 1, most, most, most] and now.tolist() == [8, 8, 8, 8]
    # (request 1 takes the free page; of request 0 six tokens have a place, of the others eight, five and seven)
    assert slots[:6].tolist() == list(range(58, 64)) and slots[most - 1:most + 7].tolist() == list(range(32, 40))
    assert slots[most + 99:most + 104].tolist() == list(range(75, 80)) and slots[most + 106:most + 113].tolist() == list(range(25, 32))
    assert int((slots >= 0).sum()) == 6 + 8 + 5 + 7 and int(slots.min()) == -1


def test_a_length_beyond_31_bits_does_not_wrap():
    """A table for more tokens than an int32 counts, all but full of them."""
    print("2^31 tokens", flush=True)
    width = 2**21 + 2
    table = torch.full((1, width), 3, dtype=torch.int32, device="cuda")
    slots, start, now, left = ints([-7] * 101), ints([-7] * 2), ints([-7]), ints([-7])
    R.rsr_cache_slots(ints([2**31 - 10]), ints([100]), table, 1024, ints([8, 5]), ints([2]), slots, start, now, left, stream())
    torch.cuda.synchronize()
    assert now.tolist() == [2**31 - 1] and start.tolist() == [0, 100] and left.item() == 1
    assert slots.tolist() == list(range(4 * 1024 - 10, 4 * 1024)) + list(range(5 * 1024, 5 * 1024 + 90)) + [-1]
    assert table[0, -3:].tolist() == [3, 5, 3]


def test_more_tokens_than_a_launch_has_workgroups():
    """2^24 wide tokens, of which a few have a slot."""
    print("many tokens", flush=True)
    count, kv_heads, dim = 2**24 + 5, 16, 128
    k, v = (torch.randn((7, kv_heads * dim), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    caches = [torch.zeros((2, kv_heads, 8, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rows, slots = torch.zeros(count, dtype=torch.int32, device="cuda"), torch.full((count,), -1, dtype=torch.int32, device="cuda")
    kept = {0: (3, 4), 1: (2, 9), 2**24 - 2: (6, 0), 2**24: (1, 15), count - 2: (5, 8), count - 1: (4, 7)}
    for at, (row, slot) in kept.items():
        rows[at], slots[at] = row, slot
    R.rsr_cache_append(R.make_cache(*caches), k, v, slots, rows, stream())
    torch.cuda.synchronize()
    for cache, x in zip(caches, (k, v)):
        want = torch.zeros_like(cache)
        for row, slot in kept.values():
            want[slot // 8, :, slot % 8] = x[row].view(kv_heads, dim)
        assert torch.equal(cache, want)
