"""rsr_tree_keep (include/rsr_decode.h) against its definition."""
import numpy as np
import pytest
import torch

import paper_2411_06360_amd as R
from oracle import decode as oracle
from tests.cache_util import draft

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Call:
    def __init__(self, drafted, chosen, parent, start, tokens=None):
        self.tokens, self.requests = len(drafted) if tokens is None else tokens, len(start) - 1
        self.lists = [list(map(int, x)) if x is not None else None for x in (drafted, chosen, parent, start)]
        self.inputs = [None if x is None else ints(x if len(x) else [0])[:len(x)] for x in self.lists]
        self.rows, self.found = (torch.full((self.tokens,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
        self.add, self.first = (torch.full((self.requests + i,), -7, dtype=torch.int32, device="cuda") for i in range(2))

    def call(self):
        drafted, chosen, parent, start = self.inputs
        R.rsr_tree_keep(drafted, chosen, parent, start, self.rows, self.found, self.add, self.first, torch.cuda.current_stream().cuda_stream)

    def check(self):
        self.call()
        torch.cuda.synchronize()
        want = oracle.keep(*self.lists, self.tokens)
        assert (self.rows.tolist(), self.found.tolist(), self.add.tolist(), self.first.tolist()) == want
        return want


def trees(seed, new, right=0.8, chain=False, words=1000):
    """Guesses of which so many are what is chosen."""
    rng = np.random.default_rng([seed, len(new)])
    start = np.concatenate([[0], np.cumsum(new)]).astype(int)
    parent = [p for n in new for p in (range(-1, n - 1) if chain else draft(rng, n))]
    drafted, chosen = rng.integers(0, words, start[-1]), rng.integers(0, words, start[-1])
    for r in range(len(new)):
        for i in range(start[r], start[r + 1]):
            if parent[i] >= 0 and rng.random() < right:
                chosen[start[r] + parent[i]] = drafted[i]
    return drafted, chosen, None if chain else parent, start


@pytest.mark.parametrize("requests", [0, 1, 2, 15, 16, 17, 63, 64, 65, 255, 256, 257, 1000, 4097])
@pytest.mark.parametrize("chain", [False, True])
def test_requests(requests, chain):
    print("requests", requests, chain, flush=True)
    rng = np.random.default_rng(requests)
    Call(*trees(requests, rng.integers(0, 20, requests).tolist(), chain=chain)).check()


@pytest.mark.parametrize("new", [1, 2, 3, 31, 32, 33, 63, 64, 65, 100])
@pytest.mark.parametrize("right", [0.0, 0.5, 1.0])
def test_trees_of_every_size(new, right):
    print("trees", new, right, flush=True)
    for chain in (False, True):
        rows, _, add, _ = Call(*trees(new, [new, 1, new, 0, new], right, chain)).check()
        if chain and right == 1.0:
            assert add == [min(new, 64), 1, min(new, 64), 0, min(new, 64)]


def test_the_first_of_equal_guesses():
    for seed in range(20):
        Call(*trees(seed, [40, 64, 7], words=2)).check()


def test_most_requests():
    Call(*trees(5, [1 + r % 3 for r in range(65535)])).check()


def test_no_tokens():
    Call([], [], [], [0]).check()
    Call([], [], [], [0, 0, 0]).check()
    Call([5, 6], [6, 7], [-1, 0], [0]).check()


def test_nothing_was_chosen():
    """A negative choice ends the path, whatever was guessed."""
    drafted, chosen, parent, start = trees(9, [30] * 6, right=1.0)
    chosen[::3], drafted[1::2] = -1, -1
    Call(drafted, chosen, parent, start).check()


@pytest.mark.parametrize("start", [[0, 50, 50], [-5, 3, 9], [4, 2, 7], [0, 1 << 30, 3], [100, 200, 300], [2, 4, 8], [-(1 << 31), (1 << 31) - 1, 5], [3, 12, 0]])
def test_trees_that_end_elsewhere(start):
    """Ends behind the last token, before the first, rows of no request."""
    drafted, chosen, parent, _ = trees(3, [12], right=1.0)
    Call(drafted, chosen, parent, start).check()


def test_parents_out_of_range():
    drafted, chosen, parent, start = trees(4, [20, 20], right=0.9)
    parent[3], parent[5], parent[8], parent[25], parent[27] = 3, 19, 1 << 30, -(1 << 31), 7
    Call(drafted, chosen, parent, start).check()


def test_trees_that_overlap_stay_within_the_rows():
    drafted, chosen, parent, _ = trees(6, [30], right=1.0)
    chain = Call(drafted, np.concatenate([drafted[1:], [0]]), None, [0, 30, 60])
    chain.inputs[3] = ints([0, 30, 0, 30])[[0, 1, 1]]  # (one request with all rows, another with none)
    chain.lists[3] = [0, 30, 30]
    chain.check()
    many = Call(drafted, np.concatenate([drafted[1:], [0]]), None, [0, 30, 0, 30, 0, 30])
    many.check()


def test_again_and_into_what_was_there():
    c = Call(*trees(8, [16] * 100))
    want = c.check()
    for _ in range(3):
        for x in (c.rows, c.found, c.add, c.first):
            x.fill_(99)
        assert c.check() == want
