"""rsr_tree_attention with the workgroups that it takes for much work, and with sets that are cut into pieces of their own, against the
definition in float64.  (How much work there could be is read from the length of the tables, which may hold little.)"""
import numpy as np
import pytest

import paper_2411_06360_amd as R
from tests.cache_util import Step

pytestmark = pytest.mark.gpu
SPARE = 1100  # pages of 64 in a row of the table that no request has: 2200 tiles of 32 for each key head


def large(held, new, **k):
    s = Step(held, new, page=64, spare=SPARE, kv_heads=2, **k)
    pieces = 1024 * 128 * ((64 if s.dim <= 64 else 128) + 2) * 4  # of 128 rows, two for each of 512 workgroups
    assert R.rsr_tree_attention_workspace(R.make_cache(s.cache_k, s.cache_v), R.make_step(s.table, s.held, s.start, s.tokens, s.max_new, s.mask), s.heads) > pieces
    return s


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [40, 64, 96, 128])
@pytest.mark.parametrize("new", [20, 33, 64])
def test_two_tiles_of_rows(kind, dim, new):
    print("two tiles", kind, dim, new, flush=True)
    large([0, 31, 700, 65, 300, 128, 1, 2000], [new, 1, new, new - 1, 0, 7, 2, new], heads=8, dim=dim, act=kind, cache=kind, seed=dim + new).check()


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_long_chains_in_large_workgroups(kind, dim):
    print("chains", kind, dim, flush=True)
    large([0, 100, 513], [333, 65, 1], heads=4, dim=dim, act=kind, cache=kind, tree=False, seed=1).check()


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("new", [24, 64])
def test_large_workgroups_are_joined(kind, new):
    print("joined", kind, new, flush=True)
    s = large([40000, 3, 9000, 700], [new, 2, new, new], heads=8, dim=128, act=kind, cache=kind, seed=2)
    first = s.check().copy()
    assert np.array_equal(s.run(), first)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [24, 64])
@pytest.mark.parametrize("held", [20, 5000])
def test_values_that_are_not_finite_in_large_workgroups(kind, dim, new, held):
    """They arrive where they are seen, and touch nothing else."""
    print("not finite", kind, dim, new, held, flush=True)
    s = large([held] * 4, [new] * 4, heads=8, dim=dim, act=kind, cache=kind, seed=3)
    want = s.check().copy()
    s.v[3, 5] = float("inf")  # token 3 of the first request, dimension 5 of the first key head
    s.v[3, 9] = float("nan")
    got = s.run()
    sees = np.array([r < new and bool(int(m) >> 3 & 1) for r, m in enumerate(s.mask.tolist())])
    assert sees.any() and not sees[:new].all()
    at = np.array([a * dim + d for a in range(4) for d in (5, 9)])
    assert (got[sees][:, at[0::2]] == np.inf).all() and np.isnan(got[sees][:, at[1::2]]).all()
    got[np.ix_(sees, at)] = want[np.ix_(sees, at)]
    assert np.array_equal(got, want)


@pytest.mark.parametrize("act,cache", [("f32", "f16"), ("bf16", "bf16")])
@pytest.mark.parametrize("requests", [2, 63, 64, 65, 130, 200])
@pytest.mark.parametrize("heads", [1, 8])
def test_sets_of_all_lengths_are_cut(act, cache, requests, heads):
    """Several requests per lane of the plan, requests without tokens, and sets of one piece beside sets of many."""
    print("cut", act, cache, requests, heads, flush=True)
    rng = np.random.default_rng([requests, heads])
    held, new = [int(x) for x in rng.integers(0, 60, requests)], [int(x) for x in rng.integers(0, 5, requests)]
    held[requests // 2], new[requests // 2], held[-1], new[-1] = 3000, 3, 1500, 1
    Step(held, new, heads=heads, kv_heads=1, dim=64, act=act, cache=cache, page=16, seed=4).check()


@pytest.mark.parametrize("dim", [128, 256])
@pytest.mark.parametrize("held", [0, 40, 700])
def test_blocks_of_a_chain_that_see_little_are_cut_like_the_others(dim, held):
    print("chain blocks", dim, held, flush=True)
    for act, cache in (("f32", "bf16"), ("f16", "f16")):
        Step([held, 3], [300, 200], heads=4, kv_heads=2, dim=dim, act=act, cache=cache, tree=False, seed=5).check()
