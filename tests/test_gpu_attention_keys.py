"""rsr_tree_attention with keys that are not finite: the results of the rows that see them are not finite, whatever the sign of the
score, and no other result changes."""
import numpy as np
import pytest
import torch

from tests.cache_util import Step, plain

pytestmark = pytest.mark.gpu
KINDS = [("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16")]
JUNK = [float("inf"), -float("inf"), float("nan")]


def check(s, want, sees):
    """The first key head's results of the rows `sees` have no finite value; all others are what they were."""
    got, touched = s.run(), np.zeros(want.shape, bool)
    touched[sees, :s.heads // s.kv_heads * s.dim] = True
    assert not np.isfinite(got[touched]).any()
    assert np.array_equal(got[~touched], want[~touched])


@pytest.mark.parametrize("act,cache", KINDS)
@pytest.mark.parametrize("dim", [64, 80, 128, 160])
@pytest.mark.parametrize("new", [3, 16])
@pytest.mark.parametrize("held", [0, 40, 3000])
def test_keys_of_new_tokens(act, cache, dim, new, held):
    """Two query heads per key head: up to 16 rows and more of them, in one piece and in several."""
    print("new keys", act, cache, dim, new, held, flush=True)
    s = Step([held, 7], [new, 2], act=act, cache=cache, heads=4, kv_heads=2, dim=dim, seed=31)
    want, keep = s.check().copy(), s.k.clone()
    for token, junk in ((0, JUNK[0]), (1, JUNK[1]), (2, JUNK[2]), (2, JUNK[1])):
        s.k.copy_(keep)
        s.k[token, 5] = junk
        check(s, want, [i for i in range(new) if int(s.mask[i]) >> token & 1])


@pytest.mark.parametrize("act,cache", KINDS)
@pytest.mark.parametrize("dim", [64, 80, 128, 160])
@pytest.mark.parametrize("new", [3, 16])
@pytest.mark.parametrize("held", [1, 40, 3000])
def test_keys_of_cached_tokens(act, cache, dim, new, held):
    print("cached keys", act, cache, dim, new, held, flush=True)
    s = Step([held, 7], [new, 2], act=act, cache=cache, heads=4, kv_heads=2, dim=dim, seed=32)
    want, keep = s.check().copy(), s.cache_k.clone()
    for junk in JUNK:
        for at in {0, held // 2, held - 1}:
            s.cache_k.copy_(keep)
            s.cache_k[int(s.table[0, at // s.page]), 0, at % s.page, dim - 1] = junk
            check(s, want, list(range(new)))


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [24, 64])
def test_keys_in_large_workgroups(kind, dim, new):
    print("large workgroups", kind, dim, new, flush=True)
    s = Step([700, 9], [new, 2], act=kind, cache=kind, heads=8, kv_heads=2, dim=dim, page=64, spare=1100, seed=33)
    want, keep, cached = s.check().copy(), s.k.clone(), s.cache_k.clone()
    for junk in JUNK:
        s.k.copy_(keep)
        s.k[1, 3] = junk
        check(s, want, [i for i in range(new) if int(s.mask[i]) >> 1 & 1])
        s.k.copy_(keep)
        s.cache_k[int(s.table[0, 3]), 0, 11, 2] = junk
        check(s, want, list(range(new)))
        s.cache_k.copy_(cached)


@pytest.mark.parametrize("act,cache", KINDS)
@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("rows", [1, 17])
def test_a_row_whose_only_score_is_minus_infinity_is_not_one_that_sees_nothing(act, cache, dim, rows):
    print("one score", act, cache, dim, rows, flush=True)
    s = Step([0], [rows], act=act, cache=cache, heads=1, kv_heads=1, dim=dim, seed=34)
    s.mask.copy_(1 << torch.arange(rows))  # a token sees itself alone
    s.mask[rows - 1] = 0 if rows > 1 else 1
    s.k[0] = -torch.sign(s.q[0]) * float("inf")
    got = s.run()
    assert not np.isfinite(got[0]).any()
    assert np.isfinite(got[1:]).all() and (rows == 1 or not got[-1].any())


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 17])
def test_scores_beyond_the_range_of_float_are_not_finite(act, rows):
    print("beyond float", act, rows, flush=True)
    for sign in (1, -1):
        s = Step([0], [rows], act=act, cache="bf16", heads=1, kv_heads=1, dim=64, seed=35)
        s.mask.copy_(1 << torch.arange(rows))
        s.q[0], s.k[0] = 1e30, sign * 1e30
        got = s.run()
        assert not np.isfinite(got[0]).any() and np.isfinite(got[1:]).all()
        alone = plain(s.v.to(s.cache_k.dtype))[1:]  # a token that sees itself alone: its own value, times its weight, by its weight
        assert (np.abs(got[1:] - alone) <= 2.0**-20 * np.abs(alone)).all()
