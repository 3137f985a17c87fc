"""rsr_tree_attention in the forms of its kernels that depend on how much work there could be: few rows with four and with eight
wavefronts, and the pages of eight wavefronts with many rows; and what a result may depend on."""
import copy

import numpy as np
import pytest
import torch

import paper_2411_06360_amd as R
from tests.cache_util import Step, plain

pytestmark = pytest.mark.gpu
KINDS = [("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16")]


def wavefronts(s):
    """Of a workgroup with up to 16 rows per key head: eight where few key heads have tables for many tiles of 32 tokens."""
    assert s.max_new * (s.heads // s.kv_heads) <= 16 and s.dim <= 128
    sets = s.held.numel() * s.kv_heads
    tiles = -(-s.table.shape[1] * s.page // 32) + -(-s.max_new // 32)
    return 8 if sets < 128 and sets * tiles > 4096 else 4


def few_rows(wide, held, new, **k):
    s = Step(held, new, page=64, spare=1100 if wide else 0, kv_heads=2, **k)
    assert wavefronts(s) == (8 if wide else 4)
    return s


@pytest.mark.parametrize("act,cache", KINDS)
@pytest.mark.parametrize("dim", [8, 40, 64, 72, 80, 96, 120, 128])
@pytest.mark.parametrize("wide", [False, True])
def test_few_rows(act, cache, dim, wide):
    print("few rows", act, cache, dim, wide, flush=True)
    few_rows(wide, [1200, 0, 77, 31], [8, 3, 1, 5], heads=4, dim=dim, act=act, cache=cache, seed=41).check()
    few_rows(wide, [600, 33], [1, 16], heads=2, dim=dim, act=act, cache=cache, tree=False, seed=42).check()


@pytest.mark.parametrize("act,cache", KINDS)
@pytest.mark.parametrize("dim", [40, 64, 80, 128])
def test_few_rows_over_a_long_cache(act, cache, dim):
    """Eight wavefronts, many pieces: of one request, and of requests of which most hold little."""
    print("long", act, cache, dim, flush=True)
    s = few_rows(True, [30011], [3], heads=6, dim=dim, act=act, cache=cache, seed=43)
    first = s.check().copy()
    assert np.array_equal(s.run(), first)
    few_rows(True, [9, 20000, 0, 700], [2, 8, 5, 8], heads=4, dim=dim, act=act, cache=cache, seed=44).check()


@pytest.mark.parametrize("act,cache", KINDS)
@pytest.mark.parametrize("new", [1, 16])
def test_one_sequence_of_twenty_heads(act, cache, new):
    print("one sequence", act, cache, new, flush=True)
    s = Step([7001], [new], heads=20, kv_heads=20, dim=128, act=act, cache=cache, seed=45)
    assert wavefronts(s) == 8
    s.check()


@pytest.mark.parametrize("act,cache", KINDS)
@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("form", ["four", "eight", "shared"])
@pytest.mark.parametrize("held", [20, 3000])
def test_infinite_values_arrive_where_they_are_seen_and_nowhere_else(act, cache, dim, form, held):
    print("infinite value", act, cache, dim, form, held, flush=True)
    if form == "shared":
        s = Step([held], [12], heads=4, kv_heads=2, dim=dim, act=act, cache=cache, seed=46)
    else:
        s = few_rows(form == "eight", [held], [8], heads=4, dim=dim, act=act, cache=cache, seed=46)
    want = s.check().copy()
    s.v[3, 5], s.v[3, 9] = float("inf"), -float("inf")  # token 3, two dimensions of the first key head
    got = s.run()
    sees = np.array([bool(int(m) >> 3 & 1) for m in s.mask.tolist()])
    assert sees.any() and not sees.all()
    at = np.array([a * dim + d for a in range(2) for d in (5, 9)])
    assert (got[np.ix_(sees, at[0::2])] == np.inf).all() and (got[np.ix_(sees, at[1::2])] == -np.inf).all()
    got[np.ix_(sees, at)] = want[np.ix_(sees, at)]
    assert np.array_equal(got, want)


def exact(s):
    """What oracle.attention gives for one request, in float64 on the GPU: many heads over long caches."""
    held, group, tokens = int(s.held[0]), s.heads // s.kv_heads, s.tokens
    side = {}
    for name in ("k", "v"):
        old = getattr(s, "cache_" + name)[s.table[0].long()].transpose(0, 1).reshape(s.kv_heads, -1, s.dim)[:, :held].double()
        new = getattr(s, name).to(s.cache_k.dtype).double().view(tokens, s.kv_heads, s.dim).transpose(0, 1)
        side[name] = torch.cat([old, new], 1)
    blind = (s.mask[:, None] >> torch.arange(tokens, device="cuda") & 1 == 0).repeat_interleave(group, 0)
    out, spread, steep = (torch.empty((tokens, s.heads, s.dim), dtype=torch.float64, device="cuda") for _ in range(3))
    for b in range(s.kv_heads):
        heads = slice(b * group, (b + 1) * group)
        q = s.q.double().view(tokens, s.heads, s.dim)[:, heads].reshape(-1, s.dim)
        k, v = side["k"][b], side["v"][b]
        score = q @ k.T.contiguous() * s.scale
        score[:, held:].masked_fill_(blind, -float("inf"))
        weight = torch.softmax(score, 1)
        out[:, heads], spread[:, heads] = ((weight @ x).view(tokens, group, s.dim) for x in (v, v.abs()))
        steep[:, heads] = ((q.abs() @ k.abs().T.contiguous()).amax(1) * abs(s.scale)).view(tokens, group, 1)
    return tuple(x.view(tokens, -1).cpu().numpy() for x in (out, spread, steep)) + (held + tokens,)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("tiles,less", [(1016, 0), (1024, 31), (1024, 0), (1032, 1), (1040, 0), (2104, 9)])
def test_eight_wavefronts_take_more_pages_than_lie_in_lds_at_once(kind, tiles, less):
    """256 rows of 32 key heads, pages of 8: eight workgroups a key head, each a run of 127, 128, 129, 130 or 263 tiles of four pages,
    of which 128 tiles' pages lie in LDS."""
    print("pages", kind, tiles, less, flush=True)
    s = Step([32 * (tiles - 2) - less], [64], heads=128, kv_heads=32, dim=8, act=kind, cache=kind, page=8, seed=47)
    got, expected = s.run(), exact(s)
    assert (np.abs(got - expected[0]) <= s.bound(expected)).all()


# ---- what a result may depend on ----
def alone(s, r, spare=0):
    """Request r of a step as a step of its own, with so many more entries in its table."""
    one, rows = copy.copy(s), slice(int(s.start[r]), int(s.start[r + 1]))
    one.table = torch.nn.functional.pad(s.table[r:r + 1], (0, spare), value=-1)
    one.held, one.start = s.held[r:r + 1].clone(), s.start[r:r + 2] - s.start[r]
    one.q, one.k, one.v, one.mask = s.q[rows], s.k[rows], s.v[rows], None if s.mask is None else s.mask[rows].contiguous()
    one.tokens = rows.stop - rows.start
    one.out, one.workspace = torch.full_like(s.out[rows], float("nan")), None
    return one


@pytest.mark.parametrize("act,cache", KINDS)
@pytest.mark.parametrize("new", [[9, 5, 2], [40, 64, 1]])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_request_gives_the_same_alone_in_a_batch_and_with_a_wider_table(act, cache, new, dim):
    """Within rounding: which tiles are added up together depends on all lengths and sizes of a step."""
    print("batch", act, cache, new, dim, flush=True)
    s = Step([3000, 70, 0], new, act=act, cache=cache, heads=4, kv_heads=2, dim=dim, seed=48)
    got, far = s.check().copy(), s.bound(s.expected())
    for r in range(3):
        rows = slice(int(s.start[r]), int(s.start[r + 1]))
        for spare in (0, 9000):
            assert (np.abs(alone(s, r, spare).check() - got[rows]) <= 2 * far[rows]).all()


def test_refused_steps_leave_the_output_alone():
    half = {"dtype": torch.float16, "device": "cuda"}
    pages = lambda *shape: torch.zeros(shape, **half)  # noqa: E731
    for changes in (
        {"scale": float("inf")}, {"scale": float("nan")}, {"max_new": 65}, {"max_new": 0}, {"heads": 3, "q": pages(4, 192), "out": pages(4, 192) * float("nan")},
        {"workspace": torch.zeros(16, dtype=torch.uint8, device="cuda")},
        {"q": pages(4, 8 * 64 + 4)[:, 4:4 + 256]},                       # not 16-byte aligned
        {"q": pages(4, 260)[:, :256]},                                   # rows 520 bytes apart
        {"cache_k": pages(5, 2, 24, 64), "cache_v": pages(5, 2, 24, 64)},  # pages of 24
        {"cache_k": pages(5, 2, 16, 68)[..., :64], "cache_v": pages(5, 2, 16, 68)[..., :64]},  # rows of the cache not 16-byte aligned
    ):
        s = Step([40], [4], dim=64, act="f16", cache="f16", seed=49)
        for name, value in changes.items():
            setattr(s, name, value)
        with pytest.raises(R.RsrError) as e:
            s.call()
        assert e.value.code == -1 and e.value.message
        torch.cuda.synchronize()
        assert np.isnan(plain(s.out)).all()
