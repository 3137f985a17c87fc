"""The operators on both sides of the attention without a GPU: their definitions on cases worked out by hand, and what the entry points
answer before anything is launched (include/rsr_decode.h)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2411_06360_amd as R
from oracle import decode as oracle

INVALID = -1
AT = 1 << 20  # an aligned address that nobody reads: all of these calls end before a launch


def rotary(**changes):
    c = R.RsrRotary(AT, AT, AT, 1e-6, 1, 64, 64, 0, 0)
    for name, value in changes.items():
        setattr(c, name, value)
    return c


def rotate(how=None, **changes):
    a = dict(q=2 * AT, q_stride=512, heads=8, k=3 * AT, k_stride=256, kv_heads=4, dtype=R.RSR_F32, position=AT, tokens=5, q_out=4 * AT, q_out_stride=512,
             k_out=5 * AT, k_out_stride=256, out_dtype=R.RSR_BF16)
    a.update(changes)
    how = rotary() if how is None else how
    return R.load().rsr_head_rotate(ctypes.addressof(how) if how else None, *a.values(), None)


@pytest.mark.parametrize("changes", [
    dict(head_dim=0), dict(head_dim=4), dict(head_dim=60), dict(head_dim=264), dict(rotated=-8), dict(rotated=72), dict(rotated=4), dict(rotated=60), dict(norm=2),
    dict(norm=-1), dict(pairs=2), dict(pairs=-1), dict(eps=-1e-6), dict(eps=math.inf), dict(eps=math.nan), dict(frequency=0)])
def test_rotations_that_are_refused(changes):
    assert rotate(rotary(**changes)) == INVALID and R.rsr_last_error()


@pytest.mark.parametrize("changes", [
    dict(q=0), dict(k=0), dict(q_out=0), dict(k_out=0), dict(position=0), dict(q=2 * AT + 8), dict(k_out=5 * AT + 4), dict(q_stride=511), dict(q_stride=514),
    dict(k_stride=252), dict(q_out_stride=500), dict(k_out_stride=260), dict(dtype=3), dict(dtype=-1), dict(out_dtype=3), dict(heads=-1), dict(heads=65536),
    dict(kv_heads=-1), dict(heads=0, kv_heads=0), dict(tokens=-1), dict(tokens=1 << 40), dict(q_out=2 * AT), dict(q_out=2 * AT, out_dtype=R.RSR_F32, q_out_stride=516),
    dict(k_out=3 * AT), dict(q_out=3 * AT, out_dtype=R.RSR_F32), dict(k_out=2 * AT, out_dtype=R.RSR_F32), dict(q_out=5 * AT)])
def test_rows_of_heads_that_are_refused(changes):
    assert rotate(**changes) == INVALID and R.rsr_last_error()


def test_a_rotation_without_its_descriptor_is_refused():
    assert R.load().rsr_head_rotate(None, AT, 512, 8, AT, 256, 4, 0, AT, 5, AT, 512, AT, 256, 0, None) == INVALID


def test_nothing_to_do_is_done_without_a_launch():
    assert rotate(tokens=0, q=0, k=0, q_out=0, k_out=0, position=0) == 0
    lib = R.load()
    assert lib.rsr_sample(0, 0, 5, 5, R.RSR_F32, None, None, None, None, 0, 0, None, None, 0, 0, None) == 0


def sample(**changes):
    a = dict(logits=AT, rows=3, columns=100, stride=100, dtype=R.RSR_F32, temperature=None, top_k=None, top_p=None, min_p=None, uniform=2 * AT, token=3 * AT,
             probability=None, kept=None, workspace=4 * AT, bytes=1 << 40)
    a.update(changes)
    return R.load().rsr_sample(*a.values(), None)


@pytest.mark.parametrize("changes", [
    dict(logits=0), dict(logits=AT + 2), dict(logits=AT + 1, dtype=R.RSR_BF16), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(columns=0), dict(columns=(1 << 22) + 1),
    dict(stride=99), dict(dtype=3), dict(uniform=0), dict(token=0), dict(workspace=0), dict(workspace=4 * AT + 128), dict(bytes=1)])
def test_samples_that_are_refused(changes):
    assert sample(**changes) == INVALID and R.rsr_last_error()


@pytest.mark.parametrize("output", ["token", "probability", "kept"])
@pytest.mark.parametrize("other", ["logits", "temperature", "top_k", "top_p", "min_p", "uniform", "workspace", "token", "probability", "kept"])
def test_samples_into_what_is_read_are_refused(output, other):
    if output != other:
        assert sample(**{output: 8 * AT, other: 8 * AT}) == INVALID and "output" in R.rsr_last_error()


def test_a_workspace_for_more_rows_or_columns_is_not_smaller():
    sizes = {(r, c): R.rsr_sample_workspace(r, c) for r in (0, 1, 2, 3, 7, 64, 255, 256, 257, 5000, 1 << 24) for c in (1, 64, 1000, 4096, 50000, 1 << 17, 1 << 22)}
    for (r, c), n in sizes.items():
        assert 0 < n <= 1 << 26
        assert all(n <= m for (r1, c1), m in sizes.items() if r <= r1 and c <= c1), (r, c)
    for bad in ((-1, 5), (5, 0), ((1 << 24) + 1, 5), (5, (1 << 22) + 1)):
        with pytest.raises(R.RsrError):
            R.rsr_sample_workspace(*bad)


def keep(**changes):
    a = dict(drafted=AT, chosen=2 * AT, parent=3 * AT, start=4 * AT, requests=2, tokens=6, rows=5 * AT, found=6 * AT, add=7 * AT, first=8 * AT)
    a.update(changes)
    return R.load().rsr_tree_keep(*a.values(), None)


@pytest.mark.parametrize("changes", [
    dict(drafted=0), dict(chosen=0), dict(start=0), dict(rows=0), dict(found=0), dict(add=0), dict(first=0), dict(requests=-1), dict(requests=65536),
    dict(tokens=-1), dict(rows=AT), dict(found=2 * AT), dict(add=4 * AT), dict(first=4 * AT), dict(rows=6 * AT), dict(first=7 * AT), dict(rows=3 * AT)])
def test_paths_that_are_refused(changes):
    assert keep(**changes) == INVALID and R.rsr_last_error()


def test_what_the_binding_refuses():
    x, f = torch.zeros((4, 64)), torch.zeros(8, dtype=torch.float64)
    for bad in (dict(frequency=f.float()), dict(frequency=torch.zeros(16, dtype=torch.float64)[::2]), dict(eps=1e-6, q_weight=torch.zeros(8)),
                dict(eps=1e-6, k_weight=torch.zeros(16, dtype=torch.float64)), dict(q_weight=torch.zeros(16))):
        with pytest.raises(ValueError):
            R.make_rotary(**{"frequency": f, "head_dim": 16, **bad})
    how, position = R.make_rotary(f, 16), torch.zeros(4, dtype=torch.int32)
    for q, k, q_out, k_out, at in ((x, x, x, None, position), (None, x, x, x, position), (x[:3], x, x, x, position), (x, x, x, x[:, :48], position),
                                   (x[:, :24], x, x[:, :24], x, position), (x, x.half(), x, x, position), (x, x, x, x.half(), position), (x, x, x, x, position.long()),
                                   (x[:, ::2], x, x[:, ::2], x, position)):
        with pytest.raises(ValueError):
            R.rsr_head_rotate(how, q, k, at, q_out, k_out)
    with pytest.raises(TypeError):
        R.rsr_head_rotate(how, x.double(), None, position, x.double(), None)
    reals, ints, space = torch.zeros(4), torch.zeros(4, dtype=torch.int32), torch.zeros(256, dtype=torch.uint8)
    for bad in (dict(uniform=reals[:3]), dict(uniform=reals.double()), dict(token=ints.long()), dict(token=ints[:3]), dict(temperature=reals[:2]), dict(top_k=reals),
                dict(top_p=ints), dict(min_p=reals.half()), dict(probability=reals.double()), dict(kept=reals), dict(logits=x[:, ::2]), dict(logits=x[0])):
        with pytest.raises(ValueError):
            R.rsr_sample(**{"logits": x, "uniform": reals, "token": ints, "workspace": space, **bad})
    with pytest.raises(TypeError):
        R.rsr_sample(x.double(), reals, ints, space)
    for at in range(8):
        call = [ints, ints.clone(), ints.clone(), ints[:3], ints.clone(), ints.clone(), ints.clone(), ints.clone()]
        call[at] = call[at].long()
        with pytest.raises(ValueError):
            R.rsr_tree_keep(*call)
    for at, n in ((1, 3), (2, 3), (4, 3), (5, 3), (6, 1), (7, 2)):
        call = [ints, ints.clone(), ints.clone(), ints[:3], ints.clone(), ints.clone(), ints.clone(), ints.clone()]
        call[at] = call[at][:n]
        with pytest.raises(ValueError):
            R.rsr_tree_keep(*call)


# ---- the definitions ----
def test_rotation_by_hand():
    x, quarter = np.array([[1.0, 2, 3, 4, 5, 6, 7, 8]]), math.pi / 2
    out, _ = oracle.rotate(x, [1], [quarter, 0, 2 * quarter, 0], 8)  # pairs (0, 4), (1, 5), (2, 6), (3, 7)
    assert np.allclose(out, [[-5, 2, -3, 4, 1, 6, -7, 8]], atol=1e-15)
    out, size = oracle.rotate(x, [-1], [quarter, 0, 2 * quarter, 0], 8, pairs=True)  # (0, 1), (2, 3), ..
    assert np.allclose(out, [[2, -1, 3, 4, -5, -6, 7, 8]], atol=1e-15) and size[0, 0] == 3 and size[0, 5] == 11
    out, _ = oracle.rotate(np.array([[3.0, 4, 0, 0, 0, 0, 0, 0]]), [7], None, 8, eps=0.0, weight=[1, 2, 1, 1, 1, 1, 1, 1])
    assert np.allclose(out, np.array([[3.0, 8, 0, 0, 0, 0, 0, 0]]) / math.sqrt(25 / 8), rtol=1e-15)


def test_sampling_by_hand():
    x = np.log([1.0, 4.0, 2.0, 1.0])  # in order: tokens 1, 2, 0, 3 with 1/2, 1/4, 1/8, 1/8
    take = lambda u, **how: oracle.sample(x, uniform=u, **how)  # noqa: E731
    assert [take(u)[0] for u in (0, 0.49, 0.51, 0.74, 0.76, 0.86, 0.88, 1.0, -3.0, math.nan)] == [1, 1, 2, 2, 0, 0, 3, 3, 1, 1]
    assert take(0.9, top_k=2) == (2, pytest.approx(1 / 3), 2) and take(0.9, top_k=9)[2] == take(0.9, top_k=-1)[2] == 4
    assert take(0.9, top_p=0.6) == (2, pytest.approx(1 / 3), 2) and take(0.9, top_p=0.8)[2] == 3 and take(0.9, top_p=0.0)[2] == take(0.9, top_p=-1.0)[2] == 1
    assert take(0.9, top_k=2, top_p=0.6)[2] == 1  # (two thirds of what the first two have)
    assert take(0.9, min_p=0.3)[2] == 2 and take(0.9, min_p=0.2)[2] == 4 and take(0.9, min_p=7.0)[2] == 1
    assert take(0.9, temperature=0.0) == take(0.9, temperature=math.nan) == (1, 1.0, 1) and take(0.9, temperature=math.inf) == (3, 0.25, 4)
    assert take(0.0, temperature=0.5) == (1, pytest.approx(16 / 22), 4)
    assert oracle.sample([-math.inf, 5.0, -math.inf], uniform=0.9) == (1, 1.0, 1) and oracle.sample([-math.inf] * 2) == (-1, 0.0, 0)
    assert oracle.sample([math.inf, 5.0, math.inf], uniform=0.9) == (2, 0.5, 3) and oracle.sample([math.nan, 5.0])[0] == -1
    assert oracle.sample([3.0, 3.0, 3.0], uniform=0.5, top_k=2)[0] == 1


def test_paths_by_hand():
    #  10 - 11 - 13      the token chosen behind 10 is 11 (the first of two), behind 11 nothing that was guessed
    #     \ 12, 11       ; the second request's guess was wrong, the third has no tokens
    drafted, parent, start = [10, 11, 12, 13, 11, 20, 21], [-1, 0, 0, 1, 0, -1, 0], [0, 5, 7, 7]
    assert oracle.keep(drafted, [11, 14, 0, 0, 0, 22, 0], parent, start, 7) == ([0, 1, 5, -1, -1, -1, -1], [11, 14, 22, -1, -1, -1, -1], [2, 1, 0], [0, 2, 3, 3])
    assert oracle.keep(drafted, [11, 13, 0, 5, 0, 21, 9], parent, start, 7) == ([0, 1, 3, 5, 6, -1, -1], [11, 13, 5, 21, 9, -1, -1], [3, 2, 0], [0, 3, 5, 5])
    assert oracle.keep([1, 2, 3], [2, 3, -1], None, [0, 3], 3) == ([0, 1, 2], [2, 3, -1], [3], [0, 3])
    assert oracle.keep([1, -1], [-1, 5], None, [0, 2], 2) == ([0, -1], [-1, -1], [1], [0, 1])
