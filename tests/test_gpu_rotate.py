"""rsr_head_rotate (include/rsr_decode.h) against its definition."""
import numpy as np
import pytest
import torch

import paper_2411_06360_amd as R
from oracle import decode as oracle
from tests.cache_util import DTYPES, ROUND, plain

pytestmark = pytest.mark.gpu


def rows(seed, tokens, width, dtype, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn((tokens, width), generator=g)).to(DTYPES[dtype]).cuda()


def frequencies(rotated, base=10000.0):
    return torch.tensor(base ** (-np.arange(rotated // 2) / max(1, rotated // 2)), dtype=torch.float64, device="cuda")


def close(got, x, position, frequency, dim, eps, weight, pairs, out):
    """Every value by the definition, in units of 2^-24 of |y_a| + |y_b|.  The sum of a head's squares is a tree of at most nine roundings, all of
    one sign, its mean and eps three more, of which a root passes on half; the reciprocal root, refined, is off by 1.5: 7.5 together; twice
    rounded, with the weight: 9.5.  (A head of 64 bits: less.)  Sine and cosine are off by 2 pi times the rounding of the turn (half a turn at most:
    1.6) and by two units in the last place of a value up to 1 (4): 5.6.  The two products and their sum are rounded once each: 18.1 in all.
    Then the rounding to the result's type, whose smallest numbers are 2^-24 apart (float16) or less."""
    want, size = oracle.rotate(plain(x), position.cpu().numpy(), None if frequency is None else frequency.cpu().numpy(), dim, eps, plain(weight), pairs)
    error, bound = np.abs(plain(got) - want), 18.1 * 2.0**-24 * size + np.abs(want) * ROUND[out] + 2.0**-25
    assert np.isfinite(plain(got)).all()
    assert (error <= bound).all(), f"off by {float((error / bound).max()):.3g} times the bound"


def check(tokens, heads, kv_heads, dim, rotated=None, norm=True, pairs=False, act="f32", out="f32", seed=0, far=5000, weights=True, stream=None):
    rotated = dim if rotated is None else rotated
    print("rotate", tokens, heads, kv_heads, dim, rotated, norm, pairs, act, out, flush=True)
    qkv = rows(seed, tokens, (heads + 2 * kv_heads) * dim, act)
    q, k = qkv[:, :heads * dim], qkv[:, heads * dim:(heads + kv_heads) * dim]
    g = torch.Generator().manual_seed(seed + 1)
    position = torch.randint(0, far + 1, (tokens,), generator=g, dtype=torch.int32).cuda()
    frequency = frequencies(rotated) if rotated else None
    w = [(1 + 0.2 * torch.randn(dim, generator=g)).cuda() if norm and weights else None for _ in range(2)]
    eps = 1e-6 if norm else None
    wide = torch.full((tokens, (heads + kv_heads) * dim + 16), float("nan"), dtype=DTYPES[out], device="cuda")
    q_out, k_out = wide[:, :heads * dim], wide[:, heads * dim + 8:(heads + kv_heads) * dim + 8]
    how = R.make_rotary(frequency, dim, eps=eps, q_weight=w[0], k_weight=w[1], pairs=pairs)
    R.rsr_head_rotate(how, q if heads else None, k if kv_heads else None, position, q_out if heads else None, k_out if kv_heads else None,
                      torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    if heads:
        close(q_out, q, position, frequency, dim, eps, w[0], pairs, out)
    if kv_heads:
        close(k_out, k, position, frequency, dim, eps, w[1], pairs, out)
    assert wide[:, heads * dim:heads * dim + 8].isnan().all() and wide[:, (heads + kv_heads) * dim + 8:].isnan().all(), "what lies between rows was written"


@pytest.mark.parametrize("dim", [8, 16, 24, 40, 64, 72, 80, 96, 112, 120, 128, 136, 160, 192, 248, 256])
@pytest.mark.parametrize("norm,pairs", [(True, False), (False, True), (True, True)])
def test_heads_of_every_width(dim, norm, pairs):
    check(5, 6, 2, dim, norm=norm, pairs=pairs, seed=dim)


@pytest.mark.parametrize("act", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("norm", [False, True])
def test_every_pair_of_types(act, out, norm):
    check(19, 5, 5, 80, rotated=48, norm=norm, act=act, out=out, seed=3)


@pytest.mark.parametrize("tokens,heads,kv_heads", [(1, 1, 0), (1, 0, 1), (1, 20, 20), (1, 64, 8), (2, 7, 3), (3, 1, 1), (63, 4, 1), (64, 20, 5), (65, 33, 1),
                                                   (511, 5, 5), (4097, 3, 1), (1000, 20, 5), (2, 300, 17)])
def test_tokens_and_heads(tokens, heads, kv_heads):
    check(tokens, heads, kv_heads, 128, act="f32", out="bf16", seed=tokens)


@pytest.mark.parametrize("rotated", [0, 8, 16, 24, 40, 56, 64, 80])
@pytest.mark.parametrize("pairs", [False, True])
def test_part_of_a_head(rotated, pairs):
    check(7, 4, 2, 80, rotated=rotated, pairs=pairs, norm=bool(rotated % 16), seed=rotated)


def test_without_weights():
    check(9, 4, 2, 64, weights=False)


@pytest.mark.parametrize("far", [1, 1 << 17, 1 << 20, 1 << 26, (1 << 31) - 2])
def test_far_positions(far):
    check(257, 2, 1, 64, far=far, seed=far % 1000)


def test_positions_before_the_first_and_frequencies_of_any_size():
    x = rows(5, 6, 64, "f32")
    position = torch.tensor([-1, -70000, -(1 << 31), (1 << 31) - 1, 0, 12345], dtype=torch.int32, device="cuda")
    for base in (1e-3, 1.0, 1e6):
        frequency = 3.7 * frequencies(64, base)
        out = torch.empty_like(x)
        R.rsr_head_rotate(R.make_rotary(frequency, 64), x, None, position, out, None, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        if base < 1:
            position, x = position[4:].contiguous(), x[4:]  # (angles beyond 2^40 have no bits left in the reference either)
            out = out[4:]
        close(out, x, position, frequency, 64, None, None, False, "f32")
        position, x = torch.tensor([-1, -70000, -(1 << 31), (1 << 31) - 1, 0, 12345], dtype=torch.int32, device="cuda"), rows(5, 6, 64, "f32")


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("norm", [False, True])
def test_in_place(act, norm):
    for tokens, dim, rotated, pairs in ((1, 128, 128, False), (333, 80, 40, True), (5000, 64, 64, False), (40, 256, 256, True)):
        print("in place", act, norm, tokens, dim, flush=True)
        qkv = rows(tokens, tokens, 8 * dim, act)
        old, position = qkv.clone(), torch.arange(tokens, dtype=torch.int32, device="cuda") + 100
        how = R.make_rotary(frequencies(rotated), dim, eps=1e-5 if norm else None, pairs=pairs)
        q, k = qkv[:, :4 * dim], qkv[:, 4 * dim:6 * dim]
        R.rsr_head_rotate(how, q, k, position, q, k, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        close(q, old[:, :4 * dim], position, frequencies(rotated), dim, how.eps if norm else None, None, pairs, act)
        close(k, old[:, 4 * dim:6 * dim], position, frequencies(rotated), dim, how.eps if norm else None, None, pairs, act)
        assert torch.equal(qkv[:, 6 * dim:], old[:, 6 * dim:])


def test_heads_of_every_size_are_normed():
    """Squares beyond the range of float, and far below it."""
    x = rows(2, 5, 64, "f32")
    x *= torch.tensor([1e-30, 1e-15, 1.0, 1e15, 1e37], device="cuda")[:, None]
    for eps in (0.0, 1e-6):
        out = torch.empty_like(x)
        position = torch.arange(5, dtype=torch.int32, device="cuda")
        R.rsr_head_rotate(R.make_rotary(frequencies(64), 64, eps=eps), x, None, position, out, None, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        close(out, x, position, frequencies(64), 64, np.float32(eps).astype(np.float64), None, False, "f32")


def test_what_is_not_finite_stays_in_its_head():
    x, position = rows(3, 4, 5 * 64, "f32"), torch.arange(4, dtype=torch.int32, device="cuda")
    bad = x.clone()
    bad[0, 70], bad[1, 3], bad[2, 300], bad[3, 128] = float("nan"), float("inf"), float("-inf"), float("nan")
    for eps in (None, 1e-6):
        got, want = torch.empty_like(x), torch.empty_like(x)
        how = R.make_rotary(frequencies(64), 64, eps=eps)
        for source, to in ((bad, got), (x, want)):
            R.rsr_head_rotate(how, source, None, position, to, None, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for row, at in ((0, 70), (1, 3), (2, 300), (3, 128)):
            head = at // 64
            assert not got[row, at].isfinite() and not got[row, head * 64 + (at % 64 + 32) % 64].isfinite()
            touched = range(64) if eps is not None else (at % 64, (at % 64 + 32) % 64)
            same = [i for i in range(320) if i // 64 != head or i % 64 not in touched]
            assert torch.equal(got[row, same], want[row, same])


def test_the_same_bits_alone_and_in_a_batch():
    x, position = rows(4, 3000, 12 * 128, "f32"), torch.arange(3000, dtype=torch.int32, device="cuda")
    how, stream = R.make_rotary(frequencies(128), 128, eps=1e-6), torch.cuda.current_stream().cuda_stream
    whole, alone = torch.empty_like(x), torch.empty_like(x[:1])
    R.rsr_head_rotate(how, x, None, position, whole, None, stream)
    for t in (0, 1, 1499, 2999):
        R.rsr_head_rotate(how, x[t:t + 1], None, position[t:t + 1], alone, None, stream)
        torch.cuda.synchronize()
        assert torch.equal(alone[0], whole[t])
