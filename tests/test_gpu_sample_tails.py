"""rsr_sample where a row's weight lies in one score and what is left of it in very many of very little: by definition the sums of those."""
from decimal import ROUND_CEILING, ROUND_FLOOR, Decimal, getcontext

import numpy as np
import pytest
import torch

import paper_2411_06360_amd as R
from oracle import decode as oracle
from tests.cache_util import DTYPES

pytestmark = pytest.mark.gpu
getcontext().prec = 60


def call(x, u, **how):
    rows, columns = x.shape
    token, kept = (torch.full((rows,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    probability = torch.full((rows,), -7.0, device="cuda")
    space = torch.zeros(R.rsr_sample_workspace(rows, columns), dtype=torch.uint8, device="cuda")
    R.rsr_sample(x, u.cuda(), token, space, probability=probability, kept=kept, stream=torch.cuda.current_stream().cuda_stream, **{name: v.cuda() for name, v in how.items()})
    torch.cuda.synchronize()
    return token.tolist(), kept.tolist(), probability.tolist()


def whole(x, rounding):
    return int(x.to_integral_value(rounding))


@pytest.mark.parametrize("rows", [2, 9, 131])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("columns,low", [(3000, -17.0), (131072, -20.75), (131072, -24.0), (262144, -25.5), (262144, -27.75), (1 << 20, -26.5), (1 << 22, -28.0), (1 << 22, -28.75)])
def test_one_score_above_a_long_tail(columns, low, dtype, rows):
    """Places in the tail, by its numbers: behind j tokens of weight w the sum is 1 + j w.  Sums are off by less than 2^-39 of theirs, and so a
    place in the tail by 2^-39 (1 + n w) / w: a sixteenth of a token with n = 131071 of -24, six tokens with 2^22 of -28.75."""
    print("tail", columns, low, dtype, rows, flush=True)
    top = columns // 3
    x = torch.full((rows, columns), low, dtype=DTYPES[dtype], device="cuda")
    x[:, top] = 0
    n, w = columns - 1, Decimal(low).exp()
    total = 1 + n * w
    off = Decimal(2.0**-39) * total / w
    u = torch.tensor(float(1 / total) + np.linspace(0.04, 0.96, rows) * float(n * w / total), dtype=torch.float64).float()

    def drawn(number, mass):
        """The first and the last token that it may be: the tail's j-th ones, 0 for the highest.  (Numbers are taken into 0 .. 1 - 2^-24.)"""
        at = (Decimal(min(number, 1 - 2.0**-24)) * mass - 1) / w
        return [0 if at + d < 0 else min(1 + whole(at + d, ROUND_FLOOR), n) for d in (-off, off)]

    place = lambda column: 0 if column == top else column + 1 if column < top else column  # noqa: E731
    token, kept, probability = call(x, u)
    for r, number in enumerate(u.tolist()):
        first, last = drawn(number, total)
        assert kept[r] == columns and first <= place(token[r]) <= last, (r, place(token[r]), first, last)
        assert probability[r] == pytest.approx(float((w if token[r] != top else 1) / total), rel=2.0**-23)
    # top_p in the tail, and the last one that it keeps
    number = 1 - 2.0**-24
    token, kept, _ = call(x, torch.full((rows,), number), top_p=u)
    for r, p in enumerate(u.tolist()):
        first, last = [1 + max(0, whole((Decimal(p) * total - 1) / w + d, ROUND_CEILING)) for d in (-off, off)]
        assert first <= kept[r] <= last, (r, kept[r], first, last)
        first, last = drawn(number, 1 + (kept[r] - 1) * w)
        assert first <= place(token[r]) <= last, (r, place(token[r]), first, last)


@pytest.mark.parametrize("rows", [3, 130])
@pytest.mark.parametrize("low", [-12.0, -18.0, -22.0])
def test_one_score_above_different_ones(low, rows):
    """The same with tails of which no two are alike."""
    print("different", low, rows, flush=True)
    columns = 131072
    x = 0.7 * torch.randn(columns, generator=torch.Generator().manual_seed(4)) + low
    x[99] = 0.0
    weight = torch.sort(x.double(), descending=True)[0].exp()
    part = torch.tensor([0.1, 0.5, 0.9])[torch.arange(rows) % 3].double()
    u = ((1 + part * weight[1:].sum()) / weight.sum()).float()
    got = call(x.cuda().expand(rows, columns).contiguous(), u, top_p=1 - (1 - u) / 2)
    want = [oracle.sample(x.double().numpy(), top_p=float(1 - (1 - u[r]) / 2), uniform=float(u[r])) for r in range(3)]
    assert list(zip(got[0], got[1])) == [(want[r % 3][0], want[r % 3][2]) for r in range(rows)]
    assert got[2] == pytest.approx([want[r % 3][1] for r in range(rows)], rel=2.0**-23)


@pytest.mark.parametrize("rows", [4, 132])
@pytest.mark.parametrize("kind", ["next to zero", "equal ones", "some next to zero", "both sides"])
def test_temperatures_that_make_steps_wide(kind, rows):
    """Less than what scores can be told apart by: the scores next to each other in a step have weights of every size, or all the same, or none."""
    print("wide steps", kind, rows, flush=True)
    columns, g = 131072, torch.Generator().manual_seed(7)
    x, temperature = torch.randn(columns, generator=g), 1e-10
    if kind == "next to zero":
        x, temperature = x * 1e-24, 5e-25
    elif kind == "equal ones":
        x = (2 * x).round()
    elif kind == "some next to zero":
        x = -1 - x.abs()
        x[5::300] = -1e-9 * torch.rand(len(x[5::300]), generator=g)
    else:
        x = torch.where(torch.rand(columns, generator=g) < 0.5, x * 1e-10, x - 9)
    u, p = torch.tensor([0.0, 0.3, 0.9, 1 - 2.0**-24]), torch.tensor([1.0, 0.999, 0.5, 1.0])
    few = torch.arange(rows) % 4
    got = call(x.cuda().expand(rows, columns).contiguous(), u[few], top_p=p[few], temperature=torch.full((rows,), temperature))
    want = [oracle.sample(x.double().numpy(), float(np.float32(temperature)), top_p=float(p[r]), uniform=float(u[r])) for r in range(4)]
    assert list(zip(got[0], got[1])) == [(want[r % 4][0], want[r % 4][2]) for r in range(rows)]
    assert got[2] == pytest.approx([want[r % 4][1] for r in range(rows)], rel=2.0**-23)
