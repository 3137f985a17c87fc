"""rsr_sample where the place of top_p and that of min_p lie next to each other, in rows whose counts tell less than they do for
others: scores near the same end of every step in which they are counted, so that what steps are off by adds up."""
import math

import numpy as np
import pytest
import torch

import paper_2411_06360_amd as R
from oracle import decode as oracle

pytestmark = pytest.mark.gpu

STEP = 33.2 / 8189  # a row from 0 down to -33.2 is counted in 8189 steps of this width


def row(columns, pieces):
    """Scores of `pieces` ((how many, how many steps below the highest) each), the others -33.2; the highest, 0, is in each of the
    16 parts of the row that are looked at first, and so is the first step's begin."""
    x = np.full(columns, -33.2, np.float32)
    looked = np.arange(1024) * (columns // 4) // 1024 * 4
    x[looked[::64]] = 0.0
    free = np.setdiff1d(np.arange(columns), np.append(looked[::64], looked[5]))
    values = np.repeat([-at * STEP for _, at in pieces], [n for n, _ in pieces])
    x[np.random.default_rng(1).choice(free, len(values), replace=False)] = values
    return x


def sums(x, kept=None):
    """Sums of weights in order, and those up to a score."""
    x = np.sort(x.astype(np.float64))[::-1][:kept]
    return np.exp((x - x[0]).astype(np.longdouble)).cumsum()


def check(x, rows, **how):
    columns, number = len(x), [0.0, 0.999, 0.25, 0.5, 0.75, 1 - 2.0**-24, 0.9, 0.1]
    print("borders", columns, rows, how, flush=True)
    how = {name: torch.full((rows,), v, dtype=torch.int32 if name == "top_k" else torch.float32) for name, v in how.items()}
    u = torch.tensor([number[r % 8] for r in range(rows)])
    token, kept = (torch.full((rows,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    space = torch.zeros(R.rsr_sample_workspace(rows, columns), dtype=torch.uint8, device="cuda")
    R.rsr_sample(torch.from_numpy(x).cuda().expand(rows, columns).contiguous(), u.cuda(), token, space, kept=kept, stream=torch.cuda.current_stream().cuda_stream,
                 **{name: v.cuda() for name, v in how.items()})
    torch.cuda.synchronize()
    want = [oracle.sample(x, uniform=float(u[r]), **{name: v[r].item() for name, v in how.items()})[::2] for r in range(min(rows, 8))]
    assert list(zip(token.tolist(), kept.tolist())) == [want[r % 8] for r in range(rows)]
    return want[0][1]


@pytest.mark.parametrize("rows", [1, 8, 130])
@pytest.mark.parametrize("columns,each,before", [(131072, 6, 1), (131072, 6, 10), (131072, 6, 20), (1 << 20, 64, 1), (1 << 20, 64, 10), (1 << 20, 64, 20), (1 << 20, 64, 200)])
def test_top_p_ends_before_min_p(columns, each, before, rows):
    """The first half of the weight is in scores just below the begin of their steps, the other half in scores just above the end of theirs,
    the same weight in each step: by counts top_p's place comes behind min_p's, by their weights `before` tokens before it.  (Of the longer
    row thousands of equal scores lie around the places.)"""
    weight = lambda s: round(each * math.exp(s * STEP))  # noqa: E731
    x = row(columns, [(weight(s), s + 0.06) for s in range(1, 500)] + [(1, 501.5)] + [(weight(s), s + 0.94) for s in range(503, 1004)])
    min_p = float(np.float32(math.exp(-501 * STEP)))
    total = sums(x)
    near = int((total[1:] - total[:-1] >= min_p).sum()) + 1
    top_p = float(np.float32((total[near - before - 1] + total[near - before - 2]) / 2 / total[-1]))
    assert check(x, rows, top_p=top_p, min_p=min_p) == near - before


@pytest.mark.parametrize("rows", [1, 8, 130])
@pytest.mark.parametrize("top_k", [600, 900, 1000])
def test_min_p_ends_before_top_p(top_k, rows):
    """The other way round, with some empty steps between: by counts top_p's place is before min_p's, by their weights one token behind."""
    x = row(131072, [(2, s + 0.94) for s in range(1, 150)] + [(2, s + 0.06) for s in range(156, 480)])
    min_p = float(np.float32(math.exp(-152.5 * STEP)))
    total = sums(x, top_k)
    near = int((total[1:] - total[:-1] >= min_p).sum()) + 1
    for part in (0.02, 0.1, 0.5):
        top_p = float(np.float32((total[near - 1] + part * (total[near] - total[near - 1])) / total[-1]))
        assert check(x, rows, top_k=top_k, top_p=top_p, min_p=min_p) == near
