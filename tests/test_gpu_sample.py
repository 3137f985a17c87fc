"""rsr_sample (include/rsr_decode.h) against its definition: tokens and counts have to be equal."""
import math

import numpy as np
import pytest
import torch

import paper_2411_06360_amd as R
from oracle import decode as oracle
from tests.cache_util import DTYPES

pytestmark = pytest.mark.gpu


def reals(x):
    return None if x is None else torch.tensor(x, dtype=torch.float32, device="cuda")


class Call:
    def __init__(self, logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None):
        rows, columns = logits.shape
        self.logits = logits
        self.given = dict(temperature=reals(temperature), top_k=None if top_k is None else torch.tensor(top_k, dtype=torch.int32, device="cuda"), top_p=reals(top_p),
                          min_p=reals(min_p), uniform=reals(uniform))
        self.token, self.kept = (torch.full((rows,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
        self.probability = torch.full((rows,), -7.0, device="cuda")
        self.workspace = torch.zeros(R.rsr_sample_workspace(rows, columns), dtype=torch.uint8, device="cuda")

    def call(self):
        given = dict(self.given)
        R.rsr_sample(self.logits, given.pop("uniform"), self.token, self.workspace, probability=self.probability, kept=self.kept,
                     stream=torch.cuda.current_stream().cuda_stream, **given)

    def results(self):
        torch.cuda.synchronize()
        return self.token.tolist(), self.kept.tolist(), self.probability.tolist()

    def expected(self):
        without = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
        given = {name: [without[name]] * len(self.token) if x is None else x.tolist() for name, x in self.given.items()}
        rows = self.logits.double().cpu().numpy()
        return [oracle.sample(rows[r], **{name: x[r] for name, x in given.items()}) for r in range(len(rows))]

    def check(self):
        self.call()
        token, kept, probability = self.results()
        for r, (t, p, n) in enumerate(self.expected()):
            assert (token[r], kept[r]) == (t, n), f"row {r}: token {token[r]} of {kept[r]}, not {t} of {n}"
            # one rounding to float, and weights off by 2^-39 of their size
            assert probability[r] == pytest.approx(p, rel=2.0**-23, abs=1e-38, nan_ok=True), r
        return self


def scores(seed, rows, columns, dtype="f32", spread=2.0, peak=8.0, few=20):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn((rows, columns), generator=g)
    if peak:
        few = max(1, min(few, columns // 3))
        x.scatter_add_(1, torch.randint(0, columns, (rows, few), generator=g), peak * torch.rand((rows, few), generator=g))
    return x.to(DTYPES[dtype]).cuda()


def numbers(seed, rows):
    return torch.rand(rows, generator=torch.Generator().manual_seed(seed)).tolist()


EVERY = dict(temperature=[0.8, 1.0, 1.0, 1.0, 0.7, 1.0, 0.0, 1.3], top_k=[50, 0, 0, 0, 40, 0, 7, 3], top_p=[1.0, 0.9, 1.0, 0.3, 0.95, 1.0, 0.5, 0.8],
             min_p=[0.0, 0.0, 0.1, 0.0, 0.02, 0.0, 0.1, 0.3])


@pytest.mark.parametrize("columns", [1, 2, 3, 4, 5, 7, 8, 63, 64, 65, 127, 255, 257, 512, 1000, 1023, 1025, 2047, 2048, 2049, 4095, 4097, 8192, 16385, 32000, 50021, 65537,
                                     131072, 262144])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_columns(columns, dtype):
    print("columns", columns, dtype, flush=True)
    Call(scores(columns, 8, columns, dtype), numbers(columns, 8), **EVERY).check()


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 255, 256, 257, 300, 600])
@pytest.mark.parametrize("columns", [300, 5003])
def test_rows(rows, columns):
    print("rows", rows, columns, flush=True)
    Call(scores(rows, rows, columns), numbers(rows, rows), **{name: [x[r % 8] for r in range(rows)] for name, x in EVERY.items()}).check()


@pytest.mark.parametrize("name,values", [("temperature", [0.01, 0.3, 1.0, 3.0, 1000.0, -1.0, 1e-30, math.inf, math.nan, 1e-45]),
                                         ("top_k", [1, 2, 17, 900, 1023, 1024, 1025, 2047, 2048, 2049, 5000, 19999, 20000, 20001, -5, 0, 1 << 30]),
                                         ("top_p", [0.0, -1.0, 1e-9, 0.1, 0.5, 0.99, 0.9999, 1 - 2.0**-24, 1.0, 2.0, math.inf, math.nan, -math.inf]),
                                         ("min_p", [0.0, -1.0, 1e-30, 1e-6, 0.001, 0.01, 0.5, 1.0, 3.0, math.inf, math.nan])])
@pytest.mark.parametrize("peak", [0.0, 10.0])
def test_one_parameter_alone(name, values, peak):
    print(name, peak, flush=True)
    rows = 4 * len(values)
    Call(scores(len(values), rows, 20000, peak=peak), numbers(7, rows), **{name: [v for v in values for _ in range(4)]}).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("spread", [0.0, 0.001, 0.1, 1.0, 30.0])
def test_flat_and_steep_scores(dtype, spread):
    """From all equal to one that has everything; many tokens next to each other."""
    print("spread", dtype, spread, flush=True)
    rows = 24
    how = dict(temperature=[1.0, 1.5, 1.0, 1.0] * 6, top_k=[0, 0, 4000, 0] * 6, top_p=[0.98, 1.0, 0.9, 1.0] * 6, min_p=[0.0, 0.0, 0.0, 0.001] * 6)
    Call(scores(5, rows, 40001, dtype, spread=spread, peak=0.0), numbers(9, rows), **how).check()


@pytest.mark.parametrize("u", [0.0, 0.25, 0.5, 1 - 2.0**-24, 1.0, 5.0, -1.0, math.nan, math.inf])
def test_equal_scores_go_to_the_lowest_column(u):
    for columns in (4, 1000, 4096, 100000):
        x = torch.full((6, columns), -3.25, device="cuda")
        Call(x, [u] * 6, temperature=[1.0, 0.0, 1.0, 1.0, 1.0, 0.5], top_k=[0, 0, columns // 2, 0, 0, 1], top_p=[1.0, 1.0, 1.0, 0.5, 1.0, 1.0],
             min_p=[0.0, 0.0, 0.0, 0.0, 1.0, 0.0]).check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_few_different_scores(dtype):
    """Runs of thousands of equal scores, with borders within them."""
    g = torch.Generator().manual_seed(11)
    x = torch.randint(-3, 2, (16, 30000), generator=g).to(DTYPES[dtype]).cuda()
    Call(x, numbers(12, 16), temperature=[1.0, 0.5] * 8, top_k=[0, 8000, 0, 12345] * 4, top_p=[0.7, 0.9, 1.0, 0.37] * 4, min_p=[0.0, 0.0, 0.1, 0.0] * 4).check()
    Call(torch.where(x == 0, -0.0, x.float()).to(DTYPES[dtype]).contiguous(), numbers(13, 16), top_k=[9000] * 16).check()  # (zeros of both signs are equal)


@pytest.mark.parametrize("rows", [1, 12, 150])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mean", [10.0, -20.0, 0.0])
def test_rounded_scores(mean, dtype, rows):
    """Scores of bfloat16, some thousand of each (float32: the same numbers), far from zero and not; each place in the middle of equal ones."""
    print("rounded", mean, dtype, rows, flush=True)
    few = (torch.arange(rows) % 12).tolist()
    how = dict(temperature=[1.0, 0.7, 1.0, 1.0, 2.0, 1.0], top_k=[0, 0, 20000, 0, 9000, 3000], top_p=[0.9, 0.95, 1.0, 1.0, 0.9, 0.99], min_p=[0.0, 0.0, 0.0, 0.01, 0.001, 0.0])
    x = (scores(6, 12, 131072, peak=0.0) + mean).bfloat16().to(DTYPES[dtype])[few].contiguous()
    c = Call(x, [numbers(8, 12)[i] for i in few], **{name: [v[i % 6] for i in few] for name, v in how.items()})
    if rows <= 12:
        c.check()
        return
    c.call()
    token, kept, _ = c.results()
    want = Call(x[:12], numbers(8, 12), **{name: v * 2 for name, v in how.items()}).expected()
    assert list(zip(token, kept)) == [(want[i][0], want[i][2]) for i in few]


@pytest.mark.parametrize("rows", [1, 12, 130])
def test_thousands_next_to_each_other(rows):
    """More tokens than are sorted at once within a step, all different: a long row's scores from 1 to 1.012, and one far away."""
    print("next to each other", rows, flush=True)
    columns = 70000
    x = 1 + torch.randperm(columns, generator=torch.Generator().manual_seed(3)).float() * 2.0**-23
    x[777] = -40.0
    few = (torch.arange(rows) % 12).tolist()
    how = dict(top_k=[0, 0, 33333, 0], top_p=[0.9, 0.3, 1.0, 1.0], min_p=[0.0, 0.0, 0.0, 0.995])
    given = {name: [v[i % 4] for i in few] for name, v in how.items()}
    c = Call(x.cuda().expand(rows, columns).contiguous(), [numbers(4, 12)[i] for i in few], **given)
    c.call()
    token, kept, _ = c.results()
    want = Call(x.cuda().expand(12, columns).contiguous(), numbers(4, 12), **{name: v * 3 for name, v in how.items()}).expected()
    assert list(zip(token, kept)) == [(want[i][0], want[i][2]) for i in few]


@pytest.mark.parametrize("seed", range(32))
def test_parameters_together(seed):
    """Whatever comes together: narrow and wide scores around zero and not, peaks, masks, with every parameter."""
    rng = np.random.default_rng(seed)
    columns, rows = int(rng.choice([1025, 1500, 5000, 50021, 131072, 152064])), int(rng.choice([1, 3, 9]))
    dtype, mean, spread, peak = rng.choice(["f32", "f32", "f16", "bf16"]), rng.choice([0, 0, 5, -10, 20]), rng.choice([0.01, 0.3, 2, 4]), rng.choice([0, 4, 12])
    print("together", seed, columns, rows, dtype, mean, spread, peak, flush=True)
    x = (scores(seed, rows, columns, spread=float(spread), peak=float(peak), few=64) + float(mean)).to(DTYPES[dtype])
    if seed % 4 == 0:
        x[:, rng.random(columns) < 0.5] = -math.inf
    how = dict(temperature=[0.3, 0.7, 1.0, 1.5, 3.0], top_k=[0, 0, 20, 1000, 5000], top_p=[1.0, 0.5, 0.9, 0.99, 0.999], min_p=[0.0, 0.0, 0.001, 0.05, 0.2])
    Call(x, numbers(seed, rows), **{name: rng.choice(v, rows).tolist() for name, v in how.items()}).check()


def test_masked_scores():
    x = scores(21, 12, 5000)
    x[0:8, ::2] = -math.inf
    x[1, 1:] = -math.inf                      # one score is left, or
    x[2, :] = -math.inf                       # none
    x[3, 3:] = -math.inf
    x[4, 70], x[5, 0], x[6, 4999] = math.inf, math.inf, math.inf
    x[6, 17] = math.inf
    x[8, 4321], x[9, 0] = math.nan, math.nan
    x[9, 1] = math.inf
    x[10, :] = torch.finfo(torch.float32).min  # the type's lowest value is a score
    x[11, 5] = torch.finfo(torch.float32).max
    for how in ({}, dict(top_k=[3000] * 12), dict(top_p=[0.9] * 12), dict(min_p=[0.05] * 12), dict(temperature=[0.0] * 12), dict(temperature=[math.inf] * 12),
                dict(temperature=[1e38] * 12)):
        Call(x, numbers(22, 12), **how).check()


def test_scores_of_any_size():
    x = scores(31, 10, 3001, peak=0.0)
    x *= torch.tensor([1e-38, 1e-30, 1e-10, 1e-3, 1.0, 100.0, 1e5, 1e10, 1e30, 1e37], device="cuda")[:, None]
    for t in (1e-30, 1.0, 1e30):
        Call(x, numbers(32, 10), temperature=[t] * 10, top_p=[0.9] * 10).check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("columns", [1, 61, 1027, 40003])
def test_rows_that_begin_anywhere(dtype, columns):
    """Slices of wider rows at every place, with neighbours that would win."""
    for lead in range(9):
        wide = torch.full((5, columns + 23), 1e4, dtype=DTYPES[dtype], device="cuda")
        wide[:, lead:lead + columns] = scores(lead, 5, columns, dtype)
        Call(wide[:, lead:lead + columns], numbers(lead, 5), top_k=[0, 3, 0, 0, 40], top_p=[1.0, 1.0, 0.8, 1.0, 0.9], min_p=[0.0, 0.0, 0.0, 0.1, 0.0]).check()


def test_rows_beyond_two_gigabytes():
    """The last row begins behind 2^31 elements."""
    columns, stride = 3000, (1 << 31) // 3 + 5
    flat = torch.zeros(3 * stride + columns, dtype=torch.float16, device="cuda")
    x = flat.as_strided((4, columns), (stride, 1))
    x.copy_(scores(41, 4, columns, "f16"))
    Call(x, numbers(42, 4), top_p=[0.9] * 4).check()


def test_outputs_that_are_not_wanted():
    x, token = scores(51, 4, 2000), torch.full((6,), -7, dtype=torch.int32, device="cuda")
    space = torch.zeros(R.rsr_sample_workspace(4, 2000), dtype=torch.uint8, device="cuda")
    R.rsr_sample(x, reals(numbers(52, 4)), token, space, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert token.tolist()[:4] == [t for t, _, _ in Call(x, numbers(52, 4)).expected()] and token.tolist()[4:] == [-7, -7]


def test_the_same_row_alone_and_in_batches():
    """A row's results depend on nothing but the row."""
    x = scores(61, 300, 30011)
    u, how = numbers(62, 300), {name: [v[r % 8] for r in range(300)] for name, v in EVERY.items()}
    whole = Call(x, u, **how)
    whole.call()
    token, kept, probability = whole.results()
    for r0, r1 in ((0, 1), (1, 2), (2, 3), (3, 4), (4, 5), (7, 8), (8, 24), (100, 200)):
        some = Call(x[r0:r1], u[r0:r1], **{name: v[r0:r1] for name, v in how.items()})
        for _ in range(2):
            some.call()
            assert some.results() == (token[r0:r1], kept[r0:r1], probability[r0:r1])


def test_frequencies_are_the_probabilities():
    """u over a grid gives every token as often as its probability says."""
    x, n = torch.tensor([0.0, 1.0, 2.0, 3.0, -1.0, 1.0], device="cuda"), 4096
    c = Call(x.expand(n, 6).contiguous(), [(i + 0.5) / n for i in range(n)], top_k=[5] * n)
    c.call()
    counts = np.bincount(c.results()[0], minlength=6)
    weight = np.exp([0.0, 1, 2, 3, -np.inf, 1])
    assert np.abs(counts / n - weight / weight.sum()).max() <= 1.0 / n


def test_one_workspace_for_calls_of_all_shapes():
    """What a call leaves behind is no other call's."""
    space = torch.zeros(R.rsr_sample_workspace(300, 131072), dtype=torch.uint8, device="cuda")
    shapes = [(1, 131072), (16, 50000), (300, 700), (2, 9), (1, 131072), (37, 30000), (256, 2000), (3, 131072)]
    calls = [Call(scores(i, r, c), numbers(i, r), **{name: [v[(i + j) % 8] for j in range(r)] for name, v in EVERY.items()}) for i, (r, c) in enumerate(shapes)]
    for c in calls:
        c.workspace = space
    for _ in range(3):
        for c in calls:
            c.call()
    for c in calls:
        token, kept, _ = c.results()
        assert list(zip(token, kept)) == [(t, n) for t, _, n in c.expected()]
