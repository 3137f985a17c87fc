"""rsr_sample at the limits of what it is given (include/rsr_decode.h)."""
import pytest
import torch

import paper_2411_06360_amd as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("columns", [8, 13])
def test_more_short_rows_than_a_launch_has(columns):
    """2^22 workgroups of 1024 threads are more than a launch has: each row's only score is its own."""
    rows = 2**22 + 5
    print("short rows", columns, flush=True)
    want = (torch.arange(rows, device="cuda") * 5 + torch.arange(rows, device="cuda") // 1024) % columns
    x = torch.full((rows, columns), -float("inf"), dtype=torch.bfloat16, device="cuda")
    x.scatter_(1, want[:, None], torch.full((rows, 1), -3.0, dtype=torch.bfloat16, device="cuda"))
    token, kept = (torch.full((rows,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    probability, u = torch.full((rows,), -7.0, device="cuda"), torch.rand(rows, generator=torch.Generator().manual_seed(columns)).cuda()
    space = torch.zeros(R.rsr_sample_workspace(rows, columns), dtype=torch.uint8, device="cuda")
    R.rsr_sample(x, u, token, space, probability=probability, kept=kept, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(token, want.int()) and bool((kept == 1).all()) and bool((probability == 1).all())
