"""rsr_head_rotate at the limits of what it is given (include/rsr_decode.h)."""
import numpy as np
import pytest
import torch

import paper_2411_06360_amd as R
from oracle import decode as oracle
from tests.test_gpu_rotate import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,pairs", [(torch.float32, False), (torch.bfloat16, True)])
def test_more_tokens_than_a_launch_has(dtype, pairs):
    """A launch has 2^26 - 4 tokens: those behind them, and around the border, as by the definition; all as in parts; nothing between the rows."""
    tokens, dim = 2**26 + 9, 8
    print("many tokens", dtype, flush=True)
    wide = torch.empty((tokens, 3 * dim), dtype=dtype, device="cuda").uniform_(-2, 2, generator=torch.Generator(device="cuda").manual_seed(3))
    old, position = wide.clone(), torch.arange(tokens, dtype=torch.int32, device="cuda") % 1000003
    frequency = torch.tensor([1.0, 0.3, 0.01, 0.0], dtype=torch.float64, device="cuda")
    how, stream = R.make_rotary(frequency, dim, eps=1e-6, pairs=pairs), torch.cuda.current_stream().cuda_stream
    q, k = wide[:, :dim], wide[:, 2 * dim:]
    R.rsr_head_rotate(how, q, k, position, q, k, stream)
    torch.cuda.synchronize()
    assert torch.equal(wide[:, dim:2 * dim], old[:, dim:2 * dim])
    for at in (0, 2**26 - 12, tokens - 12):
        for rows, source in ((q, old[:, :dim]), (k, old[:, 2 * dim:])):
            want, size = oracle.rotate(source[at:at + 12].double().cpu().numpy(), position[at:at + 12].cpu().numpy(), frequency.cpu().numpy(), dim, np.float32(1e-6).astype(np.float64), None, pairs)
            # (at most 18.1 units of 2^-24 of |a| + |b|, as for a few tokens, and the rounding to the type)
            bound = 18.1 * 2.0**-24 * size + np.abs(want) * torch.finfo(dtype).eps / 2
            assert (np.abs(rows[at:at + 12].double().cpu().numpy() - want) <= bound).all(), at
    part = torch.empty((2**25, dim), dtype=dtype, device="cuda")
    for rows, source in ((q, old[:, :dim]), (k, old[:, 2 * dim:])):
        for at in range(0, tokens, 2**25):
            n = min(2**25, tokens - at)
            R.rsr_head_rotate(how, source[at:at + n], None, position[at:at + n], part[:n], None, stream)
            assert torch.equal(rows[at:at + n], part[:n]), at


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,norm,pairs", [(4099, True, False), (2500, False, True)])
def test_prompts_of_sixteen_bits(act, tokens, norm, pairs):
    check(tokens, 8, 2, 128, norm=norm, pairs=pairs, act=act, out=act, seed=tokens, far=131072)
