"""The limits of the operators on both sides of the attention, without a GPU (include/rsr_decode.h)."""
import pytest

import paper_2411_06360_amd as R
from tests.test_decode_api import INVALID, rotate


@pytest.mark.parametrize("tokens", [2**31, 2**31 + 5, 2**62, 2**63 - 1])
def test_more_tokens_than_positions_are_numbered_for_are_refused(tokens):
    assert rotate(tokens=tokens) == INVALID and "2^31" in R.rsr_last_error()
