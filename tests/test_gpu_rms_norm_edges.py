"""The norm of hidden states at the ends of its ranges."""

import math

import pytest
import torch

from paper_2509_00195_amd import make_norm, tts_rms_norm
from tests import _layer as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [(1 << 31) - 8, (1 << 31) - 7, (1 << 31) - 1])
def test_the_longest_rows(k):
    """Every row length that an int32 holds. The squares are ones, and a thread adds at most 2^23 of them, so that its
    sum is exact; the 256 threads' add up to 2^31 - 8 or 2^31, at most 2^-24 of itself off."""
    x = torch.ones((1, k), dtype=torch.bfloat16, device=L.DEV)
    x[0, k // 3::7] = -1.0
    out = torch.full((1, k), math.nan, dtype=torch.bfloat16, device=L.DEV)
    tts_rms_norm(make_norm(k, 0.0), 1, x, None, out)
    assert torch.equal(out.view(torch.int16), x.view(torch.int16))  # 1 to within 2^-23, which bf16 rounds to 1
