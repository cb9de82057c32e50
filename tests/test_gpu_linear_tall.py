"""Products of more rows than tiles of sixteen of them cover in one launch."""

import pytest
import torch

from paper_2509_00195_amd import make_linear, tts_gated_linear, tts_linear
from tests import _layer as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gated", [False, True])
def test_rows_by_the_hundred_million(gated):
    """Small whole numbers, whose products and sums bf16 holds exactly: up to 8 x 3 x 3, gated (relu) up to 8 x 2 x 1 = 16
    squared."""
    m, k, n = (1 << 28) + 33, 8, 4
    g = L.generator(1)
    most = 2 if gated else 3
    x = torch.randint(-most, most + 1, (m, k), generator=g, device=L.DEV, dtype=torch.int8).to(torch.bfloat16)
    w, u = (torch.randint(-1 if gated else -3, 2 if gated else 4, (n, k), generator=g, device=L.DEV).to(torch.bfloat16)
            for _ in range(2))
    out = torch.full((m + 1, n), 7.0, dtype=torch.bfloat16, device=L.DEV)
    if gated:
        tts_gated_linear(make_linear(k, n, act="relu"), m, x, w, u, out)
    else:
        tts_linear(make_linear(k, n), m, x, w, out)
    for at in range(0, m, 1 << 26):
        y = x[at:at + (1 << 26)].float()
        want = (y @ w.float().t()).relu_() * (y @ u.float().t()) if gated else y @ w.float().t()
        assert torch.equal(out[at:min(m, at + (1 << 26))].float(), want), at
    assert bool((out[m] == 7.0).all())
