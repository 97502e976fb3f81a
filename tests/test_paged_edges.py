"""The paged cache's calls at the ends of what their documentation allows."""
import numpy as np
import pytest
import torch

from gpu_pipeline import say

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("no GPU", allow_module_level=True)

import paper_2502_17139_amd as fc  # noqa: E402,F401
from test_paged import bf16, make_pool, trees  # noqa: E402
from test_paged_scores import check  # noqa: E402


@pytest.mark.parametrize("R,H", [(1, 4), (5, 2), (20, 1), (40, 1), (65, 2), (130, 1)])
def test_positions_past_32_bits(R, H):
    """prefix_len + pos_ids is a sum of two 32-bit numbers: rows just below 2^31,
    past it, and before 0."""
    rng = np.random.default_rng(R)
    pool, table = make_pool(rng, 3, 1), np.array([[2, 0, 1]] * 2, np.int32)
    t = trees(rng, 2, R)
    t["pos_ids"] = (2 ** 31 - 1 - rng.integers(0, 300, (2, R))).astype(np.int32)
    t["pos_ids"][1, ::3] = -2 ** 31 + rng.integers(0, 300, len(t["pos_ids"][1, ::3]))
    row = lambda h, s=1.0: bf16(rng, 2, R, h, 128, scale=s)  # noqa: E731
    say(f"positions past 32 bits R={R}")
    check(row(H, 3.0), row(1), row(1), pool, table, [150, 60], t)
