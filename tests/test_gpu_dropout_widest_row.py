"""mar_dropout of the widest row there is: 2^31 - 1 columns, whose last group of eight ends beyond it."""
import numpy as np
import pytest
import torch

import paper_2101_08358_amd as mar
from oracle import philox

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_the_widest_row_ends_where_it_ends():
    dim, seed, step = 2 ** 31 - 1, 21, 6
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    x = torch.full((dim + 64,), 1.0, dtype=torch.bfloat16, device=DEV)
    mar.mar_dropout(x, dim, 1, dim, mar.DTYPE_BF16, 0.5, seed, step, x, dim)
    torch.cuda.synchronize()
    assert (x[dim:] == 1.0).all()
    for g0 in (0, 2 ** 27 - 3, 2 ** 28 - 40):
        g = np.arange(g0, g0 + 40)
        words = philox.philox4x32_10_np(np.zeros_like(g), g, step, 0xC0000000, seed, 0)
        u = np.stack([half for w in words for half in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1).reshape(-1)[:dim - 8 * g0]
        got = x[8 * g0:8 * g0 + u.size].float().cpu().numpy()
        assert np.array_equal(got, (u >= 32768) * np.float32(2.0)), g0
