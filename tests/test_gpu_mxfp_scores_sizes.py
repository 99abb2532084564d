"""Scores of 4-bit tables at sizes between the smallest and the largest, where a lane holds two rows; queries and rows at the ends checked."""
import numpy as np
import pytest
import torch

import mxfp_util as mu
from test_gpu_mxfp_scores import DEV, KINDS, TYPES, check, scores, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", (31, 64, 100, 190, 256, 300, 383, 400))
def test_two_rows_a_lane(dim, kind):
    T, V = (1537, 22_003) if kind == "mxfp4" else (515, 25_003)
    g = np.random.default_rng(dim)
    codes, scales_ = table(g, V, dim)
    c, s = torch.from_numpy(codes).to(DEV), torch.from_numpy(scales_).to(DEV)
    out = ("fp32", "bf16", "fp16")[dim % 3]
    rows = np.unique(np.concatenate((np.arange(300), g.integers(0, V, 700), np.arange(V - 600, V))))
    some = np.unique(np.concatenate((np.arange(40), g.integers(0, T, 60), np.arange(T - 40, T))))
    w = mu.values(codes[rows], scales_[rows], dim)
    if kind == "mxfp4":
        qc, qs = table(g, T, dim)
        got = scores(torch.from_numpy(qc).to(DEV), c, s, dim, kind, out, 0.5, dim % 2, dim % 2, torch.from_numpy(qs).to(DEV))
        q = mu.values(qc, qs, dim)
    else:
        x = torch.from_numpy(g.standard_normal((T, dim)) * np.exp2(g.integers(-6, 3, (T, 1)))).to(TYPES[kind][0])
        got = scores(x.to(DEV), c, s, dim, kind, out, 0.5, dim % 2, dim % 2)
        q = x.double().numpy()
    check(got[torch.from_numpy(some).to(DEV)][:, torch.from_numpy(rows).to(DEV)], q[some], w, kind, out, 0.5)
