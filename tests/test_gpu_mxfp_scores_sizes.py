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


@pytest.mark.parametrize("T,V,dim", ((1, 300, 100), (20, 5000, 33), (32, 70_001, 400), (40, 600, 100), (130, 9001, 200), (1537, 22_003, 64)))
def test_blocks_of_4_bit_queries_that_are_not_finite(T, V, dim):
    """Scale byte 255 in some blocks of some queries and rows: their scores are NaN, all others what they are."""
    g = np.random.default_rng(T)
    codes, scales_ = table(g, V, dim)
    qc, qs = table(g, T, dim)
    bad_q, bad_r = sorted({0, T // 2} if T > 2 else {0}), (7, V - 1)
    for j, q in enumerate(bad_q):
        qs[q, j % qs.shape[1]] = 255
    for j, r in enumerate(bad_r):
        scales_[r, -1 - j] = 255
    qc[bad_q[0]] = 0                                          # as quantisation leaves such a block
    got = scores(torch.from_numpy(qc).to(DEV), torch.from_numpy(codes).to(DEV), torch.from_numpy(scales_).to(DEV), dim, "mxfp4", q_scales=torch.from_numpy(qs).to(DEV))
    bad = np.zeros((T, V), dtype=bool)
    bad[bad_q] = True
    bad[:, bad_r] = True
    got = got.cpu().numpy()
    assert np.array_equal(np.isnan(got), bad)
    clear = lambda a: np.where(a == 255, 0, a).astype(np.uint8)
    want, bound = mu.score_bound(mu.values(qc, clear(qs), dim), mu.values(codes, clear(scales_), dim), "mxfp4", 1.0, 2.0 ** -24)
    assert (np.abs(got - want)[~bad] <= bound[~bad]).all()
