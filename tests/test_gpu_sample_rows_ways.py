"""Draws from sizes and scores at which a query's way is chosen, against extended precision; queries of a batch checked at its ends."""
import numpy as np
import pytest
import torch

from test_gpu_sample_rows import DEV, check, sample, scores_of, uniforms_of

pytestmark = pytest.mark.gpu


def check_some(s, u, some, **f):
    """All queries in one call; those named are compared with their definition and, bit by bit, with what the call gave."""
    got = sample(s, u, **f)
    for q in some:
        want = check(s[q:q + 1], u[q:q + 1].contiguous(), **f)
        assert all(torch.equal(a[q:q + 1], b) for a, b in zip(got, want)), q


@pytest.mark.parametrize("Q,V,top_ks", ((1000, 50_000, (513, 600, 2048)), (500, 60_000, (600, 1500)), (300, 100_000, (800, 1500)), (700, 140_000, (1500,)), (2048, 17_000, (600, 2000))))
def test_large_top_k_of_batches(Q, V, top_ks):
    s, u = scores_of(Q, Q, V, torch.float32), uniforms_of(Q, Q, 3)
    for k in top_ks:
        check_some(s, u, (0, Q // 2, Q - 1), top_k=k)
        check_some(s, u, (1, Q - 2), top_k=k, top_p=0.9)
