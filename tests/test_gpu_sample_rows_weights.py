"""Draws of rows that weigh next to nothing: which rows are kept, and that what is kept can be drawn, whatever way a query goes.

A number of 0 names the first kept row by id and a number of 1 the last one, however little they weigh."""
import numpy as np
import pytest
import torch

from test_gpu_sample_rows import DEV, TYPES, check

pytestmark = pytest.mark.gpu

# rows and top-k of every way that looks at the best rows alone: short list and longer one of up to 16,384 rows, of more
WAYS = ((2, 1), (300, 5), (3000, 50), (16_384, 128), (16_384, 129), (14_951, 600), (16_385, 50), (20_000, 600), (40_001, 1500), (40_001, 200), (40_001, 400), (30_000, 9000))


def steep(Q, V, top_k, depth, dtype, seed=1):
    """Q rows of scores: one at 0, top-k others from -depth up by exactly representable steps, the rest far below them, spread."""
    g = np.random.default_rng(seed + V)
    s = -4.0 * depth - 200.0 * g.random((Q, V))
    for q in range(Q):
        at = g.permutation(V)[:max(2, min(top_k, V))]
        s[q, at] = -depth + 0.25 * (np.arange(len(at)) % 16)
        best = np.sort(at)[len(at) // 2]                     # kept rows on both sides of it where there are three
        s[q, best] = 0.0
    return torch.from_numpy(s).to(dtype).to(DEV)


@pytest.mark.parametrize("tname", TYPES)
@pytest.mark.parametrize("V,top_k", WAYS)
def test_kept_rows_of_next_to_no_weight_can_be_drawn(V, top_k, tname):
    """2^-55 of the best row each: the outermost ids belong to such rows."""
    s = steep(3, V, top_k, 38.0, TYPES[tname][0])
    u = torch.tensor([[0.0, 1.0, 0.5, 0.25, 2.0 ** -149, 1.0 - 2.0 ** -24]] * 3, device=DEV)
    check(s, u, top_k=top_k)
    check(s, u, top_k=top_k, min_p=2.0 ** -60)
    check(s, u, top_k=top_k, top_p=0.5)


@pytest.mark.parametrize("tname", TYPES)
@pytest.mark.parametrize("V,top_k", WAYS + ((3000, 0), (16_384, 0), (16_385, 0), (40_001, 0)))
def test_min_p_goes_by_the_weights_themselves(V, top_k, tname):
    """Rows at e^-64 .. e^-60 weigh nothing as integers; min_p between them and those far below, and among them."""
    s = steep(3, V, top_k or 70, 64.0, TYPES[tname][0])
    u = torch.tensor([[0.5, 0.25]] * 3, device=DEV)
    for min_p in (1e-30, 1e-37, 2e-27, 5e-27, 2.0 ** -149):
        for f in (dict(), dict(top_p=0.9)):
            check(s, u, top_k=top_k, min_p=min_p, **f)
