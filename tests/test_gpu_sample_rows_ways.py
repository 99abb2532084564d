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


@pytest.mark.parametrize("V,top_ks", ((16_385, (1024, 1025, 1500, 2047, 2048)), (17_000, (1152, 1153, 2048)), (20_001, (1281, 2000)), (30_000, (1920, 1921, 2048))))
def test_large_top_k_of_few_rows(V, top_ks):
    """As few groups as eight rows each make."""
    for dt in (torch.float32, torch.bfloat16):
        s = scores_of(V, 3, V, dt)
        for k in top_ks:
            check(s, uniforms_of(V, 3, 5), top_k=k)
            check(s, uniforms_of(V, 3, 5), top_k=k, top_p=0.95, min_p=0.001)


def test_large_top_k_where_few_rows_count():
    """Fewer groups with a row that counts than top-k; and as many rows as top-k."""
    V = 20_000
    g = np.random.default_rng(1)
    allowed = np.zeros((4, V), dtype=bool)
    allowed[0, :900] = True
    allowed[1, g.permutation(V)[:1500]] = True
    allowed[2, g.permutation(V)[:2100]] = True
    allowed[3, 12_000:14_000] = True
    s = scores_of(5, 4, V, torch.float32)
    for k in (1000, 1500, 2000, 2048):
        check(s, uniforms_of(5, 4, 6), allowed, top_k=k)
        check(s, uniforms_of(5, 4, 6), allowed, top_k=k, top_p=0.8)


@pytest.mark.parametrize("V", (16_385, 17_000, 40_000))
@pytest.mark.parametrize("equal", (1023, 1024, 1100, 2500, 2501, 8192, 8193))
def test_equal_rows_at_the_border_of_top_p_of_few_rows(V, equal):
    """More of them than a sixteenth of the rows, up to more than a workgroup's list holds."""
    g = np.random.default_rng(equal + V)
    s = np.full((3, V), -25.0, dtype=np.float32)
    for q in range(3):
        at = g.permutation(V)[:equal + 1]
        s[q, at] = 1.0
        s[q, at[0]] = 1.0 + np.log(equal)
    s = torch.from_numpy(s).to(DEV)
    for top_p in (0.4999, 0.75, 0.999):
        check(s, uniforms_of(equal, 3, 8), top_p=top_p)
    check(s, uniforms_of(equal, 3, 8), top_p=0.75, temperature=0.9, min_p=0.5 / equal)


@pytest.mark.parametrize("spread", (0.05, 0.3))
@pytest.mark.parametrize("far", (-30.0, -1e4, -60_000.0))
@pytest.mark.parametrize("how", ("one", "few", "half", "first", "nearly all"))
def test_flat_scores_with_others_far_below(how, far, spread):
    """Soft masks: finite scores far below, alone, spread, in one piece, nearly everywhere; beside rows that do not count."""
    V = 200_003
    g = np.random.default_rng(4)
    soft = {"one": np.arange(V) == V // 3, "few": g.random(V) < 0.0005, "half": g.random(V) < 0.5, "first": np.arange(V) < 120_000, "nearly all": g.random(V) < 0.97}[how]
    s = scores_of(3, 3, V, torch.float32, spread=spread)
    s[:, torch.from_numpy(soft).to(DEV)] = far
    s[2, ::7] = -float("inf")
    for f in (dict(top_p=0.9), dict(top_p=0.4, min_p=0.5), dict(top_p=0.9, temperature=0.02), dict(top_p=0.9, temperature=50.0)):
        check(s, uniforms_of(9, 3, 4), **f)
        check(s.half(), uniforms_of(9, 3, 4), **f)


@pytest.mark.parametrize("V,top_k", ((5000, 100), (16_000, 2023), (40_000, 240), (40_000, 2023), (200_000, 3000)))
def test_the_same_bits_again(V, top_k):
    """Rows whose weights sum to a power of two, but for roundings: the integers' scale does not follow the order in which rows are listed."""
    g = np.random.default_rng(V)
    s = np.full((4, V), -40.0, dtype=np.float32) - g.random((4, V)).astype(np.float32)
    ones = 1023 if top_k > 1000 else 63
    for q in range(4):
        at = g.permutation(V)[:top_k]
        s[q, at[:ones]] = 3.0
        s[q, at[ones:]] = 3.0 - np.log(top_k - ones) + (q - 1.5) * 2.0 ** -20
    s = torch.from_numpy(s).to(DEV)
    u = uniforms_of(V, 4, 200)
    for f in (dict(top_k=top_k), dict(top_k=top_k, top_p=0.9995)):
        want = check(s, u, **f)
        for _ in range(20):
            assert all(torch.equal(a, b) for a, b in zip(sample(s, u, **f), want))
