"""Draws from more rows than a workgroup holds in registers: the ways that only such tables take, and their borders, against extended precision."""
import numpy as np
import pytest
import torch

from test_gpu_sample_rows import DEV, FILTERS, TYPES, check, sample, scores_of, uniforms_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", (16_383, 16_384, 16_385, 18_431, 18_433, 65_536, 131_072, 300_001))
def test_around_the_borders_between_ways(V):
    s = scores_of(V, 2, V, torch.float32)
    for f in FILTERS + (dict(top_k=2048), dict(top_k=2049, top_p=0.9), dict(top_k=V), dict(top_k=V - 1, top_p=0.99), dict(top_k=V + 5), dict(top_k=128), dict(top_k=129, min_p=0.2)):
        check(s, uniforms_of(V, 2, 6), **f)


@pytest.mark.parametrize("Q,V", ((3, 17_000), (300, 20_011), (2100, 16_500)))
def test_many_queries(Q, V):
    """One chunk a query and several; every query with parameters of its own."""
    s = scores_of(Q, Q, V, torch.bfloat16)
    g = np.random.default_rng(Q)
    arrays = tuple(tuple(g.choice(v, Q).tolist()) for v in ((0.0, 0.5, 1.0, 1.4), (0, 0, 1, 7, 300, 2500), (1.0, 0.3, 0.9, 0.99), (0.0, 0.0, 0.02)))
    check(s, uniforms_of(Q, Q, 2), arrays=arrays)


@pytest.mark.parametrize("tname", TYPES)
def test_equal_scores(tname):
    """More equal rows than any list holds: all of them, or a level of few."""
    V = 70_000
    g = np.random.default_rng(5)
    s = torch.from_numpy(np.stack((np.full(V, 1.5), g.integers(0, 3, V) * 0.5, np.where(g.random(V) < 0.001, 3.0, 0.25), np.where(g.random(V) < 0.3, -1.0, -9.0)))).to(TYPES[tname][0]).to(DEV)
    u = uniforms_of(9, 4, 8)
    for f in (dict(), dict(top_k=1), dict(top_k=50), dict(top_k=40_000), dict(top_p=0.5), dict(top_p=0.01), dict(top_p=0.5, top_k=1000), dict(min_p=1.0), dict(min_p=0.9, top_p=0.97)):
        check(s, u, **f)


@pytest.mark.parametrize("tname", TYPES)
def test_masks_infinities_and_nan(tname):
    V = 40_000
    inf, nan = float("inf"), float("nan")
    big = torch.finfo(TYPES[tname][0]).max
    s = scores_of(3, 9, V, TYPES[tname][0])
    s[0, 39_999] = inf
    s[1, [5, 20_000]] = inf
    s[2] = -inf
    s[3] = nan
    s[4, ::2], s[4, 1::2] = big, -big
    s[5, :39_000] = nan
    s[6] = -inf
    s[6, 31_234] = -big
    s[7, ::3], s[7, 1::3] = nan, -inf
    for f in (dict(), dict(temperature=1e-3), dict(temperature=1e38), dict(top_k=3), dict(top_p=0.9), dict(top_p=0.9, min_p=0.3), dict(top_k=5000, top_p=0.6)):
        got = check(s, uniforms_of(4, 9, 5), **f)
        assert (got[0][2:4] == -1).all()
    g = np.random.default_rng(1)
    allowed = np.stack([g.random(V) < p for p in (0.5, 0.9, 1.0, 0.001, 0.5, 0.5, 1.0, 0.5, 0.0)])
    for f in (dict(), dict(top_k=30, top_p=0.9), dict(top_p=0.8), dict(min_p=0.01)):
        check(s, uniforms_of(4, 9, 5), allowed, **f)


def test_special_parameters():
    nan, inf = float("nan"), float("inf")
    T = (1.0, 0.0, -1.0, nan, inf, 1e-30, 1e30, 0.5, 2.0, 1e-45, 0.9, 1.0, 1.0, 1.0, 1.0, inf)
    k = (0, 0, 5, 5, 0, 0, 7, -3, 1 << 30, 0, 20, 0, 0, 0, 0, 0)
    p = (1.0, 0.5, 0.9, 1.0, 0.3, 0.9, 0.5, 2.0, nan, 0.9, 0.0, -1.0, 0.9999999, 1e-20, 0.5, 0.9)
    m = (0.0, 0.5, 0.0, 0.0, 0.0, 0.0, 0.1, -1.0, nan, 0.0, 0.0, 0.0, 0.0, 0.0, 1.0, 0.0)
    for tname in TYPES:
        s = scores_of(5, 16, 33_333, TYPES[tname][0])
        check(s, uniforms_of(5, 16, 4), arrays=(T, k, p, m))
        s[0] = torch.randn(33_333, generator=torch.Generator().manual_seed(2)) * 1e-30
        check(s, uniforms_of(6, 16, 4), arrays=(T, None, p, m), top_k=100)


@pytest.mark.parametrize("spread,temperature,top_p", ((0.001, 1.0, 0.9), (20.0, 1.0, 0.999), (3.0, 0.05, 0.7), (8.0, 2.0, 0.5), (1.0, 1.0, 0.00001)))
def test_borders_of_top_p_wherever_they_lie(spread, temperature, top_p):
    """Flat rows, whose border lies in the first bins, and steep ones; ten queries of 100,000 rows."""
    for dt in (torch.float32, torch.bfloat16):
        s = scores_of(7, 10, 100_003, dt, spread=spread)
        check(s, uniforms_of(7, 10, 4), temperature=temperature, top_p=top_p)
        check(s, uniforms_of(8, 10, 4), temperature=temperature, top_p=top_p, min_p=0.05)


def test_results_do_not_depend_on_the_call():
    """One row alone, among others, with a stride, and drawn again: the same ids."""
    s = scores_of(11, 40, 50_001, torch.float32)
    u = uniforms_of(11, 40, 3)
    for f in (dict(top_p=0.9), dict(top_k=100, top_p=0.8), dict(min_p=0.02), dict()):
        want = sample(s, u, **f)
        assert all(torch.equal(x, y) for x, y in zip(sample(s, u, **f), want))
        wide = torch.full((40, 50_010), float("nan"), device=DEV)[:, 3:50_004]
        wide.copy_(s)
        assert all(torch.equal(x, y) for x, y in zip(sample(wide, u, **f), want))
        one = sample(s[7:8], u[7:8].contiguous(), **f)
        assert torch.equal(one[0], want[0][7:8]) and torch.equal(one[2], want[2][7:8])


@pytest.mark.parametrize("f", (dict(top_k=50), dict(top_k=600, top_p=0.9), dict(top_k=1900), dict(top_p=0.8, min_p=0.001), dict(min_p=0.01), dict(top_k=3000)), ids=str)
def test_more_segments_than_fit_beside_the_borders(f):
    for dt in (torch.float32, torch.bfloat16):
        check(scores_of(21, 2, 2_000_003, dt), uniforms_of(21, 2, 40), **f)


@pytest.mark.parametrize("V", (9_000, 16_384, 140_000))
@pytest.mark.parametrize("equal", (1, 2, 255, 256, 257, 2048, 2049, 8192, 8193))
def test_equal_rows_at_the_border_of_top_p(V, equal):
    """The border among so many equal rows: it goes by id whichever way has room for them."""
    g = np.random.default_rng(equal)
    s = np.full((3, V), -25.0, dtype=np.float32)
    for q in range(3):                                        # a row above them, the equal ones, and too little below to matter
        at = g.permutation(V)[:equal + 1]
        s[q, at] = 1.0
        s[q, at[0]] = 1.0 + np.log(equal)
    s = torch.from_numpy(s).to(DEV)
    for top_p in (0.4999, 0.75, 0.999):
        check(s, uniforms_of(equal, 3, 8), top_p=top_p)
    check(s, uniforms_of(equal, 3, 8), top_p=0.75, temperature=0.9, min_p=0.5 / equal)


@pytest.mark.parametrize("equal", (2048, 2049, 5000, 8193, 60_000, 124_999, 125_001))
def test_more_equal_rows_than_a_workgroup_holds(equal):
    """Neighbours, so that one chunk alone has more than its list; from 125,000 on, more than the query's list in memory."""
    V = 4_000_000
    s = torch.full((1, V), -30.0, device=DEV)
    s[0, 1_000_001:1_000_001 + equal] = 0.5
    s[0, 3_999_999] = 0.5 + float(np.log(equal))
    for top_p in (0.4999, 0.75):
        check(s, uniforms_of(equal, 1, 5), top_p=top_p)
    check(s, uniforms_of(equal, 1, 5), top_p=0.75, min_p=0.5 / equal)


@pytest.mark.parametrize("spread", (0.1, 0.3, 1.0))
def test_flat_scores_over_many_rows(spread):
    for dt in (torch.float32, torch.bfloat16):
        check(scores_of(13, 1, 3_000_000, dt, spread=spread), uniforms_of(13, 1, 5), top_p=0.6)


@pytest.mark.parametrize("top_k,top_p", ((600, 1.0), (1500, 0.9), (2048, 0.5), (40, 0.9)))
def test_many_queries_go_other_ways_to_the_same_rows(top_k, top_p):
    """Chunks and groups of rows follow the number of queries, what is drawn does not."""
    s, u = scores_of(17, 300, 200_003, torch.float32, spread=2.0), uniforms_of(17, 300, 3)
    got = sample(s, u, top_k=top_k, top_p=top_p)
    for first in (0, 151, 297):
        want = check(s[first:first + 3], u[first:first + 3], top_k=top_k, top_p=top_p)
        assert torch.equal(got[0][first:first + 3].cpu(), torch.as_tensor(want[0]).cpu())
        assert torch.equal(got[2][first:first + 3].cpu(), torch.as_tensor(want[2]).cpu())


@pytest.mark.parametrize("tname", TYPES)
def test_equal_scores_of_a_workgroup(tname):
    """More equal rows than the list of those that reach top-k's bound; rows that do not count among them."""
    V = 16_384
    g = np.random.default_rng(8)
    s = torch.from_numpy(np.stack((np.full(V, 0.25), np.where(g.random(V) < 0.3, -np.inf, 0.25), np.where(g.random(V) < 0.02, 2.0, 0.25), g.integers(0, 40, V) * 0.125))).to(TYPES[tname][0]).to(DEV)
    u = uniforms_of(21, 4, 6)
    for f in (dict(top_k=129), dict(top_k=300, top_p=0.9), dict(top_k=2000), dict(top_k=16_383, top_p=0.5), dict(top_k=12_000, min_p=0.5), dict(top_p=0.7), dict(top_p=0.3, min_p=0.9)):
        check(s, u, **f)
