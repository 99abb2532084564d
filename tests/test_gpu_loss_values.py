"""GPU parity of mar_softmax_loss with 64 bits where values are out of the ordinary: queries that do not count, of any size, beside
others, the ends of the floats' range, answers with all of the probability."""
import pytest
import torch

import softmax_util as su

pytestmark = pytest.mark.gpu
DEV = su.DEV
LARGE = {"fp32": (1e5, 1e8, 1e12, 1e30, 3.0e38), "bf16": (1e5, 1e8, 1e30, 3.0e38), "fp16": (6e4,)}


def make(T, V, d, tname, std=0.3):
    g = su.gen(T * 11 + V + d)
    dt = su.TYPES[tname][0]
    q, w = su.rows(g, T, d, dt, std), su.rows(g, V, d, dt, std)
    return g, q, w, torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)


def signs(g, n, d):
    return torch.randint(0, 2, (n, d), generator=g, device=DEV).float() * 2 - 1


@pytest.mark.parametrize("tname,value", [(t, v) for t in LARGE for v in LARGE[t]])
@pytest.mark.parametrize("T,V,d", ((300, 777, 60), (1000, 5000, 20), (140, 900, 300)))
def test_large_queries_that_do_not_count_touch_no_other(T, V, d, tname, value):
    """Finite values of any size in queries without an answer and in queries without weight; several in a block of eight."""
    print("case", T, V, d, tname, value, flush=True)
    g, q, w, targets = make(T, V, d, tname)
    weights = torch.rand(T, generator=g, device=DEV) + 0.5
    targets[::5] = -1
    targets[3::50] = V
    weights[4::16] = 0.0
    weights[6::48] = 2.0 ** -120
    none = (targets < 0) | (targets >= V) | (weights < 2.0 ** -100)
    n = int(none.sum())
    q[none] = (signs(g, n, d) * value * (0.5 + 0.5 * torch.rand((n, d), generator=g, device=DEV))).to(q.dtype)
    assert torch.isfinite(q).all()
    out = su.run_loss(q, w, tname, targets, weights)
    assert (out[0][none] == 0).all() and (out[2][none] == 0).all()
    clean, kept = q.clone(), ~none
    clean[none] = 0
    u = torch.where(none, torch.zeros_like(weights), weights)
    su.check_loss((out[0], None, out[2], out[3]), clean, w, tname, targets, u, 1.0)
    ref = torch.logsumexp(su.scores(q[kept], w, 1.0), 1)
    err = (out[1].double()[kept] - ref).abs()
    assert (err <= su.score_error(q[kept], w, 1.0) + su.sum_error(V) + ref.abs() * 2.0 ** -23).all(), float(err.max())
    if value <= 1e5:                                         # their own scores stay below 2^23
        ref = torch.logsumexp(su.scores(q[none], w, 1.0), 1)
        err = (out[1].double()[none] - ref).abs()
        assert (err <= su.score_error(q[none], w, 1.0) + su.sum_error(V) + ref.abs() * 2.0 ** -23).all(), float(err.max())


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
def test_queries_that_do_not_count_beside_rows_that_are_not_finite(tname):
    """Their weight is zero by itself, not zero times their probabilities."""
    g, q, w, targets = make(200, 300, 40, tname)
    targets[:] = -1
    w[17], w[40, 3] = float("inf"), float("nan")
    loss, _, gq, gw = su.run_loss(q, w, tname, targets)
    assert not loss.any() and not gq.any() and not gw.any()


@pytest.mark.parametrize("up,down", ((100, -100), (-100, 100), (60, -60), (0, -100), (-100, 0), (88, -88)))
@pytest.mark.parametrize("T,V,d", ((70, 3000, 100), (300, 700, 40), (20, 15_000, 16)))
def test_values_towards_the_ends_of_the_range(T, V, d, up, down):
    """fp32: one matrix 2^up times and the other 2^down times what is usual; weights and their sums stay inside the floats' range."""
    print("case", T, V, d, up, down, flush=True)
    g, q, w, targets = make(T, V, d, "fp32", std=1.0)
    q, w = q * 2.0 ** up, w * 2.0 ** down
    weights = torch.rand(T, generator=g, device=DEV) + 0.5
    su.check_loss(su.run_loss(q, w, "fp32", targets, weights), q, w, "fp32", targets, weights, 1.0)


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
def test_no_loss_is_negative(tname):
    """Answers with all of the probability: the log-sum-exp, in 32 bits, may come out below the answer's score in 64."""
    g, q, w, targets = make(2000, 500, 64, tname, std=1.0)
    q.copy_((w[targets.long()].float() * (1.0 + torch.rand((2000, 1), generator=g, device=DEV))).to(q.dtype))
    out = su.run_loss(q, w, tname, targets)
    assert (out[0] >= 0).all(), float(out[0].min())
    su.check_loss(out, q, w, tname, targets, None, 1.0)


@pytest.mark.parametrize("T,V,d", ((300, 1200, 100), (40, 3000, 300)))
def test_rows_2_17_times_as_large_as_their_neighbours(T, V, d):
    """fp32 rows share an exponent by eights: beside rows 2^16 times as large, of which the queries see a zero column, scores are as
    exact as the others' own size allows."""
    g, q, w, targets = make(T, V, d, "fp32")
    large = torch.arange(V, device=DEV) % 8 == 5
    q[:, 0] = 0
    w[large] = 0
    plain = w.clone()
    w[large, 0] = 2.0 ** 15
    loss, lse, _, gw = su.run_loss(q, w, "fp32", targets)
    su.check_loss((loss, lse, None, gw), q, plain, "fp32", targets, None, 1.0)


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
def test_scores_towards_2_23(tname):
    """As large as they may be: results stay finite, and log-sum-exps as exact as the scores."""
    g, q, w, targets = make(150, 900, 64, tname, std=1.0)
    size = (2.0 ** 22.9 / float(su.scores(q, w, 1.0).abs().max())) ** 0.5
    q, w = (q.float() * size * 0.99).to(q.dtype), (w.float() * size * 0.99).to(w.dtype)
    loss, lse, gq, gw = su.run_loss(q, w, tname, targets)
    lp, en, ids, tp = su.run_log_probs(q, w, tname, targets, top=5)
    assert all(torch.isfinite(x).all() for x in (loss, lse, gq, gw, lp, en, tp))
    s = su.scores(q, w, 1.0)
    ref, bound = torch.logsumexp(s, 1), su.score_error(q, w, 1.0) + su.sum_error(900)
    at = s[torch.arange(150, device=DEV), targets.long()]
    assert ((lse.double() - ref).abs() <= bound + ref.abs() * 2.0 ** -23).all()
    assert ((lp.double() - (at - ref)).abs() <= bound + (at - ref).abs() * 2.0 ** -23).all()
    assert torch.equal(ids.long(), s.sort(dim=1, descending=True, stable=True).indices[:, :5])
