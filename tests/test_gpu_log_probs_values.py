"""GPU parity of mar_log_probs with 64 bits where values are out of the ordinary: rows that a mask takes out, of any size, beside
others, rows of very different size, scores that 32 bits cannot tell apart, queries that are
not finite, distributions with nearly all probability in one row."""
import math

import pytest
import torch

import softmax_util as su
from test_gpu_log_probs import check

pytestmark = pytest.mark.gpu
DEV = su.DEV
LARGE = {"fp32": (1e8, 1e12, 1e30, 3.0e38), "bf16": (1e8, 1e30, 3.0e38), "fp16": (6e4,)}


@pytest.mark.parametrize("tname,value", [(t, v) for t in LARGE for v in LARGE[t]])
@pytest.mark.parametrize("T,V,d", ((20, 1500, 20), (100, 3000, 100), (300, 2000, 60), (600, 2500, 300), (7, 900, 400)))
def test_large_rows_that_do_not_count_touch_no_other(T, V, d, tname, value):
    """Finite values of any size in rows that no query's mask allows, in each of the three ways that rows come."""
    print("case", T, V, d, tname, value, flush=True)
    g = su.gen(V + d)
    dt = su.TYPES[tname][0]
    q, w = su.rows(g, T, d, dt), su.rows(g, V, d, dt)
    bad = torch.rand(V, generator=g, device=DEV) < 0.2
    bad[3] = True
    n = int(bad.sum())
    sign = torch.randint(0, 2, (n, d), generator=g, device=DEV).float() * 2 - 1
    w[bad] = (sign * value * (0.5 + 0.5 * torch.rand((n, d), generator=g, device=DEV))).to(dt)
    allowed = (torch.rand((T, V), generator=g, device=DEV) < 0.7) & ~bad
    targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    words = su.pack(allowed)
    out = su.run_log_probs(q, w, tname, targets, words, words.shape[1], top=10)
    clean = w.clone()
    clean[bad] = 0
    check(q, clean, tname, targets, allowed, 10, 1.0, out)


@pytest.mark.parametrize("T", (9, 100, 300))
def test_small_rows_and_queries_beside_large_ones(T):
    """fp32 scores are as exact as their own row and query allow: rows 2^40 times as large, of which the query sees a zero column,
    change nothing of the others' scores; nor do neighbouring queries 2^20 times as large."""
    g = su.gen(T)
    V, d = 2000, 48
    q, w = su.rows(g, T, d, torch.float32), su.rows(g, V, d, torch.float32)
    q[:, 0] = 0
    plain = w.clone()
    large = torch.arange(V, device=DEV) % 8 == 5
    w[large] = 0
    plain[large] = 0
    w[large, 0] = 2.0 ** 40
    targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    check(q, plain, "fp32", targets, None, 0, 1.0, su.run_log_probs(q, w, "fp32", targets))
    q[3::8] *= 2.0 ** 20                                     # the others, by themselves, as exact as they are
    out = su.run_log_probs(q, plain, "fp32", targets)
    kept = torch.arange(T, device=DEV) % 8 != 3
    check(q[kept], plain, "fp32", targets[kept], None, 0, 1.0, tuple(x[kept] for x in out))


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
@pytest.mark.parametrize("T,V,top,shared", ((5, 70_000, 10, 256.0), (100, 30_000, 32, 128.0), (600, 20_000, 10, 128.0), (1700, 6_000, 5, 240.0), (3, 300_000, 10, 200.0)))
def test_best_rows_that_32_bits_cannot_tell_apart(T, V, top, shared, tname):
    """A column that all share makes the scores large, and their differences small beside what a 32-bit score is off."""
    print("case", T, V, top, shared, tname, flush=True)
    g = su.gen(V)
    dt, d = su.TYPES[tname][0], 32
    q, w = su.rows(g, T, d, dt, std=0.05), su.rows(g, V, d, dt, std=0.05)
    q[:, 7] = shared
    w[:, 7] = shared
    out = su.run_log_probs(q, w, tname, top=top)
    check(q, w, tname, None, None, top, 1.0, (None, out[1], out[2], out[3]))
    allowed = torch.rand((T, V), generator=g, device=DEV) < 0.5
    words = su.pack(allowed)
    out = su.run_log_probs(q, w, tname, None, words, words.shape[1], top=top)
    check(q, w, tname, None, allowed, top, 1.0, (None, out[1], out[2], out[3]))


@pytest.mark.parametrize("T", (3, 300, 900, 1600))
def test_best_rows_that_all_score_the_same(T):
    """Copies of one row, and a query of zeros: every group of rows may hold the best, and the lowest ids are it."""
    g = su.gen(T)
    q, w = su.rows(g, T, 30, torch.bfloat16), su.rows(g, 1, 30, torch.bfloat16).expand(9000, 30).contiguous()
    q[1] = 0
    ids = su.run_log_probs(q, w, "bf16", top=12)[2]
    assert torch.equal(ids, torch.arange(12, device=DEV, dtype=torch.int32).expand(T, 12))
    w[4321] = 2 * q[2]                                       # one that stands out for its query, at the end for those that it repels
    s = su.scores(q, w, 1.0)
    s[:, torch.arange(9000, device=DEV) != 4321] = s[:, :1].clone()
    want = s.sort(dim=1, descending=True, stable=True).indices[:, :12]
    assert torch.equal(su.run_log_probs(q, w, "bf16", top=12)[2].long(), want)


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
@pytest.mark.parametrize("T", (30, 200, 2000))
def test_no_log_probability_is_positive(T, tname):
    g = su.gen(T)
    dt, V, d = su.TYPES[tname][0], 500, 64
    w = su.rows(g, V, d, dt, std=1.0)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    q = (w[targets.long()].float() * (1.0 + torch.rand((T, 1), generator=g, device=DEV))).to(dt)
    lp, en, ids, tp = su.run_log_probs(q, w, tname, targets, top=3)
    assert (lp <= 0).all() and (tp <= 0).all() and (en >= 0).all(), (float(lp.max()), float(tp.max()))
    check(q, w, tname, targets, None, 3, 1.0, (lp, en, ids, tp))


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
@pytest.mark.parametrize("T", (32, 250, 1500))
def test_entropy_of_confident_queries(T, tname):
    """One row has nearly all of the probability.  A sum of weights 1 + x takes some 16 roundings of 2^-24 (a lane's 16 scores, the
    joins of halves, waves and parts): together, root mean square, 16^0.5 / 3^0.5 = 2.3 of them; twice that is allowed.  What is
    left is as exact as the weights of the other rows."""
    g = su.gen(T)
    dt, V, d = su.TYPES[tname][0], 60, 64
    w = su.rows(g, V, d, dt, std=0.25)
    q = su.rows(g, T, d, dt, std=0.25)
    at = torch.randint(0, V, (T,), generator=g, device=DEV)
    q.copy_((q.float() + w[at].float() * (2.5 + 1.5 * torch.rand((T, 1), generator=g, device=DEV))).to(dt))
    en = su.run_log_probs(q, w, tname)[1].double()
    logp = torch.log_softmax(su.scores(q, w, 1.0), 1)
    H = -(logp.exp() * logp).sum(1)
    confident = H < 1e-2
    assert int(confident.sum()) > T // 4
    err = (en - H).abs()[confident]
    size = H[confident] * (4 * su.score_error(q, w, 1.0) + 2.0 ** -20)
    assert float((err - size).clamp(min=0).square().mean().sqrt()) <= 4.6 * 2.0 ** -24, float(err.square().mean().sqrt())


@pytest.mark.parametrize("T", (5, 70, 400))
def test_entropy_of_a_query_that_is_not_finite(T):
    g = su.gen(T)
    q, w = su.rows(g, T, 40, torch.float32), su.rows(g, 300, 40, torch.float32)
    q[2, 5], q[4, 0] = float("nan"), float("inf")
    en = su.run_log_probs(q, w, "fp32", top=3)[1]
    assert not torch.isfinite(en[2]) and not torch.isfinite(en[4])
    kept = torch.ones(T, dtype=torch.bool, device=DEV)
    kept[2] = kept[4] = False
    assert (en[kept] > 0).all()


def test_the_largest_table_and_many_queries():
    """Both matrices' layout takes more than one launch: all rows are zeros but one for every query, with nearly all probability (the
    zeros' part, 2^29 of e^40, and what their sum is off lie below 2^-24)."""
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    V, T, d = 0x1fffff00, 600, 8
    g = su.gen(1)
    q = su.rows(g, T, d, torch.bfloat16, std=1.0)
    w = torch.zeros((V, d), dtype=torch.bfloat16, device=DEV)
    targets = torch.linspace(0, V - 1, T, dtype=torch.float64, device=DEV).long()
    planted = (q.float() * (45.0 / q.float().square().sum(1, keepdim=True))).to(torch.bfloat16)
    w[targets] = planted
    lp = su.run_log_probs(q, w, "bf16", targets.to(torch.int32))[0].double()
    s = su.scores(q, planted, 1.0)
    ref = s.diagonal() - torch.logsumexp(torch.cat([s, torch.full((T, 1), math.log(V - T), dtype=torch.float64, device=DEV)], 1), 1)
    err = (lp - ref).abs()
    assert (err <= 2 * su.score_error(q, planted, 1.0) + 256 * 2.0 ** -24 + ref.abs() * 2.0 ** -23).all(), float(err.max())
