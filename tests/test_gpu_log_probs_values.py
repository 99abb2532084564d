"""GPU parity of mar_log_probs with 64 bits where values are out of the ordinary: rows that a mask takes out, of any size, beside
others, rows of very different size."""
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
