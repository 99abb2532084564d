"""GPU parity of mar_log_probs with 64 bits: sizes at and beside tiles, stripes and widths, every type, strides, masks that leave a
row empty, ties, values that are not finite, streams and graphs."""
import math

import pytest
import torch

import paper_2101_08358_amd as mar
import softmax_util as su

pytestmark = pytest.mark.gpu
DEV = su.DEV

SIZES = ((1, 1, 1), (1, 31, 3), (5, 33, 8), (3, 100, 17), (130, 257, 50), (64, 1000, 75), (129, 2049, 100), (33, 5000, 128), (7, 700, 200),
         (40, 1000, 256), (70, 999, 400), (600, 300, 52), (1, 40_000, 100), (17, 70_001, 64), (513, 4097, 96), (2, 3000, 129), (32, 64, 112),
         (65, 2000, 193), (300, 1025, 33))


def check(q, w, tname, targets, allowed, top, scale, out, copies=None):
    """copies: rows that are the same; the 64-bit product gives those of fp32 rows scores 5e-15 apart, by where they lie."""
    lp, en, ids, tp = out
    T, V = q.shape[0], w.shape[0]
    clean = torch.nan_to_num(w.double(), posinf=0.0, neginf=0.0).to(w.dtype) if allowed is not None else w
    s = su.scores(q, clean, scale)
    if copies is not None:
        s[:, copies] = s[:, copies[:1]].clone()
    if allowed is not None:
        s = s.masked_fill(~allowed, -math.inf)
    empty = torch.isinf(s).all(1) if allowed is not None else torch.zeros(T, dtype=torch.bool, device=DEV)
    lse = torch.logsumexp(s, 1)
    delta, total = su.score_error(q, clean, scale), su.sum_error(V)
    if targets is not None:
        has = (targets >= 0) & (targets < V)
        ref = s[torch.arange(T, device=DEV), targets.long().clamp(0, V - 1)] - lse
        ref = torch.where(torch.isnan(ref), torch.full_like(ref, -math.inf), ref)
        ref = torch.where(has, ref, torch.zeros_like(ref))
        inf = torch.isinf(ref)
        assert torch.equal(torch.isinf(lp), inf)
        err = (lp.double() - ref).abs()[~inf]
        assert (err <= 2 * delta + total + ref.abs()[~inf] * 2.0 ** -23).all(), float(err.max())
    p = torch.exp(s - lse[:, None])
    logp = (s - lse[:, None]).masked_fill(torch.isinf(s), 0.0)
    H = torch.where(empty, torch.zeros_like(lse), -(p * logp).sum(1))
    bound = (2 * delta + total) * (2 + math.log(V) + logp.abs().amax(1)) + H.abs() * 2.0 ** -23
    err = (en.double() - H).abs()
    assert (torch.where(empty, en.double() == 0.0, err <= bound)).all(), float(err.max())
    if top:
        k = min(top, V)
        best, order = s.sort(dim=1, descending=True, stable=True)
        want = torch.where(torch.isinf(best[:, :k]), torch.full_like(order[:, :k], -1), order[:, :k])
        assert torch.equal(ids[:, :k].long(), want)
        assert (ids[:, k:] == -1).all() and torch.isinf(tp[:, k:]).all()
        none = want < 0
        assert (tp[:, :k][none] == -math.inf).all()
        ref = best[:, :k] - lse[:, None]
        err = (tp[:, :k].double() - ref)[~none].abs()
        assert (err <= 2 * delta + total + ref[~none].abs() * 2.0 ** -23).all(), float(err.max())


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
@pytest.mark.parametrize("T,V,d", SIZES)
def test_against_64_bits(T, V, d, tname):
    print("case", T, V, d, tname, flush=True)
    g = su.gen(T * 7 + V + d)
    dt = su.TYPES[tname][0]
    odd = (T + V) % 2
    q = su.rows(g, T, d, dt, stride=d + 3 * odd, offset=odd)
    w = su.rows(g, V, d, dt, stride=d + 5 * odd, offset=3 * odd)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    targets[0] = -1 if T > 1 else V - 1
    top = (0, 1, 10, 32)[(T + d) % 4]
    scale = (1.0, 0.7, 2.5)[V % 3]
    check(q, w, tname, targets, None, top, scale, su.run_log_probs(q, w, tname, targets, top=top, scale=scale))


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
@pytest.mark.parametrize("T", (20, 100, 300, 520))
@pytest.mark.parametrize("d", (9, 50, 100, 128, 150, 250, 300, 400))
def test_every_width_however_the_rows_come(d, T, tname):
    """Few queries (a wave each), some (rows staged), many (images): every width there is a kernel for."""
    g = su.gen(d + T)
    dt, V = su.TYPES[tname][0], 4500
    q, w = su.rows(g, T, d, dt), su.rows(g, V, d, dt, stride=d + 1, offset=1)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    check(q, w, tname, targets, None, 10, 1.0, su.run_log_probs(q, w, tname, targets, top=10))


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
@pytest.mark.parametrize("T,V,d,shared", ((1, 1, 4, 0), (9, 65, 20, 0), (140, 1000, 100, 0), (33, 3333, 75, 1), (515, 700, 64, 0), (4, 9000, 400, 0)))
def test_masks(T, V, d, shared, tname):
    """Rows that do not count hold NaN and infinities; one query has no allowed row, one a single row."""
    print("case", T, V, d, tname, flush=True)
    g = su.gen(V + d)
    dt = su.TYPES[tname][0]
    q, w = su.rows(g, T, d, dt), su.rows(g, V, d, dt)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    allowed = torch.rand((1 if shared else T, V), generator=g, device=DEV) < (0.5 if d % 2 else 0.02)
    bad = torch.rand(V, generator=g, device=DEV) < 0.1
    allowed &= ~bad
    if not shared:
        allowed[T // 2] = False
        if T > 2:
            allowed[1] = False
            allowed[1, V - 1] = True
            bad[V - 1] = False
    w[bad] = torch.tensor([float("nan"), float("inf"), -float("inf")], device=DEV)[torch.randint(0, 3, (int(bad.sum()), d), generator=g, device=DEV)].to(dt)
    words = su.pack(allowed)
    out = su.run_log_probs(q, w, tname, targets, words, 0 if shared else words.shape[1], top=12)
    check(q, w, tname, targets, allowed.expand(T, V), 12, 1.0, out)


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
@pytest.mark.parametrize("T,V,d,top", ((2050, 3001, 40, 32), (2001, 700, 270, 32), (2300, 9000, 33, 20), (1000, 2500, 60, 32), (300, 20_000, 20, 32), (256, 70_000, 16, 32), (257, 140_000, 8, 32)))
def test_many_best_rows_of_many_queries(T, V, d, top, tname):
    """The most best rows there can be, where a wave, a workgroup of 256 and one of 1,024 look for them; half of the rows masked; half
    of the rows close to one another, so that many groups reach the threshold."""
    print("case", T, V, d, top, tname, flush=True)
    g = su.gen(T + V)
    dt = su.TYPES[tname][0]
    q, w = su.rows(g, T, d, dt), su.rows(g, V, d, dt)
    w[::2] = w[0]
    copies = torch.arange(0, V, 2, device=DEV)
    allowed = torch.rand((T, V), generator=g, device=DEV) < 0.5
    words = su.pack(allowed)
    check(q, w, tname, None, allowed, top, 1.0, su.run_log_probs(q, w, tname, None, words, words.shape[1], top=top), copies)
    check(q, w, tname, None, None, top, 1.0, su.run_log_probs(q, w, tname, top=top), copies)


def test_mask_rows_with_a_stride_of_their_own():
    g = su.gen(5)
    q, w = su.rows(g, 20, 40, torch.bfloat16), su.rows(g, 100, 40, torch.bfloat16)
    allowed = torch.rand((20, 100), generator=g, device=DEV) < 0.5
    wide = torch.full((20, 9), 0x55555555, dtype=torch.int32, device=DEV)
    wide[:, :4] = su.pack(allowed)
    wide[:, 3] |= -16                                        # bits beyond the last row (row 100 on) are not looked at
    targets = torch.zeros(20, dtype=torch.int32, device=DEV)
    check(q, w, "bf16", targets, allowed, 7, 1.0, su.run_log_probs(q, w, "bf16", targets, wide, 9, top=7))


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
def test_ties_go_to_the_lowest_id(tname):
    """All scores equal; half of the rows copies of one another; small whole numbers with many equal scores."""
    g = su.gen(11)
    dt = su.TYPES[tname][0]
    for V in (50, 4000):
        q = su.rows(g, 40, 24, dt)
        zero = torch.zeros((V, 24), dtype=dt, device=DEV)
        _, en, ids, tp = su.run_log_probs(q, zero, tname, top=32)
        assert torch.equal(ids, torch.arange(32, device=DEV, dtype=torch.int32).expand(40, 32))
        assert ((tp + math.log(V)).abs() <= su.sum_error(V) + 1e-6).all() and ((en - math.log(V)).abs() <= 20 * su.sum_error(V)).all()
        w = su.rows(g, V, 24, dt)
        w[V // 2:] = w[:V - V // 2].clone()
        check(q, w, tname, None, None, 32, 1.0, su.run_log_probs(q, w, tname, top=32))
        wi = torch.randint(-1, 2, (V, 24), generator=g, device=DEV).to(dt)
        qi = torch.randint(-1, 2, (40, 24), generator=g, device=DEV).to(dt)
        check(qi, wi, tname, None, None, 32, 0.25, su.run_log_probs(qi, wi, tname, top=32, scale=0.25))


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
def test_large_and_small_scores(tname):
    """Scores of hundreds, all negative scores, one row far above the others, fp32 rows of very different size."""
    g = su.gen(3)
    dt = su.TYPES[tname][0]
    q, w = su.rows(g, 70, 100, dt, std=2.0), su.rows(g, 3000, 100, dt, std=3.0)
    targets = torch.randint(0, 3000, (70,), generator=g, device=DEV, dtype=torch.int32)
    check(q, w, tname, targets, None, 10, 1.0, su.run_log_probs(q, w, tname, targets, top=10))
    qa, wa = q.abs(), -w.abs()
    check(qa, wa, tname, targets, None, 10, 1.0, su.run_log_probs(qa, wa, tname, targets, top=10))
    wb = w.clone()
    wb[1234] = 30 * q[5]
    check(q, wb, tname, targets, None, 10, 0.01, su.run_log_probs(q, wb, tname, targets, top=10, scale=0.01))
    if tname == "fp32":
        wc = w * torch.exp2(torch.randint(-60, 1, (3000, 1), generator=g, device=DEV).float())
        check(q, wc, tname, targets, None, 32, 1.0, su.run_log_probs(q, wc, tname, targets, top=32))
        big, small = q * 2.0 ** 100, w * 2.0 ** -100
        check(big, small, tname, targets, None, 10, 1.0, su.run_log_probs(big, small, tname, targets, top=10))


def test_a_query_that_is_not_finite_touches_no_other():
    g = su.gen(8)
    q, w = su.rows(g, 66, 48, torch.float32), su.rows(g, 500, 48, torch.float32)
    q[7, 3], q[40, 0] = float("nan"), float("inf")
    targets = torch.randint(0, 500, (66,), generator=g, device=DEV, dtype=torch.int32)
    lp, en, ids, tp = su.run_log_probs(q, w, "fp32", targets, top=5)
    assert not torch.isfinite(lp[7]) and not torch.isfinite(lp[40])
    keep = torch.ones(66, dtype=torch.bool, device=DEV)
    keep[7] = keep[40] = False
    check(q[keep], w, "fp32", targets[keep], None, 5, 1.0, (lp[keep], en[keep], ids[keep], tp[keep]))


def test_offsets_beyond_32_bits():
    """2,100 rows a million elements apart: the last begin beyond 2^31 elements."""
    stride = 1 << 20
    g = su.gen(2)
    buf = torch.empty(2100 * stride, dtype=torch.bfloat16, device=DEV)
    w = buf.view(2100, stride)[:, :64]
    w.copy_(torch.randn((2100, 64), generator=g, device=DEV) * 0.3)
    q = su.rows(g, 10, 64, torch.bfloat16)
    targets = torch.full((10,), 2099, dtype=torch.int32, device=DEV)
    check(q, w.contiguous(), "bf16", targets, None, 10, 1.0, su.run_log_probs(q, w, "bf16", targets, top=10))


def test_outputs_that_are_not_asked_for_and_no_queries():
    g = su.gen(4)
    q, w = su.rows(g, 12, 30, torch.float16), su.rows(g, 90, 30, torch.float16)
    p = su.problem(q, w, "fp16")
    ws = su.workspace(mar.mar_log_probs_workspace_bytes(p, 0))
    en = torch.empty(12, device=DEV)
    mar.mar_log_probs(p, q, w, None, None, 0, 0, None, en, None, None, ws, ws.numel())
    assert torch.equal(en, su.run_log_probs(q, w, "fp16", top=3)[1])
    p.num_queries = 0
    mar.mar_log_probs(p, None, w, None, None, 0, 4, None, None, None, None, ws, ws.numel())
    torch.cuda.synchronize()


def test_equal_bits_on_another_stream_and_in_a_replayed_graph():
    g = su.gen(6)
    q, w = su.rows(g, 200, 100, torch.float32), su.rows(g, 6000, 100, torch.float32)
    targets = torch.randint(0, 6000, (200,), generator=g, device=DEV, dtype=torch.int32)
    want = su.run_log_probs(q, w, "fp32", targets, top=10)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = su.run_log_probs(q, w, "fp32", targets, top=10)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    p = su.problem(q, w, "fp32")
    ws = [su.workspace(mar.mar_log_probs_workspace_bytes(p, 10)) for _ in range(2)]
    outs, graphs = [], []
    for i in range(2):                                       # two graphs, a workspace each
        out = [torch.zeros_like(x) for x in want]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            mar.mar_log_probs(p, q, w, targets, None, 0, 10, out[0], out[1], out[2], out[3], ws[i], ws[i].numel())
        outs.append(out)
        graphs.append(graph)
    for seed in range(4):
        q.copy_(su.rows(su.gen(100 + seed), 200, 100, torch.float32))
        want = su.run_log_probs(q, w, "fp32", targets, top=10)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(x, y) for x, y in zip(out, want)), seed
