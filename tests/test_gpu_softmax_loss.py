"""GPU parity of mar_softmax_loss with 64 bits and with differences: sizes at and beside tiles, stripes and widths, every type,
strides, queries without an answer, weights of either sign, confident queries, streams and graphs."""
import pytest
import torch

import paper_2101_08358_amd as mar
import softmax_util as su

pytestmark = pytest.mark.gpu
DEV = su.DEV

SIZES = ((1, 1, 1), (1, 31, 3), (5, 33, 8), (3, 100, 17), (130, 257, 50), (64, 1000, 75), (129, 2049, 100), (33, 5000, 128), (7, 700, 200),
         (40, 1000, 256), (70, 999, 400), (600, 300, 52), (1, 40_000, 100), (4097, 129, 64), (513, 4097, 96), (2, 3000, 129), (32, 64, 112),
         (300, 1025, 33), (2000, 31, 400), (65, 2000, 193), (1500, 600, 384), (400, 900, 150))


def make(T, V, d, tname, odd, hot=False):
    g = su.gen(T * 7 + V + d)
    dt = su.TYPES[tname][0]
    q = su.rows(g, T, d, dt, stride=d + 3 * odd, offset=odd)
    w = su.rows(g, V, d, dt, stride=d + 5 * odd, offset=3 * odd)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    if hot:
        targets[::2] = V // 2
    return g, q, w, targets


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
@pytest.mark.parametrize("T,V,d", SIZES)
def test_against_64_bits(T, V, d, tname):
    print("case", T, V, d, tname, flush=True)
    odd = (T + V) % 2
    g, q, w, targets = make(T, V, d, tname, odd, hot=T % 3 == 0)
    weights = torch.randn(T, generator=g, device=DEV) if T % 2 else None
    scale = (1.0, 0.7, 2.5)[V % 3]
    gq = su.rows(g, T, d, q.dtype, stride=d + 7 * odd, offset=odd)
    gw = su.rows(g, V, d, w.dtype, stride=d + 1 * odd, offset=odd)
    out = su.run_loss(q, w, tname, targets, weights, scale, gq=gq, gw=gw)
    su.check_loss(out, q, w, tname, targets, weights, scale)


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
def test_queries_without_an_answer(tname):
    """Their values, NaN and infinities among them, touch nothing; every id outside the table counts as none."""
    g, q, w, targets = make(300, 777, 60, tname, 1)
    targets[::5] = -1
    targets[3::50] = 777
    targets[4::50] = 2 ** 31 - 1
    targets[6::50] = -2 ** 31
    none = (targets < 0) | (targets >= 777)
    q[none] = torch.tensor([float("nan"), float("inf"), 1e4], device=DEV).to(q.dtype).repeat(20)
    out = su.run_loss(q, w, tname, targets)
    assert (out[0][none] == 0).all() and (out[2][none] == 0).all()
    kept = ~none
    ref = su.run_loss(q[kept].contiguous(), w, tname, targets[kept].contiguous())
    su.check_loss(ref, q[kept], w, tname, targets[kept], None, 1.0)
    clean = q.clone()
    clean[none] = 0
    su.check_loss((out[0], None, out[2], out[3]), clean, w, tname, targets, None, 1.0)
    targets[:] = -1
    loss, _, gq, gw = su.run_loss(q, w, tname, targets)
    assert not loss.any() and not gq.any() and not gw.any()


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
def test_confident_queries(tname):
    """Every query's answer has nearly all of its probability: p - 1 cancels, and the gradient is what is left."""
    g, q, w, targets = make(200, 400, 64, tname, 0)
    dt = q.dtype
    q.copy_((w[targets.long()].float() * 6.0).to(dt))
    s = su.scores(q, w, 1.0)
    p = torch.exp(s - torch.logsumexp(s, 1, keepdim=True))[torch.arange(200, device=DEV), targets.long()]
    assert float(p.median()) > 0.99
    out = su.run_loss(q, w, tname, targets)
    su.check_loss(out, q, w, tname, targets, None, 1.0)
    # the bound above takes the answer's weight for 2: here it is 1 - p, known to 2^-20 of itself and of p
    _, _, D, A = su.loss_reference(q, w, targets, None, 1.0)
    ref, eps = D @ w.double(), su.WEIGHT_EPS[tname]
    size = D.abs() @ w.double().abs()
    noise = (2 * (su.score_error(q, w, 1.0) + su.sum_error(400)) + 2.0 ** -20) * (A @ w.double().abs())
    err = (out[2].double() - ref).abs()
    assert (err <= size * eps + noise + ref.abs() * su.half_step(dt) + 1e-7).all(), float((err / (size * eps + noise + 1e-7)).max())


def test_weights_of_any_size():
    """Gradients are proportional to the weights, from 2^-30 to 2^30, of either sign, zeros among them."""
    for tname in ("fp32", "bf16"):
        g, q, w, targets = make(500, 900, 100, tname, 0)
        u = torch.randn(500, generator=g, device=DEV) * torch.exp2(torch.randint(-30, 31, (500,), generator=g, device=DEV).float())
        u[::7] = 0.0
        su.check_loss(su.run_loss(q, w, tname, targets, u), q, w, tname, targets, u, 1.0)


def test_weights_that_count_as_none():
    """Below 2^-100, the smallest floats among them: zero, also where the query is not finite."""
    for tname in ("fp32", "bf16", "fp16"):
        g, q, w, targets = make(130, 300, 48, tname, 0)
        u = torch.ones(130, device=DEV)
        u[::4], u[1::8] = 2.0 ** -149, -(2.0 ** -101)
        clean = u.clone()
        clean[u.abs() < 2.0 ** -100] = 0.0
        q[4] = float("nan")
        loss, _, gq, gw = su.run_loss(q, w, tname, targets, u)
        assert not loss[clean == 0].any() and not gq[clean == 0].any()
        q[4] = 0
        su.check_loss((loss, None, gq, gw), q, w, tname, targets, clean, 1.0)


def test_two_calls_at_once():
    """Two streams, a workspace each, enqueued one beside the other: the bits of either alone."""
    cases = [make(900, 4000, 100, "fp32", 0)[1:], make(1200, 3000, 64, "bf16", 0)[1:]]
    want = [su.run_loss(q, w, t, targets) for (q, w, targets), t in zip(cases, ("fp32", "bf16"))]
    probs = [su.run_log_probs(q, w, t, targets, top=7) for (q, w, targets), t in zip(cases, ("fp32", "bf16"))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for st, (q, w, targets), t in zip(streams, cases, ("fp32", "bf16")):
            with torch.cuda.stream(st):
                got.append((su.run_loss(q, w, t, targets), su.run_log_probs(q, w, t, targets, top=7)))
        torch.cuda.synchronize()
        for (a, b), x, y in zip(got, want, probs):
            assert all(torch.equal(m, n) for m, n in zip(a, x)) and all(torch.equal(m, n) for m, n in zip(b, y))


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
def test_large_scores(tname):
    g, q, w, targets = make(150, 2100, 100, tname, 0)
    q *= 6
    w *= 6
    su.check_loss(su.run_loss(q, w, tname, targets), q, w, tname, targets, None, 1.0)
    su.check_loss(su.run_loss(q.abs(), -w.abs(), tname, targets), q.abs(), -w.abs(), tname, targets, None, 1.0)


def test_rows_of_very_different_size():
    """fp32 rows from 1 to 2^-40 beside one another, blocks of zeros, queries likewise."""
    g, q, w, targets = make(260, 1100, 100, "fp32", 0)
    w *= torch.exp2(torch.randint(-40, 1, (1100, 1), generator=g, device=DEV).float())
    q *= torch.exp2(torch.randint(-40, 1, (260, 1), generator=g, device=DEV).float())
    w[64:96] = 0
    q[8:16] = 0
    su.check_loss(su.run_loss(q, w, "fp32", targets), q, w, "fp32", targets, None, 1.0)
    su.check_loss(su.run_loss(q, w * 0, "fp32", targets), q, w * 0, "fp32", targets, None, 1.0)


def test_gradients_against_differences():
    """Central differences of the losses' sum that the operator itself returns (fp32, a step of 2^-5: the third derivative's part,
    h^2 / 6 |f'''| <= 2^-10 / 6 of order 1 quantities, and 300 losses' rounding, 2^-20 / 2^-5 each)."""
    T, V, d = 30, 70, 12
    g, q, w, targets = make(T, V, d, "fp32", 0)
    weights = torch.rand(T, generator=g, device=DEV) + 0.5
    _, _, gq, gw = su.run_loss(q, w, "fp32", targets, weights, 1.3)
    step = 2.0 ** -5
    for matrix, grad in ((q, gq), (w, gw)):
        for r, c in ((0, 0), (3, 5), (29, 11), (17, 2)):
            at = matrix[r, c].clone()
            sums = []
            for sign in (1, -1):
                matrix[r, c] = at + sign * step
                sums.append(su.run_loss(q, w, "fp32", targets, weights, 1.3, want=("loss",))[0].double().sum())
            matrix[r, c] = at
            assert abs(float(sums[0] - sums[1]) / (2 * step) - float(grad[r, c])) < 2e-3, (r, c)


def test_outputs_that_are_not_asked_for_and_no_queries():
    g, q, w, targets = make(100, 300, 40, "bf16", 0)
    full = su.run_loss(q, w, "bf16", targets)
    for want in (("loss",), ("lse",), ("gq",), ("gw",), ("loss", "gw"), ()):
        got = su.run_loss(q, w, "bf16", targets, want=want)
        for name, a, b in zip(("loss", "lse", "gq", "gw"), got, full):
            assert (a is None) == (name not in want) and (a is None or torch.equal(a, b))
    none = q[:0]
    _, _, _, gw = su.run_loss(none, w, "bf16", targets[:0])
    assert not gw.any()
    big = torch.full((300, 48), 5.0, dtype=torch.bfloat16, device=DEV)          # only the rows' own columns are written
    su.run_loss(q, w, "bf16", targets, gw=big[:, :40])
    assert torch.equal(big[:, :40], full[3]) and (big[:, 40:] == 5.0).all()


@pytest.mark.parametrize("tname", ("fp32", "bf16", "fp16"))
def test_equal_bits_on_another_stream_and_in_a_replayed_graph(tname):
    g, q, w, targets = make(700, 3000, 100, tname, 0, hot=True)
    want = su.run_loss(q, w, tname, targets)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = su.run_loss(q, w, tname, targets)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    p = su.problem(q, w, tname)
    ws = su.workspace(mar.mar_softmax_loss_workspace_bytes(p))
    out = [torch.zeros_like(x) for x in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mar.mar_softmax_loss(p, q, w, targets, None, out[0], out[1], out[2], 100, out[3], 100, ws, ws.numel())
    for seed in range(4):
        q.copy_(su.rows(su.gen(100 + seed), 700, 100, q.dtype))
        want = su.run_loss(q, w, tname, targets)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)), seed
