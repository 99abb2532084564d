"""GPU parity of mar_sample_rows with its definition in extended precision: ids and counts are equal, log probabilities to their rounding."""
import numpy as np
import pytest
import torch

import mxfp_util as mu
import paper_2101_08358_amd as mar

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": (torch.float32, mar.DTYPE_FP32), "bf16": (torch.bfloat16, mar.DTYPE_BF16), "fp16": (torch.float16, mar.DTYPE_FP16)}


def words(allowed):
    """Rows of truth values as rows of 32-bit words."""
    n, V = allowed.shape
    bits = np.zeros((n, (V + 31) // 32 * 32), dtype=np.uint8)
    bits[:, :V] = allowed
    return np.packbits(bits, axis=1, bitorder="little").view(np.uint32).view(np.int32)


def on_device(values, dtype):
    return None if values is None else torch.tensor(values, dtype=dtype, device=DEV)


def sample(s, uniforms, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, allowed=None, shared_mask=False, arrays=(None,) * 4, stream=None, outputs=True):
    """s: device rows of any stride; allowed: device words or None."""
    Q, V = s.shape
    n = uniforms.shape[1]
    dtype = {t: d for t, d in TYPES.values()}[s.dtype]
    p = mar.MarSampling(V, s.stride(0) if Q > 1 else V, Q, n, dtype, top_k, temperature, top_p, min_p, 0)
    ws = torch.full((mar.mar_sample_rows_workspace_bytes(p),), 0xA5, dtype=torch.uint8, device=DEV)
    ids = torch.full((Q, n), -9, dtype=torch.int32, device=DEV)
    lp = torch.full((Q, n), 9.0, device=DEV) if outputs else None
    kept = torch.full((Q,), -9, dtype=torch.int32, device=DEV) if outputs else None
    arrays = [on_device(a, torch.int32 if i == 1 else torch.float32) for i, a in enumerate(arrays)]
    stride = 0 if allowed is None or shared_mask else allowed.stride(0) if Q > 1 else allowed.shape[1]
    mar.mar_sample_rows(p, s, allowed, stride, *arrays, uniforms, ids, lp, kept, ws, ws.numel(), stream)
    torch.cuda.synchronize()
    return ids, lp, kept


def check(s, uniforms, allowed=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, arrays=(None,) * 4):
    """allowed: truth values [Q, V] or [1, V] (shared) or None."""
    mask = None if allowed is None else torch.from_numpy(words(allowed)).to(DEV)
    Q = s.shape[0]
    shared = allowed is not None and allowed.shape[0] == 1
    got = sample(s, uniforms, temperature, top_k, top_p, min_p, mask, shared, arrays)
    ids, lp, kept = (t.cpu().numpy() for t in got)
    host, u = s.double().cpu().numpy(), uniforms.double().cpu().numpy()
    one = (np.float32(temperature), top_k, np.float32(top_p), np.float32(min_p))
    for i in range(Q):
        par = [float(np.float32(a[i])) if a is not None else float(o) for a, o in zip(arrays, one)]
        par[1] = int(par[1])
        ok = None if allowed is None else allowed[0 if shared else i]
        want_ids, want_lp, want_kept = mu.draws(host[i], ok, *par, u[i])
        assert kept[i] == want_kept, (i, par, kept[i], want_kept)
        assert np.array_equal(ids[i], want_ids), (i, par, np.nonzero(ids[i] != want_ids)[0][:5], ids[i][:5], want_ids[:5])
        inf = np.isinf(want_lp)
        assert np.array_equal(np.isinf(lp[i]), inf)
        # one rounding to fp32 of a difference whose terms are below 2^7 in 64 bits
        assert (np.abs(lp[i][~inf] - want_lp[~inf]) <= np.abs(want_lp[~inf]) * 2.0 ** -24 + 2.0 ** -40).all()
    return got


def scores_of(seed, Q, V, dtype, spread=2.5, pad=0, offset=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((Q, V), generator=g) * spread).to(dtype)
    buf = torch.full((offset + Q * (V + pad),), float("nan"), dtype=dtype, device=DEV)
    s = buf[offset:].view(Q, V + pad)[:, :V]
    s.copy_(x)
    return s


def uniforms_of(seed, Q, n):
    return torch.rand((Q, n), generator=torch.Generator().manual_seed(seed + 1000)).to(DEV)


SIZES = ((1, 1, 1), (3, 2, 5), (2, 7, 4), (2, 31, 8), (2, 33, 8), (3, 511, 16), (3, 512, 16), (2, 513, 33), (4, 1000, 20), (2, 4097, 50), (3, 14_951, 64), (2, 40_001, 17), (1, 200_003, 40))
FILTERS = (dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05), dict(temperature=1.3, top_k=300, top_p=0.8, min_p=0.01),
           dict(top_k=3000, top_p=0.95), dict(temperature=0.0), dict(temperature=0.05, top_p=0.5))


@pytest.mark.parametrize("tname", TYPES)
@pytest.mark.parametrize("Q,V,n", SIZES)
def test_draws(Q, V, n, tname):
    odd = V % 2
    s = scores_of(Q + V, Q, V, TYPES[tname][0], pad=3 * odd, offset=odd)
    u = uniforms_of(V, Q, n)
    for f in FILTERS:
        check(s, u, **f)


@pytest.mark.parametrize("tname", TYPES)
@pytest.mark.parametrize("V", (65, 3001, 20_000))
def test_masks(V, tname):
    """Half of the rows, all but a few, a few, one, none; masked rows may hold anything."""
    g = np.random.default_rng(V)
    allowed = np.stack((g.random(V) < 0.5, g.random(V) < 0.98, g.random(V) < 3 / V, np.arange(V) == V - 1, np.zeros(V, dtype=bool), np.ones(V, dtype=bool)))
    s = scores_of(V, 6, V, TYPES[tname][0])
    bad = torch.from_numpy(~allowed).to(DEV)
    s.masked_fill_(bad, float("nan"))
    s[:, ::3] = torch.where(bad[:, ::3], torch.full((), float("inf"), dtype=s.dtype, device=DEV), s[:, ::3])
    for f in (dict(), dict(top_k=40, top_p=0.9), dict(min_p=0.1), dict(temperature=0.0), dict(top_p=0.7)):
        got = check(s, uniforms_of(V, 6, 9), allowed, **f)
        assert (got[0][4] == -1).all() and got[2][4] == 0
        check(s[:1].expand(1, V), uniforms_of(V, 1, 9), allowed[:1], **f)
    shared = g.random((1, V)) < 0.3
    check(scores_of(V + 1, 4, V, TYPES[tname][0]), uniforms_of(V, 4, 9), shared, top_p=0.9)


def test_every_query_has_its_own_parameters():
    """Special values among them: what is off, and what leaves the best row alone."""
    nan, inf = float("nan"), float("inf")
    T = (1.0, 0.0, -1.0, nan, inf, 1e-30, 1e30, 0.5, 2.0, 1e-45, 0.9, 1.0, 1.0, 1.0, 1.0, 1.0)
    k = (0, 0, 5, 5, 0, 0, 7, -3, 1 << 30, 0, 20, 0, 0, 0, 0, 100)
    p = (1.0, 0.5, 0.9, 1.0, 0.3, 0.9, 0.5, 2.0, nan, 0.9, 0.0, -1.0, 0.9999999, 1e-20, 0.5, 0.999)
    m = (0.0, 0.5, 0.0, 0.0, 0.0, 0.0, 0.1, -1.0, nan, 0.0, 0.0, 0.0, 0.0, 0.0, 1.0, 2.0)
    for tname in TYPES:
        s = scores_of(5, 16, 3000, TYPES[tname][0])
        check(s, uniforms_of(5, 16, 12), arrays=(T, k, p, m))
        check(s, uniforms_of(6, 16, 12), arrays=(None, k, None, m), temperature=0.8, top_p=0.9)
        check(s, uniforms_of(7, 16, 12), arrays=(T, None, p, None), top_k=60, min_p=0.02)


@pytest.mark.parametrize("tname", TYPES)
def test_equal_scores_go_by_id(tname):
    """Rows that score alike: all of them, and groups across the borders of top-k and top-p."""
    V = 5000
    g = np.random.default_rng(4)
    s = torch.from_numpy(np.stack((np.full(V, 1.5), g.integers(0, 4, V) * 0.5, np.where(g.random(V) < 0.01, 3.0, 0.25), g.integers(-3, 3, V) * 1.0, np.full(V, -0.0)))).to(TYPES[tname][0]).to(DEV)
    s[4, ::2] = 0.0                                           # 0 and -0 are one
    u = uniforms_of(4, 5, 30)
    for f in (dict(), dict(top_k=1), dict(top_k=60), dict(top_k=1234), dict(top_k=4999), dict(top_p=0.5), dict(top_p=0.25, top_k=2000), dict(top_p=1e-9),
              dict(min_p=1.0), dict(min_p=1.0, top_k=7), dict(top_p=0.75, min_p=0.5)):
        check(s, u, **f)


@pytest.mark.parametrize("tname", TYPES)
def test_infinities_nan_and_the_ends_of_the_range(tname):
    inf, nan = float("inf"), float("nan")
    big = torch.finfo(TYPES[tname][0]).max
    s = torch.zeros((8, 700), dtype=TYPES[tname][0], device=DEV)
    s[0, 5], s[0, 6] = inf, nan                               # one infinite score takes all
    s[1, 5], s[1, 600] = inf, inf
    s[2] = -inf
    s[2, 699] = -big
    s[3] = nan
    s[4] = -inf
    s[5, :350], s[5, 350:] = big, -big
    s[6, ::7], s[6, 1::7] = nan, -inf
    s[7] = torch.randn(700, generator=torch.Generator().manual_seed(1)) * 30
    for f in (dict(), dict(temperature=1e-3), dict(temperature=1e38), dict(top_k=3), dict(top_p=0.9), dict(min_p=0.3)):
        got = check(s, uniforms_of(3, 8, 20), **f)
        assert (got[0][3:5] == -1).all()


def test_given_numbers_at_their_ends():
    """0, the largest below 1, and numbers outside [0, 1); a number on a border belongs to the row above it."""
    s = scores_of(2, 2, 900, torch.float32)
    s[1, :] = -float("inf")
    s[1, [100, 300, 600, 800]] = 2.0                          # four rows of a quarter each
    u = torch.tensor([[0.0, 1.0 - 2.0 ** -24, 1.0, 5.0, -1.0, float("nan"), 2.0 ** -149, 2.0 ** -30, 0.5, float("inf")]] * 2, device=DEV)
    check(s, u)
    # floats below 3/4 lie 2^-24 apart: 3/4 - 2^-25 is rounded to 3/4
    ids = sample(s[1:].clone(), torch.tensor([[0.0, 0.25 - 2.0 ** -26, 0.25, 0.5, 0.75 - 2.0 ** -25, 0.75, 1.0, 0.75 - 2.0 ** -24]], device=DEV))[0]
    assert ids.tolist() == [[100, 100, 300, 600, 800, 800, 800, 600]]


def test_few_outputs_and_repeated_calls():
    s = scores_of(9, 5, 3000, torch.bfloat16)
    u = uniforms_of(9, 5, 8)
    want = sample(s, u, top_k=100, top_p=0.9)
    assert torch.equal(sample(s, u, top_k=100, top_p=0.9, outputs=False)[0], want[0])
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(sample(s, u, top_k=100, top_p=0.9), want))


def test_frequencies_follow_the_weights():
    """60,000 draws: every row's count within five standard deviations of what its weight says."""
    s = torch.tensor([[0.0, 1.0, 2.0, -1.0, 0.5, 1.5]], device=DEV)
    n = 60_000
    ids = sample(s, uniforms_of(1, 1, n), temperature=0.8)[0]
    p = torch.softmax(s[0].cpu() / 0.8, 0).numpy()
    count = np.bincount(ids[0].cpu().numpy(), minlength=6)
    assert (np.abs(count - n * p) <= 5 * np.sqrt(n * p * (1 - p))).all()


def test_a_long_row_with_a_heavy_best_row():
    """Ten million rows below a best one that outweighs each of them by e^14: their draws still fall where 64 bits say."""
    V = 10_000_019
    g = torch.Generator(device=DEV).manual_seed(3)
    s = torch.randn((1, V), generator=g, device=DEV) * 0.01
    s[0, 77] = 14.0
    u = uniforms_of(8, 1, 200)
    check(s, u)
    check(s, u, top_p=0.8)


def test_offsets_beyond_32_bits():
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    far, V = 3 << 30, 3000
    x = torch.empty(2 * far + V, dtype=torch.bfloat16, device=DEV)
    s = torch.as_strided(x, (3, V), (far, 1))
    s.copy_(torch.randn((3, V), generator=torch.Generator().manual_seed(3)) * 2)
    check(s, uniforms_of(8, 3, 20), top_k=100, top_p=0.9)


def test_no_queries():
    p = mar.MarSampling(100, 100, 0, 1, mar.DTYPE_FP32, 0, 1.0, 1.0, 0.0, 0)
    ws = torch.empty(mar.mar_sample_rows_workspace_bytes(p), dtype=torch.uint8, device=DEV)
    mar.mar_sample_rows(p, None, None, 0, None, None, None, None, None, None, None, None, ws, ws.numel())
    torch.cuda.synchronize()
