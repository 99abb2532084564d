"""Queries whose blocks hold magnitudes far apart, against rows that leave the large ones out: what the small ones give has to stay.

Bounds: a score may be off by its sums in fp32 and by 2^-24 of every value, as a plain product would be.  Queries here have blocks that
take further images, or values that enter with all their bits."""
import numpy as np
import pytest
import torch

import mxfp_util as mu
import paper_2101_08358_amd as mar
from test_gpu_mxfp_scores import DEV, TYPES, scores, table

pytestmark = pytest.mark.gpu
COUNTS = (1, 5, 8, 9, 16, 31, 32, 33, 70, 200)               # few queries in one image and in several; many


def rows_without(g, V, dim, outliers):
    """A table whose odd rows have code 0 at the outliers' columns."""
    codes, scales = table(g, V, dim)
    v = np.stack((codes & 15, codes >> 4), axis=2).reshape(V, -1)
    for c in outliers:
        v[1::2, c] = 0
    return (v[:, 0::2] | (v[:, 1::2] << 4)).astype(np.uint8), scales


def check(x, codes, scales, kind):
    """x: 64-bit queries, whose values differ by less than 2 from the largest of their image or enter with all their bits."""
    T, dim = x.shape
    q = torch.from_numpy(x).to(TYPES[kind][0])
    x = q.double().numpy()
    w = mu.values(codes, scales, dim)
    got = scores(q.to(DEV), torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), dim, kind).double().cpu().numpy()
    size = np.abs(x) @ np.abs(w).T
    # a step of 64 columns rounds its sum twice at most, four images have a sum of such steps each or their steps one after the other; a slice
    # adds 1/31 of the one before it.  24 bits below an image's largest of [2^e, 2^(e + 1)) leave half of 2^(e - 23): 2^-24 of such a value
    bound = size * ((2 * 4 * ((dim + 63) // 64) + 4) * 2.0 ** -23 * (32 / 31) + 2.0 ** -24)
    off = np.abs(got - x @ w.T)
    assert (off <= bound).all(), (float((off / np.maximum(bound, 1e-300)).max()), np.argwhere(off > bound)[:3])


@pytest.mark.parametrize("kind", ("fp32", "bf16", "fp16"))
def test_a_large_value_beside_ones(kind):
    """Whole numbers: every score is exact."""
    power = {"fp32": 26, "bf16": 20, "fp16": 15}[kind]
    V, dim = 200, 32
    codes, scales = np.full((V, 16), 0x22, dtype=np.uint8), np.full((V, 1), 127, dtype=np.uint8)       # ones
    codes[:, 0] = 0x20                                       # 0 in column 0
    for T in COUNTS:
        x = np.ones((T, dim))
        x[:, 0] = 2.0 ** power
        got = scores(torch.from_numpy(x).to(TYPES[kind][0]).to(DEV), torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), dim, kind)
        assert (got == 31).all()
    small = 2.0 ** -24 if kind == "fp16" else 2.0 ** -40     # the least of fp16 beside its largest power
    x = np.full((3, dim), small)
    x[:, 0] = 2.0 ** 15
    got = scores(torch.from_numpy(x).to(TYPES[kind][0]).to(DEV), torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), dim, kind)
    assert (got.double() == 31 * small).all()


@pytest.mark.parametrize("dim", (32, 50, 75, 128, 200, 400))
@pytest.mark.parametrize("kind,power", [(k, p) for k in ("fp32", "bf16", "fp16") for p in (7, 10, 13, 20, 40, 100, 200) if k != "fp16" or p <= 13])
def test_outliers_do_not_take_their_neighbours_bits(dim, kind, power):
    """A value or two 2^power times the others, in some blocks of some queries."""
    g = np.random.default_rng(dim + power)
    V = 700
    columns = [c for c in (3, 17, 40, 130, 131, 350) if c < dim]
    codes, scales = rows_without(g, V, dim, columns)
    for T in COUNTS:
        x = (1.0 + g.random((T, dim))) * np.where(g.random((T, dim)) < 0.5, -1.0, 1.0)       # magnitudes 1 .. 2
        if power > 100: x *= 2.0 ** -90
        for c in columns:
            x[g.random(T) < 0.7, c] *= 2.0 ** power
        check(x, codes, scales, kind)


@pytest.mark.parametrize("kind", ("fp32", "bf16"))
def test_several_sizes_in_a_block(kind):
    """Four of them, each far below the last, and rows that have codes for one of them alone."""
    g = np.random.default_rng(1)
    dim, V = 96, 400
    size = np.exp2(np.array([80.0, 45.0, 10.0, -30.0]))[np.arange(dim) % 4]
    codes, scales = table(g, V, dim)
    v = np.stack((codes & 15, codes >> 4), axis=2).reshape(V, -1)
    v[(np.arange(dim)[None, :] % 4) != (np.arange(V)[:, None] % 4)] = 0
    codes = (v[:, 0::2] | (v[:, 1::2] << 4)).astype(np.uint8)
    for T in COUNTS:
        check((1.0 + g.random((T, dim))) * size, codes, scales, kind)


@pytest.mark.parametrize("kind", ("bf16", "fp16"))
@pytest.mark.parametrize("T,dim", ((3, 75), (40, 200), (100, 400)))
def test_16_bit_queries_enter_with_all_their_bits(T, dim, kind):
    """Magnitudes over 13 binary orders (fp16) and 16 (bf16): with their own bits these are the 24 below a block's largest."""
    g = np.random.default_rng(T)
    x = (1.0 + g.random((T, dim))) * np.exp2(-g.integers(0, 13 if kind == "fp16" else 16, (T, dim)).astype(np.float64))
    codes, scales = table(g, 900, dim)
    check(x * np.where(g.random((T, dim)) < 0.5, -1.0, 1.0), codes, scales, kind)


@pytest.mark.parametrize("kind", ("fp32", "bf16", "fp16"))
def test_values_that_are_not_finite_beside_outliers(kind):
    g = np.random.default_rng(3)
    dim, V = 130, 300
    codes, scales = rows_without(g, V, dim, (5, 100))
    for T in (4, 20, 50):
        x = 1.0 + g.random((T, dim))
        x[:, 5] *= 2.0 ** 13
        x[1, 40], x[3, 129], x[T - 1, 2] = np.inf, np.nan, -np.inf
        q = torch.from_numpy(x).to(TYPES[kind][0])
        got = scores(q.to(DEV), torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), dim, kind)
        bad = torch.zeros(T, dtype=torch.bool)
        bad[[1, 3, T - 1]] = True
        assert torch.equal(torch.isnan(got).all(1).cpu(), bad) and torch.equal(torch.isnan(got).any(1).cpu(), bad)
        check(np.where(bad.numpy()[:, None], 0.0, x), codes, scales, kind)


@pytest.mark.parametrize("kind", ("fp32", "bf16", "fp16"))
@pytest.mark.parametrize("T", (1, 9, 32, 40, 100))
def test_captured_with_other_queries_later(T, kind):
    """A graph captured with ordinary queries serves others that have outliers, and ordinary ones again; its workspace holds anything."""
    g = np.random.default_rng(T)
    V, dim = 900, 200
    codes, scales_ = rows_without(g, V, dim, (3, 70))
    c, s = torch.from_numpy(codes).to(DEV), torch.from_numpy(scales_).to(DEV)
    q = torch.zeros((T, dim), dtype=TYPES[kind][0], device=DEV)
    out = torch.zeros((T, V), device=DEV)
    p = mar.MarMxfp(V, codes.shape[1], scales_.shape[1], dim, 0, V, T, dim, TYPES[kind][1], mar.DTYPE_FP32, 1.0, 0)
    ws = torch.zeros(mar.mar_mxfp_scores_workspace_bytes(p) + 256, dtype=torch.uint8, device=DEV)

    def call():
        mar.mar_mxfp_scores(p, q, None, c, s, out, ws, ws.numel() - 256)

    def queries(turn):
        x = torch.randn((T, dim), generator=torch.Generator().manual_seed(turn))
        if turn % 2:
            x[::2, 3] *= 2.0 ** 12
            x[::3, 70] *= 2.0 ** 12
        return x.to(q.dtype)

    q.copy_(queries(0))
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(1, 6):
        q.copy_(queries(turn))
        call()
        torch.cuda.synchronize()
        want = out.clone()
        out.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and (ws[-256:] == 0xFF).all()
        x = q.double().cpu().numpy()
        w = mu.values(codes, scales_, dim)
        # sums as in check.  Half of the values of a block that is not wide are 2^-6 of its largest or more, and hardly one half of 32 normal values
        # is above 2: such a block's largest is below 2^7, and 2^-24 of that is cut off a value at most; a wide one's remainder is less
        bound = np.abs(x) @ np.abs(w).T * (2 * 4 * 4 + 4) * 2.0 ** -23 * (32 / 31) + 2.0 ** -17 * np.abs(w).sum(1)
        assert (np.abs(want.double().cpu().numpy() - x @ w.T) <= bound).all()
