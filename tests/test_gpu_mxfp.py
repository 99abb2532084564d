"""GPU parity of mar_mxfp_quantise and mar_mxfp_rows with their definition in 64 bits: codes, scales and values are exact."""
import numpy as np
import pytest
import torch

import mxfp_util as mu
import paper_2101_08358_amd as mar

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": (torch.float32, mar.DTYPE_FP32), "bf16": (torch.bfloat16, mar.DTYPE_BF16), "fp16": (torch.float16, mar.DTYPE_FP16)}


def strided(x, stride, offset):
    """The rows of x (host, 64 bits) on the device with a stride and an offset in elements; what lies between them is NaN."""
    rows, dim = x.shape
    buf = torch.full((offset + rows * stride,), float("nan"), dtype=x.dtype, device=DEV)
    view = buf[offset:].view(rows, stride)[:, :dim]
    view.copy_(x)
    return view


def same(got, want):
    """Equal values, infinities among them, and NaN in the same places."""
    none = torch.isnan(want)
    return torch.equal(torch.isnan(got), none) and torch.equal(got.masked_fill(none, 5.0), want.masked_fill(none, 5.0))


def quantise(x, codes_pad=0, scales_pad=0):
    rows, dim = x.shape
    nb = mu.blocks_of(dim)
    codes = torch.full((rows, 16 * nb + codes_pad), 0xA5, dtype=torch.uint8, device=DEV)
    scales = torch.full((rows, nb + scales_pad), 0x5A, dtype=torch.uint8, device=DEV)
    dtype = {t: d for t, d in TYPES.values()}[x.dtype]
    mar.mar_mxfp_quantise(x, max(x.stride(0), dim), rows, dim, dtype, codes, codes.shape[1], scales, scales.shape[1])
    return codes, scales


def check(x, codes_pad=0, scales_pad=0):
    codes, scales = quantise(x, codes_pad, scales_pad)
    nb = mu.blocks_of(x.shape[1])
    want_codes, want_scales = mu.quantise(x.double().cpu().numpy())
    assert np.array_equal(scales[:, :nb].cpu().numpy(), want_scales)
    assert np.array_equal(codes[:, :16 * nb].cpu().numpy(), want_codes)
    assert (codes[:, 16 * nb:] == 0xA5).all() and (scales[:, nb:] == 0x5A).all()
    return codes, scales


@pytest.mark.parametrize("tname", TYPES)
@pytest.mark.parametrize("rows,dim,stride,offset", ((1, 1, 1, 0), (3, 7, 9, 1), (1000, 50, 50, 0), (65, 31, 31, 3), (65, 32, 40, 0), (65, 33, 33, 1),
                                                    (257, 100, 101, 1), (129, 400, 400, 0), (77, 401, 403, 2), (5, 4099, 4099, 1), (2, 3, 1000, 5)))
def test_codes_and_scales_are_exact(rows, dim, stride, offset, tname):
    g = torch.Generator().manual_seed(rows * 1000 + dim)
    x = torch.randn((rows, dim), generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-12, 6, (rows, 1), generator=g).double())
    check(strided(x.to(TYPES[tname][0]), stride, offset), 16 * (rows % 3), rows % 5)


@pytest.mark.parametrize("tname", ("bf16", "fp16"))
def test_every_16_bit_value_alone_and_beside_a_larger_one(tname):
    """All 65,536 bit patterns, subnormals, infinities and NaN among them: as their block's largest value, and as a smaller one."""
    bits = torch.arange(65536, dtype=torch.int32, device=DEV).to(torch.int16).view(TYPES[tname][0])
    alone = torch.zeros((65536, 33), dtype=bits.dtype, device=DEV)
    alone[:, 5] = bits
    check(alone)
    x = torch.zeros((65536, 32), dtype=bits.dtype, device=DEV)
    x[:, 7] = bits
    x[:, 30] = (bits.float() * 1.75).to(bits.dtype)
    x[:, 3] = -(bits.float() * 0.3125).to(bits.dtype)
    check(x)


def test_thresholds_and_ties():
    """Every level, every border between two levels and their neighbours in fp32, at scales from the smallest to the largest."""
    border = np.concatenate((mu.LEVELS, mu.MIDS, [6.5, 7.0, 7.5, 7.9999995]))
    v = np.concatenate([np.nextafter(border.astype(np.float32), np.float32(t)) for t in (-np.inf, np.inf)] + [border.astype(np.float32)]).astype(np.float64)
    v = np.concatenate((v, -v))
    rows = []
    for e in (-127, -126, -125, -120, -60, -1, 0, 1, 60, 120, 124, 125):
        for part in range(0, len(v), 31):
            row = np.zeros(32)
            row[1:1 + len(v[part:part + 31])] = v[part:part + 31]
            row[0] = 4.0                                      # fixes the block's scale at 2^e
            rows.append(row * 2.0 ** e)
    check(torch.from_numpy(np.stack(rows)).to(torch.float32).to(DEV))    # 8 2^125 is infinite


def test_subnormals_zeros_and_values_that_are_not_finite():
    tiny = 2.0 ** -149
    x = torch.zeros((12, 70), device=DEV)
    x[1, 3] = tiny
    x[2, 3], x[2, 4] = 2.0 ** -127, -(2.0 ** -128)            # the smallest scale: levels 2^-127 apart
    x[3, :64] = -0.0
    x[4, 69] = float("inf")
    x[5, 0] = float("nan")
    x[6, 33] = -float("inf")
    x[6, 0] = 1.0
    x[7, 0], x[7, 1] = torch.finfo(torch.float32).max, -1.0e38
    x[8] = tiny
    x[9, 5] = 2.0 ** -126
    x[10, 5], x[10, 6] = 2.0 ** -125, 2.0 ** -130
    codes, scales = check(x)
    assert scales[4].tolist() == [0, 0, 255] and scales[6, 1] == 255 and scales[6, 0] != 255
    for tname in TYPES:
        out = torch.empty((12, 70), dtype=TYPES[tname][0], device=DEV)
        mar.mar_mxfp_rows(codes, 48, scales, 3, 12, 70, None, 12, TYPES[tname][1], out, 70)
        want = torch.from_numpy(mu.values(codes.cpu().numpy(), scales.cpu().numpy(), 70)).to(out.dtype)
        assert same(out.cpu(), want)


@pytest.mark.parametrize("tname", TYPES)
@pytest.mark.parametrize("rows,dim,n,stride,offset", ((1, 1, 1, 1, 0), (10, 7, 33, 9, 1), (1000, 50, 777, 50, 0), (300, 100, 1000, 101, 3), (50, 400, 200, 400, 0), (9, 4099, 20, 4100, 1)))
def test_rows_are_the_values_of_their_codes(rows, dim, n, stride, offset, tname):
    """Random codes and scales over fp32's whole range, ids that come twice and ids outside the table."""
    g = np.random.default_rng(rows + dim)
    nb = mu.blocks_of(dim)
    codes = g.integers(0, 256, (rows, 16 * nb + 16), dtype=np.uint8)
    scales = g.integers(0, 256, (rows, nb + 2), dtype=np.uint8)
    scales[::2] = g.integers(100, 140, scales[::2].shape, dtype=np.uint8)
    ids = g.integers(-2, rows + 2, n).astype(np.int32)
    dt, code = TYPES[tname]
    c, s = torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV)
    buf = torch.full((offset + n * stride,), 5.0, dtype=dt, device=DEV)
    out = buf[offset:].view(n, stride)[:, :dim]
    mar.mar_mxfp_rows(c, codes.shape[1], s, scales.shape[1], rows, dim, torch.from_numpy(ids).to(DEV), n, code, out, stride)
    want = np.zeros((n, dim))
    inside = (ids >= 0) & (ids < rows)
    want[inside] = mu.values(codes[:, :16 * nb], scales[:, :nb], dim)[ids[inside]]
    want = torch.from_numpy(want).to(torch.float32).to(dt)    # two bits of mantissa: the first rounding is exact or infinite
    assert same(out.cpu(), want)
    assert (buf[:offset] == 5.0).all() and (buf[offset:].view(n, stride)[:, dim:] == 5.0).all()


def test_nothing_to_do_and_an_empty_table():
    mar.mar_mxfp_quantise(None, 8, 0, 8, mar.DTYPE_FP32, None, 16, None, 1)
    mar.mar_mxfp_rows(None, 16, None, 1, 5, 8, None, 0, mar.DTYPE_FP32, None, 8)
    out = torch.full((3, 8), 5.0, device=DEV)
    mar.mar_mxfp_rows(None, 16, None, 1, 0, 8, torch.zeros(3, dtype=torch.int32, device=DEV), 3, mar.DTYPE_FP32, out, 8)
    torch.cuda.synchronize()
    assert (out == 0).all()


def test_offsets_beyond_32_bits():
    """Rows 2^31 bytes and elements apart, and a table of more than 2^32 bytes of codes."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    far = 3 << 30
    x = torch.empty(2 * far + 100, dtype=torch.bfloat16, device=DEV)
    rows = torch.as_strided(x, (3, 100), (far, 1))
    rows.copy_(torch.randn((3, 100), generator=torch.Generator().manual_seed(3)))
    codes = torch.empty(2 * far + 64, dtype=torch.uint8, device=DEV)
    scales = torch.empty(2 * far + 4, dtype=torch.uint8, device=DEV)
    mar.mar_mxfp_quantise(x, far, 3, 100, mar.DTYPE_BF16, codes, far, scales, far)
    want_codes, want_scales = mu.quantise(rows.double().cpu().numpy())
    assert np.array_equal(torch.as_strided(codes, (3, 64), (far, 1)).cpu().numpy(), want_codes)
    assert np.array_equal(torch.as_strided(scales, (3, 4), (far, 1)).cpu().numpy(), want_scales)
    ids = torch.tensor([2, 0, 2, 1], dtype=torch.int32, device=DEV)
    mar.mar_mxfp_rows(codes, far, scales, far, 3, 100, ids, 3, mar.DTYPE_BF16, x, far)
    want = torch.from_numpy(mu.values(want_codes, want_scales, 100)[[2, 0, 2]]).to(torch.bfloat16)
    assert torch.equal(rows.cpu(), want)
