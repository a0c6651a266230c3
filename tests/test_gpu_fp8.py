"""8-bit linear layers (f3dc_quantize_fp8, f3dc_gemm_fp8, f3dc_norm_residual) against
a plain 64-bit evaluation: every size where a tile, a block or a vector ends, the
epilogues, strides, pad rows, non-finite values, streams, graphs, and the three
together as the MLP half of a transformer block."""
import numpy as np
import pytest
import torch

import fp8_ref as R
from paper_2511_22533_gb300 import f3dc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(*shape, seed, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen(seed), device=DEV) * scale).to(dtype)


def quantize(x, q=None, s=None, **kw):
    rows, cols = x.shape
    if q is None:
        q, s = R.storage(rows, cols)
    f3dc.quantize_fp8(x, x.stride(0), q, q.stride(0), s, s.stride(0), rows, cols, **kw)
    return q, s


def gemm8(A, sa, B, sb, K, epi, bias=None, gate=None, out=None, out_scales=None, **kw):
    M, N = A.shape[0], B.shape[0]
    f3dc.gemm_fp8(A, A.stride(0), sa, sa.stride(0), B, B.stride(0), sb, sb.stride(0), bias, gate, out, out.stride(0),
                  out_scales, out_scales.stride(0) if out_scales is not None else 0, M, N, K, epi, **kw)


# ------------------------------------------------------------------ quantiser

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 127), (2, 129), (5, 1000), (7, 1024), (1, 4097), (33, 512),
                                       (130, 777), (1000, 640)])
def test_quantize_is_exact(rows, cols, dtype):
    # block maxima from 2^-60 to 2^60, some exactly at and next to 448 2^e
    x = randn(rows, cols, seed=rows + cols)
    x = x * torch.exp2(torch.randint(-60, 60, (rows, 1), generator=gen(1), device=DEV).float())
    x[0, 0] = 448.0
    if rows > 1:
        x[1] = 0.0
        x[rows - 1, cols - 1] = 450.0
    x = x.to(dtype)
    q, s = quantize(x)
    rq, rs = R.quantized(x.double())
    assert torch.equal(s[:, :R.nblocks(cols)], rs)
    assert torch.equal(q[:, :cols], rq)
    # the bytes between the rows stay
    assert torch.all(q[:, cols:] == 0x55) and torch.all(s[:, R.nblocks(cols):] == 0x33)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [0, 1])
def test_quantize_range_ends_and_non_finite(dtype, shift):
    # largest and smallest values, subnormals, signed zeros, NaN and infinities; rows
    # that start aligned and not (both kernels)
    big = torch.zeros((6, 256 + shift), dtype=dtype, device=DEV)
    x = big[:, shift:]
    x[0, ::3] = torch.finfo(dtype).max
    x[1, ::5] = 2.0 ** -126
    x[1, 128:] = 2.0 ** -133
    x[2, :128] = randn(128, seed=3).to(dtype)
    x[2, 5], x[2, 6], x[2, 7] = float("nan"), float("inf"), float("-inf")
    x[3, :] = -0.0
    x[4, :128] = float("nan")
    x[4, 128:] = float("inf")
    x[5, 130] = -3.0
    q, s = quantize(x)
    rq, rs = R.quantized(x.double())
    assert torch.equal(s[:, :2], rs)
    got, want = (v.view(torch.float8_e4m3fn).float() for v in (q[:, :256].contiguous(), rq.contiguous()))
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    assert torch.all(torch.signbit(got[3]))


def test_quantize_strides():
    # columns of a wider matrix, aligned and not, into strided bytes
    wide = randn(37, 3000, seed=4, dtype=torch.bfloat16)
    for c0, cols in ((1024, 1024), (1000, 1111), (3, 5)):
        x = wide[:, c0:c0 + cols]
        q, s = R.storage(37, cols, pad=3)
        quantize(x, q, s)
        rq, rs = R.quantized(x.double())
        assert torch.equal(q[:, :cols], rq) and torch.equal(s[:, :R.nblocks(cols)], rs)
        assert torch.all(q[:, cols:] == 0x55) and torch.all(s[:, R.nblocks(cols):] == 0x33)


def test_quantize_offsets_past_32_bits():
    # a stride that puts the last row behind 4 GiB of input and of output
    rows, cols, ld = 3, 256, 1 << 30
    x = torch.empty(2 * ld + cols, dtype=torch.bfloat16, device=DEV).as_strided((rows, cols), (ld, 1))
    x.copy_(randn(rows, cols, seed=5))
    ldq = 5 << 29
    q = torch.empty(2 * ldq + cols, dtype=torch.uint8, device=DEV).as_strided((rows, cols), (ldq, 1))
    s = torch.zeros((rows, 4), dtype=torch.uint8, device=DEV)
    quantize(x, q, s)
    rq, rs = R.quantized(x.double())
    assert torch.equal(q.contiguous(), rq) and torch.equal(s[:, :2], rs)


def test_quantize_longest_row():
    # the last block of a row of 2^31 - 1 elements, and the first
    cols = 2 ** 31 - 1
    x = torch.zeros((1, cols), dtype=torch.bfloat16, device=DEV)
    x[0, :256], x[0, -300:] = randn(256, seed=6).bfloat16(), randn(300, seed=7).bfloat16()
    q = torch.full((1, cols + 1), 0x55, dtype=torch.uint8, device=DEV)
    s = torch.full((1, R.nblocks(cols) + 1), 0x33, dtype=torch.uint8, device=DEV)
    quantize(x, q, s)
    for lo in (0, cols - cols % 128 - 256):
        rq, rs = R.quantized(x[:, lo:lo + 512].double())
        assert torch.equal(q[:, lo:min(lo + 512, cols)], rq)
        assert torch.equal(s[:, lo // 128:lo // 128 + rs.shape[1]], rs)
    assert q[0, -1] == 0x55 and s[0, -1] == 0x33


# more blocks than one step of the grid takes (fp32: two groups of four per warp), a whole
# number of groups and not, aligned rows and not
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,shift", [(6001, 1300, 0), (6000, 1280, 0), (6001, 1280, 1), (60001, 128, 0), (70000, 40, 0)])
def test_quantize_more_than_a_wave(rows, cols, shift, dtype):
    x = randn(rows, cols + 4, seed=rows + cols, dtype=dtype)[:, shift:shift + cols]
    x.mul_(torch.exp2(torch.randint(-20, 20, (rows, 1), generator=gen(2), device=DEV).float()).to(dtype))
    q, s = quantize(x)
    rq, rs = R.quantized(x.double())
    assert torch.equal(s[:, :R.nblocks(cols)], rs) and torch.equal(q[:, :cols], rq)
    assert torch.all(q[:, cols:] == 0x55) and torch.all(s[:, R.nblocks(cols):] == 0x33)


def test_quantize_no_rows():
    x, (q, s) = torch.zeros((0, 64), device=DEV), R.storage(1, 64)
    f3dc.quantize_fp8(x, 64, q, 64, s, 4, 0, 64)
    assert torch.all(q == 0x55)


# ------------------------------------------------------------------ product

def operands(M, N, K, seed):
    a = randn(M, K, seed=seed) * torch.exp(randn(M, 1, seed=seed + 1))
    a[:, ::97] *= 30.0  # blocks of quite different scales
    b = randn(N, K, seed=seed + 2, scale=K ** -0.5) * torch.exp(0.5 * randn(N, 1, seed=seed + 3))
    return (*quantize(a), *quantize(b))


# below, at and above the sizes of a row pair, a column unit, a scale block and a set of
# four; one row; ragged N; full waves with a rest (76 clusters: 80, 96 and 256 tiles); long
# sums of few tiles (units of 128 and of 256 columns shared by two pairs, a K that leaves
# the second an uneven number of blocks)
SHAPES = [(1, 8, 1), (1, 128, 128), (2, 64, 31), (5, 72, 129), (8, 1024, 4096), (9, 136, 1500), (17, 4096, 1024), (32, 264, 640),
          (33, 264, 640), (127, 256, 512), (128, 264, 513), (129, 200, 640),
          (255, 1000, 1374), (256, 256, 128), (257, 512, 2048), (300, 1088, 700), (64, 4096, 1024), (1229, 4096, 384), (300, 1000, 3200), (260, 2048, 4100),
          (1229, 1024, 4096), (70, 2056, 8000), (5, 8200, 4096), (8, 40000, 1100), (1, 16384, 2900), (12, 16400, 300), (7, 512, 8100),
          (1300, 4096, 256), (4096, 4096, 128), (2600, 1960, 1100)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("epi", [f3dc.EPI_BIAS, f3dc.EPI_GELU, f3dc.EPI_RESID])
def test_gemm_fp8(M, N, K, epi):
    A, sa, B, sb = operands(M, N, K, M + N + K)
    bias = randn(N, seed=7, dtype=torch.bfloat16)
    y, err = R.gemm(A, sa, B, sb, K, bias)
    if epi == f3dc.EPI_RESID:
        gate, x0 = randn(N, seed=8), randn(M, N, seed=9)
        out = x0.clone()
        gemm8(A, sa, B, sb, K, epi, bias, gate, out)
        ref = x0.double() + gate.double() * y
        bound = gate.double().abs() * err + R.U32 * ((gate.double() * y).abs() + ref.abs())
        assert torch.all((out.double() - ref).abs() <= 1.01 * bound)
    else:
        out = torch.full((M, N), 7.0, dtype=torch.bfloat16, device=DEV)
        gemm8(A, sa, B, sb, K, epi, bias, None, out)
        if epi == f3dc.EPI_GELU:
            y, err = R.gelu(y), R.gelu_bound(y, err)
        assert torch.all((out.double() - y).abs() <= R.U_BF16 * y.abs() + 1.01 * err)
    assert f3dc.gemm_status() == 0


# sums so long that two pairs share tiles of 256 columns too
@pytest.mark.parametrize("M,N,K", [(300, 1040, 7400), (1229, 1024, 10500), (260, 2000, 16384)])
@pytest.mark.parametrize("epi", [f3dc.EPI_GELU, f3dc.EPI_RESID, "out8"])
def test_gemm_fp8_very_long_sums(M, N, K, epi):
    A, sa, B, sb = operands(M, N, K, M + N + K)
    bias = randn(N, seed=7, dtype=torch.bfloat16)
    y, err = R.gemm(A, sa, B, sb, K, bias)
    if epi == f3dc.EPI_RESID:
        x0 = randn(M, N, seed=9)
        out = x0.clone()
        gemm8(A, sa, B, sb, K, epi, bias, None, out)
        ref = x0.double() + y
        assert torch.all((out.double() - ref).abs() <= 1.01 * (err + R.U32 * (y.abs() + ref.abs())))
    elif epi == "out8":
        q, s = R.storage(M, N, pad=1)
        gemm8(A, sa, B, sb, K, f3dc.EPI_BIAS, bias, None, q, s)
        R.check_out8(q, s, y, err)
        assert torch.all(q[:, N:] == 0x55) and torch.all(s[:, R.nblocks(N):] == 0x33)
    else:
        out = torch.full((M, N), 7.0, dtype=torch.bfloat16, device=DEV)
        gemm8(A, sa, B, sb, K, epi, bias, None, out)
        y, err = R.gelu(y), R.gelu_bound(y, err)
        assert torch.all((out.double() - y).abs() <= R.U_BF16 * y.abs() + 1.01 * err)
    assert f3dc.gemm_status() == 0


@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (3, 128, 128), (1, 4096, 1024), (11, 1040, 1300), (32, 144, 4096),
                                   (33, 144, 300), (129, 144, 300), (255, 1008, 1374), (300, 4096, 512), (300, 1040, 6200), (7, 8208, 4000), (2, 40000, 700),
                                   (955, 1152, 1024), (4000, 2048, 256)])
@pytest.mark.parametrize("epi", [f3dc.EPI_BIAS, f3dc.EPI_GELU])
def test_gemm_fp8_8bit_output(M, N, K, epi):
    A, sa, B, sb = operands(M, N, K, M + N + K)
    bias = randn(N, seed=7, dtype=torch.bfloat16)
    q, s = R.storage(M, N, pad=1)
    gemm8(A, sa, B, sb, K, epi, bias, None, q, s)
    y, err = R.gemm(A, sa, B, sb, K, bias)
    if epi == f3dc.EPI_GELU:
        y, err = R.gelu(y), R.gelu_bound(y, err)
    R.check_out8(q, s, y, err)
    assert torch.all(q[:, N:] == 0x55) and torch.all(s[:, R.nblocks(N):] == 0x33)
    assert f3dc.gemm_status() == 0


def gelu_exact(x):
    # without the cancellation of 1 + tanh
    return x * torch.sigmoid(2 * (2 / np.pi) ** 0.5 * (x + 0.044715 * x ** 3))


# GELU keeps its relative accuracy where it is small: sums around a bias far below zero, each
# kernel, bf16 and 8-bit output (where every value of a block may be small).  The bound: what the
# error of the sum moves the result (it is monotonic below -0.76; above, its slope is at most 1.13),
# 2^-14 relative for the evaluation (twice what the roundings of the exponent, at most 128 * 3 *
# 2^-24 * ln 2, and two approximations within 2^-21 can give), the output's rounding.
@pytest.mark.parametrize("centre", [1.5, 0.0, -0.5, -1.6, -3.0, -4.0, -5.0, -6.5, -8.0, -9.0])
@pytest.mark.parametrize("M,N,K", [(4, 256, 512), (33, 144, 640), (300, 512, 512), (300, 1024, 7400)])
@pytest.mark.parametrize("out8", [False, True])
def test_gemm_fp8_gelu_of_negative_sums(M, N, K, centre, out8):
    A, sa = quantize(randn(M, K, seed=1))
    B, sb = quantize(randn(N, K, seed=2, scale=0.1 * K ** -0.5))
    bias = (centre + randn(N, seed=3, scale=0.05)).to(torch.bfloat16)
    y, err = R.gemm(A, sa, B, sb, K, bias)
    g = gelu_exact(y)
    moved = torch.where(y < -1.0, torch.maximum((gelu_exact(y + err) - g).abs(), (gelu_exact(y - err) - g).abs()), 1.13 * err)
    bound = moved + 2.0 ** -14 * g.abs()
    if out8:
        q, s = R.storage(M, N)
        gemm8(A, sa, B, sb, K, f3dc.EPI_GELU, bias, None, q, s)
        R.check_out8(q, s, g, bound)
    else:
        out = torch.zeros((M, N), dtype=torch.bfloat16, device=DEV)
        gemm8(A, sa, B, sb, K, f3dc.EPI_GELU, bias, None, out)
        assert torch.all((out.double() - g).abs() <= (1 + 2.0 ** -7) * bound + R.U_BF16 * g.abs())


@pytest.mark.parametrize("M", [4, 300])
def test_gemm_fp8_gelu_of_extremes(M):
    N, K = 128, 128
    A, sa, B, sb = operands(M, N, K, 9)
    bias = torch.zeros(N, dtype=torch.bfloat16, device=DEV)
    bias[:6] = torch.tensor([float("inf"), float("nan"), 3e38, -3e38, 1e10, -1e10])
    out = torch.full((M, N), 7.0, dtype=torch.bfloat16, device=DEV)
    gemm8(A, sa, B, sb, K, f3dc.EPI_GELU, bias, None, out)
    assert torch.all(torch.isposinf(out[:, 0])) and torch.all(torch.isnan(out[:, 1]))
    assert torch.all(out[:, 2] == bias[2]) and torch.all(out[:, 4] == bias[4])
    assert torch.all(out[:, 3] == 0) and torch.all(out[:, 5] == 0) and torch.all(torch.isfinite(out[:, 6:].float()))


def test_gemm_fp8_without_bias_and_gate_and_strided():
    M, N, K = 333, 520, 900
    A, sa, B, sb = operands(M, N, K, 3)
    Aw, saw = torch.full((M, 2048), 0x7F, dtype=torch.uint8, device=DEV), torch.full((M, 20), 0xFF, dtype=torch.uint8, device=DEV)
    Aw[:, 512:512 + K], saw[:, 4:4 + R.nblocks(K)] = A[:, :K], sa[:, :R.nblocks(K)]  # NaN all around the operand
    Av, sav = Aw[:, 512:512 + K], saw[:, 4:12]
    y, err = R.gemm(A, sa, B, sb, K)
    buf = torch.full((M, 640), 3.0, dtype=torch.float32, device=DEV)
    gemm8(Av, sav, B, sb, K, f3dc.EPI_RESID, None, None, buf[:, 64:64 + N])
    got = buf[:, 64:64 + N].double() - 3.0
    assert torch.all((got - y).abs() <= 1.01 * err + 2 * R.U32 * (y.abs() + 3.0))
    assert torch.all(buf[:, :64] == 3.0) and torch.all(buf[:, 64 + N:] == 3.0)
    out = torch.full((M, 1024), 5.0, dtype=torch.bfloat16, device=DEV)
    gemm8(Av, sav, B, sb, K, f3dc.EPI_BIAS, None, None, out[:, :N])
    assert torch.all((out[:, :N].double() - y).abs() <= R.U_BF16 * y.abs() + 1.01 * err)
    assert torch.all(out[:, N:] == 5.0)


def test_gemm_fp8_scales_of_both_operands_apply_to_their_blocks():
    # one block of one row at a time carries a large scale: the sum must follow
    # exactly (every product and sum is a whole number below 2^24)
    M, N, K = 256, 256, 1152
    A = torch.full((M, K), 0x38, dtype=torch.uint8, device=DEV)  # 1.0
    B = torch.full((N, K), 0x38, dtype=torch.uint8, device=DEV)
    sa = torch.randint(127, 130, (M, 12), generator=gen(1), device=DEV).to(torch.uint8)
    sb = torch.randint(127, 131, (N, 12), generator=gen(2), device=DEV).to(torch.uint8)
    out = torch.zeros((M, N), device=DEV)
    gemm8(A, sa, B, sb, K, f3dc.EPI_RESID, None, None, out)
    y = 128.0 * (R.pow2(sa[:, :9]) @ R.pow2(sb[:, :9]).T)
    assert torch.equal(out.double(), y)


@pytest.mark.parametrize("M", [3, 64])
def test_gemm_fp8_scale_range(M):
    # scales far apart whose products are moderate, zero rows under the smallest scale
    N, K = 64, 256
    A, sa, B, sb = operands(M, N, K, 5)
    for da, db in ((100, -100), (-110, 110), (60, -20)):
        sa2, sb2 = (sa.int() + da).clamp(0, 254).to(torch.uint8), (sb.int() + db).clamp(0, 254).to(torch.uint8)
        out = torch.zeros((M, N), device=DEV)
        gemm8(A, sa2, B, sb2, K, f3dc.EPI_RESID, None, None, out)
        y, err = R.gemm(A, sa2, B, sb2, K)
        assert torch.all((out.double() - y).abs() <= 1.01 * err + R.U32 * y.abs())


@pytest.mark.parametrize("M", [16, 200])
def test_gemm_fp8_nan_stays_in_its_row_and_column(M):
    N, K, last = 136, 512, M - 2
    A, sa, B, sb = operands(M, N, K, 6)
    A[3, 77] = 0x7F          # a NaN value
    sa[last, 2] = 0xFF       # a NaN scale
    B[70, 300] = 0xFF
    out = torch.zeros((M, N), dtype=torch.bfloat16, device=DEV)
    gemm8(A, sa, B, sb, K, f3dc.EPI_BIAS, None, None, out)
    want = torch.zeros((M, N), dtype=torch.bool, device=DEV)
    want[3], want[last], want[:, 70] = True, True, True
    assert torch.equal(torch.isnan(out), want)
    # 8-bit output: NaN elements, and a scale from the finite ones
    q, s = R.storage(M, 144)
    Bp, sbp = torch.zeros((144, K), dtype=torch.uint8, device=DEV), torch.full((144, 4), 127, dtype=torch.uint8, device=DEV)
    Bp[:N], sbp[:N] = B[:, :K], sb[:, :4]
    gemm8(A, sa, Bp, sbp, K, f3dc.EPI_BIAS, None, None, q, s)
    v = R.values(q, s, 144)
    assert torch.equal(torch.isnan(v[:, :N]), want)
    y, err = R.gemm(A, sa, Bp, sbp, K)
    row = 9
    keep = ~torch.isnan(y[row])
    assert torch.all((v[row] - y[row])[keep].abs() <= (R.U_E4M3 * y[row].abs() + 0.5 * R.E4M3_MIN * R.pow2(
        s[row, :2]).repeat_interleave(128)[:144] + 1.1 * err[row])[keep])


def test_gemm_fp8_is_deterministic_and_no_rows():
    for M, K in ((10, 2000), (300, 5000), (777, 2000)):  # each kernel
        A, sa, B, sb = operands(M, 1024, K, 8)
        outs = []
        for _ in range(3):
            out = torch.zeros((M, 1024), device=DEV)
            gemm8(A, sa, B, sb, K, f3dc.EPI_RESID, None, None, out)
            outs.append(out)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    out = torch.full((1, 1024), 2.0, device=DEV)
    f3dc.gemm_fp8(A, A.stride(0), sa, sa.stride(0), B, B.stride(0), sb, sb.stride(0), None, None, out, 1024, None, 0, 0,
                  1024, 2000, f3dc.EPI_RESID)
    assert torch.all(out == 2.0)


@pytest.mark.parametrize("M,N,K", [(1229, 1024, 4096), (1, 1024, 4096), (100, 512, 8192)])
def test_gemm_fp8_long_positive_sums(M, N, K):
    # positive products: the tensor core's truncation adds up
    A, sa = quantize(randn(M, K, seed=1).abs())
    B, sb = quantize(randn(N, K, seed=2).abs())
    out = torch.zeros((M, N), device=DEV)
    gemm8(A, sa, B, sb, K, f3dc.EPI_RESID, None, None, out)
    y, err = R.gemm(A, sa, B, sb, K)
    assert torch.all((out.double() - y).abs() <= err + R.U32 * y)


# Sums of one sign, however long, stay within 2^-14 with fp32 output and 2^-12 with others: the
# tensor core may drop 2^-23 of the sum at each 32 K, no accumulator takes more than 16384 or 65536
# K, and the pieces add one rounding each, fewer than 2^5 of them here (the few rows' kernel adds
# rounded blocks: with 16 warps fewer than 2^8).  Few tiles (shared by two pairs), many, few rows; just
# above the longest single sums; an uneven last piece.
def piece_error(fp32):
    return (2.0 ** -14 if fp32 else 2.0 ** -12) + 2.0 ** 8 * R.U32


@pytest.mark.parametrize("M,N,K", [(4, 64, 1 << 18), (70, 136, 1 << 18), (300, 520, 1 << 17), (1300, 2048, 40000), (2600, 2056, 16400),
                                   (2600, 2048, 32768), (300, 1024, 32896), (300, 1024, 40000), (1300, 2048, 65664)])
@pytest.mark.parametrize("out8", [False, True])
def test_gemm_fp8_sums_of_one_sign_however_long(M, N, K, out8):
    N = N // 16 * 16 if out8 else N
    A, sa = quantize(randn(M, K, seed=1).abs())
    B, sb = quantize(randn(N, K, seed=2).abs())
    y, _ = R.gemm(A, sa, B, sb, K)
    err = piece_error(not out8) * y
    if out8:
        q, s = R.storage(M, N, pad=1)
        gemm8(A, sa, B, sb, K, f3dc.EPI_BIAS, None, None, q, s)
        R.check_out8(q, s, y, err)
        assert torch.all(q[:, N:] == 0x55) and torch.all(s[:, R.nblocks(N):] == 0x33)
    else:
        out = torch.zeros((M, N), device=DEV)
        gemm8(A, sa, B, sb, K, f3dc.EPI_RESID, None, None, out)
        assert torch.all((out.double() - y).abs() <= err + R.U32 * y)
    assert f3dc.gemm_status() == 0


# sums in pieces with each epilogue, of either sign, with bias and gate, and again
@pytest.mark.parametrize("M,N,K", [(70, 264, 66000), (300, 1040, 140000), (1229, 3000, 16500), (1229, 2056, 66100), (9, 8200, 16640),
                                   (300, 1040, 70000)])
@pytest.mark.parametrize("epi", [f3dc.EPI_BIAS, f3dc.EPI_GELU, f3dc.EPI_RESID, "out8"])
def test_gemm_fp8_sums_in_pieces(M, N, K, epi):
    N = N // 16 * 16 if epi == "out8" else N
    A, sa, B, sb = operands(M, N, K, M + N + K)
    bias, gate, x0 = randn(N, seed=7, dtype=torch.bfloat16), randn(N, seed=8), randn(M, N, seed=9)
    y, _ = R.gemm(A, sa, B, sb, K, bias)
    mag = R.values(A, sa, K).abs() @ R.values(B, sb, K).abs().T
    err = piece_error(epi == f3dc.EPI_RESID) * mag + R.U32 * (mag + bias.double().abs())
    outs = []
    for _ in range(2):
        if epi == "out8":
            q, s = R.storage(M, N, pad=1)
            gemm8(A, sa, B, sb, K, f3dc.EPI_GELU, bias, None, q, s)
            outs.append(torch.cat([q.flatten(), s.flatten()]))
        else:
            out = x0.clone() if epi == f3dc.EPI_RESID else torch.zeros((M, N), dtype=torch.bfloat16, device=DEV)
            gemm8(A, sa, B, sb, K, epi, bias, gate if epi == f3dc.EPI_RESID else None, out)
            outs.append(out)
    assert torch.equal(outs[0], outs[1])
    g = gelu_exact(y)
    moved = 1.13 * err + 2.0 ** -14 * g.abs()
    if epi == "out8":
        step = R.pow2(s[:, :R.nblocks(N)]).repeat_interleave(R.BLOCK, 1)[:, :N]
        bound = R.U_E4M3 * g.abs() + 0.5 * R.E4M3_MIN * step + (1 + R.U_E4M3) * moved
        assert torch.all((R.values(q, s, N) - g).abs() <= bound)
        assert torch.all(q[:, N:] == 0x55) and torch.all(s[:, R.nblocks(N):] == 0x33)
    elif epi == f3dc.EPI_GELU:
        assert torch.all((out.double() - g).abs() <= (1 + 2.0 ** -7) * moved + R.U_BF16 * g.abs())
    elif epi == f3dc.EPI_BIAS:
        assert torch.all((out.double() - y).abs() <= (1 + 2.0 ** -7) * err + R.U_BF16 * y.abs())
    else:
        ref = x0.double() + gate.double() * y
        bound = gate.double().abs() * err + R.U32 * ((gate.double() * y).abs() + ref.abs())
        assert torch.all((out.double() - ref).abs() <= 1.01 * bound)
    assert f3dc.gemm_status() == 0


# in two captured graphs replayed at once on two streams (the first launches of these kernels may
# be the captured ones)
@pytest.mark.parametrize("M,N,K", [(300, 512, 40000), (1300, 2048, 16640)])
def test_gemm_fp8_sums_in_pieces_in_graphs(M, N, K):
    jobs = [(operands(M, N, K, 50 + i), torch.zeros((M, N), device=DEV), torch.cuda.CUDAGraph(), torch.cuda.Stream()) for i in range(2)]
    torch.cuda.synchronize()
    for ops, out, g, _ in jobs:
        with torch.cuda.graph(g):
            gemm8(*ops, K, f3dc.EPI_RESID, None, None, out)
    torch.cuda.synchronize()
    for _, out, g, st in jobs:
        with torch.cuda.stream(st):
            g.replay()
    torch.cuda.synchronize()
    for ops, out, _, _ in jobs:
        again = torch.zeros_like(out)
        gemm8(*ops, K, f3dc.EPI_RESID, None, None, again)
        y, _ = R.gemm(*ops, K)
        mag = R.values(ops[0], ops[1], K).abs() @ R.values(ops[2], ops[3], K).abs().T
        assert torch.all((out.double() - y).abs() <= piece_error(True) * mag + R.U32 * y.abs())
        assert torch.equal(out, again)
    assert f3dc.gemm_status() == 0


def test_gemm_fp8_longest_sum():
    # ones: every partial sum is a whole number, the last one 2^26
    M, N, K = 65, 8, 1 << 26
    A, B = (torch.full((r, K), 0x38, dtype=torch.uint8, device=DEV) for r in (M, N))
    sa, sb = (torch.full((r, K // 128), 127, dtype=torch.uint8, device=DEV) for r in (M, N))
    out = torch.zeros((M, N), device=DEV)
    gemm8(A, sa, B, sb, K, f3dc.EPI_RESID, None, None, out)
    assert torch.all(out == float(K))
    assert f3dc.gemm_status() == 0


# rows and scales more than 4 GiB apart from the first, in both kernels
@pytest.mark.parametrize("M,N,K", [(3, 40, 200), (200, 264, 200), (300, 256, 4096)])
@pytest.mark.parametrize("out8", [False, True])
def test_gemm_fp8_offsets_past_32_bits(M, N, K, out8):
    if out8:
        N = N // 16 * 16
    A, sa, B, sb = operands(M, N, K, 5)
    bias = randn(N, seed=7, dtype=torch.bfloat16)
    y, err = R.gemm(A, sa, B, sb, K, bias)

    def wide(v, most=1 << 32):
        ld = most // (v.shape[0] - 1) // 64 * 64 + 64
        return torch.empty((v.shape[0], ld), dtype=v.dtype, device=DEV)[:, :v.shape[1]].copy_(v)
    ops = [wide(t) for t in (A, sa, B, sb)]
    if out8:
        q, s = (wide(t) for t in R.storage(M, N))
        gemm8(*ops, K, f3dc.EPI_BIAS, bias, None, q, s)
        R.check_out8(q, s, y, err)
    else:
        out = wide(torch.full((M, N), 7.0, dtype=torch.bfloat16, device=DEV))
        gemm8(*ops, K, f3dc.EPI_BIAS, bias, None, out)
        assert torch.all((out.double() - y).abs() <= R.U_BF16 * y.abs() + 1.01 * err)
    assert f3dc.gemm_status() == 0


# scales whose rows start 4, 8 and 16 bytes aligned are read in pieces of as many
@pytest.mark.parametrize("align", [4, 8, 16])
@pytest.mark.parametrize("M,N,K", [(70, 264, 5000), (600, 1024, 4200), (300, 520, 4200)])
def test_gemm_fp8_scale_alignment(M, N, K, align):
    A, sa, B, sb = operands(M, N, K, 6)
    y, err = R.gemm(A, sa, B, sb, K)

    def at(v):
        ld = -(-v.shape[1] // 16) * 16 + align
        buf = torch.full((16 + v.shape[0] * ld,), 0xFF, dtype=torch.uint8, device=DEV)
        return buf[align % 16:][:v.shape[0] * ld].view(-1, ld)[:, :v.shape[1]].copy_(v)
    out = torch.zeros((M, N), dtype=torch.bfloat16, device=DEV)
    gemm8(A, at(sa), B, at(sb), K, f3dc.EPI_BIAS, None, None, out)
    assert torch.all((out.double() - y).abs() <= R.U_BF16 * y.abs() + 1.01 * err)
    assert f3dc.gemm_status() == 0


# the few rows' kernel, whole and split sums: at once on two streams and in two graphs
# replayed at once, and captured by a process's very first call
@pytest.mark.parametrize("M,N,K,epi", [(1, 1024, 4096, 0), (16, 512, 1024, 1), (300, 1024, 4096, 0), (600, 1024, 6400, 1), (2000, 1024, 640, 0)])
@pytest.mark.parametrize("out8", [False, True])
def test_gemm_fp8_streams_and_graphs(M, N, K, epi, out8):
    jobs = []
    for i in range(2):
        A, sa, B, sb = operands(M, N, K, 40 + i)
        o = R.storage(M, N) if out8 else (torch.zeros((M, N), dtype=torch.bfloat16, device=DEV), None)
        gemm8(A, sa, B, sb, K, epi, None, None, *o)
        jobs.append(((A, sa, B, sb), o, o[0].clone(), o[1].clone() if out8 else None))
    streams = [torch.cuda.Stream() for _ in jobs]

    def check():
        torch.cuda.synchronize()
        for _, o, q, s in jobs:
            assert torch.equal(o[0], q) and (s is None or torch.equal(o[1], s))
            for t in o:
                if t is not None:
                    t.zero_()
        torch.cuda.synchronize()
    check()
    for _ in range(4):
        for (ops, o, _, _), st in zip(jobs, streams):
            gemm8(*ops, K, epi, None, None, *o, stream=st.cuda_stream)
    torch.cuda.synchronize()
    if out8:
        pad = [(o[0][:, N:].clone(), q[:, N:], o[1][:, R.nblocks(N):], s[:, R.nblocks(N):]) for _, o, q, s in jobs]
        assert all(torch.all(a == 0) and torch.all(b == 0x55) and torch.all(c == 0) and torch.all(d == 0x33) for a, b, c, d in pad)
        for _, o, q, s in jobs:
            o[0][:, N:], o[1][:, R.nblocks(N):] = 0x55, 0x33
    check()
    graphs = []
    for ops, o, _, _ in jobs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            gemm8(*ops, K, epi, None, None, *o)
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    if out8:
        for _, o, _, _ in jobs:
            o[0][:, N:], o[1][:, R.nblocks(N):] = 0x55, 0x33
    check()
    assert f3dc.gemm_status() == 0


# A CTA's barriers are awaited to their last arrival before it leaves: one, two, three and more
# sets of scales (512 K each), whole and shared sums, launch upon launch with other kernels in
# between whose CTAs take over the same shared memory
def test_gemm_fp8_back_to_back_with_other_kernels():
    N = 512
    jobs = []
    for i, (M, K) in enumerate([(300, 300), (70, 900), (300, 1400), (300, 4096), (1300, 2100)]):
        ops = operands(M, N, K, 60 + i)
        out = torch.zeros((M, N), dtype=torch.bfloat16, device=DEV)
        gemm8(*ops, K, f3dc.EPI_BIAS, None, None, out)
        y, err = R.gemm(*ops, K)
        assert torch.all((out.double() - y).abs() <= R.U_BF16 * y.abs() + 1.01 * err)
        jobs.append((ops, K, out, out.clone()))
    a, b = randn(256, 512, seed=70, dtype=torch.bfloat16), randn(N, 512, seed=71, dtype=torch.bfloat16)
    plain = torch.zeros((256, N), dtype=torch.bfloat16, device=DEV)
    f3dc.gemm(a, b, None, None, plain, 256, N, 512, f3dc.EPI_BIAS)
    want = plain.clone()
    for _ in range(100):
        for ops, K, out, _ in jobs:
            gemm8(*ops, K, f3dc.EPI_BIAS, None, None, out)
            f3dc.gemm(a, b, None, None, plain, 256, N, 512, f3dc.EPI_BIAS)
    assert f3dc.gemm_status() == 0
    assert torch.equal(plain, want)
    for _, _, out, first in jobs:
        assert torch.equal(out, first)


# Two pairs share a sum: each writes its partial sums where the other's operands were.  Many
# launches in a row, the operands of one being another's (a stage written too early, or sums
# read too early, would show)
@pytest.mark.parametrize("M,N,K,epi", [(300, 1024, 4096, 0), (600, 1024, 10500, 0), (300, 1040, 7400, 2)])
def test_gemm_fp8_shared_sums_in_a_row(M, N, K, epi):
    ops = [operands(M, N, K, 80 + i) for i in range(3)]
    dtype = torch.float32 if epi == 2 else torch.bfloat16
    outs = [torch.zeros((M, N), dtype=dtype, device=DEV) for _ in range(60)]
    for i, out in enumerate(outs):
        gemm8(*ops[i % 3], K, epi, None, None, out)
    for i in range(3):
        y, err = R.gemm(*ops[i], K)
        bound = 1.01 * err + (R.U32 if epi == 2 else R.U_BF16) * y.abs()
        assert torch.all((outs[i].double() - y).abs() <= bound)
    for i, out in enumerate(outs):
        assert torch.equal(out, outs[i % 3])
    assert f3dc.gemm_status() == 0


# The even CTA's tensor core reads scales that the odd one has written: launches in a row whose
# scales are all different, in whole numbers that any stale scale would change
@pytest.mark.parametrize("M,N,K", [(256, 128, 512), (512, 256, 1664), (2048, 1024, 2560)])
def test_gemm_fp8_scales_of_launches_in_a_row(M, N, K):
    A, B = (torch.full((r, K), 0x38, dtype=torch.uint8, device=DEV) for r in (M, N))  # 1.0
    blocks = R.nblocks(K)
    scales = [[torch.randint(124, 131, (r, -(-blocks // 4) * 4), generator=gen(90 + 2 * i + j), device=DEV).to(torch.uint8)
               for j, r in enumerate((M, N))] for i in range(40)]
    outs = [torch.zeros((M, N), device=DEV) for _ in scales]
    for (sa, sb), out in zip(scales, outs):
        gemm8(A, sa, B, sb, K, f3dc.EPI_RESID, None, None, out)
    assert f3dc.gemm_status() == 0
    for (sa, sb), out in zip(scales, outs):
        # every sum is 128 times a multiple of 2^-6 and at most 128 * 20 * 2^6: exact in 24 bits
        assert torch.equal(out.double(), 128.0 * (R.pow2(sa[:, :blocks]) @ R.pow2(sb[:, :blocks]).T))


FIRST_CALL_CAPTURED = """
import sys
sys.path[:0] = [%r, %r]
import torch
import fp8_ref as R
from test_gpu_fp8 import *
f3dc.lib()
A = torch.full((%d, 4096), 0x38, dtype=torch.uint8, device=DEV)
B = torch.full((256, 4096), 0x38, dtype=torch.uint8, device=DEV)
sa, sb = (torch.full((t.shape[0], 32), 127, dtype=torch.uint8, device=DEV) for t in (A, B))
out = torch.zeros((A.shape[0], 256), dtype=torch.bfloat16, device=DEV)
x, (q, s) = torch.ones((4, 256), device=DEV), R.storage(4, 256)
h = torch.zeros((4, 256), dtype=torch.bfloat16, device=DEV)
layer = f3dc.NormLayer(256, pre=f3dc.NORM_RMS, eps=0.0)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    gemm8(A, sa, B, sb, 4096, f3dc.EPI_BIAS, None, None, out)
    quantize(x, q, s)
    f3dc.norm_residual(layer, x, 256, None, 0, None, 0, None, None, None, 0, None, 1, h, 256, None, 0, 4)
g.replay()
torch.cuda.synchronize()
assert torch.all(out == 4096.0) and f3dc.gemm_status() == 0
assert torch.all(h == 1.0) and torch.all(s[:, :2] == 119) and torch.all(q == 0x78)
print("captured")
"""


@pytest.mark.parametrize("M", [4, 300])
def test_first_call_of_a_process_in_a_capture(M):
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    code = FIRST_CALL_CAPTURED % (here, os.path.dirname(here), M)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


# ------------------------------------------------------------------ norms

def norm_case(rows, W, post, pre, affine, mod, groups, out8, y=True, x_out=True, h=True, seed=0, alpha=0.875, eps=1e-6,
              pads=True, pad_cols=0):
    """Runs a case and checks every output against 64 bits."""
    x = randn(rows, W + 4 * pad_cols, seed=seed + 1, scale=2.0)[:, :W]
    yt = randn(rows, W + 8 * pad_cols, seed=seed + 2).mul_(torch.exp(randn(rows, 1, seed=seed + 3))).to(torch.bfloat16)[:, :W] if y else None
    vec = [randn(W, seed=seed + 4 + i, scale=0.1).add_(1.0 if i % 2 == 0 else 0.0).to(torch.bfloat16) if affine else None
           for i in range(4)]
    m = randn(groups, 3, W, seed=seed + 9, scale=0.4) if mod else None
    gate, scale, shift = (m[:, 0] if y else None, m[:, 1], m[:, 2]) if mod else (None, None, None)
    group = None
    if groups > 1 or pads:
        group = torch.randint(-1 if pads else 0, groups, (rows,), generator=gen(seed + 10), device=DEV).to(torch.int32)
    xo = torch.full((rows, W + 4 * pad_cols), 9.0, device=DEV) if x_out else None
    if out8:
        hq, hs = R.storage(rows, W, pad=1)
    else:
        hq, hs = torch.full((rows, W + 8 * pad_cols), 5.0, dtype=torch.bfloat16, device=DEV), None
    layer = f3dc.NormLayer(W, post, pre, *vec, eps=eps, res_scale=alpha)
    f3dc.norm_residual(layer, x, x.stride(0), xo, xo.stride(0) if x_out else 0, yt, yt.stride(0) if y else 0, gate, scale,
                       shift, 3 * W, group, groups, hq if h else None, hq.stride(0), hs if h else None,
                       hs.stride(0) if out8 else 0, rows)
    g = group.long() if group is not None else torch.zeros(rows, dtype=torch.long, device=DEV)
    live, gi = g >= 0, g.clamp(min=0)
    s = alpha32 = float(np.float32(alpha))
    xd = x.double()
    ref, err = alpha32 * xd, R.U32 * (s * xd).abs()
    if y:
        n, ne = R.norm(yt.double(), torch.zeros_like(xd), post, vec[0], vec[1], eps)
        if mod:
            gd = gate[gi].double()
            n, ne = n * gd, ne * gd.abs() + R.U32 * (n * gd).abs()
        ref = ref + n
        err = err + ne + R.U32 * ref.abs()
    err = 1.01 * err
    if x_out:
        assert torch.all((xo[:, :W].double() - ref).abs()[live] <= err[live])
        assert torch.all(xo[~live] == 9.0) and torch.all(xo[:, W:] == 9.0)
    if h:
        r, e = R.norm(ref, err, pre, vec[2], vec[3], eps)
        if mod:
            sc, sh = 1.0 + scale[gi].double(), shift[gi].double()
            e = e * sc.abs() + 2 * R.U32 * (r * sc).abs()
            r = r * sc + sh
            e = e + R.U32 * r.abs()
        e = 1.01 * e
        if out8:
            R.check_out8(hq[live], hs[live], r[live], e[live])
            assert torch.all(hq[~live] == 0x55) and torch.all(hs[~live] == 0x33)
            assert torch.all(hq[:, W:] == 0x55) and torch.all(hs[:, R.nblocks(W):] == 0x33)
        else:
            assert torch.all((hq[:, :W].double() - r).abs()[live] <= (R.U_BF16 * r.abs() + 1.01 * e)[live])
            assert torch.all(hq[~live] == 5.0) and torch.all(hq[:, W:] == 5.0)
    assert f3dc.gemm_status() == 0


@pytest.mark.parametrize("rows,W", [(1, 8), (1, 128), (3, 136), (5, 256), (4, 264), (9, 512), (2, 520), (700, 1024),
                                    (6, 1032), (3, 2048), (2, 2056), (3, 4096), (2, 4104), (2, 8192)])
@pytest.mark.parametrize("out8", [False, True])
def test_norm_widths(rows, W, out8):
    norm_case(rows, W, f3dc.NORM_RMS, f3dc.NORM_LAYER, True, True, 2, out8, seed=W)


# rows in pairs, an odd number of them, of different groups and pads within a pair
@pytest.mark.parametrize("W", [8, 128, 264, 512, 520, 1024, 1032, 2056, 4096, 4104])
@pytest.mark.parametrize("out8", [False, True])
def test_norm_many_rows(W, out8):
    norm_case(1301, W, f3dc.NORM_LAYER, f3dc.NORM_RMS, True, True, 3, out8, seed=W + 1, pad_cols=0 if out8 else 1)


# and so many that pairs of rows are taken at every width
@pytest.mark.parametrize("rows,W", [(16001, 136), (9000, 264), (4201, 520), (2101, 1024), (2100, 1032), (600, 4096), (70001, 32)])
@pytest.mark.parametrize("out8", [False, True])
def test_norm_pairs_of_rows(rows, W, out8):
    norm_case(rows, W, f3dc.NORM_LAYER, f3dc.NORM_LAYER, True, True, 5, out8, seed=W + 2)
    norm_case(rows, W, f3dc.NORM_RMS, f3dc.NORM_NONE, False, False, 1, out8, seed=W + 3, alpha=1.0, pads=False)


@pytest.mark.parametrize("rows", [2001, 16001])
def test_norm_bad_groups_in_many_rows(rows):
    W = 136
    x, y = randn(rows, W, seed=1), randn(rows, W, seed=2, dtype=torch.bfloat16)
    group = torch.randint(-2, 5, (rows,), generator=gen(3), device=DEV).to(torch.int32)  # 3 and 4 are behind the last
    m = randn(3, 3, W, seed=4)
    xo = torch.full((rows, W), 9.0, device=DEV)
    q, s = R.storage(rows, W)
    layer = f3dc.NormLayer(W, f3dc.NORM_RMS, f3dc.NORM_NONE)
    f3dc.norm_residual(layer, x, W, xo, W, y, W, m[:, 0], m[:, 1], m[:, 2], 3 * W, group, 3, q, q.stride(0), s, s.stride(0), rows)
    assert f3dc.gemm_status() == 2
    left = (group < 0) | (group > 2)
    assert torch.all(xo[left] == 9.0) and torch.all(q[left] == 0x55) and torch.all(s[left] == 0x33)
    g = group.clamp(0, 2).long()
    n, ne = R.norm(y.double(), torch.zeros_like(y.double()), 2, None, None, 1e-6)
    ref = x.double() + m[g, 0].double() * n
    bound = 1.01 * (ne * m[g, 0].double().abs() + R.U32 * ((m[g, 0].double() * n).abs() + ref.abs()))
    assert torch.all(((xo.double() - ref).abs() <= bound)[~left])


@pytest.mark.parametrize("rows", [3, 1300, 9001])
def test_norm_offsets_past_32_bits(rows):
    W = 256
    ld = (1 << 31) // (rows - 1) // 8 * 8 + 64  # the last row lies behind 8, 4 and 2 GiB
    def wide(v):
        t = torch.empty((rows - 1) * ld + W, dtype=v.dtype, device=DEV).as_strided((rows, W), (ld, 1))
        return t.copy_(v)
    x, y = randn(rows, W, seed=1), randn(rows, W, seed=2, dtype=torch.bfloat16)
    m = randn(2, W, seed=3)
    mw = torch.empty((1 << 31) + W, device=DEV).as_strided((2, W), (1 << 31, 1)).copy_(m)
    group = torch.randint(0, 2, (rows,), generator=gen(4), device=DEV).to(torch.int32)
    layer = f3dc.NormLayer(W, f3dc.NORM_LAYER, f3dc.NORM_RMS)
    h, xo = torch.zeros((rows, W), dtype=torch.bfloat16, device=DEV), torch.zeros((rows, W), device=DEV)
    f3dc.norm_residual(layer, x, W, xo, W, y, W, m, None, m, W, group, 2, h, W, None, 0, rows)
    hw, xow = wide(torch.zeros_like(h)), wide(torch.zeros_like(xo))
    f3dc.norm_residual(layer, wide(x), ld, xow, ld, wide(y), ld, mw, None, mw, 1 << 31, group, 2, hw, ld, None, 0, rows)
    assert torch.equal(hw, h) and torch.equal(xow, xo)
    assert f3dc.gemm_status() == 0


@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("pre", [0, 1, 2])
@pytest.mark.parametrize("affine,mod", [(True, True), (False, True), (True, False), (False, False)])
def test_norm_kinds(post, pre, affine, mod):
    norm_case(37, 384, post, pre, affine, mod, 3, (post + pre) % 2 == 1, seed=100 + post + pre)


@pytest.mark.parametrize("y,x_out,h", [(False, True, True), (False, False, True), (True, False, True), (True, True, False)])
def test_norm_optional_parts(y, x_out, h):
    norm_case(50, 1000, 1, 2, True, True, 2, False, y=y, x_out=x_out, h=h, seed=7, pad_cols=3)
    norm_case(50, 1000, 2, 1, True, True, 1, h, y=y, x_out=x_out, h=h, seed=8, alpha=1.0, pads=False)


def test_norm_in_place():
    W, rows = 512, 40
    x, y = randn(rows, W, seed=1), randn(rows, W, seed=2, dtype=torch.bfloat16)
    layer = f3dc.NormLayer(W, f3dc.NORM_RMS, f3dc.NORM_LAYER, res_scale=0.5)
    outs = []
    for in_place in (False, True):
        xi = x.clone()
        xo = xi if in_place else torch.empty_like(x)
        h = torch.empty((rows, W), dtype=torch.bfloat16, device=DEV)
        f3dc.norm_residual(layer, xi, W, xo, W, y, W, None, None, None, 0, None, 1, h, W, None, 0, rows)
        outs.append((xo, h))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_norm_bad_group_and_non_finite_rows():
    # a group outside its range leaves its row and is recorded; NaN and infinities of
    # a row, or of a pad row, stay there
    W, rows = 256, 12
    x, y = randn(rows, W, seed=1), randn(rows, W, seed=2, dtype=torch.bfloat16)
    group = torch.zeros(rows, dtype=torch.int32, device=DEV)
    group[4], group[5], group[6] = 2, -1, 2 ** 31 - 1
    x[5], y[5] = float("nan"), float("inf")
    y[7, 3], x[8, 200] = float("nan"), float("inf")
    xo, h = torch.full((rows, W), 9.0, device=DEV), torch.full((rows, W), 5.0, dtype=torch.bfloat16, device=DEV)
    layer = f3dc.NormLayer(W, f3dc.NORM_LAYER, f3dc.NORM_RMS)
    f3dc.norm_residual(layer, x, W, xo, W, y, W, None, None, None, 0, group, 2, h, W, None, 0, rows)
    assert f3dc.gemm_status() == 2  # F3DC_DEV_BAD_INDEX
    left = torch.tensor([4, 5, 6], device=DEV)
    assert torch.all(xo[left] == 9.0) and torch.all(h[left] == 5.0)
    assert torch.all(torch.isnan(xo[7])) and torch.all(torch.isnan(h[7])) and torch.isinf(xo[8, 200])
    rest = torch.tensor([0, 1, 2, 3, 9, 10, 11], device=DEV)
    assert torch.all(torch.isfinite(xo[rest])) and torch.all(torch.isfinite(h[rest].float()))
    assert f3dc.gemm_status() == 0


def test_norm_no_rows_and_constant_row():
    W = 128
    layer = f3dc.NormLayer(W, f3dc.NORM_LAYER, f3dc.NORM_LAYER)
    x, h = torch.full((2, W), 3.0, device=DEV), torch.full((2, W), 5.0, dtype=torch.bfloat16, device=DEV)
    f3dc.norm_residual(layer, x, W, None, 0, None, 0, None, None, None, 0, None, 1, h, W, None, 0, 0)
    assert torch.all(h == 5.0)
    y = torch.zeros((2, W), dtype=torch.bfloat16, device=DEV)
    xo = torch.empty_like(x)
    f3dc.norm_residual(layer, x, W, xo, W, y, W, None, None, None, 0, None, 1, h, W, None, 0, 2)
    assert torch.equal(xo, x) and torch.all(h == 0.0)  # no variance: eps keeps it finite


# ------------------------------------------------------------- used together

def mlp(W, hidden, rows, seed):
    """The MLP half of a block in 8 bits: norm -> fc1 + GELU -> fc2 -> norm."""
    g = randn(2, 3, W, seed=seed + 1, scale=0.3)
    group = torch.randint(-1, 2, (rows,), generator=gen(seed), device=DEV).to(torch.int32)
    return dict(W=W, hidden=hidden, rows=rows, group=group, mod=g, x=randn(rows, W, seed=seed + 2),
                y=randn(rows, W, seed=seed + 3, dtype=torch.bfloat16),
                w1=quantize(randn(hidden, W, seed=seed + 4, scale=W ** -0.5)),
                w2=quantize(randn(W, hidden, seed=seed + 5, scale=hidden ** -0.5)),
                b1=randn(hidden, seed=seed + 6, dtype=torch.bfloat16), b2=randn(W, seed=seed + 7, dtype=torch.bfloat16),
                l1=f3dc.NormLayer(W, f3dc.NORM_NONE, f3dc.NORM_LAYER),
                l2=f3dc.NormLayer(W, f3dc.NORM_RMS, f3dc.NORM_LAYER, res_scale=0.9),
                h8=tuple(torch.zeros_like(t) for t in R.storage(rows, W)), a8=tuple(torch.zeros_like(t) for t in R.storage(rows, hidden)),
                x1=torch.zeros((rows, W), device=DEV), x2=torch.zeros((rows, W), device=DEV),
                z=torch.zeros((rows, W), dtype=torch.bfloat16, device=DEV), h=torch.zeros((rows, W), dtype=torch.bfloat16, device=DEV))


def run_mlp(m, stream=None):
    W, rows, mod = m["W"], m["rows"], m["mod"]
    gate, scale, shift = mod[:, 0], mod[:, 1], mod[:, 2]
    (hq, hs), (aq, as_) = m["h8"], m["a8"]
    f3dc.norm_residual(m["l1"], m["x"], W, m["x1"], W, m["y"], W, gate, scale, shift, 3 * W, m["group"], 2, hq, hq.stride(0), hs,
                       hs.stride(0), rows, stream=stream)
    gemm8(hq, hs, *m["w1"], W, f3dc.EPI_GELU, m["b1"], None, aq, as_, stream=stream)
    gemm8(aq, as_, *m["w2"], m["hidden"], f3dc.EPI_BIAS, m["b2"], None, m["z"], stream=stream)
    f3dc.norm_residual(m["l2"], m["x1"], W, m["x2"], W, m["z"], W, gate, scale, shift, 3 * W, m["group"], 2, m["h"], W, None, 0,
                       rows, stream=stream)


def test_mlp_block_in_8_bits():
    m = mlp(256, 1024, 300, 5)
    run_mlp(m)
    assert f3dc.gemm_status() == 0
    live = m["group"] >= 0
    gi = m["group"].clamp(min=0).long()
    gate, scale, shift = (m["mod"][gi, i].double() for i in range(3))
    # stage by stage, each from the library's own input to it
    x1 = m["x"].double() + gate * m["y"].double()
    assert torch.all((m["x1"].double() - x1).abs()[live] <= (3 * R.U32 * (x1.abs() + (gate * m["y"].double()).abs()))[live])
    r, e = R.norm(x1, 3 * R.U32 * (x1.abs() + 1), 1, None, None, 1e-6)
    r, e = r * (1 + scale) + shift, e * (1 + scale).abs() + 4 * R.U32 * (r.abs() + 1)
    R.check_out8(m["h8"][0][live], m["h8"][1][live], r[live], e[live])
    a, ae = R.gemm(*m["h8"], *m["w1"], 256, m["b1"])
    R.check_out8(*m["a8"], R.gelu(a), R.gelu_bound(a, ae))
    z, ze = R.gemm(*m["a8"], *m["w2"], 1024, m["b2"])
    assert torch.all((m["z"].double() - z).abs() <= R.U_BF16 * z.abs() + 1.01 * ze)
    n, ne = R.norm(m["z"].double(), torch.zeros_like(z), 2, None, None, 1e-6)
    x2 = float(np.float32(0.9)) * m["x1"].double() + gate * n
    assert torch.all((m["x2"].double() - x2).abs()[live] <= (gate.abs() * ne + 4 * R.U32 * (x2.abs() + n.abs()))[live])
    # and the whole against a block in 64 bits that is not quantised at all: two
    # 8-bit activations and two 8-bit weights, each off by up to 2^-4 relative
    # (rms 2.6e-2), give about 2.6e-2 sqrt(2) after each product
    w1, w2 = R.values(*m["w1"], 256), R.values(*m["w2"], 1024)
    full = R.gelu(r @ w1.T + m["b1"].double()) @ w2.T + m["b2"].double()
    full = float(np.float32(0.9)) * x1 + gate * R.norm(full, torch.zeros_like(full), 2, None, None, 1e-6)[0]
    assert ((m["x2"].double() - full)[live].norm() / full[live].norm()).item() < 0.0625
    assert torch.all(m["x2"][~live] == 0) and torch.all(m["h"][~live] == 0)


def test_mlp_block_on_streams_and_in_graphs():
    # three blocks, eager for reference; then at once on two streams and replayed
    # from two captured graphs that share the library and nothing else
    want = []
    for i in range(3):
        m = mlp(256, 512, 200 + i, 20 + i)
        run_mlp(m)
        want.append((m["x2"].clone(), m["h"].clone()))
    torch.cuda.synchronize()
    ms = [mlp(256, 512, 200 + i, 20 + i) for i in range(3)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for m, st in zip(ms[:2], streams):
        run_mlp(m, stream=st.cuda_stream)
    torch.cuda.synchronize()
    for m, (x2, h) in zip(ms[:2], want):
        assert torch.equal(m["x2"], x2) and torch.equal(m["h"], h)
    graphs = []
    for m in ms[1:]:
        m["x2"].zero_(), m["h"].zero_()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run_mlp(m)
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for m, (x2, h) in zip(ms[1:], want[1:]):
        assert torch.equal(m["x2"], x2) and torch.equal(m["h"], h)
    assert f3dc.gemm_status() == 0


def test_tensors_of_another_device_are_refused():
    x, (q, s) = torch.zeros((4, 64)), R.storage(4, 64)
    with pytest.raises(f3dc.F3dcError) as e:
        f3dc.quantize_fp8(x, 64, q, 64, s, 4, 4, 64)
    assert e.value.status == 1
    with pytest.raises(f3dc.F3dcError) as e:
        f3dc.quantize_fp8(x.to(DEV).half(), 64, q, 64, s, 4, 4, 64)
    assert e.value.status == 1
    for vec in (torch.ones(64, dtype=torch.bfloat16), torch.ones(64, device=DEV), torch.ones(32, dtype=torch.bfloat16, device=DEV)):
        with pytest.raises(f3dc.F3dcError) as e:
            f3dc.NormLayer(64, pre_g=vec)
        assert e.value.status == 1
