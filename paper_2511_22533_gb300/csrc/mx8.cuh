// mx8.cuh -- device helpers of the 8-bit linear layers: tcgen05 MMAs with block
// scales (kind::mxf8f6f4), the copy of scales into tensor memory, and conversion to
// e4m3 under one power-of-two (E8M0) scale per block of 128 elements.
#pragma once

#include "common.cuh"

namespace f3dc {

// A stage of operands of a CTA pair, under one election of a converged warp: TMA loads of a
// 2-D box of A and of B into this CTA's shared memory, whose bytes an mbarrier of the even
// CTA counts (full_cluster, a shared::cluster address).  expect != 0: that CTA, which first
// arrives there, announcing both CTAs' bytes.  Returns whether the phase `parity` of `next`
// is complete, read ahead of the loads so that nothing waits for the answer.  (Address
// arithmetic in a loop run by one lane, two loads and a wait took some 490 clocks a stage.)
F3DC_DEV bool tma_load_stage_pair(uint32_t dst_a, const CUtensorMap *map_a, int row_a, uint32_t dst_b,
                                  const CUtensorMap *map_b, int row_b, int x, uint32_t full, uint32_t full_cluster,
                                  uint32_t expect, uint32_t next, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred e, q, r;\n"
        " mbarrier.test_wait.parity.shared::cta.b64 r, [%11], %12;\n"
        " elect.sync _|e, 0xffffffff;\n setp.ne.b32 q, %10, 0;\n and.pred q, q, e;\n"
        " @q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%8], %10;\n"
        " @e cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%1], [%2, {%7, %3}], [%9];\n"
        " @e cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%4], [%5, {%7, %6}], [%9];\n"
        " selp.u32 %0, 1, 0, r;\n}\n"
        : "=r"(ok)
        : "r"(dst_a), "l"((uint64_t)map_a), "r"(row_a), "r"(dst_b), "l"((uint64_t)map_b), "r"(row_b), "r"(x), "r"(full),
          "r"(full_cluster), "r"(expect), "r"(next), "r"(parity)
        : "memory");
    return ok != 0;
}

// Arrival on an mbarrier of either CTA that publishes no memory: what it orders are TMEM
// reads (waited for) or an allocation of TMEM, which tcgen05.fence::before_thread_sync
// covers.  (A release at cluster scope takes about 1000 clocks behind global stores.)
F3DC_DEV void mbar_arrive_relaxed(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// Arrival that publishes this CTA's shared memory, already made visible to the async proxy
// (fence_proxy_async_smem), on an mbarrier of the same CTA: a release at CTA scope.
F3DC_DEV void mbar_arrive_own_smem(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.release.cta.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// 16 bytes into the shared memory of a CTA of the cluster
F3DC_DEV void store_cluster16(uint32_t cluster_addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_addr), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}

// mbar_wait by a whole warp for what other CTAs of the cluster have read or written before
// their arrivals (mbar_arrive_cluster): a last look at the phase, which is over, acquires at
// cluster scope.
F3DC_DEV bool warp_wait_cluster(uint64_t *bar, uint32_t parity, volatile int *abort, uint32_t *err)
{
    const bool ok = warp_wait(bar, parity, abort, err);
    asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%0], %1;\n}\n" ::"r"(
                     smem_u32(bar)),
                 "r"(parity)
                 : "memory");
    return ok;
}

// 16 bytes of global memory into shared memory, and the wait for this thread's
F3DC_DEV void cp_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
F3DC_DEV void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// the two halves of a cluster barrier that publishes nothing, for whole warps
F3DC_DEV void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
F3DC_DEV void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// D (+)= A B^T over a CTA pair (mma_bf16_pair_128k says which rows lie where), e4m3
// operands with one E8M0 scale per row and 128 K.  The scales lie in tensor memory
// (tmem_cp_scales_pair); each MMA takes the byte of a scale column that its instruction
// descriptor names for all of its 32 K.  The four MMAs of 128 K (32 K further is 2
// descriptor units) and their commit to `bar` (of the CTAs in `mask`) under one election.
// Returns whether the phases of next0 and next1 are complete, read ahead of the MMAs so that
// nothing waits for the answer.
#define F3DC_MXF8(D, A, B, SA, SB, I, P) \
    " @e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [" D "], " A ", " B ", " I ", [" SA "], [" SB "], " P ";\n"
#define F3DC_MXF8_NEXT " add.s64 a, a, 2;\n add.s64 b, b, 2;\n"
F3DC_DEV bool mma_mxf8_pair_128k(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t sfa_tmem,
                                 uint32_t sfb_tmem, uint32_t idesc, uint32_t accumulate, uint64_t *bar, uint16_t mask,
                                 uint64_t *next0, uint32_t parity0, uint64_t *next1, uint32_t parity1)
{
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p, e, t, r0, r1;\n .reg .b64 a, b;\n"
        " mbarrier.test_wait.parity.shared::cta.b64 r0, [%10], %11;\n"
        " mbarrier.test_wait.parity.shared::cta.b64 r1, [%12], %13;\n"
        " elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %7, 0;\n setp.eq.b32 t, 0, 0;\n"
        F3DC_MXF8("%1", "%2", "%3", "%4", "%5", "%6", "p")
        " add.s64 a, %2, 2;\n add.s64 b, %3, 2;\n" F3DC_MXF8("%1", "a", "b", "%4", "%5", "%6", "t")
        F3DC_MXF8_NEXT F3DC_MXF8("%1", "a", "b", "%4", "%5", "%6", "t")
        F3DC_MXF8_NEXT F3DC_MXF8("%1", "a", "b", "%4", "%5", "%6", "t")
        " @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%8], %9;\n"
        " and.pred r0, r0, r1;\n selp.u32 %0, 1, 0, r0;\n"
        "}\n" : "=r"(ok) : "r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(sfa_tmem), "r"(sfb_tmem), "r"(idesc), "r"(accumulate), "r"(smem_u32(bar)), "h"(mask),
        "r"(smem_u32(next0)), "r"(parity0), "r"(smem_u32(next1)), "r"(parity1)
        : "memory");
    return ok != 0;
}
#undef F3DC_MXF8
#undef F3DC_MXF8_NEXT

// Copies 32 rows of 16 bytes (512 consecutive bytes of shared memory, row r at 16 r)
// of each CTA of the pair into 4 columns of its own tensor memory, the same 32 lanes
// four times: the scale bytes of 128 matrix rows, of which row i is lane i % 32,
// column i / 32.
F3DC_DEV void tmem_cp_scales_pair(uint32_t taddr, uint64_t sdesc)
{
    asm volatile(
        "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n"
        " @e tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n}\n" ::"r"(taddr),
        "l"(sdesc)
        : "memory");
}

// Instruction descriptor, kind::mxf8f6f4 with block scales: e4m3 A and B (bits 7-9,
// 10-12 = 0), both K-major, N >> 3 in bits 17-22, E8M0 scales (bit 23 = 1), M >> 4 in
// bits 24-28; the byte of the scale columns to take, for B in bits 4-5, for A in 29-30.
__host__ __device__ constexpr uint32_t make_idesc_mxf8(int M, int N, int scale_byte)
{
    return ((uint32_t)scale_byte << 4) | ((uint32_t)(N >> 3) << 17) | (1u << 23) | ((uint32_t)(M >> 4) << 24) |
           ((uint32_t)scale_byte << 29);
}

// ---- GELU, 0.5 x (1 + tanh(sqrt(2 / pi) (x + 0.044715 x^3))), as x / (1 + 2^-z) with z = 2
// sqrt(2 / pi) log2(e) (x + 0.044715 x^3): with tanh the sum cancels for negative x, and below -4
// little that is right is left.  The quotient is within 2^-15 of the value (the rounding of
// z, at most 128 where it counts, and both approximations); results below 2^-120 may
// become zeros.  2^-z is infinite for very negative x, whose quotient is then zero.
constexpr float kGelu1 = -2.302208198f, kGelu3 = kGelu1 * 0.044715f;  // -z of x and of x^3
F3DC_DEV float rcp_fast(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
F3DC_DEV f32x2 gelu2(f32x2 x)
{
    const f32x2 z = fmul2(x, ffma2(fmul2(x, x), {kGelu3, kGelu3}, {kGelu1, kGelu1}));
    const f32x2 d = fadd2({exp2_fast(z.x), exp2_fast(z.y)}, {1.f, 1.f});
    return fmul2(x, {rcp_fast(d.x), rcp_fast(d.y)});
}
F3DC_DEV float gelu1(float x) { return x * rcp_fast(1.f + exp2_fast(x * fmaf(x * x, kGelu3, kGelu1))); }

// ---- e4m3 with one E8M0 (power-of-two) scale per block of 128.
// Scale byte of a block whose largest finite magnitude is `top`: the smallest e with
// top <= 448 2^e = 1.75 2^(8 + e), as e + 127, read off top's exponent and mantissa.
// A normal top gives 0 <= byte <= 247; smaller ones clamp to 2^-127.
F3DC_DEV uint32_t e8m0_byte(float top)
{
    const uint32_t u = __float_as_uint(top);
    const int b = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(b, 0);
}
// 2^-e of such a byte (at most 247): multiplying by it is exact but for results
// below fp32's range, which e4m3 cannot hold either
F3DC_DEV float e8m0_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// four floats (at most 448 in magnitude, or NaN) to e4m3, round to nearest even, `a` in the lowest byte
F3DC_DEV uint32_t pack_e4m3x4(float a, float b, float c, float d)
{
    uint32_t r;
    asm("{\n .reg .b16 lo, hi;\n cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n"
        " mov.b32 %0, {lo, hi};\n}\n"
        : "=r"(r)
        : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// Quantises N consecutive values of each of R rows, the share of this lane in a block of
// each that `LANES` neighbouring lanes hold together: v becomes the quotients (at most 448
// in magnitude; NaN for NaN and for infinities, which e4m3 does not have), byte the scale
// bytes.  Every lane of the warp calls it; absent values are zeros.  fmaxf passes over
// NaN, so the plain maximum is infinite only with an infinity among the values: the rare
// block that has one takes the maximum of the finite ones.
template <int R, int N, int LANES>
F3DC_DEV void quantize_blocks(float (&v)[R][N], uint32_t (&byte)[R])
{
    const float inf = __int_as_float(0x7F800000);
    float top[R];
    auto maxima = [&] {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            top[i] = 0.f;
#pragma unroll
            for (int j = 0; j + 1 < N; j += 2) top[i] = fmax3(top[i], fabsf(v[i][j]), fabsf(v[i][j + 1]));
        }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < R; ++i) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], o));
    };
    maxima();
    bool some = false;
#pragma unroll
    for (int i = 0; i < R; ++i) some |= top[i] == inf;
    if (__any_sync(0xffffffffu, some)) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (fabsf(v[i][j]) == inf) v[i][j] = __int_as_float(0x7FC00000);
        maxima();
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        byte[i] = e8m0_byte(top[i]);
        const float inv = e8m0_inverse(byte[i]);
#pragma unroll
        for (int j = 0; j + 1 < N; j += 2) {
            const f32x2 q = fmul2({v[i][j], v[i][j + 1]}, {inv, inv});
            v[i][j] = q.x, v[i][j + 1] = q.y;
        }
    }
}
template <int N, int LANES>
F3DC_DEV uint32_t quantize_block(float (&v)[N])
{
    static_assert(N % 2 == 0, "pairs");
    uint32_t byte[1];
    quantize_blocks<1, N, LANES>(reinterpret_cast<float (&)[1][N]>(v), byte);
    return byte[0];
}

}  // namespace f3dc
