// k_quant.cu -- quantisation to e4m3 with one power-of-two scale per block of 128
// elements of a row (f3dc_quantize_fp8).
//
// q = x 2^-e rounded to nearest even, e the smallest integer with max |x| <= 448 2^e
// over the block.  The quotient by a power of two is exact, so the one rounding is
// the conversion's and the result is the same bit for bit in whatever order.
//
// Bound by memory: x is read once, one byte and 1/128 written per element.  A block
// is held by 8 lanes, 16 elements each (rows that start on 16 bytes), or by a whole
// warp (any other row).
#include "kernels.h"
#include "mx8.cuh"

namespace f3dc {

namespace {

constexpr int kQuantThreads = 256;

// 16 consecutive elements of a row from 16-byte aligned memory, zeros from n on
template <bool F32>
F3DC_DEV void load16(const void *row, int col, int n, float (&v)[16])
{
    if (n >= 16) {
        if constexpr (F32) {
            const float4 *p = reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(row) + col);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 u = __ldcs(p + q);
                v[4 * q] = u.x, v[4 * q + 1] = u.y, v[4 * q + 2] = u.z, v[4 * q + 3] = u.w;
            }
        } else {
            const uint4 *p = reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(row) + col);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint4 u = __ldcs(p + q);
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[8 * q + 2 * j] = bf16_bits_to_f32(w[j] & 0xFFFFu);
                    v[8 * q + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
                }
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        v[j] = 0.f;
        if (j < n)
            v[j] = F32 ? reinterpret_cast<const float *>(row)[col + j]
                       : bf16_bits_to_f32(reinterpret_cast<const uint16_t *>(row)[col + j]);
    }
}

// Rows that start on 16 bytes (x, q): a warp takes four blocks at a time.
template <bool F32>
__global__ void __launch_bounds__(kQuantThreads) k_quantize(const QuantArgs a)
{
    griddep_launch();
    griddep_wait();
    const int lane = threadIdx.x & 31;
    const int chunks = (a.cols + 511) / 512;  // of four blocks
    const int64_t items = (int64_t)a.rows * chunks;
    const int64_t step = (int64_t)gridDim.x * (kQuantThreads / 32);
    for (int64_t it = (int64_t)blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5); it < items; it += step) {
        const int64_t row = it / chunks;
        const int col = (int)(it - row * chunks) * 512 + lane * 16;
        const int n = a.cols - col;  // this lane's elements (more than 16, or none, too)
        float v[16];
        load16<F32>(reinterpret_cast<const uint8_t *>(a.x) + row * a.ldx * (F32 ? 4 : 2), col, n, v);
        const uint32_t byte = quantize_block<16, 8>(v);
        uint4 u;
        u.x = pack_e4m3x4(v[0], v[1], v[2], v[3]);
        u.y = pack_e4m3x4(v[4], v[5], v[6], v[7]);
        u.z = pack_e4m3x4(v[8], v[9], v[10], v[11]);
        u.w = pack_e4m3x4(v[12], v[13], v[14], v[15]);
        uint8_t *q = a.q + row * a.ldq + col;
        if (n >= 16) {
            *reinterpret_cast<uint4 *>(q) = u;
        } else {
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (j < n) q[j] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
        }
        if (lane % 8 == 0 && n > 0) a.scales[row * a.lds + col / kScaleBlock] = (uint8_t)byte;
    }
}

// Any rows: a warp takes four blocks, element 32 i + lane of the 512 in lane `lane`, so
// that single-element loads and stores are whole sectors.
template <bool F32>
__global__ void __launch_bounds__(kQuantThreads) k_quantize_any(const QuantArgs a)
{
    griddep_launch();
    griddep_wait();
    const int lane = threadIdx.x & 31;
    const int chunks = (a.cols + 511) / 512;
    const int64_t items = (int64_t)a.rows * chunks;
    const int64_t step = (int64_t)gridDim.x * (kQuantThreads / 32);
    for (int64_t it = (int64_t)blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5); it < items; it += step) {
        const int64_t row = it / chunks;
        const int col0 = (int)(it - row * chunks) * 512;
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int col = col0 + 32 * i + lane;
            v[i] = 0.f;
            if (col < a.cols)
                v[i] = F32 ? __ldcs(reinterpret_cast<const float *>(a.x) + row * a.ldx + col)
                           : bf16_bits_to_f32(__ldcs(reinterpret_cast<const uint16_t *>(a.x) + row * a.ldx + col));
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            float w[4] = {v[4 * b], v[4 * b + 1], v[4 * b + 2], v[4 * b + 3]};
            const uint32_t byte = quantize_block<4, 32>(w);
            const uint32_t u = pack_e4m3x4(w[0], w[1], w[2], w[3]);
            const int col = col0 + kScaleBlock * b + lane;
            uint8_t *q = a.q + row * a.ldq;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (col + 32 * j < a.cols) q[col + 32 * j] = (uint8_t)(u >> (8 * j));
            if (lane == 0 && col < a.cols) a.scales[row * a.lds + col / kScaleBlock] = (uint8_t)byte;
        }
    }
}

}  // namespace

cudaError_t launch_quantize(const QuantArgs &a, bool f32, int num_sms, cudaStream_t s)
{
    const int64_t items = (int64_t)a.rows * ((a.cols + 511) / 512), per = kQuantThreads / 32;
    const int64_t most = (int64_t)num_sms * 8;  // resident CTAs
    const int grid = (int)((items + per - 1) / per < most ? (items + per - 1) / per : most);
    const bool aligned = ((uintptr_t)a.x & 15) == 0 && (a.ldx * (f32 ? 4 : 2)) % 16 == 0 &&
                         ((uintptr_t)a.q & 15) == 0 && a.ldq % 16 == 0;
    if (aligned)
        return f32 ? launch_k(k_quantize<true>, dim3(grid), dim3(kQuantThreads), 0, s, a)
                   : launch_k(k_quantize<false>, dim3(grid), dim3(kQuantThreads), 0, s, a);
    return f32 ? launch_k(k_quantize_any<true>, dim3(grid), dim3(kQuantThreads), 0, s, a)
               : launch_k(k_quantize_any<false>, dim3(grid), dim3(kQuantThreads), 0, s, a);
}

}  // namespace f3dc
