// k_quant.cu -- quantisation to e4m3 with one power-of-two scale per block of 128
// elements of a row (f3dc_quantize_fp8).
//
// q = x 2^-e rounded to nearest even, e the smallest integer with max |x| <= 448 2^e
// over the block.  The quotient by a power of two is exact, so the one rounding is
// the conversion's and the result is the same bit for bit in whatever order.
//
// Bound by memory: x is read once, one byte and 1/128 written per element.  A block
// is held by 8 lanes, 16 elements each; a warp takes four blocks at a time, wherever
// rows end, and of fp32, with more than a wave of work, twice four (16384 x 4096: 56 us
// with one group in flight, 50 with two; 600 x 4096 3.7 and 3.3, but 400 x 4096 3.0 and
// 3.1; bf16, 32768 x 4096, 61 and 75).  32768 x 4096 of bf16 in 61 us: 6.6 TB/s, 97 % of
// what a plain copy reaches.  Rows that do not start on 16 bytes take twice the load and store
// instructions (a third piece per 32 bytes, row ends element by element) and 1.4 times the
// sectors: 32768 x 4095 83 us, x 1001 24 (39 and 64 % above their bytes at the copy's rate).
#include "kernels.h"
#include "mx8.cuh"

namespace f3dc {

namespace {

constexpr int kQuantThreads = 256;

// 16 elements as 32-bit words: 8 of bf16 pairs, 16 of fp32
template <bool F32>
struct Words {
    static constexpr int kN = F32 ? 16 : 8;
    uint32_t w[kN];
};

F3DC_DEV uint4 load_stream(const void *p) { return __ldcs(reinterpret_cast<const uint4 *>(p)); }

// Elements col .. col + 15 of a row, zeros from n on.  ALIGNED: the row starts on 16
// bytes.  Otherwise the 16-byte pieces that hold the elements are read and shifted
// into place; `edge` (the matrix's first and last elements, whose pieces may reach out
// of it) and a row's last elements are read one by one.
template <bool F32, bool ALIGNED>
F3DC_DEV void load16(const uint8_t *row, int col, int n, bool edge, Words<F32> &x)
{
    constexpr int N = Words<F32>::kN;
    const uint8_t *p = row + (int64_t)col * (F32 ? 4 : 2);
    if (n < 16 || (!ALIGNED && edge)) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if constexpr (F32) {
                x.w[j] = j < n ? reinterpret_cast<const uint32_t *>(p)[j] : 0u;
            } else {
                const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
                x.w[j] = (2 * j < n ? (uint32_t)h[2 * j] : 0u) | (2 * j + 1 < n ? (uint32_t)h[2 * j + 1] << 16 : 0u);
            }
        }
        return;
    }
    if constexpr (ALIGNED) {
#pragma unroll
        for (int c = 0; c < N / 4; ++c) {
            const uint4 u = load_stream(p + 16 * c);
            x.w[4 * c] = u.x, x.w[4 * c + 1] = u.y, x.w[4 * c + 2] = u.z, x.w[4 * c + 3] = u.w;
        }
    } else {
        const uint32_t off = (uint32_t)(uintptr_t)p & 15u;
        const uint8_t *a = p - off;
        uint32_t w[N + 4];
#pragma unroll
        for (int c = 0; c < N / 4; ++c) {
            const uint4 u = *reinterpret_cast<const uint4 *>(a + 16 * c);
            w[4 * c] = u.x, w[4 * c + 1] = u.y, w[4 * c + 2] = u.z, w[4 * c + 3] = u.w;
        }
        w[N] = w[N + 1] = w[N + 2] = w[N + 3] = 0u;
        if (off) {
            const uint4 u = *reinterpret_cast<const uint4 *>(a + 4 * N);
            w[N] = u.x, w[N + 1] = u.y, w[N + 2] = u.z, w[N + 3] = u.w;
        }
        if (off & 8u) {
#pragma unroll
            for (int j = 0; j < N + 2; ++j) w[j] = w[j + 2];
        }
        if (off & 4u) {
#pragma unroll
            for (int j = 0; j < N + 1; ++j) w[j] = w[j + 1];
        }
#pragma unroll
        for (int j = 0; j < N; ++j) x.w[j] = F32 ? w[j] : __funnelshift_r(w[j], w[j + 1], 8 * (off & 2u));
    }
}

template <bool F32>
F3DC_DEV void unpack(const Words<F32> &x, float (&v)[16])
{
#pragma unroll
    for (int j = 0; j < 16; ++j)
        v[j] = __uint_as_float(F32 ? x.w[j & (Words<F32>::kN - 1)] : (j & 1 ? x.w[j / 2] & 0xFFFF0000u : x.w[j / 2] << 16));
}

// Resident CTAs per SM: 40 registers for bf16, up to 80 for the 64 bytes per lane of fp32.
constexpr int quant_ctas(bool f32) { return f32 ? 3 : 6; }

// ALIGNED: rows of x start on 16 bytes.  WIDE: rows of q do; otherwise bytes are stored
// one by one.  U groups of four blocks per warp and step.
template <bool F32, bool ALIGNED, bool WIDE, int U>
__global__ void __launch_bounds__(kQuantThreads, quant_ctas(F32)) k_quantize(const QuantArgs a)
{
    // (a next launch's CTAs would take the places that two groups leave, and its work would then
    // lie unevenly on the SMs: 16384 x 4096 of fp32, back to back, 54 us instead of 50)
    if (U == 1) griddep_launch();
    griddep_wait();
    const int lane = threadIdx.x & 31;
    const int per_row = (a.cols - 1) / kScaleBlock + 1;
    const int64_t groups = ((int64_t)a.rows * per_row + 3) / 4;  // of four blocks
    const int64_t warps = (int64_t)gridDim.x * (kQuantThreads / 32);
    const int64_t first = (int64_t)blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5);
    // block i of the matrix is block i % per_row of row i / per_row; the one that is
    // 4 `warps` further is found without a division (a 64-bit one is as long as the rest of
    // the loop), the first with one of 32 bits: the grid is one wave, a few thousand warps
    const uint32_t step = 4u * (uint32_t)warps, mine = 4u * (uint32_t)first + (lane >> 3);
    const int64_t step_rows = step / (uint32_t)per_row;
    const int step_blocks = (int)(step % (uint32_t)per_row);
    int64_t next_row = mine / (uint32_t)per_row;
    int next_block = (int)(mine % (uint32_t)per_row);
    for (int64_t group = first; group < groups; group += U * warps) {
        Words<F32> x[U];
        int64_t row[U];
        int col[U], n[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = next_row;
            col[u] = next_block * kScaleBlock + (lane & 7) * 16;
            n[u] = next_row < a.rows ? a.cols - col[u] : 0;  // this lane's elements (more than 16, or none, too)
            next_row += step_rows;
            next_block += step_blocks;
            if (next_block >= per_row) {
                next_block -= per_row;
                ++next_row;
            }
            const bool edge = (row[u] == 0 && col[u] == 0) || (row[u] == a.rows - 1 && n[u] < 32);
            load16<F32, ALIGNED>(reinterpret_cast<const uint8_t *>(a.x) + row[u] * a.ldx * (F32 ? 4 : 2), col[u], n[u], edge, x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[16];
            unpack<F32>(x[u], v);
            const uint32_t byte = quantize_block<16, 8>(v);
            const uint32_t w[4] = {pack_e4m3x4(v[0], v[1], v[2], v[3]), pack_e4m3x4(v[4], v[5], v[6], v[7]),
                                   pack_e4m3x4(v[8], v[9], v[10], v[11]), pack_e4m3x4(v[12], v[13], v[14], v[15])};
            uint8_t *q = a.q + row[u] * a.ldq + col[u];
            if (WIDE && n[u] >= 16) {
                __stcs(reinterpret_cast<uint4 *>(q), make_uint4(w[0], w[1], w[2], w[3]));
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (j < n[u]) q[j] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
            }
            if (lane % 8 == 0 && n[u] > 0) a.scales[row[u] * a.lds + col[u] / kScaleBlock] = (uint8_t)byte;
        }
    }
}

template <bool F32>
cudaError_t launch_type(const QuantArgs &a, int num_sms, cudaStream_t s)
{
    const int64_t groups = ((int64_t)a.rows * ((a.cols - 1) / kScaleBlock + 1) + 3) / 4, per = kQuantThreads / 32;
    const int64_t ctas = (groups + per - 1) / per, most = (int64_t)num_sms * quant_ctas(F32);
    const dim3 g((unsigned)(ctas < most ? ctas : most)), b(kQuantThreads);
    const bool aligned = ((uintptr_t)a.x & 15) == 0 && (a.ldx * (F32 ? 4 : 2)) % 16 == 0;
    const bool wide = ((uintptr_t)a.q & 15) == 0 && a.ldq % 16 == 0;
    if (!wide) return launch_k(k_quantize<F32, false, false, 1>, g, b, 0, s, a);
    if constexpr (F32) {
        if (ctas > most)
            return aligned ? launch_k(k_quantize<F32, true, true, 2>, g, b, 0, s, a)
                           : launch_k(k_quantize<F32, false, true, 2>, g, b, 0, s, a);
    }
    return aligned ? launch_k(k_quantize<F32, true, true, 1>, g, b, 0, s, a)
                   : launch_k(k_quantize<F32, false, true, 1>, g, b, 0, s, a);
}

}  // namespace

cudaError_t launch_quantize(const QuantArgs &a, bool f32, int num_sms, cudaStream_t s)
{
    return f32 ? launch_type<true>(a, num_sms, s) : launch_type<false>(a, num_sms, s);
}

}  // namespace f3dc
