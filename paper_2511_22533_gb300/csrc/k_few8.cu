// k_few8.cu -- the 8-bit product of f3dc_gemm_fp8 for a few rows (single tokens, small
// batches of them):
//
//   out[m, n] = epilogue( sum_k A[m, k] 2^ea[m, k / 128] B[n, k] 2^eb[n, k / 128] ),  M small
//
// Bound by the weights' bytes and, for one layer, by latency: a 256-row tensor-memory
// tile would be nearly empty and its pipeline takes 4 us to fill and drain.  So a warp
// takes 16 weight rows and one scale block at a time, straight from global memory into
// registers, converts e4m3 to fp16 (exactly) and multiplies with mma.m16n8k16 (products
// exact, fp32 sums): the weights are the 16 rows, the tokens the 8 columns.  K may be
// permuted within an MMA as long as both operands are: a lane's 16 consecutive bytes of a
// row serve four MMAs, so nothing is rearranged.  The sums of a block are scaled in fp32
// and added up; the warps of a CTA share the K of their 16 weight rows and their sums are
// added in order.  The next two blocks of a warp are on their way (of up to 8 tokens; one
// ahead 8192 x 8192 took 24.9 us).  1 x 4096 x 1024 takes 2.7 us (1.6 TB/s), of which the
// launch, the first loads and the sums' way through shared memory are 1.8; 1 x 8192 x 8192
// 18.5 (3.6 TB/s), 1 x 32768 x 8192 59 (4.5), 67 % of a plain copy's rate.  There 128 registers
// leave room for 16 warps on an SM (13 on average: 512 CTAs are 1.7 waves), and instructions
// issue in 46 % of the cycles; which of these bounds it has not been shown (without the
// conversions it was no faster).
#include "kernels.h"
#include "mx8.cuh"

namespace f3dc {

namespace {

constexpr int kFewWarps = 16;  // at most
constexpr int kFewCols = 16;  // weight rows (output columns) per CTA

// bytes from K on become zeros (e4m3 0); k: the first byte's index
F3DC_DEV uint4 cut(uint4 u, int k, int K)
{
    if (k + 16 <= K) return u;
    uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int left = K - k - 4 * j;
        w[j] = left >= 4 ? w[j] : (left <= 0 ? 0u : w[j] & ((1u << (8 * left)) - 1u));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// 16 e4m3 values to eight pairs of fp16 (exact)
F3DC_DEV void to_half(uint4 u, uint32_t (&h)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %2;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n cvt.rn.f16x2.e4m3x2 %1, hi;\n}\n"
            : "=r"(h[2 * j]), "=r"(h[2 * j + 1])
            : "r"(w[j]));
}

F3DC_DEV void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

F3DC_DEV float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // 2^e, -126 <= e <= 127

// s 2^(ea + eb - 254) for any two scale bytes, in two steps where the power leaves fp32's
// normal range
F3DC_DEV float scaled(float s, uint32_t ea, uint32_t eb)
{
    if (ea == 255u || eb == 255u) return __int_as_float(0x7FC00000);
    const int e = (int)ea + (int)eb - 254, e1 = max(-126, min(127, e)), e2 = max(-126, min(127, e - e1));
    return s * power(e1) * power(e2);
}

F3DC_DEV void store_cluster(float *p, uint32_t rank, float v)
{
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_shared(smem_u32(p), rank)), "f"(v) : "memory");
}

// A scale block's operands: 64 K per half, 16 bytes per lane of two weight rows and of NT
// token rows.
template <int NT>
struct Block {
    uint4 w[2][2], x[2][NT];
    uint32_t eb[2], ea[NT][2];
};

// NT: tiles of 8 tokens.  OUT8: the eight CTAs of a cluster hold a scale block's 128 columns.
template <int EPI, int NT, bool OUT8>
__global__ void __launch_bounds__(32 * kFewWarps) k_few8(const FewArgs a)
{
    constexpr int kTok = 8 * NT, kStride = kFewCols + 1;
    __shared__ float part[kFewWarps][kTok * kStride];
    __shared__ float tops[kTok][8];  // OUT8: a token's maximum in each CTA of the cluster
    griddep_launch();
    if (OUT8) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // this CTA runs
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, ks = blockDim.x >> 5;
    const int g = lane >> 2, q = lane & 3;
    const int m0 = blockIdx.y * kTok;  // this CTA's tokens
    const int n0 = blockIdx.x * kFewCols, blocks = (a.K + kScaleBlock - 1) / kScaleBlock;
    const bool lo = n0 + g < a.N, hi = n0 + g + 8 < a.N;  // N is a multiple of 8
    const uint8_t *wr[2] = {a.B + (int64_t)(n0 + g) * a.ldb + 16 * q, a.B + (int64_t)(n0 + g + 8) * a.ldb + 16 * q};
    const uint8_t *er[2] = {a.sb + (int64_t)(n0 + g) * a.ldbs, a.sb + (int64_t)(n0 + g + 8) * a.ldbs};
    auto token = [&](int m) { return (int64_t)min(m0 + m, a.M - 1); };  // rows from M on repeat the last, unused

    auto load = [&](Block<NT> &b, int block) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = block * kScaleBlock + 64 * h;
            const bool in = k + 16 * q < a.K;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                b.w[h][r] = make_uint4(0u, 0u, 0u, 0u);
                if (in && (r ? hi : lo)) b.w[h][r] = __ldcs(reinterpret_cast<const uint4 *>(wr[r] + k));
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                b.x[h][t] = make_uint4(0u, 0u, 0u, 0u);
                if (in) b.x[h][t] = *reinterpret_cast<const uint4 *>(a.A + token(8 * t + g) * a.lda + 16 * q + k);
            }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) b.eb[r] = (r ? hi : lo) ? er[r][block] : 127u;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) b.ea[t][i] = a.sa[token(8 * t + 2 * q + i) * a.ldas + block];
    };

    float acc[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] = 0.f;
    // blocks ahead, as far as there are registers for them
    constexpr int kAhead = NT == 1 ? 2 : 1;
    Block<NT> cur, next[kAhead];
    if (warp < blocks) load(cur, warp);
#pragma unroll
    for (int i = 0; i < kAhead - 1; ++i)
        if (warp + (i + 1) * ks < blocks) load(next[i], warp + (i + 1) * ks);
    for (int block = warp; block < blocks; block += ks) {
        if (block + kAhead * ks < blocks) load(next[kAhead - 1], block + kAhead * ks);
        float c[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) c[t][i] = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = block * kScaleBlock + 64 * h + 16 * q;
            uint32_t w0[8], w1[8], x[8];
            to_half(cut(cur.w[h][0], k, a.K), w0);
            to_half(cut(cur.w[h][1], k, a.K), w1);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                to_half(cut(cur.x[h][t], k, a.K), x);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    mma16816(c[t], w0[2 * j], w1[2 * j], w0[2 * j + 1], w1[2 * j + 1], x[2 * j], x[2 * j + 1]);
            }
        }
        bool plain = cur.eb[0] - 64u <= 126u && cur.eb[1] - 64u <= 126u;  // products of scales are normal numbers
#pragma unroll
        for (int t = 0; t < NT; ++t) plain &= cur.ea[t][0] - 64u <= 126u && cur.ea[t][1] - 64u <= 126u;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t ea = cur.ea[t][i & 1], eb = cur.eb[i >> 1];
                acc[t][i] = plain ? fmaf(c[t][i], __uint_as_float(ea << 23) * __uint_as_float(eb << 23), acc[t][i])
                                  : acc[t][i] + scaled(c[t][i], ea, eb);
            }
        cur = next[0];
#pragma unroll
        for (int i = 0; i < kAhead - 1; ++i) next[i] = next[i + 1];
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[warp][(8 * t + 2 * q + (i & 1)) * kStride + g + 8 * (i >> 1)] = acc[t][i];
    __syncthreads();

    // thread i: column i % 16 of token i / 16, and so on for the tokens that are left
    const int threads = blockDim.x;
    auto value = [&](int i) {
        const int m = i / kFewCols, n = n0 + i % kFewCols;
        float s = 0.f;
        for (int w = 0; w < ks; ++w) s += part[w][m * kStride + i % kFewCols];
        if (a.bias && n < a.N) s += __bfloat162float(a.bias[n]);
        return EPI == kEpiGelu ? gelu1(s) : s;
    };
    if constexpr (!OUT8) {
        for (int i = threadIdx.x; i < kTok * kFewCols; i += threads) {
            const int64_t m = m0 + i / kFewCols;
            const int n = n0 + i % kFewCols;
            if (n >= a.N || m >= a.M) continue;
            const float s = value(i);
            if constexpr (EPI == kEpiResid) {
                float *o = reinterpret_cast<float *>(a.out) + m * a.ldo + n;
                *o = fmaf(a.gate ? a.gate[n] : 1.f, s, *o);
            } else {
                reinterpret_cast<bf16 *>(a.out)[m * a.ldo + n] = __float2bfloat16_rn(s);
            }
        }
    } else {
        const float inf = __int_as_float(0x7F800000);
        const uint32_t rank = cluster_rank();
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // and so do the others
        // every token's maximum over this CTA's columns goes to all CTAs of the cluster;
        // whole half warps (16 columns) work on a token
        for (int i = threadIdx.x; i < kTok * kFewCols; i += threads) {
            const int m = i / kFewCols, n = n0 + i % kFewCols;
            float s = n < a.N ? value(i) : 0.f;
            if (fabsf(s) == inf) s = __int_as_float(0x7FC00000);
            part[0][m * kStride + i % kFewCols] = s;  // the only thread that reads this place
            float top = fmaxf(fabsf(s), 0.f);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (i % kFewCols < 8) store_cluster(&tops[m][rank], i % kFewCols, top);
        }
        cluster_sync();
        for (int i = threadIdx.x; i < kTok * 4; i += threads) {  // four columns of a token
            const int m = i / 4, c = 4 * (i % 4);
            if (n0 + c >= a.N || m0 + m >= a.M) continue;
            const int64_t row = m0 + m;
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, tops[m][j]);
            const uint32_t byte = e8m0_byte(top);
            const float inv = e8m0_inverse(byte);
            const float *s = &part[0][m * kStride + c];
            *reinterpret_cast<uint32_t *>(reinterpret_cast<uint8_t *>(a.out) + row * a.ldo + n0 + c) =
                pack_e4m3x4(s[0] * inv, s[1] * inv, s[2] * inv, s[3] * inv);
            if (c == 0 && n0 % kScaleBlock == 0) a.out_scales[row * a.ldos + n0 / kScaleBlock] = (uint8_t)byte;
        }
    }
}

template <int EPI, int NT, bool OUT8>
cudaError_t launch_one(const FewArgs &a, int num_sms, cudaStream_t s)
{
    const int blocks = (a.K + kScaleBlock - 1) / kScaleBlock;
    const unsigned groups = (unsigned)((a.M + 8 * NT - 1) / (8 * NT));
    unsigned ctas = (unsigned)((a.N + kFewCols - 1) / kFewCols);
    // Half of the warps where several CTAs share an SM, and fewer yet where there are many, so
    // that each warp has blocks to load ahead: with 16 / 8 warps 1 x 1024 x 4096 (64 CTAs) takes
    // 4.1 / 5.3 us, 1 x 4096 x 4096 (256) 8.1 / 5.6; with 8 / 4 1 x 16384 x 4096 (1024) 21.3 / 17.7;
    // with 8 / 2 1 x 65536 x 1024 (4096) 31.8 / 19.9
    const int64_t all = (int64_t)ctas * groups, share = (24 * (int64_t)num_sms - 1) / all + 1;
    const int most = all <= num_sms ? kFewWarps : (int)(share < 2 ? 2 : (share < kFewWarps / 2 ? share : kFewWarps / 2));
    if (OUT8) ctas = (ctas + 7) / 8 * 8;  // whole clusters
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas, groups);
    cfg.blockDim = dim3(32 * (blocks < most ? blocks : most));
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 8;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = OUT8 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_few8<EPI, NT, OUT8>, a);
}

template <int EPI, bool OUT8>
cudaError_t launch_rows(const FewArgs &a, int num_sms, cudaStream_t s)
{
    return a.M <= 8 ? launch_one<EPI, 1, OUT8>(a, num_sms, s) : launch_one<EPI, 2, OUT8>(a, num_sms, s);
}

}  // namespace

cudaError_t launch_few8(const FewArgs &a, int epi, int num_sms, cudaStream_t s)
{
    const bool out8 = a.out_scales != nullptr;
    switch (epi) {
    case kEpiBias: return out8 ? launch_rows<kEpiBias, true>(a, num_sms, s) : launch_rows<kEpiBias, false>(a, num_sms, s);
    case kEpiGelu: return out8 ? launch_rows<kEpiGelu, true>(a, num_sms, s) : launch_rows<kEpiGelu, false>(a, num_sms, s);
    case kEpiResid: return out8 ? cudaErrorInvalidValue : launch_rows<kEpiResid, false>(a, num_sms, s);
    default: return cudaErrorInvalidValue;
    }
}

}  // namespace f3dc
