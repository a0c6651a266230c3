// k_norm.cu -- the norm after a block, its gate and residual scale, the residual sum
// and the norm before the next block in one pass over the rows (f3dc_norm_residual):
//
//   n = post(y) g + b,  x' = alpha x + gate n,  h = (pre(x') g + b) (1 + scale) + shift
//
// with post and pre none, LayerNorm or RMSNorm; x' in fp32, h in bf16 or in e4m3 with
// one power-of-two scale per block of 128.
//
// Bound by memory: x, y read and x', h written once (12 bytes per element, 11 with
// 8-bit h).  A row stays in registers between its two norms: a warp holds a row of up
// to 1024 values (8 consecutive ones per lane and step, so that 16 lanes hold a scale
// block), four warps a wider one.  Means, then mean squared deviations from them, in
// fp32.
#include "kernels.h"
#include "mx8.cuh"

namespace f3dc {

namespace {

constexpr int kNormThreads = 128;

struct V8 {
    float v[8];
};

F3DC_DEV V8 load_f32x8(const float *p)
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}

F3DC_DEV V8 load_bf16x8(const bf16 *p)
{
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    V8 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        r.v[2 * j] = bf16_bits_to_f32(w[j] & 0xFFFFu);
        r.v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
    return r;
}

// Sum over the TPR threads of a row.
template <int TPR>
F3DC_DEV float row_sum(float v, float *sh)
{
    v = warp_sum(v);
    if constexpr (TPR > 32) {
        __syncthreads();  // the last sum has been read
        if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < TPR / 32; ++i) v += sh[i];
    }
    return v;
}

// v becomes its norm times g plus b; vectors from `nv` on are zeros and stay out of the sums.
template <int NV, int TPR>
F3DC_DEV void normalise(V8 (&v)[NV], int t, int W, int kind, const bf16 *g, const bf16 *b, float eps, float *sh)
{
    if (kind != kNormNone) {
        float mean = 0.f;
        if (kind == kNormLayer) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) s += v[i].v[j];
            mean = row_sum<TPR>(s, sh) / (float)W;
        }
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((t + TPR * i) * 8 < W) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[i].v[j] -= mean;
                    ss += v[i].v[j] * v[i].v[j];
                }
            }
        const float r = rsqrtf(row_sum<TPR>(ss, sh) / (float)W + eps);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i].v[j] *= r;
    }
    if (!g && !b) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (t + TPR * i) * 8;
        if (col >= W) continue;
        if (g) {
            const V8 u = load_bf16x8(g + col);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i].v[j] *= u.v[j];
        }
        if (b) {
            const V8 u = load_bf16x8(b + col);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i].v[j] += u.v[j];
        }
    }
}

// NV vectors of 8 per thread, TPR threads per row (32: a warp; kNormThreads: the CTA).
template <int NV, int TPR>
__global__ void __launch_bounds__(kNormThreads) k_norm_residual(const NormArgs a)
{
    __shared__ float sh[kNormThreads / 32];
    griddep_launch();
    griddep_wait();
    constexpr int kRows = kNormThreads / TPR;
    const int t = threadIdx.x % TPR, W = a.width;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; row < a.rows; row += (int64_t)gridDim.x * kRows) {
        const int g = a.group ? a.group[row] : 0;
        if (g < 0) continue;
        if (g >= a.groups) {
            if (t == 0) raise_error(a.err, kDevBadIndex);
            continue;
        }
        V8 x[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (t + TPR * i) * 8;
            x[i] = V8{};
            if (col < W) x[i] = load_f32x8(a.x + row * a.ldx + col);
        }
        if (a.y) {
            V8 y[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int col = (t + TPR * i) * 8;
                y[i] = V8{};
                if (col < W) y[i] = load_bf16x8(a.y + row * a.ldy + col);
            }
            normalise<NV, TPR>(y, t, W, a.post, a.post_g, a.post_b, a.eps, sh);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int col = (t + TPR * i) * 8;
                if (col >= W) continue;
                V8 gate;
                if (a.gate) gate = load_f32x8(a.gate + g * a.ldmod + col);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[i].v[j] = a.res_scale * x[i].v[j] + (a.gate ? gate.v[j] * y[i].v[j] : y[i].v[j]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i].v[j] *= a.res_scale;
        }
        if (a.x_out) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int col = (t + TPR * i) * 8;
                if (col >= W) continue;
                float4 *p = reinterpret_cast<float4 *>(a.x_out + row * a.ldxo + col);
                p[0] = make_float4(x[i].v[0], x[i].v[1], x[i].v[2], x[i].v[3]);
                p[1] = make_float4(x[i].v[4], x[i].v[5], x[i].v[6], x[i].v[7]);
            }
        }
        if (!a.h) continue;
        normalise<NV, TPR>(x, t, W, a.pre, a.pre_g, a.pre_b, a.eps, sh);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (t + TPR * i) * 8;
            const bool in = col < W;
            if (in && a.scale) {
                const V8 u = load_f32x8(a.scale + g * a.ldmod + col);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i].v[j] *= 1.0f + u.v[j];
            }
            if (in && a.shift) {
                const V8 u = load_f32x8(a.shift + g * a.ldmod + col);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i].v[j] += u.v[j];
            }
            const float(&v)[8] = x[i].v;
            if (a.h_scales) {
                float w[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
                const uint32_t byte = quantize_block<8, 16>(w);
                if (in) {
                    *reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(a.h) + row * a.ldh + col) =
                        make_uint2(pack_e4m3x4(w[0], w[1], w[2], w[3]), pack_e4m3x4(w[4], w[5], w[6], w[7]));
                    if (t % 16 == 0) a.h_scales[row * a.ldhs + col / kScaleBlock] = (uint8_t)byte;
                }
            } else if (in) {
                uint4 u;
                u.x = pack_bf16x2(v[0], v[1]);
                u.y = pack_bf16x2(v[2], v[3]);
                u.z = pack_bf16x2(v[4], v[5]);
                u.w = pack_bf16x2(v[6], v[7]);
                *reinterpret_cast<uint4 *>(reinterpret_cast<bf16 *>(a.h) + row * a.ldh + col) = u;
            }
        }
    }
}

template <int NV, int TPR>
cudaError_t launch_rows(const NormArgs &a, int num_sms, cudaStream_t s)
{
    constexpr int kRows = kNormThreads / TPR;
    const int64_t ctas = ((int64_t)a.rows + kRows - 1) / kRows, most = (int64_t)num_sms * 16;
    return launch_k(k_norm_residual<NV, TPR>, dim3((unsigned)(ctas < most ? ctas : most)), dim3(kNormThreads), 0, s, a);
}

}  // namespace

cudaError_t launch_norm_residual(const NormArgs &a, int num_sms, cudaStream_t s)
{
    if (a.width <= 256) return launch_rows<1, 32>(a, num_sms, s);
    if (a.width <= 512) return launch_rows<2, 32>(a, num_sms, s);
    if (a.width <= 1024) return launch_rows<4, 32>(a, num_sms, s);
    if (a.width <= 2048) return launch_rows<2, kNormThreads>(a, num_sms, s);
    if (a.width <= 4096) return launch_rows<4, kNormThreads>(a, num_sms, s);
    return launch_rows<8, kNormThreads>(a, num_sms, s);
}

}  // namespace f3dc
