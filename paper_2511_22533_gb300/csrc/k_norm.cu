// k_norm.cu -- the norm after a block, its gate and residual scale, the residual sum
// and the norm before the next block in one pass over the rows (f3dc_norm_residual):
//
//   n = post(y) g + b,  x' = alpha x + gate n,  h = (pre(x') g + b) (1 + scale) + shift
//
// with post and pre none, LayerNorm or RMSNorm; x' in fp32, h in bf16 or in e4m3 with
// one power-of-two scale per block of 128.
//
// Bound by memory: x, y read and x', h written once (12 bytes per element, 11 with
// 8-bit h).  A CTA has one thread per 8 columns, so that 16 threads hold a scale block,
// and takes R rows at once: their loads are in flight together, their sums share the
// shuffles and the barrier, and a gain or a modulation is read once for all of them
// (from L1: with one row at a time these vectors, 20 bytes per element, are more than
// the rows themselves).  The rows stay in registers between the two norms.  Means, then
// mean squared deviations from them, in fp32.  32768 x 1024 with a gate, modulations and
// 8-bit h take 69 us: 5.35 TB/s, 79 % of a plain copy's rate (one row per CTA 82 us, four
// 81); instructions issue in 64 % of the cycles, and the rows' loads do not overlap their
// CTA's sums.  One row of 128 takes 1.9 us.
#include "kernels.h"
#include "mx8.cuh"

namespace f3dc {

namespace {

constexpr int kNormRows = 2;
constexpr int kNormThreadsPerSm = 1024;

struct V8 {
    f32x2 v[4];
};

F3DC_DEV V8 from_bf16(uint4 u)
{
    return V8{{{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u)},
               {__uint_as_float(u.y << 16), __uint_as_float(u.y & 0xFFFF0000u)},
               {__uint_as_float(u.z << 16), __uint_as_float(u.z & 0xFFFF0000u)},
               {__uint_as_float(u.w << 16), __uint_as_float(u.w & 0xFFFF0000u)}}};
}
// gains, biases, modulations: read by every CTA, kept in L1.  Issued where they stand, ahead
// of the sums that run before their use (a null p: nothing is read).
F3DC_DEV uint4 vec_load16(const void *p)
{
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if (p) asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
    return u;
}
struct Vec {  // 8 fp32
    uint4 lo, hi;
    F3DC_DEV f32x2 pair(int j) const
    {
        const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        return {__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1])};
    }
};
F3DC_DEV Vec vec_f32(const float *p) { return Vec{vec_load16(p), vec_load16(p ? p + 4 : nullptr)}; }
// rows: read once
F3DC_DEV uint4 row_load16(const void *p)
{
    uint4 u;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
    return u;
}
F3DC_DEV f32x2 both(float a) { return {a, a}; }

// Sums of R values over the CTA's NW warps, in every thread.  Two values share a step that
// halves what a lane holds; a warp's sums lie in sh[i][warp].
template <int R, int NW>
F3DC_DEV void row_sums(float (&s)[R], float (*sh)[NW])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if constexpr (R == 1) {
        const float v = warp_sum(s[0]);
        if constexpr (NW == 1) {
            s[0] = v;
            return;
        }
        if (lane == 0) sh[0][warp] = v;
    } else {
#pragma unroll
        for (int i = 0; i < R; i += 2) {
            const bool up = lane & 16;
            float v = up ? s[i + 1] : s[i];
            v += __shfl_xor_sync(0xffffffffu, up ? s[i] : s[i + 1], 16);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (NW == 1) {
                s[i] = __shfl_sync(0xffffffffu, v, 0);
                s[i + 1] = __shfl_sync(0xffffffffu, v, 16);
            } else if ((lane & 15) == 0) {
                sh[i + (lane >> 4)][warp] = v;
            }
        }
    }
    if constexpr (NW > 1) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float v = 0.f;
            if constexpr (NW == 2) {
                const float2 u = *reinterpret_cast<const float2 *>(sh[i]);
                v = u.x + u.y;
            } else {
#pragma unroll
                for (int w = 0; w < NW; w += 4) {
                    const float4 u = *reinterpret_cast<const float4 *>(sh[i] + w);
                    v += (u.x + u.y) + (u.z + u.w);
                }
            }
            s[i] = v;
        }
    }
}

// v[i] becomes its norm times g plus b.  `in`: this thread has columns of the row (its
// values are zeros otherwise, and stay out of the sums).
template <int R, int NW>
F3DC_DEV void normalise(V8 (&v)[R], bool in, float inv_w, int kind, const bf16 *g, const bf16 *b, float eps,
                        float (*sh)[R][NW], int &turn)
{
    const uint4 gain = vec_load16(in ? g : nullptr), bias = vec_load16(in ? b : nullptr);
    if (kind != kNormNone) {
        float s[R];
        if (kind == kNormLayer) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const f32x2 t = fadd2(fadd2(v[i].v[0], v[i].v[1]), fadd2(v[i].v[2], v[i].v[3]));
                s[i] = t.x + t.y;
            }
            row_sums<R, NW>(s, sh[turn]);
            turn ^= 1;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const f32x2 m = both(in ? -s[i] * inv_w : 0.f);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i].v[j] = fadd2(v[i].v[j], m);
            }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            f32x2 t = fmul2(v[i].v[0], v[i].v[0]);
#pragma unroll
            for (int j = 1; j < 4; ++j) t = ffma2(v[i].v[j], v[i].v[j], t);
            s[i] = t.x + t.y;
        }
        row_sums<R, NW>(s, sh[turn]);
        turn ^= 1;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const f32x2 r = both(rsqrtf(s[i] * inv_w + eps));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i].v[j] = fmul2(v[i].v[j], r);
        }
    }
    if (g && in) {
        const V8 u = from_bf16(gain);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i].v[j] = fmul2(v[i].v[j], u.v[j]);
    }
    if (b && in) {
        const V8 u = from_bf16(bias);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i].v[j] = fadd2(v[i].v[j], u.v[j]);
    }
}

// R rows per CTA, at most NW warps (a power of two)
template <int R, int NW>
__global__ void __launch_bounds__(32 * NW, kNormThreadsPerSm / (32 * NW)) k_norm_residual(const NormArgs a)
{
    __shared__ __align__(16) float sh[2][R][NW];  // by turns: one barrier per sum
    griddep_launch();
    // the sums of warps that the CTA does not have
    if (NW > 2 && blockDim.x < 32 * NW && threadIdx.x < 2 * R * NW && threadIdx.x % NW >= blockDim.x / 32)
        (&sh[0][0][0])[threadIdx.x] = 0.f;
    griddep_wait();
    const int col = threadIdx.x * 8;
    const bool in = col < a.width;
    const float inv_w = 1.0f / (float)a.width;
    const int64_t row0 = (int64_t)blockIdx.x * R;
    int turn = 0;

    int g[R];  // group of each row; -1: left as it is
    bool any = false;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        g[i] = -1;
        if (row0 + i < a.rows) g[i] = a.group ? a.group[row0 + i] : 0;
        if (g[i] >= a.groups) {
            if (threadIdx.x == 0) raise_error(a.err, kDevBadIndex);
            g[i] = -1;
        }
        any |= g[i] >= 0;
    }
    if (!any) return;  // the same for every thread of the CTA

    uint4 xr[R][2], yr[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        xr[i][0] = xr[i][1] = yr[i] = make_uint4(0u, 0u, 0u, 0u);
        if (in && g[i] >= 0) {
            const float *p = a.x + (row0 + i) * a.ldx + col;
            xr[i][0] = row_load16(p);
            xr[i][1] = row_load16(p + 4);
            if (a.y) yr[i] = row_load16(a.y + (row0 + i) * a.ldy + col);
        }
    }
    V8 x[R];
    const f32x2 alpha = both(a.res_scale);
    if (a.y) {
        // the gate of the first row's group (a batch's rows are rarely of two)
        Vec gate = vec_f32(a.gate && in && g[0] >= 0 ? a.gate + g[0] * a.ldmod + col : nullptr);
        int of = g[0];  // the group whose vector `gate` is
        V8 y[R];
#pragma unroll
        for (int i = 0; i < R; ++i) y[i] = from_bf16(yr[i]);
        normalise<R, NW>(y, in, inv_w, a.post, a.post_g ? a.post_g + col : nullptr, a.post_b ? a.post_b + col : nullptr,
                         a.eps, sh, turn);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float *f = reinterpret_cast<const float *>(xr[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i].v[j] = fmul2({f[2 * j], f[2 * j + 1]}, alpha);
            if (a.gate && in && g[i] >= 0) {
                if (g[i] != of) gate = vec_f32(a.gate + g[i] * a.ldmod + col);
                of = g[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i].v[j] = ffma2(gate.pair(j), y[i].v[j], x[i].v[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i].v[j] = fadd2(y[i].v[j], x[i].v[j]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float *f = reinterpret_cast<const float *>(xr[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i].v[j] = fmul2({f[2 * j], f[2 * j + 1]}, alpha);
        }
    }
    if (a.x_out) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (in && g[i] >= 0) {
                float4 *p = reinterpret_cast<float4 *>(a.x_out + (row0 + i) * a.ldxo + col);
                p[0] = make_float4(x[i].v[0].x, x[i].v[0].y, x[i].v[1].x, x[i].v[1].y);
                p[1] = make_float4(x[i].v[2].x, x[i].v[2].y, x[i].v[3].x, x[i].v[3].y);
            }
    }
    if (!a.h) return;
    const bool mod0 = in && g[0] >= 0;
    Vec sc = vec_f32(a.scale && mod0 ? a.scale + g[0] * a.ldmod + col : nullptr);
    Vec sf = vec_f32(a.shift && mod0 ? a.shift + g[0] * a.ldmod + col : nullptr);
    normalise<R, NW>(x, in, inv_w, a.pre, a.pre_g ? a.pre_g + col : nullptr, a.pre_b ? a.pre_b + col : nullptr, a.eps, sh,
                     turn);
    if (a.scale || a.shift) {
        int of = g[0];  // the group whose vectors sc and sf are
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (!in || g[i] < 0) continue;
            if (g[i] != of) {
                sc = vec_f32(a.scale ? a.scale + g[i] * a.ldmod + col : nullptr);
                sf = vec_f32(a.shift ? a.shift + g[i] * a.ldmod + col : nullptr);
            }
            of = g[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i].v[j] = ffma2(x[i].v[j], fadd2(sc.pair(j), both(1.0f)), sf.pair(j));
        }
    }
    if (a.h_scales) {
        float f[R][8];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f[i][2 * j] = in ? x[i].v[j].x : 0.f;
                f[i][2 * j + 1] = in ? x[i].v[j].y : 0.f;
            }
        uint32_t byte[R];
        quantize_blocks<R, 8, 16>(f, byte);
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (in && g[i] >= 0) {
                *reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(a.h) + (row0 + i) * a.ldh + col) =
                    make_uint2(pack_e4m3x4(f[i][0], f[i][1], f[i][2], f[i][3]), pack_e4m3x4(f[i][4], f[i][5], f[i][6], f[i][7]));
                if (threadIdx.x % 16 == 0) a.h_scales[(row0 + i) * a.ldhs + col / kScaleBlock] = (uint8_t)byte[i];
            }
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (in && g[i] >= 0)
                *reinterpret_cast<uint4 *>(reinterpret_cast<bf16 *>(a.h) + (row0 + i) * a.ldh + col) =
                    make_uint4(pack_bf16x2(x[i].v[0].x, x[i].v[0].y), pack_bf16x2(x[i].v[1].x, x[i].v[1].y),
                               pack_bf16x2(x[i].v[2].x, x[i].v[2].y), pack_bf16x2(x[i].v[3].x, x[i].v[3].y));
    }
}

template <int R, int NW>
cudaError_t launch_rows(const NormArgs &a, cudaStream_t s)
{
    const unsigned threads = (unsigned)((a.width + 255) / 256 * 32);
    const unsigned ctas = (unsigned)(((int64_t)a.rows + R - 1) / R);
    return launch_k(k_norm_residual<R, NW>, dim3(ctas), dim3(threads), 0, s, a);
}

template <int R>
cudaError_t launch_width(const NormArgs &a, cudaStream_t s)
{
    if (a.width <= 256) return launch_rows<R, 1>(a, s);
    if (a.width <= 512) return launch_rows<R, 2>(a, s);
    if (a.width <= 1024) return launch_rows<R, 4>(a, s);
    if (a.width <= 2048) return launch_rows<R, 8>(a, s);
    if (a.width <= 4096) return launch_rows<R, 16>(a, s);
    return launch_rows<1, 32>(a, s);
}

}  // namespace

// One row per CTA while all of them run at once: with one / two, us, of width 1024: 600 rows
// 4.2 / 4.3, 1000 4.4 / 5.1, 1400 5.6 / 5.5, 2400 7.4 / 6.0; of width 256: 600 rows 2.2 / 2.4,
// 1400 3.5 / 2.7.
cudaError_t launch_norm_residual(const NormArgs &a, int num_sms, cudaStream_t s)
{
    return a.rows >= 8 * num_sms ? launch_width<kNormRows>(a, s) : launch_width<1>(a, s);
}

}  // namespace f3dc
