// k_norm.cu -- the norm after a block, its gate and residual scale, the residual sum
// and the norm before the next block in one pass over the rows (f3dc_norm_residual):
//
//   n = post(y) g + b,  x' = alpha x + gate n,  h = (pre(x') g + b) (1 + scale) + shift
//
// with post and pre none, LayerNorm or RMSNorm; x' in fp32, h in bf16 or in e4m3 with
// one power-of-two scale per block of 128.
//
// Bound by memory: x, y read and x', h written once (12 bytes per element, 11 with
// 8-bit h).  One thread per 8 columns, so that 16 threads hold a scale block; the rows stay
// in registers between the two norms.  Means, then mean squared deviations from them, in
// fp32.  Two kernels:
//   k_norm_rows, for many rows: a CTA takes two, whose loads are in flight together, whose
//     sums share the shuffles and the barrier, and for which a gain or a modulation is read
//     once (from L1: with one row at a time these vectors, 20 bytes per element, are more
//     than the rows themselves).  32768 x 1024 with a gate, modulations and 8-bit h take 69
//     us: 5.4 TB/s, 80 % of a plain copy's rate (one row per CTA 82 us, four 81, runs of
//     rows with the next one's loads in flight 79); the chain of four sums per row is as
//     long as its loads, and instructions issue in 61 % of the cycles.
//   k_norm_runs, for few: a CTA takes a run of consecutive rows, mostly one, with everything
//     loaded at once at the start and the next row ahead.  955 x 1024 take 4.1 us (4.6 with all
//     norms, gains and modulations and 8-bit h), one row of 128 1.8.
#include "kernels.h"
#include "mx8.cuh"

namespace f3dc {

namespace {

constexpr int kNormThreadsPerSm = 1024;     // k_norm_rows: 64 registers
constexpr int kNormRunThreadsPerSm = 640;   // k_norm_runs: 96

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

// Gain and bias of a norm at this thread's columns, as bf16 pairs.
struct Affine {
    uint4 gain, bias;
    bool some;
};
F3DC_DEV Affine affine(const bf16 *g, const bf16 *b, int col, bool in)
{
    const uint32_t one = 0x3F803F80u;
    return Affine{g ? vec_load16(in ? g + col : nullptr) : make_uint4(one, one, one, one), vec_load16(in && b ? b + col : nullptr),
                  g != nullptr || b != nullptr};
}

// v[i] becomes its norm times the gain plus the bias.  `in`: this thread has columns of the
// row (its values are zeros otherwise, and stay out of the sums).
template <int R, int NW>
F3DC_DEV void normalise(V8 (&v)[R], bool in, float inv_w, int kind, const Affine &w, float eps, float (*sh)[R][NW], int &turn)
{
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
    if (w.some) {
        const V8 m = from_bf16(w.gain), c = from_bf16(w.bias);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i].v[j] = ffma2(v[i].v[j], m.v[j], c.v[j]);
    }
}

// R rows per CTA, at most NW warps (a power of two)
template <int R, int NW>
__global__ void __launch_bounds__(32 * NW, kNormThreadsPerSm / (32 * NW)) k_norm_rows(const NormArgs a)
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

    // rows are loaded while their groups are
    int g[R];  // group of each row; -1: left as it is
    uint4 xr[R][2], yr[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const bool there = row0 + i < a.rows;
        g[i] = there ? (a.group ? a.group[row0 + i] : 0) : -1;
        xr[i][0] = xr[i][1] = yr[i] = make_uint4(0u, 0u, 0u, 0u);
        if (in && there) {
            const float *p = a.x + (row0 + i) * a.ldx + col;
            xr[i][0] = row_load16(p);
            xr[i][1] = row_load16(p + 4);
            if (a.y) yr[i] = row_load16(a.y + (row0 + i) * a.ldy + col);
        }
    }
    bool any = false;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (g[i] >= a.groups) {
            if (threadIdx.x == 0) raise_error(a.err, kDevBadIndex);
            g[i] = -1;
        }
        any |= g[i] >= 0;
    }
    if (!any) return;  // the same for every thread of the CTA

    V8 x[R];
    const f32x2 alpha = both(a.res_scale);
    if (a.y) {
        // the gate of the first row's group (a batch's rows are rarely of two)
        Vec gate = vec_f32(a.gate && in && g[0] >= 0 ? a.gate + g[0] * a.ldmod + col : nullptr);
        int of = g[0];  // the group whose vector `gate` is
        V8 y[R];
#pragma unroll
        for (int i = 0; i < R; ++i) y[i] = from_bf16(yr[i]);
        normalise<R, NW>(y, in, inv_w, a.post, affine(a.post_g, a.post_b, col, in), a.eps, sh, turn);
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
    normalise<R, NW>(x, in, inv_w, a.pre, affine(a.pre_g, a.pre_b, col, in), a.eps, sh, turn);
    if (a.scale || a.shift) {
        int of = g[0];  // the group whose vectors sc and sf are
        f32x2 m[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) m[j] = fadd2(sc.pair(j), both(1.0f));
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (!in || g[i] < 0) continue;
            if (g[i] != of) {
                sc = vec_f32(a.scale ? a.scale + g[i] * a.ldmod + col : nullptr);
                sf = vec_f32(a.shift ? a.shift + g[i] * a.ldmod + col : nullptr);
#pragma unroll
                for (int j = 0; j < 4; ++j) m[j] = fadd2(sc.pair(j), both(1.0f));
            }
            of = g[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i].v[j] = ffma2(x[i].v[j], m[j], sf.pair(j));
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

// Each CTA a run of consecutive rows, the next one's loads in flight while a row is worked on;
// gains, and the modulations of the rows' group, stay in registers.
template <int NW>
__global__ void __launch_bounds__(32 * NW, kNormRunThreadsPerSm / (32 * NW)) k_norm_runs(const NormArgs a)
{
    __shared__ __align__(16) float sh[2][1][NW];
    griddep_launch();
    // the sums of warps that the CTA does not have
    if (NW > 2 && blockDim.x < 32 * NW && threadIdx.x < 2 * NW && threadIdx.x % NW >= blockDim.x / 32)
        (&sh[0][0][0])[threadIdx.x] = 0.f;
    const int col = threadIdx.x * 8;
    const bool in = col < a.width;
    const float inv_w = 1.0f / (float)a.width;
    const int64_t row0 = (int64_t)a.rows * blockIdx.x / gridDim.x, end = (int64_t)a.rows * (blockIdx.x + 1) / gridDim.x;
    const f32x2 alpha = both(a.res_scale);
    griddep_wait();
    struct Row {
        uint4 x[2], y;
        int g;
    };
    const float *px = a.x + row0 * a.ldx + col;
    const bf16 *py = a.y ? a.y + row0 * a.ldy + col : nullptr;
    const int32_t *pg = a.group ? a.group + row0 : nullptr;
    auto load = [&](Row &r) {
        r.x[0] = r.x[1] = r.y = make_uint4(0u, 0u, 0u, 0u);
        r.g = a.group ? *pg++ : 0;
        if (in) {
            r.x[0] = row_load16(px);
            r.x[1] = row_load16(px + 4);
            if (a.y) r.y = row_load16(py);
        }
        if (a.y) py += a.ldy;
        px += a.ldx;
    };
    Row cur, next;
    if (row0 < end) load(cur);
    const Affine post = affine(a.post_g, a.post_b, col, in), pre = affine(a.pre_g, a.pre_b, col, in);
    Vec gate, sc, sf;
    int of = -1, turn = 0;
    for (int64_t row = row0; row < end; ++row, cur = next) {
        if (row + 1 < end) load(next);
        const int g = cur.g;
        if (g < 0) continue;
        if (g >= a.groups) {
            if (threadIdx.x == 0) raise_error(a.err, kDevBadIndex);
            continue;
        }
        if (g != of) {
            of = g;
            const int64_t m = (int64_t)g * a.ldmod + col;
            gate = vec_f32(a.gate && in ? a.gate + m : nullptr);
            sc = vec_f32(a.scale && in ? a.scale + m : nullptr);
            sf = vec_f32(a.shift && in ? a.shift + m : nullptr);
        }
        const float *f = reinterpret_cast<const float *>(cur.x);
        V8 xs[1], &x = xs[0];
#pragma unroll
        for (int j = 0; j < 4; ++j) x.v[j] = fmul2({f[2 * j], f[2 * j + 1]}, alpha);
        if (a.y) {
            V8 ys[1] = {from_bf16(cur.y)}, &y = ys[0];
            normalise<1, NW>(ys, in, inv_w, a.post, post, a.eps, sh, turn);
#pragma unroll
            for (int j = 0; j < 4; ++j) x.v[j] = a.gate ? ffma2(gate.pair(j), y.v[j], x.v[j]) : fadd2(y.v[j], x.v[j]);
        }
        if (a.x_out && in) {
            float4 *p = reinterpret_cast<float4 *>(a.x_out + row * a.ldxo + col);
            p[0] = make_float4(x.v[0].x, x.v[0].y, x.v[1].x, x.v[1].y);
            p[1] = make_float4(x.v[2].x, x.v[2].y, x.v[3].x, x.v[3].y);
        }
        if (!a.h) continue;
        normalise<1, NW>(xs, in, inv_w, a.pre, pre, a.eps, sh, turn);
        if (a.scale || a.shift) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x.v[j] = ffma2(x.v[j], fadd2(sc.pair(j), both(1.0f)), sf.pair(j));
        }
        if (a.h_scales) {
            float q[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[2 * j] = in ? x.v[j].x : 0.f, q[2 * j + 1] = in ? x.v[j].y : 0.f;
            const uint32_t byte = quantize_block<8, 16>(q);
            if (in) {
                *reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(a.h) + row * a.ldh + col) =
                    make_uint2(pack_e4m3x4(q[0], q[1], q[2], q[3]), pack_e4m3x4(q[4], q[5], q[6], q[7]));
                if (threadIdx.x % 16 == 0) a.h_scales[row * a.ldhs + col / kScaleBlock] = (uint8_t)byte;
            }
        } else if (in) {
            *reinterpret_cast<uint4 *>(reinterpret_cast<bf16 *>(a.h) + row * a.ldh + col) =
                make_uint4(pack_bf16x2(x.v[0].x, x.v[0].y), pack_bf16x2(x.v[1].x, x.v[1].y), pack_bf16x2(x.v[2].x, x.v[2].y),
                           pack_bf16x2(x.v[3].x, x.v[3].y));
        }
    }
}

template <int R, int NW>
cudaError_t launch_rows(const NormArgs &a, cudaStream_t s)
{
    const unsigned threads = (unsigned)((a.width + 255) / 256 * 32);
    const unsigned ctas = (unsigned)(((int64_t)a.rows + R - 1) / R);
    return launch_k(k_norm_rows<R, NW>, dim3(ctas), dim3(threads), 0, s, a);
}

template <int NW>
cudaError_t launch_runs(const NormArgs &a, int num_sms, cudaStream_t s)
{
    const unsigned threads = (unsigned)((a.width + 255) / 256 * 32), most = (unsigned)num_sms * (kNormRunThreadsPerSm / (32 * NW));
    return launch_k(k_norm_runs<NW>, dim3((unsigned)a.rows < most ? (unsigned)a.rows : most), dim3(threads), 0, s, a);
}

// Runs up to 2^21 elements.  Runs / pairs of rows, us: of width 1024 600 rows 3.2 / 4.3, 955
// 4.1 / 5.1, 1800 5.5 / 5.9, 2400 7.0 / 6.0, 4800 14.0 / 13.7; of width 4096 300 rows 4.6 / 6.1,
// 600 8.0 / 6.8, 2400 33 / 26; of width 128 64 rows 2.0 / 2.3, 2400 3.7 / 3.3.
template <int NW>
cudaError_t launch_width(const NormArgs &a, int num_sms, cudaStream_t s)
{
    return (int64_t)a.rows * a.width <= 1 << 21 ? launch_runs<NW>(a, num_sms, s) : launch_rows<2, NW>(a, s);
}

}  // namespace

cudaError_t launch_norm_residual(const NormArgs &a, int num_sms, cudaStream_t s)
{
    if (a.width <= 256) return launch_width<1>(a, num_sms, s);
    if (a.width <= 512) return launch_width<2>(a, num_sms, s);
    if (a.width <= 1024) return launch_width<4>(a, num_sms, s);
    if (a.width <= 2048) return launch_width<8>(a, num_sms, s);
    if (a.width <= 4096) return launch_width<16>(a, num_sms, s);
    return launch_rows<1, 32>(a, s);  // (more threads than two rows, or a run, leave registers for)
}

}  // namespace f3dc
