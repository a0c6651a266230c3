// k_kv_append.cu -- f3dc_kv_append_fp8: the keys and values of new tokens into the pages of
// their sequences, e4m3 with one power-of-two scale per page and head, keys and queries
// rotated by their positions on the way.
//
//   k'_p = R(p) k_p:  (a, b) -> (a cos - b sin, b cos + a sin), angle 2 pi p turns_j / 2^64
//   byte = smallest e with max |k'| <= 448 2^e over the page's new tokens, at least the
//          page's own where it already holds tokens; q = k' 2^-e to nearest even
//
// One pass over the rows.  A CTA takes one page of one sequence: it computes the angles'
// cosines and sines of the page's new tokens once, into shared memory, and uses them for all of
// its heads; it holds as many heads of the page as fit its threads' registers (a "round"),
// takes their maxima, and writes them.  An angle is a position times a 64-bit
// fraction of a turn, modulo 2^64: exact modulo a turn, so only the last step (top 32 bits to
// fp32) rounds, to 2^-25 of a turn.
#include "kv.cuh"

namespace f3dc {

namespace {

constexpr int kThreads = 256, kUnits = 4;  // a unit: 16 elements of a token and head
constexpr int kMaxHeads = 256;             // of a round

// The 16 elements of a unit: two 16-byte vectors of bf16.
struct Unit {
    uint4 a, b;
};

F3DC_DEV void widen(uint4 u, float *f)
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

F3DC_DEV uint4 narrow(const float *f)
{
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// kind of a round: 0 keys, 1 values, 2 queries
template <int DH>
__global__ void __launch_bounds__(kThreads) k_kv_append(const KvAppendArgs a)
{
    constexpr int kPer = DH / 16;  // units of a token and head
    extern __shared__ float angles[];  // cosines, then sines: [tokens][pairs] each
    __shared__ uint32_t top[kMaxHeads], new_byte[kMaxHeads], old_byte[kMaxHeads];
    griddep_launch();
    griddep_wait();
    const int slots = a.slots, b = blockIdx.x / slots, slot = blockIdx.x - b * slots, tid = threadIdx.x;
    const KvSeq s = kv_seq(a.batch, a.cache, b, a.err);
    if (s.n <= 0) return;
    if (s.n > s.length) {
        raise_error(a.err, kDevBadIndex);
        return;
    }
    const int page = a.cache.page, held = s.length - s.n;  // tokens before this call
    const int j = held / page + slot;                      // page of the sequence
    const int lo = max(held, j * page), hi = min(s.length, (j + 1) * page);
    if (lo >= hi) return;
    const int nt = hi - lo, row0 = s.row0 + lo - held, place0 = lo - j * page;
    const int p = kv_page(a.batch, a.cache, b, j, a.err);
    const int pairs = a.dims / 2, heads_k = a.cache.heads;

    // heads of a round, and rounds of keys (as many of values) and of queries
    const int per_round = min(kMaxHeads, kThreads * kUnits / (nt * kPer));
    const int rounds_k = (heads_k + per_round - 1) / per_round;
    const int rounds_q = a.q ? (a.heads + per_round - 1) / per_round : 0;
    const int rounds = 2 * rounds_k + rounds_q;

    float *const cosines = angles, *const sines = angles + page * pairs;
    if (pairs > 0) {
        const int of_axis = pairs / a.axes;
        for (int i = tid; i < nt * pairs; i += kThreads) {
            const int t = i / pairs, pr = i - t * pairs, axis = pr / of_axis;
            float sn = 0.f, cs = 1.f;
            if (axis < a.axes) {
                const int at = a.positions ? a.positions[(int64_t)(row0 + t) * a.axes + axis] : lo + t;
                const uint64_t turn = (uint64_t)(int64_t)at * a.turns[pr];
                sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &sn, &cs);
            }
            cosines[t * pairs + pr] = cs;
            sines[t * pairs + pr] = sn;
        }
        __syncthreads();
    }

#pragma unroll 1
    for (int r = blockIdx.y; r < rounds; r += gridDim.y) {
        const int kind = r < rounds_k ? 0 : (r < 2 * rounds_k ? 1 : 2);
        if (kind < 2 && p < 0) continue;
        const int all = kind < 2 ? heads_k : a.heads;
        const int h0 = (kind == 0 ? r : (kind == 1 ? r - rounds_k : r - 2 * rounds_k)) * per_round;
        const int nh = min(per_round, all - h0), units = nh * nt * kPer;
        const bf16 *const src = kind == 0 ? a.k : (kind == 1 ? a.v : a.q);
        const int64_t ld = kind == 0 ? a.ldk : (kind == 1 ? a.ldv : a.ldq);
        const int turning = kind == 1 ? 0 : a.dims / 16;  // a token's units that rotate

        // unit i: head, token and first elements of its two vectors
        auto where = [&](int i, int &head, int &t, int &c, int &e0, int &e1) {
            c = i % kPer;
            const int x = i / kPer;
            head = x / nt;
            t = x - head * nt;
            const bool split = c < turning && !a.interleaved;
            e0 = split ? 8 * c : 16 * c;
            e1 = split ? pairs + 8 * c : 16 * c + 8;
        };
        if (kind < 2) {
            if (tid < nh) top[tid] = 0u;
            __syncthreads();
        }
        Unit u[kUnits];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int i = tid + k * kThreads;
            u[k].a = u[k].b = make_uint4(0u, 0u, 0u, 0u);
            if (i < units) {
                int head, t, c, e0, e1;
                where(i, head, t, c, e0, e1);
                const bf16 *x = src + (int64_t)(row0 + t) * ld + (h0 + head) * DH;
                u[k].a = *reinterpret_cast<const uint4 *>(x + e0);
                u[k].b = *reinterpret_cast<const uint4 *>(x + e1);
            }
        }
        float f[kUnits][16];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int i = tid + k * kThreads;
            widen(u[k].a, f[k]);
            widen(u[k].b, f[k] + 8);
            int head = 0, t, c, e0, e1;
            if (i < units) {
                where(i, head, t, c, e0, e1);
                if (c < turning) {
                    const float *cs = cosines + t * pairs + 8 * c, *sn = sines + t * pairs + 8 * c;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (a.interleaved) {
                            const float p0 = f[k][2 * e], p1 = f[k][2 * e + 1];
                            f[k][2 * e] = p0 * cs[e] - p1 * sn[e];
                            f[k][2 * e + 1] = p1 * cs[e] + p0 * sn[e];
                        } else {
                            const float p0 = f[k][e], p1 = f[k][8 + e];
                            f[k][e] = p0 * cs[e] - p1 * sn[e];
                            f[k][8 + e] = p1 * cs[e] + p0 * sn[e];
                        }
                    }
                }
            }
            if (kind < 2) {
                // the unit's largest finite magnitude; an infinity becomes NaN, which fmaxf passes over
                const float inf = __int_as_float(0x7F800000);
                float m = 0.f;
#pragma unroll
                for (int e = 0; e < 16; e += 2) m = fmax3(m, fabsf(f[k][e]), fabsf(f[k][e + 1]));
                if (m == inf) {
                    m = 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        if (fabsf(f[k][e]) == inf) f[k][e] = __int_as_float(0x7FC00000);
                        m = fmaxf(m, fabsf(f[k][e]));
                    }
                }
                // one atomic a warp where its units are of one head
                const int h = i < units ? head : -1;
                const uint32_t bits = __float_as_uint(m);
                const int h_first = __shfl_sync(0xffffffffu, h, 0);
                if (__all_sync(0xffffffffu, h == h_first)) {
                    const uint32_t most = __reduce_max_sync(0xffffffffu, bits);
                    if (h >= 0 && (tid & 31) == 0) atomicMax(&top[h], most);
                } else if (h >= 0) {
                    atomicMax(&top[h], bits);
                }
            }
        }
        if (kind == 2) {
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const int i = tid + k * kThreads;
                if (i >= units) continue;
                int head, t, c, e0, e1;
                where(i, head, t, c, e0, e1);
                bf16 *y = a.q_out + (int64_t)(row0 + t) * a.ldqo + (h0 + head) * DH;
                *reinterpret_cast<uint4 *>(y + e0) = narrow(f[k]);
                *reinterpret_cast<uint4 *>(y + e1) = narrow(f[k] + 8);
            }
            continue;
        }
        uint8_t *const scales = (kind == 0 ? a.cache.ks : a.cache.vs) + (int64_t)p * a.cache.scale_stride + h0;
        uint8_t *const pool = (kind == 0 ? a.cache.k : a.cache.v) + (int64_t)p * a.cache.page_stride +
                              (int64_t)h0 * page * DH;
        __syncthreads();
        if (tid < nh) {
            uint32_t byte = e8m0_byte(__uint_as_float(top[tid])), old = byte;
            if (place0 > 0) {  // the page goes on
                old = scales[tid];
                byte = max(byte, old);
            }
            old_byte[tid] = old;
            new_byte[tid] = byte;
            scales[tid] = (uint8_t)byte;
        }
        __syncthreads();
        // tokens that a larger scale rounds anew
        if (place0 > 0) {
            for (int i = tid; i < nh * place0 * kPer; i += kThreads) {
                const int head = i / (place0 * kPer);
                const int down = (int)new_byte[head] - (int)old_byte[head];
                if (down == 0) continue;
                uint4 *at = reinterpret_cast<uint4 *>(pool + (int64_t)head * page * DH) + (i - head * place0 * kPer);
                const uint4 w = *at;
                const float by = pow2(-down);
                auto moved = [&](uint32_t x) {
                    uint32_t l, h;
                    e4m3x4_to_half2(x, l, h);
                    const float2 g0 = __half22float2(*reinterpret_cast<const __half2 *>(&l));
                    const float2 g1 = __half22float2(*reinterpret_cast<const __half2 *>(&h));
                    return pack_e4m3x4(g0.x * by, g0.y * by, g1.x * by, g1.y * by);
                };
                *at = make_uint4(moved(w.x), moved(w.y), moved(w.z), moved(w.w));
            }
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int i = tid + k * kThreads;
            if (i >= units) continue;
            int head, t, c, e0, e1;
            where(i, head, t, c, e0, e1);
            const float by = pow2(127 - (int)new_byte[head]);
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[e] = pack_e4m3x4(f[k][4 * e] * by, f[k][4 * e + 1] * by, f[k][4 * e + 2] * by, f[k][4 * e + 3] * by);
            uint8_t *y = pool + ((int64_t)head * page + place0 + t) * DH;
            if (e1 == e0 + 8) {
                *reinterpret_cast<uint4 *>(y + e0) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                *reinterpret_cast<uint2 *>(y + e0) = make_uint2(w[0], w[1]);
                *reinterpret_cast<uint2 *>(y + e1) = make_uint2(w[2], w[3]);
            }
        }
        __syncthreads();  // top, new_byte: the next round's
    }
}

template <int DH>
cudaError_t launch_dh(const KvAppendArgs &a, dim3 grid, size_t smem, cudaStream_t s)
{
    static std::atomic<uint64_t> devices{0};
    const cudaError_t e = ask_smem(k_kv_append<DH>, 128 * DH * sizeof(float), devices);
    return e == cudaSuccess ? launch_k(k_kv_append<DH>, grid, dim3(kThreads), smem, s, a) : e;
}

}  // namespace

cudaError_t launch_kv_append(const KvAppendArgs &args, int num_sms, cudaStream_t s)
{
    KvAppendArgs a = args;
    const int page = a.cache.page;
    // pages that a sequence's rows can touch, starting anywhere in one
    a.slots = (a.batch.max_rows + page - 2) / page + 1;
    const int64_t ctas = (int64_t)a.slots * a.batch.batch;
    if (ctas > INT32_MAX) return cudaErrorInvalidValue;
    // rounds of a full page
    const int tokens = a.batch.max_rows < page ? a.batch.max_rows : page, per = kThreads * kUnits / (tokens * (a.cache.dh / 16));
    const int per_round = per < kMaxHeads ? per : kMaxHeads;
    const int rounds = 2 * ((a.cache.heads + per_round - 1) / per_round) + (a.q ? (a.heads + per_round - 1) / per_round : 0);
    int64_t split = (4 * (int64_t)num_sms + ctas - 1) / ctas;
    if (split > rounds) split = rounds;
    const size_t smem = (size_t)page * a.dims * sizeof(float);
    const dim3 grid((unsigned)ctas, (unsigned)split);
    switch (a.cache.dh) {
    case 32: return launch_dh<32>(a, grid, smem, s);
    case 64: return launch_dh<64>(a, grid, smem, s);
    case 128: return launch_dh<128>(a, grid, smem, s);
    default: return cudaErrorInvalidValue;
    }
}

}  // namespace f3dc
