// k_kv_append.cu -- f3dc_kv_append_fp8: the keys and values of new tokens into the pages of
// their sequences, e4m3 with one power-of-two scale per page and head, keys and queries
// rotated by their positions on the way.
//
//   k'_p = R(p) k_p:  (a, b) -> (a cos - b sin, b cos + a sin), angle 2 pi p turns_j / 2^64
//   byte = smallest e with max |k'| <= 448 2^e over the page's new tokens, at least the
//          page's own where it already holds tokens; q = k' 2^-e to nearest even
//
// One pass over the rows.  A CTA takes one page of one sequence: it computes the cosines and sines of the
// page's new tokens once, into shared memory, and uses them for all of its heads.  A head of the page is the
// work of 1 to 256 threads, two or four units of 16 elements each, in registers; the next head's are on their way
// meanwhile.  Up to a warp's threads meet in shuffles, more in a barrier
// of their own, so heads do not wait for one another.  An angle is a position times a 64-bit
// fraction of a turn, modulo 2^64: exact modulo a turn, so only the last step (top 32 bits to
// fp32) rounds, to 2^-25 of a turn.
// What bounds it: bytes, at 77 % of a plain copy's rate: 32768 tokens of 16 heads of 64 (keys, values and
// queries, 336 MB) take 64 us, and 513 CTAs, two to an SM, are 1.7 rounds of them.  8192 tokens of 32 and 8 heads of 128 33 us (81 %),
// eight samples of up to 955 rows 16.8, one token 2.9, 64 tokens of 32 and 8 heads of 128 3.6.  Without the ring, the next
// head on its way in registers: 76 us, 43, 17.6, 3.3 and 4.0; with it, but two barriers a head, 67 us, 33, 17.6, 2.9 and 3.6, and
// then two places or four instead of three 71 and 68 us.  Three CTAs to an
// SM (80 registers): 82 us, and 14.4 for the samples.  (Pages of 128 with heads of 128 and neighbours rotated spill 96 bytes of a thread.)  Equal shares of all pages' heads for the CTAs that fit the SMs: 72 us, a pause
// at each change of page.
#include <algorithm>

#include "kv.cuh"

namespace f3dc {

namespace {

constexpr int kThreads = 256;
constexpr int kPerSm = 2;                  // CTAs, where shared memory has room for them
constexpr size_t kMostShared = 112 * 1024;  // for each of them

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

// threads that share a head of `units` units, at most `most` each: a power of two
__host__ __device__ inline int head_threads(int units, int most)
{
    int t = 1;
    while (t < units && t < 32) t *= 2;
    while (t * most < units) t *= 2;
    return t;
}
// heads on their way: a place of the ring holds a thread's units of one
template <int kUnits>
struct Ring {
    static constexpr int kPlaces = 3, kPlace = kUnits * 2 * kThreads;  // 16-byte vectors
    static constexpr int kBytes = kPlaces * kPlace * 16;
};
// units of a thread, at most: a page's head has up to 1024
inline int units_of(int page, int dh) { return page * (dh / 16) > 2 * kThreads ? 4 : 2; }

// INTER: pairs are neighbours
template <int DH, bool INTER, int kUnits>
__global__ void __launch_bounds__(kThreads, kPerSm) k_kv_append(const KvAppendArgs a)
{
    constexpr int kPer = DH / 16;  // units of a token and head
    constexpr int kPlaces = Ring<kUnits>::kPlaces, kPlace = Ring<kUnits>::kPlace;
    extern __shared__ __align__(16) uint4 ring[];  // [places][units][2][threads]: a thread reads what it has brought in itself
    float *const angles = reinterpret_cast<float *>(ring + kPlaces * kPlace);  // cosines, then sines: [tokens][pairs] each
    __shared__ float tops[2][kThreads / 32];  // in turn, so that one barrier a head is enough
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
    if ((uint32_t)slot * page >= (uint32_t)s.n + page) return;  // (the bound on rows may be far above n: no token's number overflows below)
    const int j = held / page + slot;                      // page of the sequence
    const int lo = max(held, j * page), hi = min(s.length, (j + 1) * page);
    if (lo >= hi) return;
    const int nt = hi - lo, row0 = s.row0 + lo - held, place0 = lo - j * page;
    const int p = kv_page(a.batch, a.cache, b, j, a.err);
    const int pairs = a.dims / 2, heads_k = a.cache.heads;

    float *const cosines = angles, *const sines = angles + page * pairs;
    // (a thread's units are of tokens `apart` tokens apart, the same elements of each)
    const int threads = head_threads(nt * kPer, kUnits), group = tid / threads, own = tid & (threads - 1);
    const int groups = kThreads / threads, token = own / kPer, apart = threads / kPer, c = own % kPer;
    const bool rotates = c < a.dims / 16;
    // The unit's two vectors of 8: one of each half of the elements that turn, or of each half of those that do not, so that
    // neighbouring threads' vectors lie side by side.
    const int e0 = rotates ? 8 * c : pairs + 8 * c, e1 = e0 + (rotates ? pairs : DH / 2 - pairs);
    const float inf = __int_as_float(0x7F800000);

    // The heads of keys, of values and of queries are shared out as one sequence, and done in that order.  (Whole warps go
    // through them together: a warp's heads are beside one another, the last perhaps not there.)
    const int own_item = blockIdx.y * groups + tid / threads, warp_item = threads < 32 ? blockIdx.y * groups + (tid & ~31) / threads : own_item;
    const int beside = own_item - warp_item, step = gridDim.y * groups, span = 31 / min(threads, 32);
    const int begin_q = 2 * heads_k, end = a.q ? begin_q + a.heads : begin_q;
    const uint32_t own_place = smem_u32(ring + tid);
    auto fetch = [&](int item, int place) {
        if (item < end && token < nt) {
            const bf16 *rows = item < heads_k ? a.k : (item < begin_q ? a.v : a.q);
            const int64_t ld = item < heads_k ? a.ldk : (item < begin_q ? a.ldv : a.ldq);
            const int head = item < heads_k ? item : (item < begin_q ? item - heads_k : item - begin_q);
            const bf16 *from = rows + (int64_t)(row0 + token) * ld + (int64_t)head * DH;
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                if (token + k * apart >= nt) break;
                const uint32_t to = own_place + (uint32_t)(place * kPlace + 2 * k * kThreads) * 16u;
                cp_async16(to, from + (int64_t)(k * apart) * ld + e0);
                cp_async16(to + kThreads * 16u, from + (int64_t)(k * apart) * ld + e1);
            }
        }
        cp_async_commit();
    };
    int coming = own_item;
#pragma unroll
    for (int i = 0; i < kPlaces - 1; ++i, coming += step) fetch(coming, i);

    if (pairs > 0) {
        // a thread's pair is the same for all of its tokens
        const int at_once = kThreads / pairs, t0 = tid / pairs, pr = tid - t0 * pairs, axis = pr / (pairs / a.axes);
        if (t0 < at_once) {
            const uint64_t turns = axis < a.axes ? a.turns[pr] : 0;
            for (int t = t0; t < nt; t += at_once) {
                int at = lo + t;
                if (a.positions) at = a.positions[(int64_t)(row0 + t) * a.axes + min(axis, a.axes - 1)];
                const uint64_t turn = (uint64_t)(int64_t)at * turns;
                sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &sines[t * pairs + pr], &cosines[t * pairs + pr]);
            }
        }
        __syncthreads();
    }

    int place = 0, turn = 0;
    auto pass = [&](auto kind_tag, int head, int count, uint8_t *pool, uint8_t *scales) {
        constexpr int kKind = decltype(kind_tag)::value;  // 0 keys, 1 values, 2 queries
        if (kKind < 2 && p < 0) return;
        const bool live = (uint32_t)head < (uint32_t)count;
        uint8_t *const scale = scales + head;
        uint32_t old = 0;
        if (kKind < 2 && live && place0 > 0) old = *scale;  // the page goes on
        float f[kUnits][16];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            uint4 u0 = make_uint4(0u, 0u, 0u, 0u), u1 = u0;
            if (live && token + k * apart < nt) {
                u0 = ring[place * kPlace + 2 * k * kThreads + tid];
                u1 = ring[place * kPlace + (2 * k + 1) * kThreads + tid];
            }
            widen(u0, f[k]);
            widen(u1, f[k] + 8);
        }
        if (kKind != 1 && rotates) {
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const int at = min(token + k * apart, nt - 1) * pairs;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // four pairs: neighbours in vector h, or elements 4 h .. of both vectors
                    const int pr = INTER ? (h ? e1 : e0) / 2 : 8 * c + 4 * h;
                    const float4 c4 = *reinterpret_cast<const float4 *>(cosines + at + pr);
                    const float4 s4 = *reinterpret_cast<const float4 *>(sines + at + pr);
                    const float co[4] = {c4.x, c4.y, c4.z, c4.w}, si[4] = {s4.x, s4.y, s4.z, s4.w};
                    if constexpr (INTER) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float &x = f[k][8 * h + 2 * e], &y = f[k][8 * h + 2 * e + 1];
                            const float p0 = x, p1 = y;
                            x = p0 * co[e] - p1 * si[e];
                            y = p1 * co[e] + p0 * si[e];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            float *const x = f[k] + 4 * h + e;
                            const f32x2 p0 = {x[0], x[1]}, p1 = {x[8], x[9]}, c2 = {co[e], co[e + 1]}, s2 = {si[e], si[e + 1]};
                            const f32x2 a2 = fmul2(p1, s2), b2 = fmul2(p0, s2);
                            const f32x2 r0 = ffma2(p0, c2, {-a2.x, -a2.y}), r1 = ffma2(p1, c2, b2);
                            x[0] = r0.x, x[1] = r0.y, x[8] = r1.x, x[9] = r1.y;
                        }
                    }
                }
            }
        }
        if constexpr (kKind == 2) {
            if (!live) return;
            bf16 *const dst = a.q_out + (int64_t)(row0 + token) * a.ldqo + (int64_t)head * DH;
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                if (token + k * apart >= nt) continue;
                bf16 *y = dst + (int64_t)(k * apart) * a.ldqo;
                *reinterpret_cast<uint4 *>(y + e0) = narrow(f[k]);
                *reinterpret_cast<uint4 *>(y + e1) = narrow(f[k] + 8);
            }
        } else {
            // The largest finite magnitude.  fmaxf passes over NaN, so the plain maximum is infinite only with an infinity
            // among the values: the rare unit that has one makes NaN of it (e4m3 has no infinity) and takes the maximum of
            // the others.
            float top = 0.f;
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
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
                top = fmaxf(top, m);
            }
            if (threads >= 32) {
                // (magnitudes order as their bits do)
                top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
            } else {
                for (int o = threads / 2; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            }
            if (threads > 32) {
                if ((tid & 31) == 0) tops[turn][tid >> 5] = top;
                asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(threads) : "memory");
                const int w0 = group * (threads >> 5);
                for (int w = 0; w < threads >> 5; ++w) top = fmaxf(top, tops[turn][w0 + w]);
                turn ^= 1;
            }
            const uint32_t byte = max(e8m0_byte(top), old);
            if (live) {
                uint8_t *const block = pool + (int64_t)head * page * DH;
                // tokens of the page that a larger scale rounds anew
                if (place0 > 0 && byte != old) {
                    const float by = pow2((int)old - (int)byte);
                    for (int i = own; i < place0 * kPer; i += threads) {
                        uint4 *at = reinterpret_cast<uint4 *>(block) + i;
                        const uint4 w = *at;
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
                const float by = pow2(127 - (int)byte);
                uint8_t *const dst = block + (place0 + token) * DH;
#pragma unroll
                for (int k = 0; k < kUnits; ++k) {
                    if (token + k * apart >= nt) continue;
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f32x2 g0 = fmul2({f[k][4 * e], f[k][4 * e + 1]}, {by, by}), g1 = fmul2({f[k][4 * e + 2], f[k][4 * e + 3]}, {by, by});
                        w[e] = pack_e4m3x4(g0.x, g0.y, g1.x, g1.y);
                    }
                    uint8_t *y = dst + k * apart * DH;
                    *reinterpret_cast<uint2 *>(y + e0) = make_uint2(w[0], w[1]);
                    *reinterpret_cast<uint2 *>(y + e1) = make_uint2(w[2], w[3]);
                }
            }
            // (all have read the old scale before the maxima were joined)
            if (live && own == 0) *scale = (uint8_t)byte;
        }
    };
    const int64_t page_at = (int64_t)p * a.cache.page_stride, scale_at = (int64_t)p * a.cache.scale_stride;
#pragma unroll 1
    for (int first = warp_item; first < end; first += step) {
        cp_async_wait<kPlaces - 2>();
        fetch(coming, place == 0 ? kPlaces - 1 : place - 1);  // (the place read last)
        coming += step;
        const int item = first + beside;
        // (a warp's last item may be of the next kind)
        if (first < heads_k) pass(std::integral_constant<int, 0>(), item, heads_k, a.cache.k + page_at, a.cache.ks + scale_at);
        if (first + span >= heads_k && first < begin_q)
            pass(std::integral_constant<int, 1>(), item - heads_k, heads_k, a.cache.v + page_at, a.cache.vs + scale_at);
        if (first + span >= begin_q) pass(std::integral_constant<int, 2>(), item - begin_q, end - begin_q, nullptr, nullptr);
        place = place + 1 == kPlaces ? 0 : place + 1;
    }
    cp_async_wait_all();
}

template <int DH, bool INTER, int U>
cudaError_t launch_one(const KvAppendArgs &a, dim3 grid, size_t smem, cudaStream_t s)
{
    static std::atomic<uint64_t> devices{0};
    const cudaError_t e = ask_smem(k_kv_append<DH, INTER, U>, 128 * DH * sizeof(float) + Ring<U>::kBytes, devices);
    return e == cudaSuccess ? launch_k(k_kv_append<DH, INTER, U>, grid, dim3(kThreads), smem + Ring<U>::kBytes, s, a) : e;
}

template <int DH>
cudaError_t launch_dh(const KvAppendArgs &a, dim3 grid, size_t smem, cudaStream_t s)
{
    if (DH == 128 && units_of(a.cache.page, DH) == 4)
        return a.interleaved ? launch_one<128, true, 4>(a, grid, smem, s) : launch_one<128, false, 4>(a, grid, smem, s);
    return a.interleaved ? launch_one<DH, true, 2>(a, grid, smem, s) : launch_one<DH, false, 2>(a, grid, smem, s);
}

}  // namespace

cudaError_t launch_kv_append(const KvAppendArgs &args, int num_sms, cudaStream_t s)
{
    KvAppendArgs a = args;
    const int page = a.cache.page;
    // pages that a sequence's rows can touch, starting anywhere in one
    a.slots = (int)(((int64_t)a.batch.max_rows + page - 2) / page + 1);
    const int64_t ctas = (int64_t)a.slots * a.batch.batch;
    if (ctas > INT32_MAX) return cudaErrorInvalidValue;
    // heads of a page are shared by CTAs where there are few pages: as many as fit the SMs at once
    const int tokens = a.batch.max_rows < page ? a.batch.max_rows : page, units = units_of(page, a.cache.dh);
    const int groups = kThreads / head_threads(tokens * (a.cache.dh / 16), units), all = 2 * a.cache.heads + (a.q ? a.heads : 0);
    const size_t smem = (size_t)page * a.dims * sizeof(float);
    const int per_sm = smem + (units == 4 ? Ring<4>::kBytes : Ring<2>::kBytes) > kMostShared ? 1 : kPerSm;
    const int64_t split = std::max<int64_t>(1, std::min<int64_t>(per_sm * (int64_t)num_sms / ctas, (all + groups - 1) / groups));
    const dim3 grid((unsigned)ctas, (unsigned)split);
    switch (a.cache.dh) {
    case 32: return launch_dh<32>(a, grid, smem, s);
    case 64: return launch_dh<64>(a, grid, smem, s);
    case 128: return launch_dh<128>(a, grid, smem, s);
    default: return cudaErrorInvalidValue;
    }
}

}  // namespace f3dc
