// k_kv_few.cu -- f3dc_kv_attention_fp8 for few query rows to a key head (single tokens, a
// few at once, groups of heads): attention over a paged 8-bit cache, and the sum of the
// parts where several CTAs share a sequence's keys.
//
//   S^T = K Q^T, x = S scale 2^(ek) + ev, w = 2^(x - r), O^T += V^T w, l += w 2^-ev
//
// Bound by the cache's bytes.  A warp takes 32 tokens at a time: their keys and values come by cp.async into a ring
// of its own (no other warp is waited for), are converted to fp16 (exactly) and multiplied with mma.m16n8k16, 16 tokens or 16
// columns of the head as the rows and 8 packed query rows as the columns, so that up to 8 query rows (a group of heads' single
// token) cost half the products and exponents of a tile of 16.  K may be permuted within an MMA as long as both
// operands are: a lane's 16 consecutive bytes of a key serve four MMAs.  The weights turn round in one movmatrix a tile, and the
// tokens behind the rows of S^T are chosen so that four lanes read four neighbouring tokens' values.  Each warp
// keeps sums and references of its own, which are joined at the end.
// One token of 32 heads of 128 to 8 key heads over 524288: 167 us (6.4 TB/s, 95 % of a plain copy's rate); 64 sequences' tokens over
// 4096 to 8192: 132 us (6.2 TB/s), where the lengths leave some SMs idle at the end; one token over 1374 of 16 heads of 64:
// 5.8 us, the launch and the latencies of page table, pages and the cluster.  With query rows as the MMA's rows, and parts joined by
// a warp one after another: 224, 190 and 13 us.
#include "kv.cuh"

namespace f3dc {

namespace {

constexpr int kWarps = 4, kChunk = 32;
constexpr float kInf = __builtin_huge_valf();
// A row's largest weight is 2^kTop where its reference was taken, and up to 2^(kTop + kLazy) before it is taken anew:
// below 2^16, with 2^-25 of it at fp16's full precision and 2^-36 at all.
constexpr float kTop = 11.f, kLazy = 4.f;

template <int DH>
struct FewCfg {
    // (one chunk ahead with dh 128, where three CTAs fit an SM, or two with two ahead: 64 tokens over up to 8192 136 us / 153, one over
    // 524288 167 / 184)
    static constexpr int kHalf = kChunk * DH, kStage = 2 * kHalf;  // bytes: keys, then values
    static constexpr int kStages = DH == 128 ? 2 : 3;
    static constexpr int kSmem = kWarps * kStages * kStage;
};

F3DC_DEV void cp_async16_or_zeros(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}

F3DC_DEV void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Places of a token's 16-byte pieces in a stage, chosen so that the reads below meet no bank twice.
// Keys: row g of each eight holds the token behind column g of S.
template <int DH>
F3DC_DEV int key_place(int token, int piece)
{
    const int row = (token & ~7) | ((token & 3) << 1) | ((token >> 2) & 1);
    if (DH == 128) piece ^= (row & 1) << 2;
    return row * DH + 16 * piece;
}
template <int DH>
F3DC_DEV int value_place(int token, int piece)
{
    if (DH == 128) piece ^= (token & 3) << 1;
    if (DH == 64) piece ^= token & 2;
    return token * DH + 16 * piece;
}

// an 8 x 8 matrix of 16-bit elements, lane (g, q) holding (g, 2 q) and (g, 2 q + 1), transposed
F3DC_DEV uint32_t transposed(uint32_t a)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}
// all ones in the halves that are no NaN
F3DC_DEV uint32_t half2_numbers(uint32_t a)
{
    return __heq2_mask(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&a));
}

// NT: tiles of 8 packed rows
// CLUSTER: the CTAs of a sequence's keys are a cluster and join their sums themselves.  (A form of its own: in one with the other it cost
// calls without a cluster 2 %.)
template <int DH, int NT, bool CLUSTER>
__global__ void __launch_bounds__(32 * kWarps) k_kv_few(const KvAttnArgs a)
{
    using Cfg = FewCfg<DH>;
    constexpr int kSteps = DH / 16, kRows = 8 * NT;
    constexpr int kStages = Cfg::kStages;
    extern __shared__ uint4 smem4[];
    uint8_t *const smem = reinterpret_cast<uint8_t *>(smem4);
    __shared__ float sm_m[kWarps][kRows], sm_l[kWarps][kRows];
    __shared__ float2 sm_ml[kRows];
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;

    uint32_t item = blockIdx.x;
    const int split = (int)(item % (uint32_t)a.splits);
    item /= (uint32_t)a.splits;
    const int rb = (int)(item % (uint32_t)a.row_blocks);
    item /= (uint32_t)a.row_blocks;
    const int hk = (int)(item % (uint32_t)a.cache.heads), b = (int)(item / (uint32_t)a.cache.heads);
    const KvSeq s = kv_seq(a.batch, a.cache, b, a.err);
    const int r0 = rb * kRows;
    const int rows = s.n * a.group;  // packed
    if (s.n <= 0 || r0 >= rows) return;
    const int row_end = min(rows, r0 + kRows);

    // tokens that the last and the first of the rows see
    const int behind = s.length - s.n + 1;
    const int most = a.causal ? max(0, behind + (row_end - 1) / a.group) : s.length;
    const int least = a.causal ? behind + r0 / a.group : s.length;
    const int chunks = (most + kChunk - 1) / kChunk;
    const int c_begin = kv_share(chunks, split, a.splits), c_end = kv_share(chunks, split + 1, a.splits);

    // ---- this warp's ring
    uint8_t *const ring = smem + warp * kStages * Cfg::kStage;
    const int page = a.cache.page, page_log2 = 31 - __clz(page);
    // where the next chunk's two runs of 16 tokens lie (-1: nowhere), and their pages
    int64_t run0 = -1, run1 = -1;
    int page0 = -1, page1 = -1;
    auto look_up = [&](int c) {
        const int t = c * kChunk;
        if (c >= c_end) return;
        page0 = kv_page(a.batch, a.cache, b, t >> page_log2, a.err);
        page1 = t + 16 < s.length ? kv_page(a.batch, a.cache, b, (t + 16) >> page_log2, a.err) : -1;
        run0 = page0 < 0 ? -1 : (int64_t)page0 * a.cache.page_stride + (int64_t)(hk * page + (t & (page - 1))) * DH;
        run1 = page1 < 0 ? -1 : (int64_t)page1 * a.cache.page_stride + (int64_t)(hk * page + ((t + 16) & (page - 1))) * DH;
    };
    // loads of chunk c; returns its scale byte of lane's kind: keys / values, first / second run
    auto load = [&](int c, int slot) {
        uint32_t scale = 127u;
        if (c < c_end) {
            const uint32_t dst = smem_u32(ring + slot * Cfg::kStage);
            const int t0 = c * kChunk;
            const bool whole = t0 + kChunk <= s.length && run0 >= 0 && run1 >= 0;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                // a run's bytes follow one another: piece p is 16 p bytes into it
                const int p = lane + 32 * i, token = p / kSteps, piece = p % kSteps;
                const int64_t run = i < kSteps / 2 ? run0 : run1;
                const int off = 16 * p - (i < kSteps / 2 ? 0 : 16 * DH);
                if (whole) {
                    cp_async16(dst + key_place<DH>(token, piece), a.cache.k + run + off);
                    cp_async16(dst + Cfg::kHalf + value_place<DH>(token, piece), a.cache.v + run + off);
                } else {
                    const bool real = t0 + token < s.length && run >= 0;
                    const int64_t at = real ? run + off : 0;
                    cp_async16_or_zeros(dst + key_place<DH>(token, piece), a.cache.k + at, real);
                    cp_async16_or_zeros(dst + Cfg::kHalf + value_place<DH>(token, piece), a.cache.v + at, real);
                }
            }
            const int pg = lane & 2 ? page1 : page0;
            if (pg >= 0) scale = (lane & 1 ? a.cache.vs : a.cache.ks)[(int64_t)pg * a.cache.scale_stride + hk];
        }
        cp_async_commit();
        return scale;
    };
    const int c0 = c_begin + warp;
    uint32_t scales[kStages - 1];
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) {
        look_up(c0 + i * kWarps);
        scales[i] = load(c0 + i * kWarps, i);
    }
    look_up(c0 + (kStages - 1) * kWarps);

    // ---- queries as the products' columns: fp16 times a power of two for each row; the k of step j are elements 16 q + 4 j
    // .. + 3 of each 64
    uint32_t qb[NT][kSteps][2];
    float factor[NT][2];  // of S, in log2, for rows 2 q and 2 q + 1
    int sees[NT][2];      // tokens
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = min(r0 + 8 * n + g, row_end - 1), token = at / a.group, head = hk * a.group + at % a.group;
        const bf16 *x = a.q + (int64_t)(s.row0 + token) * a.ldq + (int64_t)head * DH;
        uint32_t w[DH / 8];
        constexpr int kRun = DH >= 64 ? 16 : 8;  // consecutive elements of a lane
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) {
            const uint4 u = *reinterpret_cast<const uint4 *>(x + (j * 8 / kRun) * 64 + kRun * q + j * 8 % kRun);
            w[4 * j] = u.x, w[4 * j + 1] = u.y, w[4 * j + 2] = u.z, w[4 * j + 3] = u.w;
        }
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < DH / 8; ++j)
            top = fmax3(top, fabsf(__uint_as_float(w[j] << 16)), fabsf(__uint_as_float(w[j] & 0xFFFF0000u)));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = query_exponent(top), sight = a.causal ? behind + token : s.length;
        const float up = pow2(e), down = a.scale_log2 * pow2(-e);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            factor[n][i] = __shfl_sync(0xffffffffu, down, 4 * (2 * q + i));
            sees[n][i] = __shfl_sync(0xffffffffu, sight, 4 * (2 * q + i));
        }
#pragma unroll
        for (int j = 0; j < 2 * kSteps; ++j)
            qb[n][j / 2][j % 2] = pack_half2(__uint_as_float(w[j] << 16) * up, __uint_as_float(w[j] & 0xFFFF0000u) * up);
    }

    // sums O^T: element (column, row): acc[n][j][e] of column g DH / 8 + 2 j + e / 2 and row 8 n + 2 q + e % 2
    float acc[NT][kSteps][4];
    float ref[NT][2], sum[NT][2];
    float widest = (float)kLeastScale;  // largest value scale so far
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][j][e] = 0.f;
        ref[n][0] = ref[n][1] = -kInf;
        sum[n][0] = sum[n][1] = 0.f;
    }

    // Chunk c, whose keys and values stand in place `slot` of the ring.  Plain: returns false, with nothing done, where a value scale is too far below the
    // largest so far; such a chunk is done in the other form.
    auto chunk = [&](int c, uint32_t scale, int slot, auto apart_tag) {
        constexpr bool kApart = decltype(apart_tag)::value;
        const uint8_t *const keys = ring + slot * Cfg::kStage, *const values = keys + Cfg::kHalf;
        const int t0 = c * kChunk;

        // S^T: 16 tokens by 8 rows each: x[n][h][e] of row 2 q + e % 2 and token 16 h + 8 (e / 2) + 4 (g & 1) + (g >> 1)
        float x[NT][2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[n][h][e] = 0.f;
#pragma unroll
            for (int v = 0; v < (DH >= 64 ? DH / 64 : 1); ++v) {
                uint32_t w[2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int row = 16 * h + 8 * i + g;
                    if constexpr (DH >= 64) {
                        const int piece = (4 * v + q) ^ (DH == 128 ? (row & 1) << 2 : 0);
                        const uint4 u = *reinterpret_cast<const uint4 *>(keys + row * DH + 16 * piece);
                        w[i][0] = u.x, w[i][1] = u.y, w[i][2] = u.z, w[i][3] = u.w;
                    } else {
                        const uint2 u = *reinterpret_cast<const uint2 *>(keys + row * DH + 8 * q);
                        w[i][0] = u.x, w[i][1] = u.y;
                    }
                }
#pragma unroll
                for (int j = 0; j < (DH >= 64 ? 4 : 2); ++j) {
                    uint32_t k[4];
                    e4m3x4_to_half2(w[0][j], k[0], k[2]);
                    e4m3x4_to_half2(w[1][j], k[1], k[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma16816(x[n][h], k, qb[n][4 * v + j][0], qb[n][4 * v + j][1]);
                }
            }
        }

        // scales of the chunk's two runs, scores in log2 with their value scales
        float ks[2];
        ValueScale vs[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            ks[h] = key_scale(__shfl_sync(0xffffffffu, scale, 2 * h));
            vs[h] = value_scale(__shfl_sync(0xffffffffu, scale, 2 * h + 1));
        }
        const bool partly = t0 + kChunk > least;
        const int own_token = t0 + 4 * (g & 1) + (g >> 1);
        widest = fmaxf(widest, fmaxf(vs[0].log2, vs[1].log2));
        const bool apart = !kApart && fminf(vs[0].log2, vs[1].log2) < widest - kScaleSpan;  // (the same for the warp)
        // (dh 128: looked at with the vote below.  A branch of its own costs 4 rows of 16 sequences of 8192 6 %, and the vote's costs heads of
        // 64 and 32 3 % and more.)
        if (DH < 128 && __builtin_expect(apart, 0)) return false;
        bool raise = DH == 128 && apart;
        float top[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float t = -kInf;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float &y = x[n][h][2 * i + r];
                        y = fmaf(y, factor[n][r] * ks[h], vs[h].log2);
                        if (partly && own_token + 16 * h + 8 * i >= sees[n][r]) y = -kInf;
                        t = fmaxf(t, y);
                    }
#pragma unroll
                for (int o = 4; o < 32; o *= 2) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
                top[n][r] = t;
                raise |= t > ref[n][r] + (kTop + kLazy);
            }
        if (__any_sync(0xffffffffu, raise)) {
            if (DH == 128 && apart) return false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float to = fmaxf(ref[n][r], top[n][r] - kTop);
                    const float half = half_factor(ref[n][r], to), by = half * half;
                    ref[n][r] = to;
                    sum[n][r] = sum[n][r] * half * half;
#pragma unroll
                    for (int j = 0; j < kSteps; ++j) {
                        acc[n][j][r] *= by;
                        acc[n][j][2 + r] *= by;
                    }
                }
        }
        uint32_t w[NT][2][2];  // weights as the second product's columns: tokens along the quad, a row for each g
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float base[2] = {ref[n][0] == -kInf ? 0.f : -ref[n][0], ref[n][1] == -kInf ? 0.f : -ref[n][1]};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = exp2_fast(x[n][h][e] + base[e & 1]);
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    if (kApart) {
                        const float at = base[r] - vs[h].log2 + kSumShift;
                        sum[n][r] = fmaf(exp2_fast(x[n][h][r] + at) + exp2_fast(x[n][h][2 + r] + at), kSumUnshift, sum[n][r]);
                    } else {
                        sum[n][r] = fmaf(p[r] + p[2 + r], vs[h].inverse, sum[n][r]);
                    }
                }
                w[n][h][0] = transposed(pack_half2(p[0], p[1]));
                w[n][h][1] = transposed(pack_half2(p[2], p[3]));
            }
        }
        const bool odd = partly || vs[0].times != kHalfOnes || vs[1].times != kHalfOnes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // sixteen tokens
            uint32_t v[4][DH / 32];  // lane's columns g DH / 8 .. of tokens 4 i + q
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int token = 16 * h + 4 * i + q;
                if constexpr (DH == 128) {
                    const uint4 u = *reinterpret_cast<const uint4 *>(values + value_place<DH>(token, g));
                    v[i][0] = u.x, v[i][1] = u.y, v[i][2] = u.z, v[i][3] = u.w;
                } else if constexpr (DH == 64) {
                    const uint2 u = *reinterpret_cast<const uint2 *>(values + value_place<DH>(token, g >> 1) + 8 * (g & 1));
                    v[i][0] = u.x, v[i][1] = u.y;
                } else {
                    v[i][0] = *reinterpret_cast<const uint32_t *>(values + token * DH + 4 * g);
                }
            }
            // pairs of tokens of the lane's columns 4 k .. 4 k + 3, two columns to an operand
            auto operands = [&](int k, uint32_t (&o)[2][4]) {
                e4m3x4_to_half2(__byte_perm(v[0][k], v[1][k], 0x5140), o[0][0], o[0][1]);
                e4m3x4_to_half2(__byte_perm(v[0][k], v[1][k], 0x7362), o[1][0], o[1][1]);
                e4m3x4_to_half2(__byte_perm(v[2][k], v[3][k], 0x5140), o[0][2], o[0][3]);
                e4m3x4_to_half2(__byte_perm(v[2][k], v[3][k], 0x7362), o[1][2], o[1][3]);
            };
            if (!odd) {
#pragma unroll
                for (int k = 0; k < DH / 32; ++k) {
                    uint32_t o[2][4];
                    operands(k, o);
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma16816(acc[n][2 * k + j], o[j], w[n][h][0], w[n][h][1]);
                }
            } else {
                // A NaN that a row does not see must not meet its weight of zero: NaN count as zeros in the product,
                // and where there are any, a second one counts for each row those that it sees.
                const uint32_t times = vs[h].times;
                uint32_t sight[NT][2];  // 1 for a token that the row sees
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t m = 0;
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            m |= own_token + 16 * h + 8 * i < sees[n][r] ? 0x3C00u << (16 * r) : 0u;
                        sight[n][i] = transposed(m);
                    }
#pragma unroll
                for (int k = 0; k < DH / 32; ++k) {
                    uint32_t o[2][4];
                    operands(k, o);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t numbers[4], all = 0xffffffffu;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            o[j][e] = half2_times(o[j][e], times);
                            numbers[e] = half2_numbers(o[j][e]);
                            o[j][e] &= numbers[e];
                            all &= numbers[e];
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma16816(acc[n][2 * k + j], o[j], w[n][h][0], w[n][h][1]);
                        if (__any_sync(0xffffffffu, all != 0xffffffffu)) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) numbers[e] = ~numbers[e] & kHalfOnes;
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                float count[4] = {0.f, 0.f, 0.f, 0.f};
                                mma16816(count, numbers, sight[n][0], sight[n][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (count[e] > 0.f) acc[n][2 * k + j][e] = __int_as_float(0x7FC00000);
                            }
                        }
                    }
                }
            }
        }
        return true;
    };
    int slot = 0, c = c0;
    uint32_t scale = 127u;
    while (true) {
#pragma unroll 1
        for (; c < c_end; c += kWarps) {
            cp_async_wait<kStages - 2>();
            __syncwarp();
            scale = scales[0];
#pragma unroll
            for (int i = 0; i < kStages - 2; ++i) scales[i] = scales[i + 1];
            const int next = c + (kStages - 1) * kWarps, next_slot = slot == 0 ? kStages - 1 : slot - 1;
            scales[kStages - 2] = load(next, next_slot);
            look_up(next + kWarps);
            if (!chunk(c, scale, slot, std::false_type())) break;
            slot = slot + 1 == kStages ? 0 : slot + 1;
        }
        if (__builtin_expect(c >= c_end, 1)) break;
        chunk(c, scale, slot, std::true_type());
        slot = slot + 1 == kStages ? 0 : slot + 1;
        c += kWarps;
    }

    // ---- the warps' sums joined.  (Only now may the next kernel's CTAs come: with them in between the launch's own would
    // not all fit at once, see kv_splits.)
    griddep_launch();
    cp_async_wait<0>();
    __syncthreads();
    float *const sums = reinterpret_cast<float *>(smem);  // [warps][rows][DH]
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float l = sum[n][r];
#pragma unroll
            for (int o = 4; o < 32; o *= 2) l += __shfl_xor_sync(0xffffffffu, l, o);
            const int row = 8 * n + 2 * q + r;
            if (g == 0) {
                sm_m[warp][row] = ref[n][r];
                sm_l[warp][row] = l;
            }
            float *o = sums + (warp * kRows + row) * DH + g * (DH / 8);
#pragma unroll
            for (int j = 0; j < kSteps; j += 2)
                *reinterpret_cast<float4 *>(o + 2 * j) =
                    make_float4(acc[n][j][r], acc[n][j][2 + r], acc[n][j + 1][r], acc[n][j + 1][2 + r]);
        }
    __syncthreads();
    const int items = (row_end - r0) * (DH / 8);  // eight elements of a row each
    auto write = [&](int row, int col, float m, float l, const float (&o)[8]) {
        const int token = (r0 + row) / a.group, head = hk * a.group + (r0 + row) % a.group;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        uint4 u;
        u.x = pack_bf16x2(o[0] * inv, o[1] * inv);
        u.y = pack_bf16x2(o[2] * inv, o[3] * inv);
        u.z = pack_bf16x2(o[4] * inv, o[5] * inv);
        u.w = pack_bf16x2(o[6] * inv, o[7] * inv);
        *reinterpret_cast<uint4 *>(a.out + (int64_t)(s.row0 + token) * a.ldo + (int64_t)head * DH + col) = u;
        if (a.lse && col == 0) a.lse[(int64_t)(s.row0 + token) * a.heads + head] = log_sum(m, l);
    };
    for (int i = threadIdx.x; i < items; i += 32 * kWarps) {
        const int row = i / (DH / 8), col = i % (DH / 8) * 8;
        float m = sm_m[0][row];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sm_m[w][row]);
        float l = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            // (a NaN sum has no reference of its own)
            const float half = half_factor(sm_m[w][row], m), by = half * half;
            l += sm_l[w][row] * half * half;
            const float *x = sums + (w * kRows + row) * DH + col;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(x[e], by, o[e]);
        }
        if (a.splits == 1) {
            write(row, col, m, l, o);
        } else if (CLUSTER) {
            // (the first warp's place, read by this thread alone)
            float *dst = sums + row * DH + col;
            *reinterpret_cast<float4 *>(dst) = make_float4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<float4 *>(dst + 4) = make_float4(o[4], o[5], o[6], o[7]);
            if (col == 0) sm_ml[row] = make_float2(m, l);
        } else {
            const int token = (r0 + row) / a.group, head = hk * a.group + (r0 + row) % a.group;
            const int64_t part = (int64_t)split * a.batch.rows * a.heads + (int64_t)(s.row0 + token) * a.heads + head;
            float *dst = a.part + part * DH + col;
            *reinterpret_cast<float4 *>(dst) = make_float4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<float4 *>(dst + 4) = make_float4(o[4], o[5], o[6], o[7]);
            if (col == 0) {
                float2 *ml = reinterpret_cast<float2 *>(a.part + (int64_t)a.splits * a.batch.rows * a.heads * DH);
                ml[part] = make_float2(m, l);
            }
        }
    }
    if constexpr (CLUSTER) {
        // each CTA joins some of the rows' elements from all CTAs' shared memory
        __syncwarp();
        cluster_sync();
        for (int i = threadIdx.x + 32 * kWarps * split; i < items; i += 32 * kWarps * a.splits) {
            const int row = i / (DH / 8), col = i % (DH / 8) * 8;
            const uint32_t ml_own = smem_u32(sm_ml + row), o_own = smem_u32(sums + row * DH + col);
            float2 p[kMostCluster];
            float4 v[kMostCluster][2];
            float m = -kInf;
#pragma unroll
            for (int k = 0; k < kMostCluster; ++k) {
                p[k] = make_float2(-kInf, 0.f);
                v[k][0] = v[k][1] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k < a.splits) {
                    const uint32_t from = mapa_shared(o_own, k);
                    p[k] = load_cluster8(mapa_shared(ml_own, k));
                    v[k][0] = load_cluster16(from);
                    v[k][1] = load_cluster16(from + 16);
                }
            }
#pragma unroll
            for (int k = 0; k < kMostCluster; ++k) m = fmaxf(m, p[k].x);
            float l = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kMostCluster; ++k) {
                const float half = half_factor(p[k].x, m), by = half * half;
                l += p[k].y * half * half;
                const float x[8] = {v[k][0].x, v[k][0].y, v[k][0].z, v[k][0].w, v[k][1].x, v[k][1].y, v[k][1].z, v[k][1].w};
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = fmaf(x[e], by, o[e]);
            }
            write(row, col, m, l, o);
        }
        __syncwarp();
        cluster_sync();  // no CTA leaves while another reads its shared memory
    }
}

// Parts of a row and head added up by WARPS warps: they take the parts in turn, several on their way at
// once, and their sums are joined in order.  (One warp for up to 16 parts, which come where many rows are shared: 1521 rows of two
// sequences over up to 1811, heads of 128, in 3 parts 28 us instead of 38 with 8 warps; 700 rows in 12 parts 20.7 instead of 25.6.)
constexpr int kJoinWarps = 8, kJoinAhead = 4;
template <int DH, int WARPS>
__global__ void __launch_bounds__(32 * kJoinWarps) k_kv_join(const KvAttnArgs a)
{
    constexpr int kPer = DH / 32;
    __shared__ float sm_o[kJoinWarps][DH], sm_m[kJoinWarps], sm_l[kJoinWarps];
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t per = (int64_t)a.batch.rows * a.heads;  // (below 2^31)
    const int first = warp / WARPS * WARPS;               // of the row's warps
    const uint32_t own = blockIdx.x * (kJoinWarps / WARPS) + warp / WARPS, at = WARPS == kJoinWarps ? own : min(own, (uint32_t)per - 1u);
    const float2 *const ml = reinterpret_cast<const float2 *>(a.part + a.splits * per * DH) + at;
    float m = -kInf, l = 0.f, o[kPer] = {};
#pragma unroll 1
    for (int i0 = warp - first; i0 < a.splits; i0 += WARPS * kJoinAhead) {
        float2 p[kJoinAhead];
        float v[kJoinAhead][kPer];
#pragma unroll
        for (int k = 0; k < kJoinAhead; ++k) {
            const int i = i0 + k * WARPS;
            p[k] = make_float2(-kInf, 0.f);
            if (i < a.splits) p[k] = ml[i * per];
#pragma unroll
            for (int e = 0; e < kPer; ++e) v[k][e] = i < a.splits ? a.part[(i * per + at) * DH + lane + 32 * e] : 0.f;
        }
        float to = m;
#pragma unroll
        for (int k = 0; k < kJoinAhead; ++k) to = fmaxf(to, p[k].x);
        // (a NaN sum may have no reference of its own)
        const float half = half_factor(m, to), by = half * half;
        l = l * half * half;
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] *= by;
        m = to;
#pragma unroll
        for (int k = 0; k < kJoinAhead; ++k) {
            const float half_k = half_factor(p[k].x, to), f = half_k * half_k;
            l += p[k].y * half_k * half_k;
#pragma unroll
            for (int e = 0; e < kPer; ++e) o[e] = fmaf(v[k][e], f, o[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) sm_o[warp][lane + 32 * e] = o[e];
    if (lane == 0) sm_m[warp] = m, sm_l[warp] = l;
    // the row's sequence: the last that starts at or before it
    const int row = (int)(at / (uint32_t)a.heads), head = (int)(at % (uint32_t)a.heads);
    int lo = 0, hi = a.batch.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (a.batch.row_start[mid] <= row ? lo : hi) = mid;
    }
    auto holds = [&](int b) {
        const KvSeq s = kv_seq(a.batch, a.cache, b, nullptr);
        return s.n > 0 && row >= s.row0 && row < s.row0 + s.n;
    };
    bool mine = holds(lo);
    // (starts of broken sequences need not be in order: a row that was not found may be any sequence's, or none's)
    if (!mine)
        for (int b = lane; b < a.batch.batch && !mine; b += 32) mine = holds(b);
    mine = __any_sync(0xffffffffu, mine);
    griddep_launch();
    __syncthreads();
    if (own >= per || !mine) return;
    float top = sm_m[first];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) top = fmaxf(top, sm_m[first + w]);
    for (int d = threadIdx.x - 32 * first; d < DH; d += 32 * WARPS) {
        float total = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float half = half_factor(sm_m[first + w], top), f = half * half;
            total += sm_l[first + w] * half * half;
            sum = fmaf(sm_o[first + w][d], f, sum);
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;
        a.out[(int64_t)row * a.ldo + (int64_t)head * DH + d] = __float2bfloat16_rn(sum * inv);
        if (a.lse && d == 0) a.lse[at] = log_sum(top, total);
    }
}

template <int DH, int NT, bool CLUSTER>
cudaError_t launch_few(const KvAttnArgs &args, cudaStream_t s)
{
    KvAttnArgs a = args;
    a.row_blocks = (int)(((int64_t)a.batch.max_rows * a.group + 8 * NT - 1) / (8 * NT));
    const int64_t ctas = (int64_t)a.splits * a.row_blocks * a.cache.heads * a.batch.batch;
    if (ctas > INT32_MAX) return cudaErrorInvalidValue;
    static std::atomic<uint64_t> devices{0};
    cudaError_t e = ask_smem(k_kv_few<DH, NT, CLUSTER>, FewCfg<DH>::kSmem, devices);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(32 * kWarps);
    cfg.dynamicSmemBytes = FewCfg<DH>::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)a.splits;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = CLUSTER ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, k_kv_few<DH, NT, CLUSTER>, a);
    return e != cudaSuccess || CLUSTER || a.splits == 1 ? e : launch_kv_join(a, s);
}

template <int DH, bool CLUSTER>
cudaError_t launch_tile(const KvAttnArgs &a, cudaStream_t s)
{
    const int tile = kv_few_rows((int64_t)a.batch.max_rows * a.group, DH);
    return tile == 8 ? launch_few<DH, 1, CLUSTER>(a, s)
                     : (tile == 16 ? launch_few<DH, 2, CLUSTER>(a, s) : launch_few<DH, DH == 128 ? 2 : 4, CLUSTER>(a, s));
}

template <int DH>
cudaError_t launch_dh(const KvAttnArgs &a, cudaStream_t s)
{
    return a.cluster ? launch_tile<DH, true>(a, s) : launch_tile<DH, false>(a, s);
}

template <int DH>
cudaError_t launch_join(const KvAttnArgs &a, cudaStream_t s)
{
    const unsigned rows = (unsigned)(a.batch.rows * (int64_t)a.heads);
    const dim3 block(32 * kJoinWarps);
    return a.splits <= 16 ? launch_k(k_kv_join<DH, 1>, dim3((rows + kJoinWarps - 1) / kJoinWarps), block, 0, s, a)
                         : launch_k(k_kv_join<DH, kJoinWarps>, dim3(rows), block, 0, s, a);
}

}  // namespace

cudaError_t launch_kv_join(const KvAttnArgs &a, cudaStream_t s)
{
    if ((int64_t)a.batch.rows * a.heads > INT32_MAX) return cudaErrorInvalidValue;
    switch (a.cache.dh) {
    case 32: return launch_join<32>(a, s);
    case 64: return launch_join<64>(a, s);
    default: return launch_join<128>(a, s);
    }
}

cudaError_t launch_kv_few(const KvAttnArgs &a, cudaStream_t s)
{
    switch (a.cache.dh) {
    case 32: return launch_dh<32>(a, s);
    case 64: return launch_dh<64>(a, s);
    case 128: return launch_dh<128>(a, s);
    default: return cudaErrorInvalidValue;
    }
}

}  // namespace f3dc
