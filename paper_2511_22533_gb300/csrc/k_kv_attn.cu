// k_kv_attn.cu -- f3dc_kv_attention_fp8 for many query rows to a key head: attention over a
// paged 8-bit cache on 5th-generation tensor cores.
//
//   S = Q K^T, x = S scale 2^(ek) + ev, w = 2^(x - m + shift), O += w V, l += w 2^-ev
//
// A CTA (512 threads) takes 256 packed rows (query row, head of the group) of one sequence and key head:
// two tiles A and B of 128 rows that share their keys, whose score / softmax / product chains run side by side.
//   warps 0, 1   tcgen05.mma issuers of tile A and of tile B.  Per key tile g of 128 tokens: S_t(g) = Q_t K^T
//                (N = 128, K = dh), O_t += P_t V(g) (N = dh, K = 128; P read from TMEM)
//   warps 4-7    the cache's pages: each thread loads 16-byte pieces of keys and values (the next half of a
//                tile while it converts this one), converts e4m3 to fp16 (exactly) and writes them to shared memory in the
//                MMA's swizzled layout; scales of the tile's pages beside them
//   warps 8-11   softmax of tile A, warps 12-15 of tile B: one thread per row.  Before the first tile they convert
//                their queries (bf16 times a power of two of the row: exact in fp16) into shared memory.
// TMEM: S_A S_B (fp32, 128 columns each) | O_A O_B (dh each) | P_A P_B (fp16 pairs, 64 each); with dh 128 there
// is no room for P beside them, and it takes the place of S_t, whose next MMA then waits for P_t V.
// fp16 weights are what the 8-bit values allow: e4m3 is exact in fp16 but needs more instructions to become bf16, and
// fp16's rounding is 2^-11.  Their range (kv.cuh) needs the running maximum: it is taken for every tile.
// A NaN that some rows do not see: where a row of the CTA sees only a part of a tile, NaN values count as
// zeros in the MMA and the rows look them up at the end.
#include "kv.cuh"

namespace f3dc {

namespace {

constexpr int kThreads = 512;
constexpr float kInf = __builtin_huge_valf();
// Registers per thread after the split: the launch has 512 x 128.
constexpr int kIssueRegs = 48, kConvertRegs = 96, kSoftmaxRegs = 184;
static_assert(128 * (kIssueRegs + kConvertRegs) + 256 * kSoftmaxRegs <= 512 * 128, "register split above the launch's total");

// Scales of a tile's eight blocks of 16 tokens (a page has at least one).
struct TileScales {
    float key[8], value_log2[8], value_inverse[8];
};

template <int DH>
struct Cfg {
    static constexpr int kRowBytes = DH == 32 ? 64 : 128;  // of a region: 32 or 64 columns
    static constexpr int kRegions = DH == 128 ? 2 : 1;
    static constexpr int kRegion = 128 * kRowBytes, kTile = kRegions * kRegion;
    static constexpr uint32_t kAtom = 8 * kRowBytes, kSwz = DH == 32 ? kSwizzle64 : kSwizzle128;
    static constexpr int kStages = DH == 128 ? 2 : 3;
    static constexpr size_t kSmem = 1024 + (size_t)kTile * (2 + 2 * kStages) + (kStages + 1) * sizeof(TileScales) + 512;
    static constexpr bool kAlias = DH == 128;  // P in the place of S
    static constexpr uint32_t kColO = 256, kColP = kAlias ? 0 : 256 + 2 * DH, kStepP = kAlias ? 128 : 64;
    static_assert(kAlias || 256 + 2 * DH + 128 <= 512, "TMEM layout");
    // byte of 16-byte piece `piece` (8 columns) of a row
    static F3DC_DEV int place(int row, int piece)
    {
        if (DH == 32) return row * 64 + ((piece ^ (row >> 1 & 3)) << 4);
        return (piece >> 3) * kRegion + row * 128 + (((piece & 7) ^ (row & 7)) << 4);
    }
};

// kind::f16 with fp16 operands: fp32 accumulator (bits 4-5 = 1), types 0
__host__ __device__ constexpr uint32_t make_idesc_f16(int M, int N, int b_mn_major)
{
    return (1u << 4) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

F3DC_DEV bool wait_bounded(uint64_t *bar, uint32_t parity, uint64_t ns)
{
    const uint64_t t0 = globaltimer();
    while (!mbar_try_wait(bar, parity))
        if (globaltimer() - t0 > ns) return false;
    return true;
}

F3DC_DEV uint32_t half2_times(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <int DH>
__global__ void __launch_bounds__(kThreads, 1) k_kv_attn(const KvAttnArgs a)
{
    using C = Cfg<DH>;
    constexpr int kStages = C::kStages;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *const smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *const sQ = smem, *const sK = sQ + 2 * C::kTile, *const sV = sK + kStages * C::kTile;
    TileScales *const scales = reinterpret_cast<TileScales *>(sV + kStages * C::kTile);
    uint64_t *const bars = reinterpret_cast<uint64_t *>(scales + kStages + 1);
    // per stage: keys / values written by the four converting warps, and read by both tiles' MMAs
    uint64_t *const k_full = bars, *const v_full = k_full + kStages, *const k_empty = v_full + kStages,
                   *const v_empty = k_empty + kStages;
    // per query tile t, once: Q_t written; once per key tile: S_t written, S_t read, P_t written, P_t V done
    // per place of `scales`: written (its next writer is behind the softmax of the tile before)
    uint64_t *const c_full = v_empty + kStages;
    uint64_t *const q_full = c_full + kStages + 1, *const s_full = q_full + 2, *const s_free = s_full + 2,
                   *const p_full = s_free + 2, *const pv_done = p_full + 2, *const drain = pv_done + 2;
    uint32_t *const tmem_holder = reinterpret_cast<uint32_t *>(drain + 1);
    volatile int *const abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    volatile int *const nan_flag = abort_flag + 1;  // NaN values counted as zeros

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    griddep_launch();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&k_full[s], 4);
            mbar_init(&v_full[s], 4);
            mbar_init(&k_empty[s], 2);
            mbar_init(&v_empty[s], 2);
        }
        for (int s = 0; s <= kStages; ++s) mbar_init(&c_full[s], 1);
        for (int t = 0; t < 2; ++t) {
            mbar_init(&q_full[t], 4);
            mbar_init(&s_full[t], 1);
            mbar_init(&s_free[t], 4);
            mbar_init(&p_full[t], 4);
            mbar_init(&pv_done[t], 1);
        }
        mbar_init(drain, 2);
        *abort_flag = 0;
        *nan_flag = 0;
        fence_mbar_init();
    }
    griddep_wait();

    // ---- this CTA's item; the blocks of rows that see most come first
    int64_t item = blockIdx.x;
    const int split = (int)(item % a.splits);
    item /= a.splits;
    const int hk = (int)(item % a.cache.heads);
    item /= a.cache.heads;
    const int b = (int)(item % a.batch.batch), rb = a.row_blocks - 1 - (int)(item / a.batch.batch);
    const KvSeq s = kv_seq(a.batch, a.cache, b, a.err);
    const int64_t rows = (int64_t)s.n * a.group;  // packed
    const int64_t r0 = (int64_t)rb * 256;
    if (s.n <= 0 || r0 >= rows) return;  // (before anything that needs an end)
    const int left = (int)min(rows - r0, (int64_t)256), tiles = left > 128 ? 2 : 1;
    const int behind = s.length - s.n + 1;
    // tokens that the last and the first of the rows see
    const int most = a.causal ? max(0, behind + (int)((r0 + left - 1) / a.group)) : s.length;
    const int least = a.causal ? behind + (int)(r0 / a.group) : s.length;
    const int all = (most + 127) / 128;
    const int g_begin = (int)((int64_t)all * split / a.splits), g_end = (int)((int64_t)all * (split + 1) / a.splits);
    const int n_tiles = g_end - g_begin;
    const int page = a.cache.page, page_log2 = 31 - __clz(page);

    if (warp == 0) {
        tmem_alloc(tmem_holder, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_holder, 0);
    auto wait = [&](uint64_t *bar, uint32_t parity) { return warp_wait(bar, parity, abort_flag, a.err); };

    if (warp < 4) {
        reg_dec<kIssueRegs>();
        if (warp < tiles && n_tiles > 0) {
            // ------------------------------------------------ MMA issuer of one query tile
            constexpr uint32_t idesc_s = make_idesc_f16(128, 128, 0), idesc_o = make_idesc_f16(128, DH, 1);
            const int t = warp;
            const uint64_t q_desc = make_sdesc(smem_u32(sQ + t * C::kTile), 16, C::kAtom, C::kSwz);
            const uint64_t k_desc = make_sdesc(smem_u32(sK), 16, C::kAtom, C::kSwz);
            // values: the head's columns lie a region apart, eight tokens an atom
            const uint64_t v_desc = make_sdesc(smem_u32(sV), C::kRegion, C::kAtom, C::kSwz);
            constexpr uint64_t kStageStep = C::kTile >> 4, kRegionStep = C::kRegion >> 4, kVStep = (16 * C::kRowBytes) >> 4;
            auto scores = [&](int g) {
                const int st = g % kStages;
                if (!wait(&k_full[st], (g / kStages) & 1)) return false;
                if (g > 0 && !(C::kAlias ? wait(&pv_done[t], (g - 1) & 1) : wait(&s_free[t], (g - 1) & 1))) return false;
                tc_fence_after();
                const uint64_t kd = k_desc + st * kStageStep;
#pragma unroll
                for (int kk = 0; kk < DH / 16; ++kk) {
                    const uint64_t at = (kk / 4) * kRegionStep + 2 * (kk % 4);
                    mma_bf16_elect(tmem + t * 128, q_desc + at, kd + at, idesc_s, kk > 0);
                }
                mma_commit_elect(&s_full[t]);
                for (int i = tiles; i <= 2; ++i) mma_commit_elect(&k_empty[st]);  // (for the tile that there is not, too)
                return true;
            };
            auto product = [&](int g) {
                const int st = g % kStages;
                if (!wait(&v_full[st], (g / kStages) & 1)) return false;
                if (!wait(&p_full[t], g & 1)) return false;
                tc_fence_after();
                const uint64_t vd = v_desc + st * kStageStep;
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                    mma_bf16_ts_elect(tmem + C::kColO + t * DH, tmem + C::kColP + t * C::kStepP + kk * 8, vd + kk * kVStep, idesc_o,
                                      kk > 0 || g > 0);
                mma_commit_elect(&pv_done[t]);
                for (int i = tiles; i <= 2; ++i) mma_commit_elect(&v_empty[st]);
                return true;
            };
            if (wait(&q_full[t], 0)) {
#pragma unroll 1
                for (int g = 0; g < n_tiles; ++g) {
                    if (!scores(g)) break;
                    if (C::kAlias) {
                        if (!product(g)) break;
                    } else {
                        if (g > 0 && !product(g - 1)) break;
                        if (g + 1 == n_tiles && !product(g)) break;
                    }
                }
            }
        }
    } else if (warp < 8) {
        // ------------------------------------------------ pages to operands
        reg_dec<kConvertRegs>();
        constexpr int kPieces = DH / 16;  // 16-byte pieces of a token, and of a thread per half of a tile
        const int i = threadIdx.x - 128;
        // lane l < 8 looks after the tile's 16 tokens from 16 l: their page and its scale bytes
        int pg = -1, pg_next = -1;
        uint32_t bytes = 0, bytes_next = 0;
        auto look_up = [&](int g, int &p, uint32_t &sb) {
            const int t0 = (g_begin + g) * 128 + 16 * (lane & 7);
            p = -1;
            sb = 127u | 127u << 8;
            if (g < n_tiles && t0 < s.length) {
                p = kv_page(a.batch, a.cache, b, t0 >> page_log2, a.err);
                if (p >= 0) {
                    const int64_t at = (int64_t)p * a.cache.scale_stride + hk;
                    sb = a.cache.ks[at] | (uint32_t)a.cache.vs[at] << 8;
                }
            }
        };
        // piece k of a half of tile g
        auto fetch = [&](const uint8_t *pool, int g, int p, int k) {
            const int x = i + 128 * k, token = x / kPieces, piece = x % kPieces, t = (g_begin + g) * 128 + token;
            const int pp = __shfl_sync(0xffffffffu, p, token >> 4);
            uint4 u = make_uint4(0u, 0u, 0u, 0u);
            if (pp >= 0 && t < s.length)
                u = *reinterpret_cast<const uint4 *>(pool + (int64_t)pp * a.cache.page_stride +
                                                     ((int64_t)hk * page + (t & (page - 1))) * DH + 16 * piece);
            return u;
        };
        auto store = [&](uint8_t *tile, int k, const uint32_t (&h)[8]) {
            const int x = i + 128 * k, token = x / kPieces, piece = x % kPieces, swap = DH == 128 ? piece >> 2 : 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int f = e ^ swap;
                // (registers are picked by selects, not by an index)
                const uint4 w = f == 0 ? make_uint4(h[0], h[1], h[2], h[3]) : make_uint4(h[4], h[5], h[6], h[7]);
                *reinterpret_cast<uint4 *>(tile + C::place(token, 2 * piece + f)) = w;
            }
        };
        look_up(0, pg, bytes);
        uint4 u[kPieces];
#pragma unroll
        for (int k = 0; k < kPieces; ++k) u[k] = fetch(a.cache.k, 0, pg, k);
#pragma unroll 1
        for (int g = 0; g < n_tiles; ++g) {
            const int st = g % kStages;
            const uint32_t parity = (g / kStages) & 1;
            look_up(g + 1, pg_next, bytes_next);
            // keys
            if (!wait(&k_empty[st], parity ^ 1)) break;
            if (warp == 4) {
                const int at = g % (kStages + 1);
                if (lane < 8) {
                    const ValueScale v = value_scale(bytes >> 8);
                    scales[at].key[lane] = key_scale(bytes & 255u);
                    scales[at].value_log2[lane] = v.log2;
                    scales[at].value_inverse[lane] = v.inverse;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&c_full[at]);
            }
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                uint32_t h[8];
                const uint32_t w[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) e4m3x4_to_half2(w[e], h[2 * e], h[2 * e + 1]);
                store(sK + st * C::kTile, k, h);
                u[k] = fetch(a.cache.v, g, pg, k);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&k_full[st]);
            // values
            if (!wait(&v_empty[st], parity ^ 1)) break;
            const uint32_t times = value_scale(bytes >> 8).times;
            const bool partly = (g_begin + g + 1) * 128 > least;
            const bool odd = partly || __any_sync(0xffffffffu, times != kHalfOnes);
            uint32_t numbers = 0xffffffffu;
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                uint32_t h[8];
                const uint32_t w[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) e4m3x4_to_half2(w[e], h[2 * e], h[2 * e + 1]);
                if (odd) {
                    const uint32_t by = __shfl_sync(0xffffffffu, times, (i + 128 * k) / kPieces >> 4);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        h[e] = half2_times(h[e], by);
                        if (partly) {
                            const uint32_t m = __heq2_mask(*reinterpret_cast<const __half2 *>(&h[e]),
                                                           *reinterpret_cast<const __half2 *>(&h[e]));
                            numbers &= m;
                            h[e] &= m;
                        }
                    }
                }
                store(sV + st * C::kTile, k, h);
                u[k] = fetch(a.cache.k, g + 1, pg_next, k);
            }
            if (numbers != 0xffffffffu) *nan_flag = 1;
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&v_full[st]);
            pg = pg_next;
            bytes = bytes_next;
        }
        // every arrival of the MMAs' completion is in before the CTA leaves
#pragma unroll 1
        for (int g = max(0, n_tiles - kStages); g < n_tiles; ++g)
            if (!wait(&k_empty[g % kStages], (g / kStages) & 1) || !wait(&v_empty[g % kStages], (g / kStages) & 1)) break;
    } else {
        // ------------------------------------------------ softmax
        reg_inc<kSoftmaxRegs>();
        const int q = warp & 3, t = (warp - 8) >> 2, row = q * 32 + lane;
        const uint32_t tl = (uint32_t)(q * 32) << 16;
        const uint32_t s_addr = tmem + tl + t * 128, o_addr = tmem + tl + C::kColO + t * DH,
                       p_addr = tmem + tl + C::kColP + t * C::kStepP;
        if (t < tiles) {
            const int r = 128 * t + row;
            const bool real = r < left;
            const int token = (int)((r0 + min(r, left - 1)) / a.group), head = hk * a.group + (int)((r0 + min(r, left - 1)) % a.group);
            const int sees = a.causal ? behind + token : s.length;
            float factor;  // of S, in log2
            {
                const bf16 *x = a.q + (int64_t)(s.row0 + token) * a.ldq + (int64_t)head * DH;
                uint4 u[DH / 8];
#pragma unroll
                for (int c = 0; c < DH / 8; ++c) u[c] = reinterpret_cast<const uint4 *>(x)[c];
                float top = 0.f;
                auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
                auto hi = [](uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); };
#pragma unroll
                for (int c = 0; c < DH / 8; ++c) {
                    top = fmax3(top, fabsf(lo(u[c].x)), fabsf(hi(u[c].x)));
                    top = fmax3(top, fabsf(lo(u[c].y)), fabsf(hi(u[c].y)));
                    top = fmax3(top, fabsf(lo(u[c].z)), fabsf(hi(u[c].z)));
                    top = fmax3(top, fabsf(lo(u[c].w)), fabsf(hi(u[c].w)));
                }
                const int e = query_exponent(top);
                const float up = pow2(e);
                factor = a.scale_log2 * pow2(-e);
#pragma unroll
                for (int c = 0; c < DH / 8; ++c) {
                    uint4 w;
                    w.x = pack_half2(lo(u[c].x) * up, hi(u[c].x) * up);
                    w.y = pack_half2(lo(u[c].y) * up, hi(u[c].y) * up);
                    w.z = pack_half2(lo(u[c].z) * up, hi(u[c].z) * up);
                    w.w = pack_half2(lo(u[c].w) * up, hi(u[c].w) * up);
                    *reinterpret_cast<uint4 *>(sQ + t * C::kTile + C::place(row, c)) = w;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&q_full[t]);
            }

            float m_ref = -kInf, l_run = 0.f;
            // Key tile g.  PARTLY: some row of the warp may not see all of it.
            auto tile = [&](int g, auto partly_tag) {
                constexpr bool kPartly = decltype(partly_tag)::value;
                if (!wait(&c_full[g % (kStages + 1)], (g / (kStages + 1)) & 1)) return false;
                if (!wait(&s_full[t], g & 1)) return false;
                tc_fence_after();
                float sv[128];
                {
                    uint32_t w[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + 32 * c, w[c]);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 128; ++c) sv[c] = __uint_as_float(w[c / 32][c % 32]);
                }
                if (!C::kAlias) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&s_free[t]);
                }
                const TileScales &sc = scales[g % (kStages + 1)];
                const int valid = sees - (g_begin + g) * 128;  // tokens of the tile that the row sees
                float mx = -kInf;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (kPartly) {
#pragma unroll
                        for (int c = 16 * k; c < 16 * k + 16; ++c)
                            if (c >= valid) sv[c] = -kInf;
                    }
                    float top = fmax3(sv[16 * k], sv[16 * k + 1], sv[16 * k + 2]);
#pragma unroll
                    for (int c = 16 * k + 3; c < 16 * k + 15; c += 2) top = fmax3(top, sv[c], sv[c + 1]);
                    top = fmaxf(top, sv[16 * k + 15]);
                    const float x = fmaf(top, factor * sc.key[k], sc.value_log2[k]);
                    mx = fmaxf(mx, kPartly && top == -kInf ? -kInf : x);
                }
                if (!C::kAlias && g > 0) {
                    if (!wait(&pv_done[t], (g - 1) & 1)) return false;  // P_t and O_t are free
                    tc_fence_after();
                }
                if (__any_sync(0xffffffffu, mx > m_ref + kLazy)) {
                    const float to = fmaxf(m_ref, mx);
                    const float by = m_ref == -kInf ? 0.f : exp2_fast(m_ref - to);
                    m_ref = to;
                    l_run *= by;
                    if (g > 0) {
#pragma unroll 1
                        for (int d = 0; d < DH; d += 16) {
                            uint32_t w[16];
                            tmem_ld16(o_addr + d, w);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * by);
                            tmem_st16(o_addr + d, w);
                        }
                    }
                }
                const float base = kWeightShift - (m_ref == -kInf ? 0.f : m_ref);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t pw[32];
#pragma unroll
                    for (int k = 4 * h; k < 4 * h + 4; ++k) {
                        const float f = factor * sc.key[k], at = base + sc.value_log2[k];
                        const f32x2 f2 = {f, f}, at2 = {at, at};
                        f32x2 s0 = {0.f, 0.f}, s1 = {0.f, 0.f};
#pragma unroll
                        for (int c = 16 * k; c < 16 * k + 16; c += 4) {
                            const f32x2 x0 = ffma2({sv[c], sv[c + 1]}, f2, at2), x1 = ffma2({sv[c + 2], sv[c + 3]}, f2, at2);
                            f32x2 e0 = {exp2_fast(x0.x), exp2_fast(x0.y)}, e1 = {exp2_fast(x1.x), exp2_fast(x1.y)};
                            if (kPartly) {
                                if (c >= valid) e0.x = 0.f;
                                if (c + 1 >= valid) e0.y = 0.f;
                                if (c + 2 >= valid) e1.x = 0.f;
                                if (c + 3 >= valid) e1.y = 0.f;
                            }
                            s0 = fadd2(s0, e0);
                            s1 = fadd2(s1, e1);
                            pw[c / 2 - 32 * h] = pack_half2(e0.x, e0.y);
                            pw[c / 2 + 1 - 32 * h] = pack_half2(e1.x, e1.y);
                        }
                        l_run = fmaf((s0.x + s0.y) + (s1.x + s1.y), sc.value_inverse[k], l_run);
                    }
                    tmem_st32(p_addr + 32 * h, pw);
                }
                tmem_wait_st();
                tc_fence_before();  // P (and a rescaled O) written before P V may start
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[t]);
                return true;
            };
            const int whole = max(0, min(n_tiles, least / 128 - g_begin));  // tiles that every row sees
            bool ok = true;
            int g = 0;
#pragma unroll 1
            for (; ok && g < whole; ++g) ok = tile(g, std::false_type());
#pragma unroll 1
            for (; ok && g < n_tiles; ++g) ok = tile(g, std::true_type());
            if (ok && n_tiles > 0) {
                // (v_full: nan_flag is what the converting warps left)
                ok = wait(&pv_done[t], (n_tiles - 1) & 1) && wait(&v_full[(n_tiles - 1) % kStages], ((n_tiles - 1) / kStages) & 1);
                tc_fence_after();
            }
            if (ok) {
                const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
                const int64_t at = (int64_t)(s.row0 + token) * a.heads + head;
                const bool rare = *nan_flag != 0;
#pragma unroll 1
                for (int d0 = 0; d0 < DH; d0 += 32) {
                    float o[32];
                    if (n_tiles > 0) {
                        uint32_t w[32];
                        tmem_ld32(o_addr + d0, w);
                        tmem_wait_ld();
#pragma unroll
                        for (int d = 0; d < 32; ++d) o[d] = __uint_as_float(w[d]);
                    } else {
#pragma unroll
                        for (int d = 0; d < 32; ++d) o[d] = 0.f;
                    }
                    if (rare && real) {
                        // NaN values of the tiles that are seen in part
                        const int stop = min(sees, g_end * 128);
#pragma unroll 1
                        for (int x = (g_begin + whole) * 128; x < stop; ++x) {
                            const int p = kv_page(a.batch, a.cache, b, x >> page_log2, a.err);
                            if (p < 0) continue;
                            const uint8_t *v = a.cache.v + (int64_t)p * a.cache.page_stride +
                                               ((int64_t)hk * page + (x & (page - 1))) * DH + d0;
                            const bool scale = a.cache.vs[(int64_t)p * a.cache.scale_stride + hk] == 255;
#pragma unroll
                            for (int d = 0; d < 32; ++d)
                                if (scale || (v[d] & 0x7F) == 0x7F) o[d] = __int_as_float(0x7FC00000);
                        }
                    }
                    if (!real) continue;
                    if (a.splits == 1) {
                        uint4 *dst = reinterpret_cast<uint4 *>(a.out + (int64_t)(s.row0 + token) * a.ldo + (int64_t)head * DH + d0);
#pragma unroll
                        for (int d = 0; d < 32; d += 8) {
                            uint4 w;
                            w.x = pack_bf16x2(o[d] * inv, o[d + 1] * inv);
                            w.y = pack_bf16x2(o[d + 2] * inv, o[d + 3] * inv);
                            w.z = pack_bf16x2(o[d + 4] * inv, o[d + 5] * inv);
                            w.w = pack_bf16x2(o[d + 6] * inv, o[d + 7] * inv);
                            dst[d / 8] = w;
                        }
                    } else {
                        float4 *dst = reinterpret_cast<float4 *>(a.part + ((int64_t)split * a.batch.rows * a.heads + at) * DH + d0);
#pragma unroll
                        for (int d = 0; d < 32; d += 4) dst[d / 4] = make_float4(o[d], o[d + 1], o[d + 2], o[d + 3]);
                    }
                }
                if (real) {
                    if (a.splits == 1) {
                        if (a.lse) a.lse[at] = log_sum(m_ref, l_run);
                    } else {
                        float2 *ml = reinterpret_cast<float2 *>(a.part + (int64_t)a.splits * a.batch.rows * a.heads * DH);
                        ml[(int64_t)split * a.batch.rows * a.heads + at] = make_float2(m_ref, l_run);
                    }
                }
                tc_fence_before();
            }
        }
    }
    __syncthreads();
    if (*abort_flag) {
        if (warp < 2) {
            mma_commit_elect(drain);  // the MMAs' issuing lane
            if (lane == 0) wait_bounded(drain, 0, 100000000ull);
        }
        __syncthreads();
    }
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <int DH>
cudaError_t launch_dh(const KvAttnArgs &args, cudaStream_t s)
{
    KvAttnArgs a = args;
    a.row_blocks = (int)(((int64_t)a.batch.max_rows * a.group + 255) / 256);
    const int64_t ctas = (int64_t)a.splits * a.row_blocks * a.cache.heads * a.batch.batch;
    if (ctas > INT32_MAX) return cudaErrorInvalidValue;
    static std::atomic<uint64_t> devices{0};
    cudaError_t e = ask_smem(k_kv_attn<DH>, (int)Cfg<DH>::kSmem, devices);
    if (e != cudaSuccess) return e;
    e = launch_k(k_kv_attn<DH>, dim3((unsigned)ctas), dim3(kThreads), Cfg<DH>::kSmem, s, a);
    return e != cudaSuccess || a.splits == 1 ? e : launch_kv_join(a, s);
}

}  // namespace

cudaError_t launch_kv_attn(const KvAttnArgs &a, cudaStream_t s)
{
    switch (a.cache.dh) {
    case 32: return launch_dh<32>(a, s);
    case 64: return launch_dh<64>(a, s);
    case 128: return launch_dh<128>(a, s);
    default: return cudaErrorInvalidValue;
    }
}

}  // namespace f3dc
