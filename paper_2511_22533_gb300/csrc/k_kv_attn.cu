// k_kv_attn.cu -- f3dc_kv_attention_fp8 for many query rows to a key head: attention over a
// paged 8-bit cache on 5th-generation tensor cores.
//
//   S = Q K^T, x = S scale 2^(ek) + ev, w = 2^(x - r), O += w V, l += w 2^-ev, out = O / l
//
// A CTA (512 threads) takes 256 packed rows (query row, head of the group) of one sequence and key head: two tiles
// A and B of 128 rows that share their keys, whose score / softmax / product chains run side by side, in steps of 64
// tokens (half of a tile of keys and values).
//   warps 0, 1   tcgen05.mma issuers of tile A and of tile B.  Step j: S_t(j) = Q_t K^T (N = 64, K = dh), O_t += P_t V(j)
//                (N = dh, K = 64; P read from TMEM).  S is two steps ahead, in the place of the P that has been used
//   warp 2       walks the page table, four tiles at a time: where each 16 tokens of a tile lie, and their scales
//   warps 4-7    the cache's pages: each thread loads 16-byte pieces of keys and values (those of the next tile
//                while it converts this one's), converts e4m3 to fp16 (exactly) and writes them to shared memory in the
//                MMA's swizzled layout
//   warps 8-11   softmax of tile A, warps 12-15 of tile B: one thread per row.  Before the first step they bring their queries
//                in (bf16 times a power of two of the row: exact in fp16)
// TMEM: two places of 64 columns each for S and P of A, then of B | O_A O_B (dh each) | Q_A Q_B (dh / 2 each, up to
// dh 64: with dh 128 the queries stay in shared memory).
// fp16 weights are what the 8-bit values allow: e4m3 is exact in fp16 but needs more instructions to become bf16, and
// fp16's rounding is 2^-11.  Their range is looked after by the sum of a step's weights, which is taken anyway.
// A NaN that some rows do not see: where a row of the CTA sees only a part of a tile, NaN values count as
// zeros in the MMA and the rows look them up at the end.
// What bounds it: a softmax warp's own latencies.  A step of 64 tokens takes it some 1300 clocks, of which the
// exponents are 260 (alone) to 520 (both tiles' warps at once): waits, tensor-memory loads and stores, votes and the
// fetch of instructions are the rest, and tensor memory has no room for more tiles with dh 128 (with dh 64, four tiles of
// one place each measured 7 % slower).  That is this loop's and no floor: k_attn.cu takes 1950 clocks for the scores and exponents of two
// steps.  With dh 128 shared memory comes next: operands read and written take 2500 of some
// 3000 clocks a pair of tiles.  32768 x 32768, 16 heads of 64: 4.94 ms = 890 TFLOP/s; causal 8192 x 8192, 32 heads of
// 128 to 8: 508 us = 1081 TFLOP/s; 1229 x 1374, 16 heads of 64: 29 us, of which 8 before the first and behind the last step.
// (dh 128: two or three registers of a thread are spilled, 8 to 12 bytes.)
// Steps that led here, prompt of 8192 / 32768 x 32768: one step of 128 tokens, its maximum always taken 872 us / 6.8 ms; no
// maximum, pages looked up by a warp of their own, steps of 64 in two places 505 / 5.24 (steps of 128 held in registers 567); queries
// in TMEM and two steps without a jump between them 502 / 4.98.  Three places of S made no difference and leave no room for the
// queries.
#include "kv.cuh"

namespace f3dc {

namespace {

constexpr int kThreads = 512;
constexpr float kInf = __builtin_huge_valf();
// Registers per thread at the launch and after the split.
constexpr int kLaunchRegs = 128;
constexpr int kIssueRegs = 40, kConvertRegs = 104, kSoftmaxRegs = 184;
static_assert(128 * (kIssueRegs + kConvertRegs) + 256 * kSoftmaxRegs <= 512 * kLaunchRegs, "register split above the launch's total");

// A row's largest weight is 2^kTop where its reference was taken.  The sum of a step's weights, which is taken
// anyway, says whether one may have left fp16's range; only then is the reference looked at again, by all rows of the warp.  64
// weights of 2^kTop are 2^9, far below kMostSum, so rows of even weights do not ask.  fp16 holds 2^-17 of a row's
// largest weight at full precision and 2^-28 at all, but 2^-14 and 2^-25 where the reference was raised by the sum of 64 weights and the
// largest may be 2^0.  A higher kTop holds more and asks more often: prompt of 8192 / 32768 x
// 32768 with keys and queries of a few large channels 502 us / 4.99 ms, with 2^6 540 / 5.10, with 2^8 576 / 5.24.
constexpr float kTop = 3.f, kMostSum = 60000.f;

// What the page table says about a tile: of each of its eight runs of 16 tokens where it starts in the pool (in 16
// bytes; inside the pool always, page 0 standing for what is not there), how many tokens there are, and what its values are multiplied by;
// and the scales of its NB blocks of 128 / NB tokens (a page has at least one).
template <int NB>
struct StepScales {  // of half a tile
    // (Where a value scale is more than kScaleSpan below the largest so far, value_log2 is infinity: the sum of a plain step then sends it
    // to the careful form, which has the scales from value_inverse.)
    float key[NB / 2], value_log2[NB / 2], value_inverse[NB / 2];
};
template <int NB>
struct TileInfo {
    uint32_t at[8], times[8];
    int32_t there[8];
    StepScales<NB> scales[2];
    int32_t complete, plain;  // every run has 16 tokens; values are multiplied by 1
};
constexpr int kGroup = 4, kGroups = 4;  // tiles looked up at once, and groups of them in shared memory
constexpr int kGroupSteps = 2 * kGroup;

template <int DH, int NB>
struct Cfg {
    static constexpr int kRowBytes = DH == 32 ? 64 : 128;  // of a region: 32 or 64 columns
    static constexpr int kRegions = DH == 128 ? 2 : 1;
    static constexpr int kRegion = 128 * kRowBytes, kTile = kRegions * kRegion;
    static constexpr uint32_t kAtom = 8 * kRowBytes, kSwz = DH == 32 ? kSwizzle64 : kSwizzle128;
    static constexpr int kStages = DH == 128 ? 2 : 4;
    static constexpr int kPlaces = 2;  // of S and P of a query tile, 64 columns each
    // Queries in TMEM, where there is room: an S MMA of 64 columns reads twice as many bytes of queries from shared memory as of keys
    // and takes 48 clocks instead of 32.
    static constexpr bool kQTmem = DH < 128;
    static constexpr uint32_t kColQ = 2 * 64 * kPlaces + 2 * DH;
    static constexpr size_t kSmem = 1024 + (size_t)kTile * (2 + 2 * kStages) + kGroups * kGroup * sizeof(TileInfo<NB>) + 256 * sizeof(float2) + 576;
    static constexpr uint32_t kColO = 2 * 64 * kPlaces;
    static_assert(kColO + 2 * DH + (kQTmem ? DH : 0) <= 512, "TMEM layout");
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

// mbarrier operations on a shared-memory address that is at hand
F3DC_DEV bool mbar_test_addr(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity)
                 : "memory");
    return ok != 0;
}
F3DC_DEV bool warp_wait_addr(uint32_t bar, uint32_t parity, volatile int *abort, uint32_t *err)
{
    if (warp_all(mbar_test_addr(bar, parity))) return true;
    return warp_wait(reinterpret_cast<uint64_t *>(__cvta_shared_to_generic(bar)), parity, abort, err);
}
// an arrival by the lanes that say so, without a branch
F3DC_DEV void mbar_arrive_if(uint32_t bar, bool me)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %1, 0;\n @p mbarrier.arrive.shared::cta.b64 _, [%0];\n}\n" ::"r"(bar),
                 "r"((uint32_t)me)
                 : "memory");
}

F3DC_DEV bool wait_bounded(uint64_t *bar, uint32_t parity, uint64_t ns)
{
    const uint64_t t0 = globaltimer();
    while (!mbar_try_wait(bar, parity))
        if (globaltimer() - t0 > ns) return false;
    return true;
}

template <int DH, int NB>
__global__ void __launch_bounds__(kThreads, 1) k_kv_attn(const KvAttnArgs a)
{
    using C = Cfg<DH, NB>;
    constexpr int kStages = C::kStages;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *const smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *const sQ = smem, *const sK = sQ + 2 * C::kTile, *const sV = sK + kStages * C::kTile;
    uint64_t *const bars = reinterpret_cast<uint64_t *>(sV + kStages * C::kTile);
    TileInfo<NB> *const infos = reinterpret_cast<TileInfo<NB> *>(bars + 72);
    // per stage: keys / values written by the four converting warps, and read by both tiles' MMAs
    uint64_t *const k_full = bars, *const v_full = k_full + kStages, *const k_empty = v_full + kStages,
                   *const v_empty = k_empty + kStages;
    // per query tile t, once: Q_t written; per step, in turn for the places: S_t written, P_t written, P_t V done
    // per group of infos: written, read by the converting and the softmax warps
    uint64_t *const i_full = v_empty + kStages, *const i_empty = i_full + kGroups;
    uint64_t *const q_full = i_empty + kGroups, *const s_full = q_full + 2, *const p_full = s_full + 2 * C::kPlaces,
                   *const pv_done = p_full + 2 * C::kPlaces, *const drain = pv_done + 2 * C::kPlaces;
    uint32_t *const tmem_holder = reinterpret_cast<uint32_t *>(drain + 1);
    volatile int *const abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    volatile int *const nan_flag = abort_flag + 1;  // NaN values counted as zeros

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    griddep_launch();
    if (warp == 0) {
        tmem_alloc(tmem_holder, 512);
        tmem_relinquish();
    }
    griddep_wait();

    // ---- this CTA's item; the blocks of rows that see most come first
    uint32_t item = blockIdx.x;
    const int split = (int)(item % (uint32_t)a.splits);
    item /= (uint32_t)a.splits;
    const int hk = (int)(item % (uint32_t)a.cache.heads);
    item /= (uint32_t)a.cache.heads;
    const int b = (int)(item % (uint32_t)a.batch.batch), rb = a.row_blocks - 1 - (int)(item / (uint32_t)a.batch.batch);
    const KvSeq s = kv_seq(a.batch, a.cache, b, a.err);
    const int rows = s.n * a.group, r0 = rb * 256;  // packed
    if (s.n <= 0 || r0 >= rows) {
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (warp == 0) tmem_dealloc(*tmem_holder, 512);
        return;
    }
    const int left = min(rows - r0, 256), tiles = left > 128 ? 2 : 1;
    const int behind = s.length - s.n + 1;
    // tokens that the last and the first of the rows see
    const int most = a.causal ? max(0, behind + (r0 + left - 1) / a.group) : s.length;
    const int least = a.causal ? behind + r0 / a.group : s.length;
    const int all = (most + 127) / 128;
    const int g_begin = kv_share(all, split, a.splits), g_end = kv_share(all, split + 1, a.splits);
    const int n_tiles = g_end - g_begin;
    // steps of 64 tokens: two to a tile, of the last one perhaps none sees the second
    const int n_steps = max(0, min(2 * n_tiles, (most + 63) / 64 - 2 * g_begin));
    const int page = a.cache.page, page_log2 = 31 - __clz(page);

    if (warp == 1) {
        // arrivals of each barrier, in the order in which they lie
        constexpr int kEmpty = 2 * kStages, kInfo = 4 * kStages, kQ = kInfo + 2 * kGroups, kS = kQ + 2, kP = kS + 2 * C::kPlaces,
                      kDone = kP + 2 * C::kPlaces, kAll = kDone + 2 * C::kPlaces + 1;
        static_assert(kAll <= 64, "room for barriers");
        for (int i = lane; i < kAll; i += 32)
            mbar_init(&bars[i], i < kEmpty ? 4 : (i < kInfo ? tiles : (i < kInfo + kGroups ? 1 : (i < kQ ? 4 + 4 * tiles : (i < kS ? 4 :
                                (i < kP ? 1 : (i < kDone ? 4 : (i < kAll - 1 ? 1 : 2))))))));
        if (lane == 0) {
            *abort_flag = 0;
            *nan_flag = 0;
        }
        fence_mbar_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_holder, 0);
    auto wait = [&](uint64_t *bar, uint32_t parity) { return warp_wait(bar, parity, abort_flag, a.err); };

    // (The softmax warps' code stands first: with the others' before it 4096 x 4096 of heads of 64 118.6 us instead of 116.4,
    // 32768 x 32768 5.02 ms instead of 4.94, with heads of 128 143 to 145 us either way.)
    if (warp >= 8) {
        // ------------------------------------------------ softmax
        reg_inc<kSoftmaxRegs>();
        const int q = warp & 3, t = (warp - 8) >> 2, row = q * 32 + lane;
        const uint32_t tl = (uint32_t)(q * 32) << 16;
        const uint32_t s_addr0 = tmem + tl + t * 64 * C::kPlaces, o_addr = tmem + tl + C::kColO + t * DH;
        if (t < tiles) {
            const int r = 128 * t + row;
            const bool real = r < left;
            const int token = (r0 + min(r, left - 1)) / a.group, head = hk * a.group + (r0 + min(r, left - 1)) % a.group;
            const int sees = a.causal ? behind + token : s.length;
            // The warp's 32 rows pass through its own rows of Q_t on the way in and out: kLanes lanes take a row's 16-byte
            // pieces side by side.  (A thread that reads or writes its own row in global memory touches a line for each lane: for
            // dh 128 that took 5000 clocks more in and 4000 out.)
            constexpr int kLanes = DH / 8, kOnce = 32 / kLanes;
            const int piece = lane % kLanes;
            uint8_t *const own_q = sQ + t * C::kTile;
            const int64_t q_at = (int64_t)(s.row0 + token) * a.ldq + (int64_t)head * DH;
            // (Loops here and at the end are kept short: what a CTA runs once costs it the fetch of its instructions.)
#pragma unroll 4
            for (int i = 0; i < kLanes; ++i) {
                const int line = i * kOnce + lane / kLanes;
                const int64_t at = __shfl_sync(0xffffffffu, q_at, line);
                cp_async16(smem_u32(own_q + C::place(32 * q + line, piece)), a.q + at + 8 * piece);
            }
            cp_async_wait_all();
            __syncwarp();
            float factor;  // of S, in log2
            {
                uint32_t tops = 0;
#pragma unroll 4
                for (int c = 0; c < DH / 8; ++c) {
                    const uint4 u = *reinterpret_cast<const uint4 *>(own_q + C::place(row, c));
                    // (magnitudes of bf16 order as their bits do)
                    tops = __vmaxu2(tops, __vmaxu2(__vmaxu2(u.x & 0x7FFF7FFFu, u.y & 0x7FFF7FFFu),
                                                   __vmaxu2(u.z & 0x7FFF7FFFu, u.w & 0x7FFF7FFFu)));
                }
                const int e = query_exponent(__uint_as_float(max(tops & 0xFFFFu, tops >> 16) << 16));
                const float up = pow2(e);
                factor = a.scale_log2 * pow2(-e);
                auto half2 = [&](uint32_t w) { return pack_half2(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xFFFF0000u) * up); };
#pragma unroll 1
                for (int c0 = 0; c0 < DH / 8; c0 += 4) {
                    uint4 u[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) u[c] = *reinterpret_cast<const uint4 *>(own_q + C::place(row, c0 + c));
#pragma unroll
                    for (int c = 0; c < 4; ++c) u[c] = make_uint4(half2(u[c].x), half2(u[c].y), half2(u[c].z), half2(u[c].w));
                    if constexpr (C::kQTmem) {
                        const uint32_t w[16] = {u[0].x, u[0].y, u[0].z, u[0].w, u[1].x, u[1].y, u[1].z, u[1].w,
                                                u[2].x, u[2].y, u[2].z, u[2].w, u[3].x, u[3].y, u[3].z, u[3].w};
                        tmem_st16(tmem + tl + C::kColQ + t * (DH / 2) + 4 * c0, w);
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c) *reinterpret_cast<uint4 *>(own_q + C::place(row, c0 + c)) = u[c];
                    }
                }
                if constexpr (C::kQTmem) {
                    tmem_wait_st();
                    tc_fence_before();
                } else {
                    fence_proxy_async_smem();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&q_full[t]);
            }

            float ref = -kInf, l_run = 0.f;
            float peak = 0.f;  // largest sum of a step's weights against the reference
            constexpr int kBlock = 128 / NB, kBlocks = 64 / kBlock;  // of a step
            // Weights of a step's scores (of its first `valid` tokens) against the reference, as pairs; adds their sum without value
            // scales to l, returns the one with them.
            auto weights = [&](const StepScales<NB> &x, const uint32_t (&sc)[64], int valid, float &l, uint32_t (&pw)[32], auto partly_tag) {
                constexpr bool kPartly = decltype(partly_tag)::value;
                const float base = ref == -kInf ? 0.f : -ref;
                float total = 0.f;
#pragma unroll
                for (int k = 0; k < kBlocks; ++k) {
                    const float f = factor * x.key[k], at = base + x.value_log2[k];
                    const f32x2 f2 = {f, f}, at2 = {at, at};
                    f32x2 s0 = {0.f, 0.f}, s1 = {0.f, 0.f};
#pragma unroll
                    for (int c = k * kBlock; c < (k + 1) * kBlock; c += 4) {
                        const f32x2 x0 = ffma2({__uint_as_float(sc[c]), __uint_as_float(sc[c + 1])}, f2, at2);
                        const f32x2 x1 = ffma2({__uint_as_float(sc[c + 2]), __uint_as_float(sc[c + 3])}, f2, at2);
                        f32x2 e0 = {exp2_fast(x0.x), exp2_fast(x0.y)}, e1 = {exp2_fast(x1.x), exp2_fast(x1.y)};
                        if (kPartly) {
                            if (c >= valid) e0.x = 0.f;
                            if (c + 1 >= valid) e0.y = 0.f;
                            if (c + 2 >= valid) e1.x = 0.f;
                            if (c + 3 >= valid) e1.y = 0.f;
                        }
                        s0 = fadd2(s0, e0);
                        s1 = fadd2(s1, e1);
                        pw[c / 2] = pack_half2(e0.x, e0.y);
                        pw[c / 2 + 1] = pack_half2(e1.x, e1.y);
                    }
                    const float sum = (s0.x + s0.y) + (s1.x + s1.y);
                    l = fmaf(sum, x.value_inverse[k], l);
                    total += sum;
                }
                return total;
            };
            const uint32_t s_bars = smem_u32(s_full + C::kPlaces * t), p_bars = smem_u32(p_full + C::kPlaces * t);
            auto product_done = [&](int j) {  // P V of step j
                return wait(&pv_done[C::kPlaces * t + j % C::kPlaces], (j / C::kPlaces) & 1);
            };
            StepScales<NB> x = {};  // of the step
            bool early = false;  // its S_t is known to be written
            // Step j, in place i (phase `phase`) of S and P.  Careful: with its maximum (of the tokens that the row sees): the first step,
            // those seen in part, and those whose weights ran away from the reference or whose value scales lie far apart; O_t and l
            // are rescaled where it is taken anew.  Plain ones take the reference as it stands; where the sum of weights says that one may have left its
            // range they return 0, and the step is done again, carefully (1: done, -1: the kernel is aborting).  What the next step
            // begins with (whether its S_t is written, its scales) is asked for under this one's exponents: a warp's own
            // latencies are what bounds it.
            auto step = [&](int j, int i, uint32_t phase, const StepScales<NB> &next, auto careful_tag) {
                constexpr bool kCareful = decltype(careful_tag)::value;
                if (__builtin_expect(!early && !warp_wait_addr(s_bars + 8 * i, phase, abort_flag, a.err), 0)) return -1;
                tc_fence_after();
                const uint32_t cols = s_addr0 + 64 * i;
                uint32_t sc[64], pw[32];
                tmem_ld32(cols, reinterpret_cast<uint32_t (&)[32]>(sc));
                tmem_ld32(cols + 32, reinterpret_cast<uint32_t (&)[32]>(sc[32]));
                const bool last = i + 1 == C::kPlaces;
                const bool ready = mbar_test_addr(s_bars + (last ? 0 : 8 * i + 8), last ? phase ^ 1 : phase);
                const StepScales<NB> now = x;
                x = next;
                tmem_wait_ld();
                float l = l_run;
                if (!kCareful) {
                    const float total = weights(now, sc, 64, l, pw, std::false_type());
                    if (__builtin_expect(__any_sync(0xffffffffu, total > kMostSum), 0)) {
                        x = now;
                        early = true;
                        return 0;
                    }
                    peak = fmaxf(peak, total);
                } else {
                    const int valid = sees - (2 * g_begin + j) * 64;
                    float mx = -kInf;
#pragma unroll
                    for (int k = 0; k < kBlocks; ++k) {
                        float most = -kInf;
#pragma unroll
                        for (int c = k * kBlock; c < (k + 1) * kBlock; c += 2)
                            most = fmax3(most, c < valid ? __uint_as_float(sc[c]) : -kInf, c + 1 < valid ? __uint_as_float(sc[c + 1]) : -kInf);
                        const float y = fmaf(most, factor * now.key[k], now.value_log2[k]);
                        mx = fmaxf(mx, most == -kInf ? -kInf : y);
                    }
                    if (__any_sync(0xffffffffu, mx > ref + (kTop + 1.f))) {
                        // (all rows of the warp, by what they have seen: the next one will be long in coming)
                        const float seen = fmaxf(ref, ref + __log2f(peak) - (kTop + 3.f));
                        const float to = fmaxf(seen, mx - kTop);
                        const float half = half_factor(ref, to), by = half * half;
                        ref = to;
                        l_run = l_run * half * half;
                        peak *= by;
                        if (j > 0) {
                            if (!product_done(j - 1)) return -1;
                            tc_fence_after();
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
                    l = l_run;
                    weights(now, sc, valid, l, pw, std::true_type());
                }
                l_run = l;
                tmem_st32(cols, pw);
                early = warp_all(ready);
                tmem_wait_st();
                tc_fence_before();  // P (and a rescaled O) written before P V may start
                __syncwarp();
                mbar_arrive_if(p_bars + 8 * i, lane == 0);
                return 1;
            };
            const int whole = max(0, min(n_steps, least / 64 - 2 * g_begin));  // steps that every row sees
            // Two plain steps stand one after another in the code: a jump back costs a warp some 200 clocks, as the instructions of the others
            // have taken the place of its own.  (All eight of a group were 10 % faster while the warps ran through them together and
            // 40 % slower with warps that had left the others' pace by a careful step.)
            bool ok = true, again = true;
            int j = 0;
            // Steps with value scales far apart: the sum of their weights without value scales, (largest score, sum against it) of the
            // row, which has taken in step `summed`; the careful form adds nothing for them.  What finds it stands behind the loop and in
            // shared memory: between the other steps' code or in their registers it costs all of them 4 to 7 %.
            float2 *const apart = reinterpret_cast<float2 *>(infos + kGroups * kGroup) + (threadIdx.x - 256);
            int summed = -1;
#pragma unroll 1
            while (true) {
#pragma unroll 1
                while (ok && j < n_steps) {
                    const int group = j / kGroupSteps % kGroups, u = j % kGroupSteps;
                    if (u == 0 && !(ok = wait(&i_full[group], (j / (kGroupSteps * kGroups)) & 1))) break;
                    const uint32_t phase = (j / C::kPlaces) & 1;
                    const StepScales<NB> *const own = infos[(j >> 1) % (kGroup * kGroups)].scales;
                    x = own[j & 1];
                    int r;
                    if (again || j >= whole) {
                        if (x.value_log2[0] == kInf) {
                            if (summed < j) break;
#pragma unroll
                            for (int k = 0; k < kBlocks; ++k) {
                                x.value_log2[k] = 127.f - (float)(__float_as_uint(x.value_inverse[k]) >> 23);
                                x.value_inverse[k] = 0.f;
                            }
                        }
                        r = step(j, j % C::kPlaces, phase, x, std::true_type());
                        if (r == 1) ++j;
                    } else {
                        static_assert(C::kPlaces == 2, "an even step is in the first place");
                        r = 1;
                        if ((j & 1) == 0) {
                            r = step(j, 0, phase, own[1], std::false_type());
                            if (r == 1) ++j;
                        }
                        if (r == 1 && j < whole) {
                            // (the scales of the step after are another tile's, perhaps another group's: read when it begins)
                            r = step(j, 1, phase, own[1], std::false_type());
                            if (r == 1) ++j;
                        }
                    }
                    again = r == 0;
                    ok = r >= 0;
                    if (r == 1 && j % kGroupSteps == 0) mbar_arrive_if(smem_u32(&i_empty[group]), lane == 0);
                }
                if (!ok || j >= n_steps) break;
                if (!early && !(ok = wait(s_full + C::kPlaces * t + j % C::kPlaces, (j / C::kPlaces) & 1))) break;
                early = true;
                tc_fence_after();
                const float *const key = infos[(j >> 1) % (kGroup * kGroups)].scales[j & 1].key;
                const int valid = sees - (2 * g_begin + j) * 64;
                // the scores of step j twice: their maximum, their sum
                float top = -kInf, sum = 0.f;
                if (summed >= 0) top = apart->x, sum = apart->y;
                const float before = top;
#pragma unroll 1
                for (int c0 = 0; c0 < 128; c0 += 16) {
                    if (c0 == 64) {
                        const float half = half_factor(before, top);
                        sum = sum * half * half;
                    }
                    uint32_t sc[16];
                    tmem_ld16(s_addr0 + 64 * (j % C::kPlaces) + c0 % 64, sc);
                    tmem_wait_ld();
                    const float f = factor * key[c0 % 64 / kBlock], base = top == -kInf ? 0.f : -top;
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        if (c0 % 64 + c >= valid) continue;
                        if (c0 < 64) top = fmaxf(top, __uint_as_float(sc[c]) * f);
                        else sum += exp2_fast(fmaf(__uint_as_float(sc[c]), f, base));
                    }
                }
                *apart = make_float2(top, sum);
                summed = j;
            }
            if (summed >= 0 && apart->y != 0.f) {
                const float half = exp2_fast(0.5f * (apart->x - ref));
                l_run += apart->y * half * half;
            }
            if (ok && n_steps > 0) {
                // (The last two products: no other wait has seen the one before the last arrive.  v_full: nan_flag is what the converting
                // warps left.)
                ok = product_done(n_steps - 1) && (n_steps == 1 || product_done(n_steps - 2)) && wait(&v_full[(n_tiles - 1) % kStages], ((n_tiles - 1) / kStages) & 1);
                tc_fence_after();
            }
            if (ok) {
                const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
                const int64_t at = (int64_t)(s.row0 + token) * a.heads + head;
                const bool rare = *nan_flag != 0;
                // All of a row in bf16, or the half of it that takes as many bytes in fp32, then its way out.
                constexpr int kCols = DH == 32 ? 16 : 32;  // at once
                const int rounds = a.splits == 1 ? 1 : 2;
                const int64_t part_at = ((int64_t)split * a.batch.rows * a.heads + at) * DH;
                const int64_t out_at = (int64_t)(s.row0 + token) * a.ldo + (int64_t)head * DH;
                const uint32_t reals = __ballot_sync(0xffffffffu, real);
#pragma unroll 1
                for (int round = 0; round < rounds; ++round) {
#pragma unroll 1
                    for (int d0 = round * (DH / 2); d0 < (rounds == 1 ? DH : (round + 1) * (DH / 2)); d0 += kCols) {
                        float o[kCols];
                        if (n_tiles > 0) {
                            uint32_t w[kCols];
                            if constexpr (kCols == 32) tmem_ld32(o_addr + d0, w);
                            else tmem_ld16(o_addr + d0, w);
                            tmem_wait_ld();
#pragma unroll
                            for (int d = 0; d < kCols; ++d) o[d] = __uint_as_float(w[d]);
                        } else {
#pragma unroll
                            for (int d = 0; d < kCols; ++d) o[d] = 0.f;
                        }
                        if (__builtin_expect(rare, 0)) {
                            // NaN values of the tiles that are seen in part
                            const int stop = min(sees, g_end * 128);
#pragma unroll 1
                            for (int x = max(g_begin * 128, least / 128 * 128); x < stop; ++x) {
                                const int p = kv_page(a.batch, a.cache, b, x >> page_log2, a.err);
                                if (p < 0) continue;
                                const uint8_t *v = a.cache.v + (int64_t)p * a.cache.page_stride +
                                                   ((int64_t)hk * page + (x & (page - 1))) * DH + d0;
                                const bool scale = a.cache.vs[(int64_t)p * a.cache.scale_stride + hk] == 255;
#pragma unroll
                                for (int d = 0; d < kCols; ++d)
                                    if (scale || (v[d] & 0x7F) == 0x7F) o[d] = __int_as_float(0x7FC00000);
                            }
                        }
                        if (rounds == 1) {
#pragma unroll
                            for (int d = 0; d < kCols; d += 8) {
                                uint4 w;
                                w.x = pack_bf16x2(o[d] * inv, o[d + 1] * inv);
                                w.y = pack_bf16x2(o[d + 2] * inv, o[d + 3] * inv);
                                w.z = pack_bf16x2(o[d + 4] * inv, o[d + 5] * inv);
                                w.w = pack_bf16x2(o[d + 6] * inv, o[d + 7] * inv);
                                *reinterpret_cast<uint4 *>(own_q + C::place(row, (d0 + d) / 8)) = w;
                            }
                        } else {
#pragma unroll
                            for (int d = 0; d < kCols; d += 4)
                                *reinterpret_cast<float4 *>(own_q + C::place(row, (d0 - round * (DH / 2) + d) / 4)) =
                                    make_float4(o[d], o[d + 1], o[d + 2], o[d + 3]);
                        }
                    }
                    __syncwarp();
#pragma unroll 4
                    for (int i = 0; i < kLanes; ++i) {
                        const int line = i * kOnce + lane / kLanes;
                        const int64_t to = __shfl_sync(0xffffffffu, rounds == 1 ? out_at : part_at, line);
                        const uint4 w = *reinterpret_cast<const uint4 *>(own_q + C::place(32 * q + line, piece));
                        if (!(reals >> line & 1)) continue;
                        if (rounds == 1) *reinterpret_cast<uint4 *>(a.out + to + 8 * piece) = w;
                        else *reinterpret_cast<uint4 *>(a.part + to + round * (DH / 2) + 4 * piece) = w;
                    }
                    __syncwarp();
                }
                if (real) {
                    if (a.splits == 1) {
                        if (a.lse) a.lse[at] = log_sum(ref, l_run);
                    } else {
                        float2 *ml = reinterpret_cast<float2 *>(a.part + (int64_t)a.splits * a.batch.rows * a.heads * DH);
                        ml[(int64_t)split * a.batch.rows * a.heads + at] = make_float2(ref, l_run);
                    }
                }
                tc_fence_before();
            }
        }
    } else if (warp < 4) {
        reg_dec<kIssueRegs>();
        if (warp < tiles && n_tiles > 0) {
            // ------------------------------------------------ MMA issuer of one query tile
            constexpr uint32_t idesc_s = make_idesc_f16(128, 64, 0), idesc_o = make_idesc_f16(128, DH, 1);
            const int t = warp;
            const uint64_t q_desc = make_sdesc(smem_u32(sQ + t * C::kTile), 16, C::kAtom, C::kSwz);
            const uint64_t k_desc = make_sdesc(smem_u32(sK), 16, C::kAtom, C::kSwz);
            // values: the head's columns lie a region apart, eight tokens an atom
            const uint64_t v_desc = make_sdesc(smem_u32(sV), C::kRegion, C::kAtom, C::kSwz);
            constexpr uint64_t kStageStep = C::kTile >> 4, kRegionStep = C::kRegion >> 4, kVStep = (16 * C::kRowBytes) >> 4;
            constexpr uint64_t kHalfStep = (64 * C::kRowBytes) >> 4;
            // step j: place j % kPlaces of S and P, whose barriers are in their phase j / kPlaces
            struct Place {
                int i = 0;
                uint32_t phase = 0;
                F3DC_DEV void next()
                {
                    if (++i == C::kPlaces) i = 0, phase ^= 1;
                }
            } ps, pp;
            uint64_t *const s_own = s_full + C::kPlaces * t, *const p_own = p_full + C::kPlaces * t, *const done = pv_done + C::kPlaces * t;
            const uint32_t tm = tmem + t * 64 * C::kPlaces;
            auto scores = [&](int j) {
                const int g = j >> 1, st = g % kStages;
                if ((j & 1) == 0 && !wait(&k_full[st], (g / kStages) & 1)) return false;
                tc_fence_after();
                const uint64_t kd = k_desc + st * kStageStep + (j & 1) * kHalfStep;
#pragma unroll
                for (int kk = 0; kk < DH / 16; ++kk) {
                    const uint64_t at = (kk / 4) * kRegionStep + 2 * (kk % 4);
                    if (C::kQTmem) mma_bf16_ts_elect(tm + ps.i * 64, tmem + C::kColQ + t * (DH / 2) + kk * 8, kd + at, idesc_s, kk > 0);
                    else mma_bf16_elect(tm + ps.i * 64, q_desc + at, kd + at, idesc_s, kk > 0);
                }
                mma_commit_elect(&s_own[ps.i]);
                if ((j & 1) || j + 1 == n_steps) mma_commit_elect(&k_empty[st]);
                ps.next();
                return true;
            };
            // P V of step j, then S of the step that takes P's place
            auto product = [&](int j) {
                const int g = j >> 1, st = g % kStages;
                if ((j & 1) == 0 && !wait(&v_full[st], (g / kStages) & 1)) return false;
                if (!wait(&p_own[pp.i], pp.phase)) return false;
                tc_fence_after();
                const uint64_t vd = v_desc + st * kStageStep + (j & 1) * kHalfStep;
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    mma_bf16_ts_elect(tmem + C::kColO + t * DH, tm + pp.i * 64 + kk * 8, vd + kk * kVStep, idesc_o, kk > 0 || j > 0);
                mma_commit_elect(&done[pp.i]);
                if ((j & 1) || j + 1 == n_steps) mma_commit_elect(&v_empty[st]);
                if (j + C::kPlaces < n_steps && !(wait(&done[pp.i], pp.phase) && scores(j + C::kPlaces))) return false;
                pp.next();
                return true;
            };
            bool ok = wait(&q_full[t], 0);
#pragma unroll 1
            for (int j = 0; ok && j < min(C::kPlaces, n_steps); ++j) ok = scores(j);
#pragma unroll 1
            for (int j = 0; ok && j < n_steps; ++j) ok = product(j);
        }
        if (warp == 2) {
            // ------------------------------------------------ the page table: a lane for 16 tokens of one of four tiles
            const int run = lane & 7;
            const uint32_t stride16 = (uint32_t)(a.cache.page_stride >> 4);
            const uint32_t own16 = (uint32_t)(hk * page + (16 * run & (page - 1))) * (DH / 16);
            int widest = kLeastScale;
#pragma unroll 1
            for (int g0 = 0, n = 0; g0 < n_tiles; g0 += kGroup, ++n) {
                const int g = g0 + (lane >> 3), t0 = (g_begin + g) * 128 + 16 * run;
                const bool mine = lane < 8 * kGroup;
                uint32_t at = own16, bytes = 127u | 127u << 8;
                int there = 0;
                if (mine && g < n_tiles && t0 < s.length) {
                    const int p = kv_page(a.batch, a.cache, b, t0 >> page_log2, a.err);
                    if (p >= 0) {
                        const int64_t of = (int64_t)p * a.cache.scale_stride + hk;
                        bytes = a.cache.ks[of] | (uint32_t)a.cache.vs[of] << 8;
                        at = (uint32_t)p * stride16 + own16;
                        there = min(16, s.length - t0);
                    }
                }
                const int slot = n % kGroups;
                if (!wait(&i_empty[slot], ((n / kGroups) & 1) ^ 1)) break;
                const ValueScale v = value_scale(bytes >> 8);
                const uint32_t tile = 0xFFu << (lane & 24);
                const uint32_t complete = __ballot_sync(0xffffffffu, there == 16), plain = __ballot_sync(0xffffffffu, v.times == kHalfOnes);
                // (the largest of all four tiles: one that comes later does no harm)
                widest = max(widest, __reduce_max_sync(0xffffffffu, (int)v.log2));
                const uint32_t apart = __ballot_sync(0xffffffffu, (int)v.log2 < widest - kScaleSpan);
                if (mine) {
                    TileInfo<NB> &x = infos[slot * kGroup + (lane >> 3)];
                    x.at[run] = at;
                    x.times[run] = v.times;
                    x.there[run] = there;
                    if (run % (8 / NB) == 0) {
                        StepScales<NB> &sc = x.scales[run >> 2];
                        const int k = (run & 3) * NB / 8;
                        sc.key[k] = key_scale(bytes & 255u);
                        sc.value_log2[k] = apart & tile ? kInf : v.log2;
                        sc.value_inverse[k] = v.inverse;
                    }
                    if (run == 0) {
                        x.complete = (complete & tile) == tile;
                        x.plain = (plain & tile) == tile;
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&i_full[slot]);
            }
        }
    } else if (warp < 8) {
        // ------------------------------------------------ pages to operands
        reg_dec<kConvertRegs>();
        // 16-byte pieces of a token, and of a thread per half of a tile: piece k is of a token 128 / kPieces further
        constexpr int kPieces = DH / 16, kTokens = 128 / kPieces;
        const int i = threadIdx.x - 128;
        // (dh 128: eight neighbouring lanes hold the same columns' half of two tokens, so that their stores meet no bank twice)
        const int piece = DH == 128 ? (i & 3) | (i >> 1 & 4) : i % kPieces;
        const int token = DH == 128 ? (i >> 4) * 2 + (i >> 2 & 1) : i / kPieces;
        const int put0 = C::place(token, 2 * piece), put1 = C::place(token, 2 * piece + 1);
        const uint4 *const k_own = reinterpret_cast<const uint4 *>(a.cache.k) + (token & 15) * kPieces + piece;
        const uint4 *const v_own = reinterpret_cast<const uint4 *>(a.cache.v) + (token & 15) * kPieces + piece;
        const int run = token >> 4;  // of piece 0
        auto info = [&](int g) -> const TileInfo<NB> & { return infos[g / kGroup % kGroups * kGroup + g % kGroup]; };
        // piece k of a half of a tile
        auto fetch = [&](const uint4 *own, const TileInfo<NB> &x, int k) { return own[x.at[run + k * (kTokens / 16)]]; };
        auto clear = [&](const TileInfo<NB> &x, uint4 (&u)[kPieces]) {
#pragma unroll
            for (int k = 0; k < kPieces; ++k)
                if ((token & 15) >= x.there[run + k * (kTokens / 16)]) u[k] = make_uint4(0u, 0u, 0u, 0u);
        };
        auto widen = [&](uint4 w, uint32_t (&h)[8]) {
            e4m3x4_to_half2(w.x, h[0], h[1]);
            e4m3x4_to_half2(w.y, h[2], h[3]);
            e4m3x4_to_half2(w.z, h[4], h[5]);
            e4m3x4_to_half2(w.w, h[6], h[7]);
        };
        auto store = [&](uint8_t *tile, int k, const uint32_t (&h)[8]) {
            tile += k * kTokens * C::kRowBytes;  // (the swizzle repeats every eight rows)
            *reinterpret_cast<uint4 *>(tile + put0) = make_uint4(h[0], h[1], h[2], h[3]);
            *reinterpret_cast<uint4 *>(tile + put1) = make_uint4(h[4], h[5], h[6], h[7]);
        };
        uint4 ku[kPieces], vu[kPieces];
        {
            // the first tile's pages looked up here too: its pieces do not wait for its scales
            const int t0 = g_begin * 128 + 16 * (lane & 7);
            uint32_t at = (uint32_t)(hk * page + (16 * (lane & 7) & (page - 1))) * kPieces;
            if (n_tiles > 0 && t0 < s.length) {
                const int p = kv_page(a.batch, a.cache, b, t0 >> page_log2, nullptr);
                if (p >= 0) at += (uint32_t)p * (uint32_t)(a.cache.page_stride >> 4);
            }
#pragma unroll
            for (int k = 0; k < kPieces; ++k) ku[k] = k_own[__shfl_sync(0xffffffffu, at, run + k * (kTokens / 16))];
#pragma unroll
            for (int k = 0; k < kPieces; ++k) vu[k] = v_own[__shfl_sync(0xffffffffu, at, run + k * (kTokens / 16))];
            if (n_tiles > 0) wait(&i_full[0], 0);
        }
#pragma unroll 1
        for (int g = 0; g < n_tiles; ++g) {
            const int st = g % kStages;
            const uint32_t parity = (g / kStages) & 1;
            const TileInfo<NB> &now = info(g);
            // (behind the last tile its own pieces are loaded once more, unused)
            const int ng = min(g + 1, n_tiles - 1);
            if (ng % kGroup == 0 && ng > g && !wait(&i_full[ng / kGroup % kGroups], (ng / kGroup / kGroups) & 1)) break;
            const TileInfo<NB> &next = info(ng);
            const bool complete = now.complete != 0;
            // keys
            if (!wait(&k_empty[st], parity ^ 1)) break;
            if (!complete) clear(now, ku);
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                uint32_t h[8];
                widen(ku[k], h);
                store(sK + st * C::kTile, k, h);
                ku[k] = fetch(k_own, next, k);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&k_full[st]);
            // values
            if (!wait(&v_empty[st], parity ^ 1)) break;
            if (!complete) clear(now, vu);
            const bool partly = (g_begin + g + 1) * 128 > least;
            if (!partly && now.plain) {
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    uint32_t h[8];
                    widen(vu[k], h);
                    store(sV + st * C::kTile, k, h);
                    vu[k] = fetch(v_own, next, k);
                }
            } else {
                uint32_t numbers = 0xffffffffu;
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    uint32_t h[8];
                    widen(vu[k], h);
                    const uint32_t by = now.times[run + k * (kTokens / 16)];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        h[e] = half2_times(h[e], by);
                        if (partly) {
                            const __half2 x = *reinterpret_cast<const __half2 *>(&h[e]);
                            const uint32_t m = __heq2_mask(x, x);
                            numbers &= m;
                            h[e] &= m;
                        }
                    }
                    store(sV + st * C::kTile, k, h);
                    vu[k] = fetch(v_own, next, k);
                }
                if (numbers != 0xffffffffu) *nan_flag = 1;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&v_full[st]);
                if (g % kGroup == kGroup - 1) mbar_arrive(&i_empty[g / kGroup % kGroups]);
            }
        }
        // every arrival of the MMAs' completion is in before the CTA leaves
#pragma unroll 1
        for (int g = max(0, n_tiles - kStages); g < n_tiles; ++g)
            if (!wait(&k_empty[g % kStages], (g / kStages) & 1) || !wait(&v_empty[g % kStages], (g / kStages) & 1)) break;
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

template <int DH, int NB>
cudaError_t launch_one(const KvAttnArgs &args, cudaStream_t s)
{
    KvAttnArgs a = args;
    a.row_blocks = (int)(((int64_t)a.batch.max_rows * a.group + 255) / 256);
    const int64_t ctas = (int64_t)a.splits * a.row_blocks * a.cache.heads * a.batch.batch;
    if (ctas > INT32_MAX) return cudaErrorInvalidValue;
    // (a register split above what the launch really has would wait for ever)
    static std::atomic<uint64_t> checked{0}, devices{0};
    cudaError_t e = once_per_device(checked, [] {
        cudaFuncAttributes f;
        const cudaError_t e = cudaFuncGetAttributes(&f, k_kv_attn<DH, NB>);
        return e != cudaSuccess ? e : (f.numRegs >= kLaunchRegs ? cudaSuccess : cudaErrorInvalidKernelImage);
    });
    if (e != cudaSuccess) return e;
    e = ask_smem(k_kv_attn<DH, NB>, (int)Cfg<DH, NB>::kSmem, devices);
    if (e != cudaSuccess) return e;
    e = launch_k(k_kv_attn<DH, NB>, dim3((unsigned)ctas), dim3(kThreads), Cfg<DH, NB>::kSmem, s, a);
    return e != cudaSuccess || a.splits == 1 ? e : launch_kv_join(a, s);
}

template <int DH>
cudaError_t launch_dh(const KvAttnArgs &a, cudaStream_t s)
{
    return a.cache.page >= 64 ? launch_one<DH, 2>(a, s) : launch_one<DH, 8>(a, s);
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
