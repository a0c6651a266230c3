// k_gemm8.cu -- the matrix product of 8-bit linear layers (f3dc_gemm_fp8):
//
//   out[m, n] = epilogue( sum_k A[m, k] 2^ea[m, k / 128] B[n, k] 2^eb[n, k / 128] )
//
// A [M, K] and B [N, K] e4m3 with one power-of-two scale per row and block of 128 K.
//
// The scales go into the tensor cores: kind::mxf8f6f4 with block scales multiplies
// every 32 K of a row by a scale byte held in tensor memory, so K up to 16384 or 65536
// (piece_most) is one fp32 sum in one accumulator, longer ones are pieces of that, and nothing
// is rescaled in registers.  A block of 128 is four MMAs that take the same byte; one 32-bit
// column of scales serves 512 K.
//
// Clusters of two CTAs (cta_group::2), persistent over tiles of 256 x 256 (narrower
// ones in the last wave), 384 threads:
//   warp 0      TMA producer: this CTA's 128 rows of A and half of the tile's rows of
//               B, 128 K (a scale block, one 128-byte swizzled line per row) per stage
//   warp 1      of the even CTA issues the MMAs for both
//   warp 2      reads scale bytes from global memory (plain rows) and lays them out
//               for the tensor memory: 512 K of A's 128 and B's 256 rows at a time
//   warp 3      allocates tensor memory; of the even CTA issues the copies of scales into it, so
//               that the MMAs' issuer, which is what bounds narrow units, has less to do; of the
//               odd one publishes its scales to the even one
//   warps 4-11  epilogue: each has 32 rows (its TMEM lanes) and half of the columns, stages
//               its output and sends it by TMA; no warp waits for another
// Tensor memory: 512 columns hold two accumulators of 256 only if nothing else is
// there, but two sets of scales need 24.  So the second accumulator starts at column
// 232: the tile after may begin as soon as the epilogue has read the 24 columns that
// the two share, which it reads first.  Sums in pieces have units of 128 columns, whose
// accumulators take turns, and the sum of the pieces so far in 128 columns more.
//
// 32768 x 4096 x 1024 takes 96 us (2.86 PFLOP/s), 110 to 117 with GELU, back to back from Python
// 129: a tile's epilogue is then longer than its sum, though neither issue (38 % of the cycles)
// nor the special functions (28 %) nor the tensor cores (56 %) are near their limit: two epilogue
// warps per scheduler do not hide one another's latencies.  8192 x 8192 x 8192 348 (3.16 PFLOP/s),
// where the board's power is the bound.  A few tiles take 4.3 us (launch, first fetches, scales
// and their way from the odd CTA to the even one, epilogue, exit) and per 128 K 0.18 of narrow
// units, what issuing their loads and MMAs takes one warp each, to 0.3 of full ones, whose MMAs
// alone are 512 clocks.
#include <atomic>

#include "kernels.h"
#include "mx8.cuh"

namespace f3dc {

namespace {

constexpr int kThreads8 = 384;
constexpr int kOperand8 = 128 * 128;        // a stage's 128 K of A, or of up to 128 rows of B, per CTA
constexpr int kMaxStages8 = 8;
constexpr int kSetBytes = 512 + 1024;       // scales of A's 128 rows, B's 256, four bytes each (512 K)
constexpr int kSets = 4;                    // such sets in shared memory
constexpr int kVecBytes8 = 8 * 2 * 128 * 4; // an epilogue warp's biases and gates of a unit
constexpr int kOutBox8 = 32 * 128;          // 32 rows of 128 bytes on their way out
constexpr int kBarBytes8 = 320;             // mbarriers and two words
constexpr uint32_t kTmemCols8 = 512;
constexpr uint32_t kAcc1 = 232;             // first column of the second accumulator
constexpr uint32_t kScaleCols = 488;        // two sets of 4 (A) + 8 (B) columns
constexpr uint32_t kSumCols = 360;          // sums in pieces: the 128 columns behind the second accumulator's
// What shared memory holds beside the scales and an output box per epilogue warp: stages of
// operands (b_bytes of B in each, this CTA's half of the widest unit's rows).
struct Depth8 {
    int stages, b_bytes;
    size_t smem() const
    {
        return 1024 + (size_t)stages * (kOperand8 + b_bytes) + kSets * kSetBytes + kVecBytes8 + 8 * kOutBox8 + kBarBytes8;
    }
};
constexpr size_t kMostSmem8 = 227 * 1024;
// As many stages as there is room for, five of full units.  (A second output box per warp instead
// of the fifth: 32768 x 4096 x 1024 107 us instead of 103, with 8-bit output 104 and 102, with
// GELU 133.4 and 132.6, 4096 x 4096 x 1024 with 8-bit output 17.4 and 16.9; 32768 x 4096 x 256
// with 8-bit output and GELU 115.0 and 115.4.)  Narrow units leave room for more: the loads'
// latency counts most where there is one unit.
inline Depth8 depth8(int width)
{
    Depth8 d{1, width / 2 * 128};
    while (d.stages < kMaxStages8 && Depth8{d.stages + 1, d.b_bytes}.smem() <= kMostSmem8) ++d.stages;
    return d;
}

// n / d and n % d for n < 2^31 (d >= 1) by a multiplication (the round-up method).
struct FastDiv {
    uint32_t d, mul, shift;
    void set(uint32_t v)
    {
        d = v;
        shift = 0;
        while ((1ull << shift) < v) ++shift;
        mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - v)) / v + 1);
    }
    F3DC_DEV int div(int n) const { return (int)((__umulhi((uint32_t)n, mul) + (uint32_t)n) >> shift); }
};

// Work units: full waves of 256 x 256 tiles, the tiles left for the last wave cut into
// 2 or 4 pieces of 128 or 64 columns where there are clusters for all of them.  Tiles
// run in bands of kBand row pairs, row-fastest within a band's columns, so that what
// the clusters work on at a time is about as many rows of A as of B.  A tile's columns
// behind N are not computed but for the rounding up of its width to 64, 128 or 256.
constexpr int kBand = 8;
struct Units8 {
    int full, sub, total, N, min_width, last_band;
    FastDiv band, last_high;  // tiles of a band, rows of the last band
    void set(int M, int N_, int clusters, int min_width_)
    {
        N = N_;
        min_width = min_width_;
        const int pairs = (M + 255) / 256, line = (N + 255) / 256, tiles = pairs * line;
        full = tiles / clusters * clusters;
        const int rest = tiles - full;
        sub = 4 * rest <= clusters && min_width <= 64 ? 4 : (2 * rest <= clusters ? 2 : 1);
        total = full + rest * sub;
        band.set((uint32_t)kBand * line);
        last_band = (pairs - 1) / kBand;
        last_high.set(pairs - last_band * kBand);
    }
    // split sums and sums in pieces: units of `width` columns (256 or 128); returns their number
    int set_single(int M, int N_, int width)
    {
        set(M, N_, 1, width);  // (every unit is that wide, also behind N)
        const int tiles = ((M + 255) / 256) * ((N + 255) / 256);
        full = width == 256 ? tiles : 0;
        sub = width == 256 ? 1 : 2;
        total = tiles * sub;
        return total;
    }
    // unit u: first row m0 of the pair, first column n0, width bn (0: nothing to do)
    F3DC_DEV void decode(int u, int &m0, int &n0, int &bn) const
    {
        int tile = u, piece = 0;
        bn = 256;
        if (u >= full) {
            const int v = u - full, log_sub = sub >> 1;
            tile = full + (v >> log_sub);
            piece = v & (sub - 1);
            bn = 256 >> log_sub;
        }
        const int b = band.div(tile), in = tile - b * (int)band.d;
        const int high = b == last_band ? (int)last_high.d : kBand;
        const int col = b == last_band ? last_high.div(in) : in / kBand;
        m0 = (b * kBand + in - col * high) * 256;
        n0 = col * 256 + piece * bn;
        const int left = N - n0;
        bn = left <= 0 ? 0 : min(bn, left <= min_width ? min_width : (left <= 128 ? 128 : 256));
    }
    // the unit after u of a cluster, ncl clusters in all; false: none
    F3DC_DEV bool next(int &u, int ncl, int &m0, int &n0, int &bn) const
    {
        do {
            u += ncl;
            if (u >= total) return false;
            decode(u, m0, n0, bn);
        } while (bn == 0);
        return true;
    }
};

F3DC_DEV bool wait_ns8(uint64_t *bar, uint32_t parity, uint64_t ns)
{
    const uint64_t t0 = globaltimer();
    while (!mbar_try_wait(bar, parity))
        if (globaltimer() - t0 > ns) return false;
    return true;
}

// Waits for this thread's TMEM loads; r's values count from here on.
F3DC_DEV void wait_chunk(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]),
                   "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                   "+r"(r[30]), "+r"(r[31])::"memory");
}

// r += 32 columns of tensor memory (fp32)
F3DC_DEV void add_sum(uint32_t (&r)[32], uint32_t taddr)
{
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
        uint32_t v[16];
        tmem_ld16(taddr + h, v);
        asm volatile("tcgen05.wait::ld.sync.aligned;"
                     : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                       "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]),
                       "+r"(v[15])::"memory");
#pragma unroll
        for (int j = 0; j < 16; ++j) r[h + j] = __float_as_uint(__uint_as_float(v[j]) + __uint_as_float(r[h + j]));
    }
}

// acc + bias and the epilogue's function of 32 columns, in place (fp32 bits); biases
// and gates from shared memory.
template <int EPI>
F3DC_DEV void apply(uint32_t (&r)[32], const float *bias, const float *gate)
{
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
        const float4 b = *reinterpret_cast<const float4 *>(bias + j);
        f32x2 x0 = fadd2({__uint_as_float(r[j]), __uint_as_float(r[j + 1])}, {b.x, b.y});
        f32x2 x1 = fadd2({__uint_as_float(r[j + 2]), __uint_as_float(r[j + 3])}, {b.z, b.w});
        if constexpr (EPI == kEpiGelu) {
            x0 = gelu2(x0);
            x1 = gelu2(x1);
        }
        if constexpr (EPI == kEpiResid) {
            const float4 g = *reinterpret_cast<const float4 *>(gate + j);
            x0 = fmul2(x0, {g.x, g.y});
            x1 = fmul2(x1, {g.z, g.w});
        }
        r[j] = __float_as_uint(x0.x), r[j + 1] = __float_as_uint(x0.y);
        r[j + 2] = __float_as_uint(x1.x), r[j + 3] = __float_as_uint(x1.y);
    }
}

// Staged output of an epilogue warp: a box of its 32 rows x 128 bytes, the 16-byte piece c
// of row r at 128 r + 16 (c ^ (r % 8)) (TMA 128B swizzle).  Lane 0 issues the stores and waits
// before the box is written again until its last store has read it.  (Stores from registers, or
// turned through shared memory into whole sectors, took 132 and 129 us instead of 115 at
// 32768 x 4096 x 1024.)
struct Stage8 {
    uint8_t *buf;
    const CUtensorMap *map;
    int row, lane;
    F3DC_DEV void begin() const
    {
        if (lane == 0) bulk_wait_read<0>();
        __syncwarp();
    }
    F3DC_DEV void put16(int c, uint4 u) const
    {
        *reinterpret_cast<uint4 *>(buf + lane * 128 + ((c ^ (lane & 7)) << 4)) = u;
    }
    template <bool kReduce>
    F3DC_DEV void send(int x) const
    {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            if (kReduce)
                tma_reduce_add_2d(map, buf, x, row);
            else
                tma_store_2d(map, buf, x, row);
            bulk_commit();
        }
    }
};

// SPLIT: a cluster is two pairs that share the K of one unit, the first taking p.split_kb
// blocks (whole scale sets).  Each pair finishes one half of the columns: its partial sums
// of the other half go to the other pair's CTA of the same rows, into operand stages that
// are no longer used, and are added to that CTA's own (two addends: their order does not
// matter).
// LONG: what a pair sums is longer than piece_most and summed in pieces of p.piece_kb blocks
// (whole scale sets), each in an accumulator as if it were a unit; the epilogue adds them up in
// order, in tensor memory, and finishes the unit with the last.
template <int EPI, bool OUT8, bool SPLIT, bool LONG>
__global__ void __launch_bounds__(kThreads8, 1)
    k_gemm8_pair(const __grid_constant__ CUtensorMap tma, const __grid_constant__ GemmPairB tmb,
                 const __grid_constant__ CUtensorMap tmo, const Units8 U, const Depth8 depth, const Gemm8Params p)
{
    const int S = depth.stages;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *sa = smem;
    uint8_t *sb = sa + S * kOperand8;
    uint8_t *ss = sb + S * depth.b_bytes;
    float *sv = reinterpret_cast<float *>(ss + kSets * kSetBytes);
    uint8_t *so = ss + kSets * kSetBytes + kVecBytes8;
    uint64_t *bars = reinterpret_cast<uint64_t *>(so + 8 * kOutBox8);
    uint64_t *full = bars, *empty = full + kMaxStages8;    // operands of a stage there (even CTA) / used (both)
    uint64_t *sfull = empty + kMaxStages8, *sempty = sfull + kSets;  // scales of a set there (even CTA) / copied (both)
    uint64_t *tfull = sempty + kSets, *tempty = tfull + 2; // scales of a set in tensor memory / used (even CTA)
    uint64_t *accf = tempty + 2, *acce = accf + 2;         // accumulator complete (both) / read (even CTA)
    uint64_t *shared_read = acce + 2;                      // its columns that the next one needs are read (even CTA)
    uint64_t *drain = shared_read + 1;                     // of the MMAs, of the copies
    uint64_t *tmem_there = drain + 2, *tmem_here = tmem_there + 1;  // tensor memory of both CTAs (even CTA), of this one
    uint64_t *other_done = tmem_here + 1, *parts = other_done + 1;  // SPLIT: the other pair's stages are free, its sums are here
    constexpr int kBars = 2 * kMaxStages8 + 2 * kSets + 4 + 4 + 1 + 2 + 2 + 2;
    static_assert(kBars * 8 + 8 <= kBarBytes8, "barriers");
    static_assert(!(OUT8 && SPLIT && LONG), "a unit of 128 columns is one scale block");
    constexpr bool kReuse = !SPLIT || LONG;    // accumulators are used again: their readers say so,
    constexpr bool kShared = !SPLIT && !LONG;  // and that they have read the columns that both have
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(bars + kBars);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t crank = __shfl_sync(0xffffffffu, cluster_rank(), 0);
    const uint32_t rank = crank & 1, pair = SPLIT ? crank >> 1 : 0, even = SPLIT ? crank & ~1u : 0;
    const uint16_t both = (uint16_t)(3u << (2 * pair));  // this pair's CTAs
    griddep_launch();

    if (threadIdx.x == 64) {
        tma_prefetch(&tma);
        for (int i = 0; i < 3; ++i) tma_prefetch(&tmb.rows[i]);
        tma_prefetch(&tmo);
    }
    if (warp == 0) {
        for (int i = lane; i < kBars; i += 32) {
            uint64_t *const b = bars + i;
            uint32_t count = 1;
            if (b >= sfull && b < sempty) count = 2 - rank;  // even: this CTA's scale warp, the odd CTA's warp 3
            if (b == tmem_there) count = 2;                  // warp 3 of each CTA
            if (b == parts) count = 8;                       // the eight epilogue warps of the other CTA
            if (b == &acce[0] || b == &acce[1]) count = 16;  // eight epilogue warps in each CTA
            if (b == shared_read) count = 8;                 // the four warps that hold the columns, in each CTA
            mbar_init(b, count);
        }
        if (lane == 0) *abort_flag = 0;
        fence_mbar_init();
    }
    __syncthreads();
    // both CTAs' barriers are initialised before any warp passes its cluster_wait(); what
    // does not need them runs before that
    cluster_arrive_relaxed();
    if (warp == 3) {
        tmem_alloc_pair(tmem_holder, kTmemCols8);
        tmem_relinquish_pair();
        tc_fence_before();
    }
    // scale blocks of a row, and the ones that this pair sums (from a whole set on)
    const int kb_all = (p.K + 127) / 128;
    const int kb_0 = SPLIT ? (int)pair * p.split_kb : 0, kb_n = SPLIT ? min(kb_all, kb_0 + p.split_kb) : kb_all;
    const int cl = blockIdx.x / (SPLIT ? 4 : 2), ncl = gridDim.x / (SPLIT ? 4 : 2);
    int t = cl - ncl, m0 = 0, n0 = 0, bn = 0;
    bool more = U.next(t, ncl, m0, n0, bn);  // this cluster's first unit

    if (warp == 0) {
        const uint32_t full_u = smem_u32(full), full_c = mapa_shared(full_u, even), empty_u = smem_u32(empty);
        const uint32_t sa_u = smem_u32(sa), sb_u = smem_u32(sb), b_bytes = (uint32_t)depth.b_bytes;
        cluster_wait();
        griddep_wait();
        int s = 0;
        uint32_t ph = 0;
        bool ok = true, ready = true;
#pragma unroll 1
        for (; more && ok; more = U.next(t, ncl, m0, n0, bn)) {
            // this CTA holds bn / 2 of the unit's B rows
            const CUtensorMap *mb = &tmb.rows[bn == 256 ? 0 : (bn == 128 ? 1 : 2)];
            const int row_a = m0 + (int)rank * 128, row_b = n0 + (int)rank * (bn / 2);
            const uint32_t bytes = rank == 0 ? 2u * (kOperand8 + (uint32_t)(bn / 2) * 128) : 0u;  // both CTAs
#pragma unroll 1
            for (int kb = kb_0; kb < kb_n; ++kb) {
                if (!warp_all(ready) && !warp_wait(&empty[s], ph ^ 1, abort_flag, p.err)) {
                    ok = false;
                    break;
                }
                const int s_next = s + 1 == S ? 0 : s + 1;
                const uint32_t ph_next = s_next == 0 ? ph ^ 1 : ph;
                ready = tma_load_stage_pair(sa_u + (uint32_t)s * kOperand8, &tma, row_a, sb_u + (uint32_t)s * b_bytes, mb, row_b,
                                            kb * 128, full_u + 8u * (uint32_t)s, full_c + 8u * (uint32_t)s, bytes,
                                            empty_u + 8u * (uint32_t)s_next, ph_next ^ 1);
                s = s_next;
                ph = ph_next;
            }
        }
        // (every arrival at this CTA's barriers is awaited before it leaves)
        for (int i = 0; i < S && ok; ++i) {
            ok = warp_wait(&empty[s], ph ^ 1, abort_flag, p.err);
            if (++s == S) {
                s = 0;
                ph ^= 1;
            }
        }
    } else if (warp == 1) {
        cluster_wait();
        griddep_wait();
        if (rank == 0 && warp_wait(tmem_there, 0, abort_flag, p.err)) {
            tc_fence_after();
            const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_holder, 0);
            const uint64_t a_desc0 = make_sdesc(smem_u32(sa), 16, 1024, kSwizzle128);
            const uint64_t b_desc0 = make_sdesc(smem_u32(sb), 16, 1024, kSwizzle128);
            int s = 0, it = 0, set = 0;
            uint32_t ph = 0;
            bool ok = true;
            // a stage's barrier (and a set's) is read while the MMAs of the stage before are issued
            bool ready = mbar_test(&full[0], 0) && mbar_test(&tfull[0], 0);
#pragma unroll 1
            while (more && ok) {
                bool another = false;
                int kb0 = kb_0;
#pragma unroll 1
                do {  // LONG: a piece of the unit
                    const int buf = it & 1;
                    if ((it > 1 && !warp_wait(&acce[buf], ((it >> 1) & 1) ^ 1, abort_flag, p.err)) ||
                        (kShared && it > 0 && !warp_wait(shared_read, (it - 1) & 1, abort_flag, p.err))) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t d = tmem + (buf ? kAcc1 : 0u);
                    const uint32_t idesc0 = make_idesc_mxf8(256, 0, 0) | ((uint32_t)(bn >> 3) << 17);
                    const int first = kb0, end = LONG ? min(kb_n, kb0 + p.piece_kb) : kb_n;
#pragma unroll 1
                    for (; kb0 < end && ok; kb0 += 4) {
                        const uint32_t sfa = tmem + kScaleCols + 12u * (uint32_t)(set & 1);
                        const uint32_t setp = (set >> 1) & 1, setp_next = ((set + 1) >> 1) & 1;
                        uint64_t *const tf = &tfull[set & 1], *const tf_next = &tfull[(set + 1) & 1];
#pragma unroll
                        for (uint32_t byte = 0; byte < 4; ++byte) {
                            const int kb = kb0 + (int)byte;
                            if (byte != 0 && kb >= kb_n) break;
                            if (!warp_all(ready) && !((byte != 0 || warp_wait(tf, setp, abort_flag, p.err)) &&
                                                      warp_wait(&full[s], ph, abort_flag, p.err))) {
                                ok = false;
                                break;
                            }
                            tc_fence_after();
                            const int s_next = s + 1 == S ? 0 : s + 1;
                            const uint32_t ph_next = s_next == 0 ? ph ^ 1 : ph;
                            const bool last = byte == 3 || kb + 1 == kb_n;
                            ready = mma_mxf8_pair_128k(d, a_desc0 + (uint64_t)s * (kOperand8 >> 4),
                                                       b_desc0 + (uint64_t)s * (uint32_t)(depth.b_bytes >> 4), sfa, sfa + 4,
                                                       idesc0 | byte << 4 | byte << 29, byte != 0 || kb0 != first, &empty[s], both,
                                                       &full[s_next], ph_next, last ? tf_next : tf, last ? setp_next : setp);
                            s = s_next;
                            ph = ph_next;
                        }
                        mma_commit_pair_elect(tf == &tfull[0] ? &tempty[0] : &tempty[1]);
                        ++set;
                        // (bn is this unit's until its last piece has begun)
                        if (kb0 == first && end == kb_n) another = U.next(t, ncl, m0, n0, bn);
                    }
                    if (ok) mma_commit_pair_mc_elect(&accf[buf], both);
                    ++it;
                } while (LONG && ok && kb0 < kb_n);
                more = another;
            }
            if (kReuse && ok && it > 0) {
                if (kShared) warp_wait(shared_read, (it - 1) & 1, abort_flag, p.err);
                for (int i = it > 1 ? it : 2; i < it + 2; ++i) warp_wait(&acce[i & 1], ((i >> 1) & 1) ^ 1, abort_flag, p.err);
            }
            if (*abort_flag) {
                // wait (bounded) for the MMAs in flight, which their issuing lane commits
                mma_commit_pair_elect(drain);
                if (lane == 0) wait_ns8(drain, 0, 100000000ull);
                __syncwarp();
            }
        }
    } else if (warp == 2) {
        // lane l: rows l, l + 32, l + 64, l + 96 of each 128, four scale bytes (512 K) of
        // each per set.  A row's bytes are read for 1, 2 or 4 sets at once, as far as
        // the rows' alignment allows: 4-byte loads of every set cost 10 % of the whole
        // product at 8192 x 8192 x 8192.  A group's loads are in flight while the sets
        // of the group before wait for their places.
        struct Group {
            uint4 a[4], b[8];
        };
        const int per = p.scale_sets;
        const uint8_t *ra[4], *rb[8];  // this lane's rows (rows from M, N on: the last one, which nothing uses)
        auto set_rows = [&] {
#pragma unroll
            for (int j = 0; j < 4; ++j) ra[j] = p.sa + (int64_t)min(m0 + (int)rank * 128 + 32 * j + lane, p.M - 1) * p.lda_s;
#pragma unroll
            for (int j = 0; j < 8; ++j) rb[j] = p.sb + (int64_t)min(n0 + 32 * j + lane, p.N - 1) * p.ldb_s;
        };
        auto load_rows = [&](Group &x, int kb, auto get) {
#pragma unroll
            for (int j = 0; j < 4; ++j) get(x.a[j], ra[j] + kb);
#pragma unroll
            for (int j = 0; j < 4; ++j) get(x.b[j], rb[j] + kb);
            if (bn > 128) {
#pragma unroll
                for (int j = 4; j < 8; ++j) get(x.b[j], rb[j] + kb);
            }
        };
        auto load = [&](Group &x, int kb) {
            if (per == 4)
                load_rows(x, kb, [](uint4 &w, const uint8_t *r) { w = *reinterpret_cast<const uint4 *>(r); });
            else if (per == 2)
                load_rows(x, kb, [](uint4 &w, const uint8_t *r) { *reinterpret_cast<uint2 *>(&w) = *reinterpret_cast<const uint2 *>(r); });
            else
                load_rows(x, kb, [](uint4 &w, const uint8_t *r) { w.x = *reinterpret_cast<const uint32_t *>(r); });
        };
        Group x, next;
        if (more) set_rows();
        griddep_wait();
        if (more) load(x, kb_0);
        cluster_wait();
        int kb = kb_0, n = 0;
        bool ok = true;
#pragma unroll 1
        while (more && ok) {
            const int sets = min(per, (kb_n - kb + 3) / 4);
            kb += 4 * per;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= sets || !ok) break;
                const int b = n % kSets;
                ok = warp_wait(&sempty[b], (n / kSets & 1) ^ 1, abort_flag, p.err);
                if (!ok) break;
                auto word = [&](const uint4 &w) { return i == 0 ? w.x : (i == 1 ? w.y : (i == 2 ? w.z : w.w)); };
                uint4 *dst = reinterpret_cast<uint4 *>(ss + b * kSetBytes) + lane;
                dst[0] = make_uint4(word(x.a[0]), word(x.a[1]), word(x.a[2]), word(x.a[3]));
                dst[32] = make_uint4(word(x.b[0]), word(x.b[1]), word(x.b[2]), word(x.b[3]));
                dst[64] = make_uint4(word(x.b[4]), word(x.b[5]), word(x.b[6]), word(x.b[7]));
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sfull[b]);
                ++n;
                if (i == 0) {
                    // behind the release, which would wait for loads in flight
                    if (kb >= kb_n) {
                        kb = kb_0;
                        more = U.next(t, ncl, m0, n0, bn);
                        if (more) set_rows();
                    }
                    if (more) load(next, kb);
                }
            }
            x = next;
        }
        for (int i = 0; i < kSets && ok; ++i, ++n) ok = warp_wait(&sempty[n % kSets], (n / kSets & 1) ^ 1, abort_flag, p.err);
    } else if (warp >= 4) {
        // warp w: rows 32 q .. 32 q + 31 of this CTA's 128 (its TMEM lanes), one half of
        // the unit's columns (of 8-bit output a whole scale block)
        const int q = warp & 3, half = (warp - 4) >> 2;
        float *bias = sv + (warp - 4) * 256, *gate = bias + 128;
        Stage8 o{so + (warp - 4) * kOutBox8, &tmo, 0, lane};
        const uint32_t acce_c = mapa_shared(smem_u32(acce), even), shared_c = mapa_shared(smem_u32(shared_read), even);
        auto arrive = [&](uint32_t bar) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_relaxed(bar);
        };
        // columns of a unit that this pair finishes, and this warp's of them (a box of 128
        // bytes is the least that a warp stores)
        auto unit_slice = [&] { return SPLIT ? bn / 2 : bn; };
        auto unit_width = [&] { return OUT8 ? 128 : (EPI == kEpiResid ? unit_slice() / 2 : max(64, unit_slice() / 2)); };
        // A unit's biases and gates of this warp's columns are on their way a unit ahead (they
        // took 1000 clocks of each unit): in registers, columns 32 i + lane, or with 8-bit output,
        // which needs its registers, as they are in the place of the gates.
        float vb[4], vg[4];
        auto load_vectors = [&] {
            const int width = unit_width(), col0 = n0 + (int)pair * unit_slice() + half * width;
            if constexpr (OUT8) {
                if (lane < 16) {
                    if (p.bias && col0 + 8 * lane < p.N)
                        cp_async16(smem_u32(gate) + 16u * (uint32_t)lane, p.bias + col0 + 8 * lane);
                    else
                        *reinterpret_cast<uint4 *>(gate + 4 * lane) = make_uint4(0u, 0u, 0u, 0u);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = 32 * i + lane;
                    const bool in = c < width && col0 + c < p.N;
                    vb[i] = in && p.bias ? __bfloat162float(p.bias[col0 + c]) : 0.f;
                    if constexpr (EPI == kEpiResid) vg[i] = in && p.gate ? p.gate[col0 + c] : 1.f;
                }
            }
        };
        auto place_vectors = [&] {
            if constexpr (OUT8) {
                cp_async_wait_all();
                __syncwarp();
                const uint2 u = *reinterpret_cast<const uint2 *>(gate + 2 * lane);
                *reinterpret_cast<float4 *>(bias + 4 * lane) =
                    make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                                __uint_as_float(u.y & 0xFFFF0000u));
            } else {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    bias[32 * i + lane] = vb[i];
                    if constexpr (EPI == kEpiResid) gate[32 * i + lane] = vg[i];
                }
            }
            __syncwarp();
        };
        griddep_wait();
        if (more) load_vectors();
        uint32_t tmem = 0;
        if (!more) cluster_wait();  // (every warp waits once)
#pragma unroll 1
        for (int it = 0; more; ++it) {
            const int slice = unit_slice(), width = unit_width(), c0 = half * width;
            const int col0 = n0 + (int)pair * slice + c0;
            o.row = m0 + (int)rank * 128 + q * 32;
            const bool mine = o.row < p.M && c0 < slice && col0 < p.N;
            place_vectors();
            // the half that holds the 24 columns which the other accumulator shares, the
            // last ones of a full first accumulator or the first of the second, reads
            // them first
            const bool from_end = !SPLIT && !LONG && bn == 256 && (it & 1) == 0;
            const bool shares = half == (from_end ? 1 : 0);
            more = U.next(t, ncl, m0, n0, bn);
            if (more) load_vectors();
            if (it == 0) cluster_wait();
            if (it == 0 && !warp_wait(tmem_here, 0, abort_flag, p.err)) break;
            if constexpr (LONG) {
                // All pieces but the last: this warp's columns of both slices are added up.
                if (it == 0) tmem = *tmem_holder + ((uint32_t)(q * 32) << 16);
                bool ok = true;
                const int last = it + (kb_n - kb_0 - 1) / p.piece_kb;
#pragma unroll 1
                for (const int first = it; it < last; ++it) {
                    ok = warp_wait(&accf[it & 1], (it >> 1) & 1, abort_flag, p.err);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = c0; c < c0 + width && c0 < slice; c += 32)
#pragma unroll 1
                        for (int h = 0; h < (SPLIT ? 2 : 1); ++h) {
                            const uint32_t x = tmem + (uint32_t)(h * slice + c);
                            uint32_t r[32];
                            tmem_ld32(x + (it & 1 ? kAcc1 : 0u), r);
                            wait_chunk(r);
                            if (it != first) add_sum(r, x + kSumCols);
                            tmem_st32(x + kSumCols, r);
                        }
                    tmem_wait_st();
                    arrive(acce_c + 8u * (uint32_t)(it & 1));
                }
                if (!ok) break;
            }
            const int buf = it & 1;
            if (!warp_wait(&accf[buf], (it >> 1) & 1, abort_flag, p.err)) break;
            tc_fence_after();
            if (!LONG && it == 0) tmem = *tmem_holder + ((uint32_t)(q * 32) << 16);
            const uint32_t acc = tmem + (buf ? kAcc1 : 0u) + (uint32_t)pair * slice + c0;
            const uint32_t sum = tmem + kSumCols + (uint32_t)pair * slice + c0;  // LONG
            // partial sums of this lane's row and this warp's columns: 16 bytes (4 columns)
            // every 128 rows
            const uint32_t part = 16u * (uint32_t)(q * 32 + lane) + 512u * (uint32_t)c0;
            if constexpr (SPLIT) {
                const uint32_t other = crank ^ 2u;  // the other pair's CTA of these rows
                // this CTA's stages, which the MMAs have read, may be written by the other one
                if (warp == 4 && lane == 0) mbar_arrive_cluster(mapa_shared(smem_u32(other_done), other));
                __syncwarp();
                if (!warp_wait_cluster(other_done, 0, abort_flag, p.err)) break;
                if (c0 < slice) {
                    const uint32_t from = (uint32_t)((pair ^ 1) * slice + c0), dst = mapa_shared(smem_u32(sa) + part, other);
#pragma unroll 1
                    for (int c = 0; c < width; c += 32) {
                        uint32_t r[32];
                        tmem_ld32(tmem + (buf ? kAcc1 : 0u) + from + c, r);
                        wait_chunk(r);
                        if constexpr (LONG) add_sum(r, tmem + kSumCols + from + c);
#pragma unroll
                        for (int j = 0; j < 32; j += 4)
                            store_cluster16(dst + 512u * (uint32_t)(c + j), r[j], r[j + 1], r[j + 2], r[j + 3]);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(mapa_shared(smem_u32(parts), other));
                if (!warp_wait_cluster(parts, 0, abort_flag, p.err)) break;
            }
            // adds the earlier pieces' and the other pair's sums of columns c .. c + 31
            auto join = [&](uint32_t (&r)[32], int c) {
                if constexpr (LONG) add_sum(r, sum + c);
                if constexpr (SPLIT) {
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 v = *reinterpret_cast<const float4 *>(sa + part + 512 * (c + j));
                        const f32x2 x0 = fadd2({__uint_as_float(r[j]), __uint_as_float(r[j + 1])}, {v.x, v.y});
                        const f32x2 x1 = fadd2({__uint_as_float(r[j + 2]), __uint_as_float(r[j + 3])}, {v.z, v.w});
                        r[j] = __float_as_uint(x0.x), r[j + 1] = __float_as_uint(x0.y);
                        r[j + 2] = __float_as_uint(x1.x), r[j + 3] = __float_as_uint(x1.y);
                    }
                }
            };
            if (!mine) {
                if (kShared && shares) arrive(shared_c);
                if (kReuse) arrive(acce_c + 8u * (uint32_t)buf);
                continue;
            }
            if constexpr (OUT8) {
                // The 128 columns are one scale block of this lane's row.  The chunk with the
                // shared columns comes first; f has the chunks in the order of their reading.
                auto chunk = [&](int i) { return from_end ? (i + 3) & 3 : i; };
                float f[128];  // columns behind N: GELU of zero sums without a bias
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t r[32];
                    tmem_ld32(acc + 32 * chunk(i), r);
                    wait_chunk(r);
                    if (kShared && i == 0 && shares) arrive(shared_c);
                    if (kReuse && i == 3) arrive(acce_c + 8u * (uint32_t)buf);
                    join(r, 32 * chunk(i));
                    apply<EPI>(r, bias + 32 * chunk(i), gate);
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[32 * i + j] = __uint_as_float(r[j]);
                }
                const uint32_t byte = quantize_block<128, 1>(f);
                if (o.row + lane < p.M) p.out_scales[(int64_t)(o.row + lane) * p.ldo_s + col0 / kScaleBlock] = (uint8_t)byte;
                o.begin();
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float *x = f + 32 * i + 16 * h;
                        o.put16(2 * chunk(i) + h,
                                make_uint4(pack_e4m3x4(x[0], x[1], x[2], x[3]), pack_e4m3x4(x[4], x[5], x[6], x[7]),
                                           pack_e4m3x4(x[8], x[9], x[10], x[11]), pack_e4m3x4(x[12], x[13], x[14], x[15])));
                    }
                o.template send<false>(col0);
            } else {
                const int chunks = width / 32;
                auto at = [&](int i) { return 32 * (from_end ? chunks - 1 - i : i); };
                // 32 columns: a box of fp32, half a box of bf16
                auto finish = [&](uint32_t (&r)[32], int c) {
                    if (col0 + c >= p.N) return;
                    join(r, c);
                    apply<EPI>(r, bias + c, gate + c);
                    if constexpr (EPI == kEpiResid) {
                        // x += gate y as an fp32 reduce-add of gate y
                        o.begin();
#pragma unroll
                        for (int i = 0; i < 8; ++i) o.put16(i, make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]));
                        o.template send<true>(col0 + c);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float *x = reinterpret_cast<const float *>(r + 8 * i);
                            o.put16(((c >> 3) & 4) + i, make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                                                   pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])));
                        }
                    }
                };
                // the next chunk's load runs while a chunk is worked on
                uint32_t a[32], b[32];
                tmem_ld32(acc + at(0), a);
                wait_chunk(a);
                if (kShared && shares) arrive(shared_c);
#pragma unroll 1
                for (int i = 0; i < chunks; i += 2) {
                    if (i + 1 < chunks)
                        tmem_ld32(acc + at(i + 1), b);
                    else if (kReuse)
                        arrive(acce_c + 8u * (uint32_t)buf);
                    if constexpr (EPI != kEpiResid) o.begin();
                    finish(a, at(i));
                    if (i + 1 < chunks) {
                        wait_chunk(b);
                        if (i + 2 < chunks)
                            tmem_ld32(acc + at(i + 2), a);
                        else if (kReuse)
                            arrive(acce_c + 8u * (uint32_t)buf);
                        finish(b, at(i + 1));
                        if (i + 2 < chunks) wait_chunk(a);
                    }
                    if constexpr (EPI != kEpiResid) o.template send<false>(col0 + (at(i) & ~63));
                }
            }
        }
        if (lane == 0) bulk_wait_all();
        __syncwarp();
    } else {
        // copies the even CTA's and its peer's sets of scales into tensor memory, by turns into
        // the half that the set before the last had, when its MMAs are over
        cluster_wait();
        griddep_wait();
        if (lane == 0) {
            const uint32_t there = mapa_shared(smem_u32(tmem_there), even);
            if (rank == 0)
                mbar_arrive_own_smem(there);  // (and tmem_holder)
            else
                mbar_arrive_relaxed(there);
            mbar_arrive(tmem_here);
        }
        __syncwarp();
        if (rank != 0) {
            // The odd CTA's scales are published to the even one, whose tensor core reads them, by a
            // release at cluster scope: here, where no loads are in flight for it to wait for (by the
            // scale warp itself 1229 x 1024 x 4096 12.5 us instead of 12.0).
            const uint32_t sfull_c = mapa_shared(smem_u32(sfull), even);
            int n = 0;
            bool ok = true;
#pragma unroll 1
            for (; more && ok; more = U.next(t, ncl, m0, n0, bn)) {
#pragma unroll 1
                for (int kb = kb_0; kb < kb_n; kb += 4, ++n) {
                    const int b = n % kSets;
                    ok = warp_wait(&sfull[b], (n / kSets) & 1, abort_flag, p.err);
                    if (!ok) break;
                    if (lane == 0) mbar_arrive_cluster(sfull_c + 8u * (uint32_t)b);
                    __syncwarp();
                }
            }
        } else if (warp_wait(tmem_there, 0, abort_flag, p.err)) {
            tc_fence_after();
            // 32 rows of 16 bytes: groups of 8 rows are 128 bytes apart
            const uint64_t s_desc0 = make_sdesc(smem_u32(ss), 16, 128, kSwizzleNone);
            const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_holder, 0);
            int n = 0;
            bool ok = true;
#pragma unroll 1
            for (; more && ok; more = U.next(t, ncl, m0, n0, bn)) {
#pragma unroll 1
                for (int kb = kb_0; kb < kb_n; kb += 4, ++n) {
                    const int b = n % kSets, h = n & 1;
                    ok = warp_wait_cluster(&sfull[b], (n / kSets) & 1, abort_flag, p.err) &&
                         (n < 2 || warp_wait(&tempty[h], ((n >> 1) & 1) ^ 1, abort_flag, p.err));
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t sd = s_desc0 + (uint64_t)b * (kSetBytes >> 4);
                    const uint32_t col = tmem + kScaleCols + 12u * (uint32_t)h;
                    tmem_cp_scales_pair(col, sd);
                    tmem_cp_scales_pair(col + 4, sd + (512 >> 4));
                    tmem_cp_scales_pair(col + 8, sd + (1024 >> 4));
                    mma_commit_pair_elect(&tfull[h]);
                    mma_commit_pair_mc_elect(&sempty[b], both);
                }
            }
            // the last commits to tempty, which no further set waits for
            for (int i = n > 2 ? n : 2; i < n + 2 && ok; ++i) ok = warp_wait(&tempty[i & 1], ((i >> 1) & 1) ^ 1, abort_flag, p.err);
            if (*abort_flag) {
                mma_commit_pair_elect(&drain[1]);
                if (lane == 0) wait_ns8(&drain[1], 0, 100000000ull);
                __syncwarp();
            }
        }
    }
    // No CTA leaves while another may still signal its barriers, (an even CTA's MMAs) write
    // its TMEM or (SPLIT) its shared memory.  All of that has been awaited above, and nothing
    // is published here: a release, which waits for the warp's stores, took 1000 clocks.
    tc_fence_before();
    cluster_arrive_relaxed();
    cluster_wait();
    if (*abort_flag) spin_ns(200000);  // loads in flight land
    if (warp == 3) {
        tc_fence_after();
        tmem_dealloc_pair(*tmem_holder, kTmemCols8);
    }
}

// Resident clusters of 2 (SPLIT: 4) CTAs on the current device.  They are counted, and the
// kernel's shared-memory attribute set, on each device's first launch (0 = not yet).
template <int EPI, bool OUT8, bool SPLIT, bool LONG>
cudaError_t resident8(int *clusters)
{
    static std::atomic<int> max_clusters_of[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    *clusters = max_clusters_of[dev & 63].load(std::memory_order_acquire);
    if (*clusters) return cudaSuccess;
    e = cudaFuncSetAttribute(k_gemm8_pair<EPI, OUT8, SPLIT, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem8);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = SPLIT ? 4 : 2;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(SPLIT ? 4 : 2);
    cfg.blockDim = dim3(kThreads8);
    cfg.dynamicSmemBytes = kMostSmem8;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, k_gemm8_pair<EPI, OUT8, SPLIT, LONG>, &cfg);
    if (e != cudaSuccess) return e;
    if (n < 1) return cudaErrorInvalidConfiguration;
    max_clusters_of[dev & 63].store(n, std::memory_order_release);
    *clusters = n;
    return cudaSuccess;
}

template <int EPI, bool OUT8, bool SPLIT, bool LONG>
cudaError_t launch_units8(const CUtensorMap *ta, const GemmPairB *tb, const CUtensorMap *to, const Gemm8Params &p,
                          const Units8 &u, int width, int clusters, cudaStream_t s)
{
    const Depth8 depth = depth8(width);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = SPLIT ? 4 : 2;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((SPLIT ? 4u : 2u) * (unsigned)clusters);
    cfg.blockDim = dim3(kThreads8);
    cfg.dynamicSmemBytes = depth.smem();
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_gemm8_pair<EPI, OUT8, SPLIT, LONG>, *ta, *tb, *to, u, depth, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}

// Width of the units of a split sum, 0: the sum is not split.  Few tiles leave clusters
// idle that may take half of the K: it costs 2 us with units of 128 columns, 4.5 with 256
// (64 KB per CTA change places), and saves 0.09 us per 128 K.  Whole / split, us:
//   300 x 1024 (units of 128) x 3200 9.2 / 9.6, x 4096 10.5 / 9.5, x 8192 16.7 / 12.7; 1229 x
//   1024 (256) x 4096 11.2 / 12.8, x 8192 17.8 to 19.2 / 17.4 to 18.1, x 16384 35.2 / 26.8; 600 x
//   1024 with 8-bit output, which needs whole scale blocks, x 8192 17.2 / 16.4, x 16384 34.7 / 26.0.
constexpr int kSplitBlocks = 24;  // no sum of fewer scale blocks is split
int split_width8(int M, int N, int kb_n, bool out8, int max_clusters)
{
    const int64_t tiles = (((int64_t)M + 255) / 256) * (((int64_t)N + 255) / 256);
    if (kb_n >= kSplitBlocks && !out8 && 2 * tiles <= max_clusters) return 128;
    return kb_n >= (out8 ? 56 : 80) && tiles <= max_clusters ? 256 : 0;
}

// A pair's sum of kb blocks, more than piece_most, is taken in pieces of that length or a little
// less.  Every MMA adds 32 K to the accumulator and drops what is below its last bit, downwards
// in magnitude (at most 2^-23), so the error of a sum of one sign grows with its length, and
// faster than that: 0.9e-6 at 4096 K, 4.8e-6 at 16384, 2.6e-5 at 65536, 1.6e-4 at 262144.
// Outputs of 16 and 8 bits, whose own rounding is 4e-3 and more, take 65536 K at once, fp32
// ones 16384: pieces have units of 128 columns only (4096 x 4096 x 32768 470 us instead of 366; of
// few tiles, narrow anyway, as long as before: 300 x 1024 x 65536 69 us).
template <int EPI>
constexpr int piece_most = EPI == kEpiResid ? 128 : 512;
inline int piece_blocks(int kb, int most)
{
    const int pieces = (kb - 1) / most + 1;
    return ((kb - 1) / pieces / 4 + 1) * 4;  // whole scale sets
}

template <int EPI, bool OUT8, bool SPLIT, bool LONG>
cudaError_t launch_sum8(const CUtensorMap *ta, const GemmPairB *tb, const CUtensorMap *to, Gemm8Params p, int width, cudaStream_t s)
{
    int max_clusters = 0;
    const cudaError_t e = resident8<EPI, OUT8, SPLIT, LONG>(&max_clusters);
    if (e != cudaSuccess) return e;
    Units8 u;
    const int n = u.set_single(p.M, p.N, width);
    // (a cluster of two pairs takes one unit)
    return launch_units8<EPI, OUT8, SPLIT, LONG>(ta, tb, to, p, u, width, SPLIT || n < max_clusters ? n : max_clusters, s);
}

template <int EPI, bool OUT8>
cudaError_t launch_one8(const CUtensorMap *ta, const GemmPairB *tb, const CUtensorMap *to, Gemm8Params p, cudaStream_t s)
{
    int max_clusters = 0;
    const int kb_n = (p.K + 127) / 128;
    cudaError_t e;
    if (kb_n >= kSplitBlocks) {
        e = resident8<EPI, OUT8, true, false>(&max_clusters);
        if (e != cudaSuccess) return e;
        const int width = split_width8(p.M, p.N, kb_n, OUT8, max_clusters);
        const int half = ((kb_n + 1) / 2 + 3) / 4 * 4;
        const bool pieces = half > piece_most<EPI>;
        if (width && !(pieces && width == 256)) {  // (pieces of 256 columns have no place in tensor memory)
            p.split_kb = half;
            // the second pair's scale bytes start there: they are read as far as that is aligned
            while (p.split_kb % (4 * p.scale_sets) != 0) p.scale_sets /= 2;
            if (!pieces) return launch_sum8<EPI, OUT8, true, false>(ta, tb, to, p, width, s);
            if constexpr (!OUT8) {
                p.piece_kb = piece_blocks(half, piece_most<EPI>);
                return launch_sum8<EPI, OUT8, true, true>(ta, tb, to, p, width, s);
            }
        }
    }
    if (kb_n > piece_most<EPI>) {
        p.piece_kb = piece_blocks(kb_n, piece_most<EPI>);
        return launch_sum8<EPI, OUT8, false, true>(ta, tb, to, p, 128, s);
    }
    e = resident8<EPI, OUT8, false, false>(&max_clusters);
    if (e != cudaSuccess) return e;
    // units: 64 columns (128 with 8-bit output) are the smallest
    constexpr int width = OUT8 ? 128 : 64;
    const int64_t units = (((int64_t)p.M + 255) / 256) * (((int64_t)p.N + width - 1) / width);
    const int clusters = units < max_clusters ? (int)units : max_clusters;
    Units8 u;
    u.set(p.M, p.N, clusters, width);
    return launch_units8<EPI, OUT8, false, false>(ta, tb, to, p, u, u.full ? 256 : 256 / u.sub, clusters, s);
}

}  // namespace

cudaError_t launch_gemm8_pair(const CUtensorMap *ta, const GemmPairB *tb, const CUtensorMap *to, const Gemm8Params &p, int epi, bool out8,
                              cudaStream_t s)
{
    switch (epi) {
    case kEpiBias: return out8 ? launch_one8<kEpiBias, true>(ta, tb, to, p, s) : launch_one8<kEpiBias, false>(ta, tb, to, p, s);
    case kEpiGelu: return out8 ? launch_one8<kEpiGelu, true>(ta, tb, to, p, s) : launch_one8<kEpiGelu, false>(ta, tb, to, p, s);
    case kEpiResid: return out8 ? cudaErrorInvalidValue : launch_one8<kEpiResid, false>(ta, tb, to, p, s);
    default: return cudaErrorInvalidValue;
    }
}

}  // namespace f3dc
