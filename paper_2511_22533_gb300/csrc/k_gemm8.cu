// k_gemm8.cu -- the matrix product of 8-bit linear layers (f3dc_gemm_fp8):
//
//   out[m, n] = epilogue( sum_k A[m, k] 2^ea[m, k / 128] B[n, k] 2^eb[n, k / 128] )
//
// A [M, K] and B [N, K] e4m3 with one power-of-two scale per row and block of 128 K.
//
// The scales go into the tensor cores: kind::mxf8f6f4 with block scales multiplies
// every 32 K of a row by a scale byte held in tensor memory, so the whole K is one
// fp32 sum in one accumulator and nothing is rescaled in registers.  A block of 128
// is four MMAs that take the same byte; one 32-bit column of scales serves 512 K.
//
// Clusters of two CTAs (cta_group::2), persistent over tiles of 256 x 256 (narrower
// ones in the last wave), 384 threads:
//   warp 0      TMA producer: this CTA's 128 rows of A and half of the tile's rows of
//               B, 128 K (one 128-byte swizzled line per row) per stage
//   warp 1      of the even CTA issues the copies of scales and the MMAs for both
//   warp 2      reads scale bytes from global memory (plain rows) and lays them out
//               for the tensor memory: 512 K of A's 128 and B's 256 rows at a time
//   warp 3      allocates tensor memory
//   warps 4-11  epilogue, two groups of four (one warp per TMEM lane quarter)
// Tensor memory: 512 columns hold two accumulators of 256 only if nothing else is
// there, but two sets of scales need 24.  So the second accumulator starts at column
// 232: the tile after may begin as soon as the epilogue has read the 24 columns that
// the two share, which it reads first.
#include <atomic>

#include <cudaTypedefs.h>

#include "kernels.h"
#include "mx8.cuh"

namespace f3dc {

namespace {

constexpr int kThreads8 = 384;
constexpr int kBK8 = 128;                   // K of a stage: one scale block
constexpr int kStages8 = 5;
constexpr int kOperand8 = 128 * kBK8;       // 128 rows of A, or up to 128 of B, per CTA
constexpr int kStageScales = 512 + 1024;    // A's 128 rows, B's 256, four scale bytes each
constexpr int kOutBuf8 = 128 * 64;          // staged output: 128 rows of 64 bytes
constexpr int kOutBytes8 = 2 * 2 * kOutBuf8;
constexpr uint32_t kTmemCols8 = 512;
constexpr uint32_t kAcc1 = 232;             // first column of the second accumulator
constexpr uint32_t kScaleCols = 488;        // two sets of 4 (A) + 8 (B) columns
constexpr size_t kSmem8 = 1024 + (size_t)kStages8 * 2 * kOperand8 + kOutBytes8 + 2 * kStageScales + 256;

// Work units: full waves of 256 x 256 tiles, the tiles left for the last wave cut into
// 2 or 4 pieces of 128 or 64 columns where there are clusters for all of them.  Units run
// column-fastest.  A tile's columns behind N are not computed but for the rounding up
// of its width to 64, 128 or 256.
struct Units8 {
    int line, full, sub, total, N, min_width;
    F3DC_DEV Units8(int M, int N_, int clusters, int min_width_) : N(N_), min_width(min_width_)
    {
        line = (N + 255) / 256;
        const int tiles = ((M + 255) / 256) * line;
        full = tiles / clusters * clusters;
        const int rest = tiles - full;
        sub = 4 * rest <= clusters && min_width <= 64 ? 4 : (2 * rest <= clusters ? 2 : 1);
        total = full + rest * sub;
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
        const int m = tile / line;
        m0 = m * 256;
        n0 = (tile - m * line) * 256 + piece * bn;
        const int left = N - n0;
        bn = left <= 0 ? 0 : min(bn, left <= min_width ? min_width : (left <= 128 ? 128 : 256));
    }
};

F3DC_DEV bool wait_ns8(uint64_t *bar, uint32_t parity, uint64_t ns)
{
    const uint64_t t0 = globaltimer();
    while (!mbar_try_wait(bar, parity))
        if (globaltimer() - t0 > ns) return false;
    return true;
}

// Staged output of a group of four epilogue warps: boxes of 128 rows x 64 bytes, the
// 16-byte piece c of row r at 64 r + 16 (c ^ ((r / 2) % 4)) (TMA 64B swizzle), in two
// buffers; the issuer sends a box when all four warps have written it and waits
// before the next is written until the store of the one before has been read.
struct Stage8 {
    uint8_t *buf;
    const CUtensorMap *map;
    int row, bar;
    bool issuer;
    int ck;
    F3DC_DEV void put16(int c, uint4 u) const
    {
        *reinterpret_cast<uint4 *>(buf + (ck & 1) * kOutBuf8 + row * 64 + ((c ^ ((row >> 1) & 3)) << 4)) = u;
    }
    template <bool kReduce>
    F3DC_DEV void emit(int x, int y)
    {
        fence_proxy_async_smem();
        if (issuer) bulk_wait_read<0>();
        asm volatile("bar.sync %0, 128;" ::"r"(bar) : "memory");
        if (issuer) {
            if (kReduce)
                tma_reduce_add_2d(map, buf + (ck & 1) * kOutBuf8, x, y);
            else
                tma_store_2d(map, buf + (ck & 1) * kOutBuf8, x, y);
            bulk_commit();
        }
        ++ck;
    }
};

// Adds the biases of 32 columns to v (N is a multiple of 8; columns from N on get none).
F3DC_DEV void add_bias(const Gemm8Params &p, int col, float (&v)[32])
{
    if (!p.bias) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (col + 8 * q >= p.N) break;
        const uint4 u = __ldg(reinterpret_cast<const uint4 *>(p.bias + col) + q);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[8 * q + 2 * j] += bf16_bits_to_f32(w[j] & 0xFFFFu);
            v[8 * q + 2 * j + 1] += __uint_as_float(w[j] & 0xFFFF0000u);
        }
    }
}

F3DC_DEV void load_acc(uint32_t taddr, float (&v)[32])
{
    uint32_t r[32];
    tmem_ld32(taddr, r);
    tmem_wait_ld();
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}

template <int EPI, bool OUT8>
__global__ void __launch_bounds__(kThreads8, 1)
    k_gemm8_pair(const __grid_constant__ CUtensorMap tma, const __grid_constant__ GemmPairB tmb,
                 const __grid_constant__ CUtensorMap tmo, const Gemm8Params p)
{
    constexpr int S = kStages8;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *sa = smem;
    uint8_t *sb = sa + S * kOperand8;
    uint8_t *so = sb + S * kOperand8;
    uint8_t *ss = so + kOutBytes8;
    uint64_t *bars = reinterpret_cast<uint64_t *>(ss + 2 * kStageScales);
    uint64_t *full = bars, *empty = full + S;          // operands of a stage there (even CTA) / used (both)
    uint64_t *sfull = empty + S, *sempty = sfull + 2;  // scales of a set there (even CTA) / used (both)
    uint64_t *accf = sempty + 2, *acce = accf + 2;     // accumulator complete (both) / read (even CTA)
    uint64_t *shared_read = acce + 2;                  // its columns that the next one needs are read (even CTA)
    uint64_t *drain = shared_read + 1;
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(drain + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = __shfl_sync(0xffffffffu, cluster_rank(), 0);
    griddep_launch();

    if (threadIdx.x == 64) {
        tma_prefetch(&tma);
        for (int i = 0; i < 3; ++i) tma_prefetch(&tmb.rows[i]);
        tma_prefetch(&tmo);
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sfull[b], 2);   // one scale warp in each CTA
            mbar_init(&sempty[b], 1);
            mbar_init(&accf[b], 1);
            mbar_init(&acce[b], 16);   // eight epilogue warps in each CTA
        }
        mbar_init(shared_read, 8);     // the group of four that holds the columns, in each CTA
        mbar_init(drain, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 3) {
        tmem_alloc_pair(tmem_holder, kTmemCols8);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    cluster_sync();  // both CTAs' barriers are initialised before any remote signal
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_holder, 0);
    const int kb_n = (p.K + kBK8 - 1) / kBK8;
    const int cl = blockIdx.x >> 1, ncl = gridDim.x >> 1;
    const Units8 U(p.M, p.N, ncl, OUT8 ? 128 : 64);
    griddep_wait();

    if (warp == 0) {
        if (lane == 0) {
            const uint32_t full_c = mapa_shared(smem_u32(full), 0);
            int s = 0;
            uint32_t ph = 0;
            bool ok = true;
#pragma unroll 1
            for (int t = cl; t < U.total && ok; t += ncl) {
                int m0, n0, bn;  // this CTA holds bn / 2 of the unit's B rows
                U.decode(t, m0, n0, bn);
                if (bn == 0) continue;
                const CUtensorMap *mb = &tmb.rows[bn == 256 ? 0 : (bn == 128 ? 1 : 2)];
                const uint32_t bytes = 2u * (kOperand8 + (uint32_t)(bn / 2) * kBK8);  // both CTAs
#pragma unroll 1
                for (int kb = 0; kb < kb_n; ++kb) {
                    if (!mbar_wait(&empty[s], ph ^ 1, abort_flag, p.err)) {
                        ok = false;
                        break;
                    }
                    if (rank == 0) mbar_arrive_expect_tx(&full[s], bytes);
                    const uint32_t fb = full_c + 8u * (uint32_t)s;
                    tma_load_2d_pair(sa + s * kOperand8, &tma, kb * kBK8, m0 + (int)rank * 128, fb);
                    tma_load_2d_pair(sb + s * kOperand8, mb, kb * kBK8, n0 + (int)rank * (bn / 2), fb);
                    if (++s == S) {
                        s = 0;
                        ph ^= 1;
                    }
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const uint64_t a_desc0 = make_sdesc(smem_u32(sa), 16, 1024, kSwizzle128);
            const uint64_t b_desc0 = make_sdesc(smem_u32(sb), 16, 1024, kSwizzle128);
            // 32 rows of 16 bytes: groups of 8 rows are 128 bytes apart
            const uint64_t s_desc0 = make_sdesc(smem_u32(ss), 16, 128, kSwizzleNone);
            int s = 0, it = 0, set = 0;
            uint32_t ph = 0, sph = 0;
            bool ok = true;
#pragma unroll 1
            for (int t = cl; t < U.total && ok; t += ncl) {
                int m0, n0, bn;
                U.decode(t, m0, n0, bn);
                if (bn == 0) continue;
                const int buf = it & 1;
                if (!warp_wait(&acce[buf], ((it >> 1) & 1) ^ 1, abort_flag, p.err)) break;
                if (it > 0 && !warp_wait(shared_read, (it - 1) & 1, abort_flag, p.err)) break;
                tc_fence_after();
                const uint32_t d = tmem + (buf ? kAcc1 : 0u);
                const uint32_t idesc0 = make_idesc_mxf8(256, 0, 0) | ((uint32_t)(bn >> 3) << 17);
#pragma unroll 1
                for (int kb = 0; kb < kb_n; ++kb) {
                    const uint32_t sfa = tmem + kScaleCols + 12u * (uint32_t)set, sfb = sfa + 4;
                    if ((kb & 3) == 0) {
                        // this set's last use is over: its scales were written after the wait for that
                        if (!warp_wait(&sfull[set], sph, abort_flag, p.err)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        const uint64_t sd = s_desc0 + (uint64_t)set * (kStageScales >> 4);
                        tmem_cp_scales_pair(sfa, sd);
                        tmem_cp_scales_pair(sfb, sd + (512 >> 4));
                        if (bn > 128) tmem_cp_scales_pair(sfb + 4, sd + (1024 >> 4));
                    }
                    if (!warp_wait(&full[s], ph, abort_flag, p.err)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t byte = (uint32_t)(kb & 3);
                    mma_mxf8_pair_128k(d, a_desc0 + (uint64_t)s * (kOperand8 >> 4), b_desc0 + (uint64_t)s * (kOperand8 >> 4),
                                       sfa, sfb, idesc0 | byte << 4 | byte << 29, kb != 0);
                    mma_commit_pair_mc_elect(&empty[s], 3);
                    if ((kb & 3) == 3 || kb + 1 == kb_n) {
                        mma_commit_pair_mc_elect(&sempty[set], 3);
                        set ^= 1;
                        if (set == 0) sph ^= 1;
                    }
                    if (++s == S) {
                        s = 0;
                        ph ^= 1;
                    }
                }
                if (ok) mma_commit_pair_mc_elect(&accf[buf], 3);
                ++it;
            }
        }
    } else if (warp == 2) {
        // lane l: rows l, l + 32, l + 64, l + 96 of each 128, four scale bytes (512 K) of each
        const uint32_t sfull_c = mapa_shared(smem_u32(sfull), 0);
        int set = 0;
        uint32_t ph = 0;
        bool ok = true;
        auto four = [&](const uint8_t *sc, int64_t ld, int row0, int rows, int byte) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = row0 + 32 * j + lane;
                w[j] = r < rows ? *reinterpret_cast<const uint32_t *>(sc + r * ld + byte) : 0x7F7F7F7Fu;
            }
            return make_uint4(w[0], w[1], w[2], w[3]);
        };
#pragma unroll 1
        for (int t = cl; t < U.total && ok; t += ncl) {
            int m0, n0, bn;
            U.decode(t, m0, n0, bn);
            if (bn == 0) continue;
#pragma unroll 1
            for (int kb = 0; kb < kb_n; kb += 4) {
                const uint4 wa = four(p.sa, p.lda_s, m0 + (int)rank * 128, p.M, kb);
                const uint4 wb0 = four(p.sb, p.ldb_s, n0, p.N, kb);
                uint4 wb1 = wb0;
                if (bn > 128) wb1 = four(p.sb, p.ldb_s, n0 + 128, p.N, kb);
                if (!warp_wait(&sempty[set], ph ^ 1, abort_flag, p.err)) {
                    ok = false;
                    break;
                }
                uint4 *dst = reinterpret_cast<uint4 *>(ss + set * kStageScales) + lane;
                dst[0] = wa;
                dst[32] = wb0;
                dst[64] = wb1;
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(sfull_c + 8u * (uint32_t)set);
                set ^= 1;
                if (set == 0) ph ^= 1;
            }
        }
    } else if (warp >= 4) {
        const int q = warp & 3, grp = (warp - 4) >> 2;
        const int row = q * 32 + lane;
        Stage8 o{so + grp * 2 * kOutBuf8, &tmo, row, 1 + grp, (int)threadIdx.x == 128 + 128 * grp, 0};
        const uint32_t acce_c = mapa_shared(smem_u32(acce), 0), shared_c = mapa_shared(smem_u32(shared_read), 0);
        auto arrive = [&](uint32_t bar) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(bar);
        };
        int it = 0;
#pragma unroll 1
        for (int t = cl; t < U.total; t += ncl) {
            int m0, n0, bn;
            U.decode(t, m0, n0, bn);
            if (bn == 0) continue;
            m0 += (int)rank * 128;
            const int buf = it & 1;
            // the group's warps meet at barriers below: they take the wait's outcome together
            const uint32_t got = mbar_wait(&accf[buf], (it >> 1) & 1, abort_flag, p.err) ? 1u : 0u;
            uint32_t all;
            asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.and.pred q, %2, 128, p;\n"
                         " selp.u32 %0, 1, 0, q;\n}\n"
                         : "=r"(all)
                         : "r"(got), "r"(o.bar)
                         : "memory");
            if (!all) break;
            tc_fence_after();
            const uint32_t acc = tmem + ((uint32_t)(q * 32) << 16) + (buf ? kAcc1 : 0u);
            // the group whose first chunk covers the 24 columns that the other
            // accumulator shares: the last ones of a full first accumulator, the
            // first ones of the second
            const bool from_end = bn == 256 && buf == 0;
            const bool shares = grp == (from_end ? 1 : 0);
            const bool rows = m0 < p.M;  // the odd CTA's rows may lie behind M
            if constexpr (OUT8) {
                // group g has columns 128 g .. 128 g + 127: a scale block of each row
                const int c0 = 128 * grp;
                if (rows && c0 < bn) {
                    float v[128];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float w[32];
                        load_acc(acc + c0 + 32 * k, w);
                        add_bias(p, n0 + c0 + 32 * k, w);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[32 * k + j] = EPI == kEpiGelu ? gelu_tanh(w[j]) : w[j];
                    }
                    if (shares) arrive(shared_c);
                    arrive(acce_c + 8u * (uint32_t)buf);
                    const int col = n0 + c0;
                    const uint32_t byte = quantize_block<128, 1>(v);
                    if (m0 + row < p.M && col < p.N)
                        p.out_scales[(int64_t)(m0 + row) * p.ldo_s + col / kScaleBlock] = (uint8_t)byte;
                    // one box of 128 rows x 128 bytes (128B swizzle) over both buffers
                    if (o.issuer) bulk_wait_read<0>();
                    asm volatile("bar.sync %0, 128;" ::"r"(o.bar) : "memory");
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        uint4 u;
                        u.x = pack_e4m3x4(v[16 * c], v[16 * c + 1], v[16 * c + 2], v[16 * c + 3]);
                        u.y = pack_e4m3x4(v[16 * c + 4], v[16 * c + 5], v[16 * c + 6], v[16 * c + 7]);
                        u.z = pack_e4m3x4(v[16 * c + 8], v[16 * c + 9], v[16 * c + 10], v[16 * c + 11]);
                        u.w = pack_e4m3x4(v[16 * c + 12], v[16 * c + 13], v[16 * c + 14], v[16 * c + 15]);
                        *reinterpret_cast<uint4 *>(o.buf + row * 128 + ((c ^ (row & 7)) << 4)) = u;
                    }
                    fence_proxy_async_smem();
                    asm volatile("bar.sync %0, 128;" ::"r"(o.bar) : "memory");
                    if (o.issuer && col < p.N) {
                        tma_store_2d(&tmo, o.buf, col, m0);
                        bulk_commit();
                    }
                } else {
                    if (shares) arrive(shared_c);
                    arrive(acce_c + 8u * (uint32_t)buf);
                }
            } else {
                const int chunks = rows ? bn / 32 : 0;
#pragma unroll 1
                for (int k = grp; k < chunks; k += 2) {
                    const int c0 = 32 * (from_end ? chunks - 1 - (k ^ 1) : k);
                    const int col = n0 + c0;
                    float v[32];
                    load_acc(acc + c0, v);
                    if (k == grp && shares) arrive(shared_c);
                    if (col >= p.N) continue;
                    add_bias(p, col, v);
                    if constexpr (EPI == kEpiGelu) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = gelu_tanh(v[j]);
                    }
                    if constexpr (EPI == kEpiResid) {
                        // x += gate y as an fp32 reduce-add of gate y, 16 columns per box
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int c = col + 16 * h + 4 * i;
                                const float *w = v + 16 * h + 4 * i;
                                const float4 g = p.gate && c < p.N ? __ldg(reinterpret_cast<const float4 *>(p.gate + c))
                                                                   : make_float4(1.f, 1.f, 1.f, 1.f);
                                o.put16(i, make_uint4(__float_as_uint(g.x * w[0]), __float_as_uint(g.y * w[1]),
                                                      __float_as_uint(g.z * w[2]), __float_as_uint(g.w * w[3])));
                            }
                            if (col + 16 * h < p.N) o.template emit<true>(col + 16 * h, m0);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint4 u;
                            u.x = pack_bf16x2(v[8 * i + 0], v[8 * i + 1]);
                            u.y = pack_bf16x2(v[8 * i + 2], v[8 * i + 3]);
                            u.z = pack_bf16x2(v[8 * i + 4], v[8 * i + 5]);
                            u.w = pack_bf16x2(v[8 * i + 6], v[8 * i + 7]);
                            o.put16(i, u);
                        }
                        o.template emit<false>(col, m0);
                    }
                }
                if (chunks == 0 && shares) arrive(shared_c);
                arrive(acce_c + 8u * (uint32_t)buf);
            }
            ++it;
        }
        if (o.issuer) bulk_wait_all();
    }
    __syncthreads();
    if (*abort_flag) {
        if (warp == 1 && rank == 0) {
            mma_commit_pair_elect(drain);  // the MMAs' issuing lane
            if (lane == 0) wait_ns8(drain, 0, 100000000ull);
        }
        if (threadIdx.x == 0) spin_ns(200000);
        __syncthreads();
    }
    // neither CTA leaves while the other may still signal its barriers or
    // (the even CTA's MMAs) write its TMEM
    cluster_sync();
    if (warp == 3) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, kTmemCols8);
    }
}

template <int EPI, bool OUT8>
cudaError_t launch_one8(const CUtensorMap *ta, const GemmPairB *tb, const CUtensorMap *to, const Gemm8Params &p,
                        cudaStream_t s)
{
    // per device: the shared-memory attribute and the resident-cluster count are
    // taken on each device's first launch (0 = not yet known)
    static std::atomic<int> max_clusters_of[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(kThreads8);
    cfg.dynamicSmemBytes = kSmem8;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int max_clusters = max_clusters_of[dev & 63].load(std::memory_order_acquire);
    if (!max_clusters) {
        e = cudaFuncSetAttribute(k_gemm8_pair<EPI, OUT8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem8);
        if (e != cudaSuccess) return e;
        int n = 0;
        e = cudaOccupancyMaxActiveClusters(&n, k_gemm8_pair<EPI, OUT8>, &cfg);
        if (e != cudaSuccess) return e;
        if (n < 1) return cudaErrorInvalidConfiguration;
        max_clusters = n;
        max_clusters_of[dev & 63].store(n, std::memory_order_release);
    }
    // units: 64 columns (128 with 8-bit output) are the smallest
    const int64_t width = OUT8 ? 128 : 64;
    const int64_t units = (((int64_t)p.M + 255) / 256) * ((p.N + width - 1) / width);
    const int clusters = units < max_clusters ? (int)units : max_clusters;
    cfg.gridDim = dim3(2 * clusters);
    cfg.stream = s;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, k_gemm8_pair<EPI, OUT8>, *ta, *tb, *to, p);
    if (e != cudaSuccess) return e;
    return cudaGetLastError();
}

}  // namespace

bool make_tmap_2d(CUtensorMap *map, CUtensorMapDataType type, const void *base, uint64_t rows, uint64_t cols,
                  uint64_t row_bytes, uint32_t box_rows, uint32_t box_cols, CUtensorMapSwizzle swizzle)
{
    static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> encoder{nullptr};
    PFN_cuTensorMapEncodeTiled_v12000 encode = encoder.load(std::memory_order_acquire);
    if (!encode) {
        cudaDriverEntryPointQueryResult q;
        void *fn = nullptr;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) !=
                cudaSuccess ||
            q != cudaDriverEntryPointSuccess || !fn)
            return false;
        encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
        encoder.store(encode, std::memory_order_release);
    }
    if (((uintptr_t)base & 15) != 0 || row_bytes % 16 != 0) return false;
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {row_bytes};
    cuuint32_t box[2] = {box_cols, box_rows};
    cuuint32_t estr[2] = {1, 1};
    return encode(map, type, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_gemm8_pair(const CUtensorMap *ta, const GemmPairB *tb, const CUtensorMap *to, const Gemm8Params &p,
                              int epi, bool out8, cudaStream_t s)
{
    switch (epi) {
    case kEpiBias: return out8 ? launch_one8<kEpiBias, true>(ta, tb, to, p, s) : launch_one8<kEpiBias, false>(ta, tb, to, p, s);
    case kEpiGelu: return out8 ? launch_one8<kEpiGelu, true>(ta, tb, to, p, s) : launch_one8<kEpiGelu, false>(ta, tb, to, p, s);
    case kEpiResid: return out8 ? cudaErrorInvalidValue : launch_one8<kEpiResid, false>(ta, tb, to, p, s);
    default: return cudaErrorInvalidValue;
    }
}

}  // namespace f3dc
