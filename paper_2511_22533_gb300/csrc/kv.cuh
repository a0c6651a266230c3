// kv.cuh -- device helpers of the paged 8-bit key / value cache (f3dc_kv_append_fp8,
// f3dc_kv_attention_fp8): a sequence's bounds, its pages, and conversions of e4m3.
#pragma once

#include <cuda_fp16.h>

#include <atomic>
#include <type_traits>

#include "kernels.h"
#include "mx8.cuh"

namespace f3dc {

// What has to succeed once on each device; a failure is tried again by the next call.
template <typename Ask>
cudaError_t once_per_device(std::atomic<uint64_t> &devices, Ask ask)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (devices.load(std::memory_order_acquire) & bit) return cudaSuccess;
    e = ask();
    if (e == cudaSuccess) devices.fetch_or(bit, std::memory_order_acq_rel);
    return e;
}

// Dynamic shared memory above 48 KB is asked for once per kernel and device.
template <typename Kernel>
cudaError_t ask_smem(Kernel kernel, int bytes, std::atomic<uint64_t> &devices)
{
    return once_per_device(devices, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
}

// Sequence b of a batch: its packed rows [row0, row0 + n) and the tokens of its pages.
// Bounds that the batch does not keep are reported and leave n = -1.
struct KvSeq {
    int row0, n, length;
};
F3DC_DEV KvSeq kv_seq(const KvBatch &t, const KvCache &c, int b, uint32_t *err)
{
    KvSeq s;
    s.row0 = t.row_start[b];
    s.n = t.row_start[b + 1] - s.row0;
    s.length = t.lengths[b];
    const bool ok = s.row0 >= 0 && s.n >= 0 && s.n <= t.max_rows && (int64_t)s.row0 + s.n <= t.rows && s.length >= 0 &&
                    s.length <= t.max_length && s.length <= t.table_stride * c.page;
    if (!ok) {
        raise_error(err, kDevBadIndex);
        s.n = -1;
    }
    return s;
}

// Page number j of sequence b, or -1 (reported) where it is not one of the pool's.
F3DC_DEV int kv_page(const KvBatch &t, const KvCache &c, int b, int j, uint32_t *err)
{
    const int p = t.table[(int64_t)b * t.table_stride + j];
    if ((uint32_t)p < (uint32_t)c.pages) return p;
    raise_error(err, kDevBadIndex);
    return -1;
}

// Where share i of n of `all` begins.
F3DC_DEV int kv_share(int all, int i, int n) { return n == 1 ? all * i : (int)((int64_t)all * i / n); }

// 2^e for any e: 0 below fp32's smallest number, infinity above its largest
F3DC_DEV float pow2(int e)
{
    if (e >= -126) return __uint_as_float((uint32_t)(min(e, 128) + 127) << 23);
    return e < -149 ? 0.f : __uint_as_float(1u << (e + 149));
}

F3DC_DEV void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
F3DC_DEV void cp_async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// 16 and 8 bytes of the shared memory of a CTA of the cluster
F3DC_DEV float4 load_cluster16(uint32_t cluster_addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_addr) : "memory");
    return v;
}
F3DC_DEV float2 load_cluster8(uint32_t cluster_addr)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(cluster_addr) : "memory");
    return v;
}
// four e4m3 values to two pairs of fp16 (exact)
F3DC_DEV void e4m3x4_to_half2(uint32_t w, uint32_t &h0, uint32_t &h1)
{
    asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %2;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n cvt.rn.f16x2.e4m3x2 %1, hi;\n}\n"
        : "=r"(h0), "=r"(h1)
        : "r"(w));
}
F3DC_DEV uint32_t half2_times(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
F3DC_DEV uint32_t pack_half2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// ---- Softmax with value scales.  With s = scale q . k in log2, the weight of a token in a page of value
// scale 2^e is kept as w = 2^(s + e - r), so the product with the page's bytes needs no scale of its own; the
// reference r of a row is such that w < 2^16, fp16's range, with the row's largest s + e some binades above r, so that fp16 holds
// weights far below the largest.  The sum of weights takes them without their value scales, w 2^-e.  A value
// scale below 2^kLeastScale counts as 2^kLeastScale with values of zero (they are below 2^-55): without that
// bound the blocks of zeros, whose scale is 2^-127, would take the sums out of fp32's range.
// Within kScaleSpan binades of the largest value scale E so far, w 2^-e loses nothing of the sum: s + e - r is at least
// s - max(s) - kScaleSpan, and the exponential's end at 2^-126 is 2^-56 of the sum's largest term.  Tokens beside a page further
// below ("apart") take a second exponential without e, 2^(s - r + kSumShift): since s + e - r <= 16, its exponent is at most
// 16 + 64 + kSumShift = 120, and since r <= max(s) + 127 the largest s stands at 2^(kSumShift - 127) or above, 2^39 above the end.
constexpr int kLeastScale = -64, kScaleSpan = 70;
constexpr float kSumShift = 40.f, kSumUnshift = 0x1p-40f;
// Square root of the factor from one reference to a larger one (none: 0).  Sums of weights are multiplied by it twice: references take
// value scales in, so that for equal scores they may lie 191 apart, and a sum is large where the factor is out of range.
F3DC_DEV float half_factor(float from, float to)
{
    return from == __int_as_float(0xFF800000) ? 0.f : exp2_fast(0.5f * (from - to));
}

struct ValueScale {
    float log2, inverse;  // e and 2^-e
    uint32_t times;       // what the values are multiplied by, two of fp16: 1, 0 or NaN
};
constexpr uint32_t kHalfOnes = 0x3C003C00u, kHalfNans = 0x7E007E00u;
F3DC_DEV ValueScale value_scale(uint32_t byte)
{
    ValueScale v;
    const int e = byte == 255u ? 0 : max((int)byte - 127, kLeastScale);
    v.log2 = (float)e;
    v.inverse = pow2(-e);
    v.times = byte == 255u ? kHalfNans : ((int)byte - 127 < kLeastScale ? 0u : kHalfOnes);
    return v;
}
F3DC_DEV float key_scale(uint32_t byte) { return byte == 255u ? __int_as_float(0x7FC00000) : pow2((int)byte - 127); }

// The power of two that brings a query row's largest magnitude into [2^14, 2^15), where fp16 holds bf16 values
// exactly down to 2^-28 of it; at most 2^126.
F3DC_DEV int query_exponent(float top)
{
    const int e = (int)(__float_as_uint(top) >> 23) - 127;  // of a normal number
    return top == 0.f ? 0 : min(14 - e, 126);
}

// ln of the sum of exp from a reference and a sum of weights; no token: -infinity
F3DC_DEV float log_sum(float r, float l) { return l == 0.f ? __int_as_float(0xFF800000) : (r + log2f(l)) * 0.6931471805599453f; }

}  // namespace f3dc
