// api_kv.cu -- the C ABI of attention over a paged 8-bit cache: f3dc_rotary_turns,
// f3dc_kv_append_fp8, f3dc_kv_attention_workspace and f3dc_kv_attention_fp8.  Arguments
// are checked before any launch; nothing here allocates, synchronises or throws.
#include <cmath>
#include <string>

#include "../../include/f3dc.h"
#include "kernels.h"

using namespace f3dc;

namespace {

// failures are reported through f3dc_last_error(NULL)
f3dc_status fail(f3dc_status st, const char *msg, cudaError_t e = cudaSuccess)
{
    try {
        set_host_error(e == cudaSuccess ? std::string(msg) : std::string(msg) + ": " + cudaGetErrorString(e));
    } catch (...) {  // out of memory: the status alone is reported
    }
    return st;
}

f3dc_status bad(const char *msg) { return fail(F3DC_ERR_INVALID_ARG, msg); }

bool misaligned(const void *p, int n) { return ((uintptr_t)p & (n - 1)) != 0; }

cudaError_t sm_count(int *sms)
{
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    return e != cudaSuccess ? e : cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
}

// what is wrong with the shape of a cache, or null
const char *cache_shape(const f3dc_kv_cache *c)
{
    if (!c) return "null cache";
    if (c->pages < 1) return "a cache needs pages >= 1";
    if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128)
        return "page_tokens must be 16, 32, 64 or 128";
    if (c->kv_heads < 1 || c->kv_heads > 1024) return "kv_heads must be 1 to 1024";
    if (c->dh != 32 && c->dh != 64 && c->dh != 128) return "dh must be 32, 64 or 128";
    if (c->page_stride < (int64_t)c->kv_heads * c->page_tokens * c->dh || c->page_stride % 16)
        return "page_stride must be a multiple of 16, at least a page's bytes";
    if (c->scale_stride < c->kv_heads) return "scale_stride is smaller than kv_heads";
    // (offsets in k and v are counted in 32 bits of 16 bytes)
    if (c->page_stride > ((int64_t)1 << 36) / c->pages || c->scale_stride > ((int64_t)1 << 62) / c->pages)
        return "the cache is too large";
    return nullptr;
}

const char *batch_shape(const f3dc_kv_batch *t)
{
    if (!t) return "null batch";
    if (t->batch < 0 || t->rows < 0 || t->max_rows < 0 || t->max_length < 0)
        return "batch, rows, max_rows and max_length must not be negative";
    if (t->table_stride < 0 || t->table_stride >= (int64_t)1 << 31) return "table_stride must be 0 to 2^31 - 1";
    return nullptr;
}

const char *cache_pointers(const f3dc_kv_cache *c)
{
    if (!c->k || !c->v || !c->k_scales || !c->v_scales) return "null pointer in the cache";
    if (misaligned(c->k, 16) || misaligned(c->v, 16)) return "the cache's k and v must be 16-byte aligned";
    return nullptr;
}

const char *batch_pointers(const f3dc_kv_batch *t)
{
    if (!t->row_start || !t->lengths || (!t->page_table && t->table_stride > 0)) return "null pointer in the batch";
    if (misaligned(t->row_start, 4) || misaligned(t->lengths, 4) || misaligned(t->page_table, 4))
        return "row_start, lengths and page_table must be 4-byte aligned";
    return nullptr;
}

// a row stride of a bf16 matrix with rows of n elements
bool row_stride(int64_t ld, int64_t n) { return ld >= n && ld % 8 == 0 && ld < (int64_t)1 << 36; }

KvCache cache_of(const f3dc_kv_cache *c)
{
    return {(uint8_t *)c->k, (uint8_t *)c->v, c->k_scales, c->v_scales, c->page_stride, c->scale_stride,
            c->pages, c->page_tokens, c->kv_heads, c->dh};
}

// rows of a sequence at most: the bound may be loose
int32_t most_rows(const f3dc_kv_batch *t) { return t->max_rows < t->rows ? t->max_rows : t->rows; }

KvBatch batch_of(const f3dc_kv_batch *t)
{
    return {t->row_start, t->lengths, t->page_table, t->table_stride, t->batch, t->rows, most_rows(t), t->max_length};
}

bool empty(const f3dc_kv_batch *t) { return t->batch == 0 || t->rows == 0 || t->max_rows == 0; }

// Whether a call within these bounds has more to count than the attention's kernels do.  (Blocks of 8 packed rows are the smallest
// that any kernel makes, and a sequence's CTAs are shared out only up to some times the SMs.)
bool attention_too_large(const f3dc_kv_cache *c, const f3dc_kv_batch *t, int32_t heads)
{
    if (empty(t)) return false;
    const int64_t packed = (int64_t)most_rows(t) * (heads / c->kv_heads);
    return (packed + 7) / 8 > INT32_MAX / 2 / ((int64_t)c->kv_heads * t->batch) || packed > INT32_MAX / 2 ||
           (int64_t)t->rows * heads > INT32_MAX || t->max_length > INT32_MAX - 1024;
}

int64_t part_bytes(const f3dc_kv_cache *c, const f3dc_kv_batch *t, int32_t heads)
{
    return (int64_t)t->rows * heads * (c->dh + 2) * (int64_t)sizeof(float);
}

// CTAs that share a sequence's keys
int splits(const f3dc_kv_cache *c, const f3dc_kv_batch *t, int32_t heads, int sms, bool *cluster)
{
    *cluster = false;
    if (empty(t)) return 1;
    return kv_splits(t->batch, most_rows(t), t->max_length, heads, c->kv_heads, c->dh, sms, cluster);
}

}  // namespace

extern "C" f3dc_status f3dc_rotary_turns(const double *inv_freq, int32_t n, uint64_t *turns_out)
{
    if (n < 0 || (n > 0 && (!inv_freq || !turns_out))) return bad("need n >= 0, inv_freq and turns_out");
    for (int32_t j = 0; j < n; ++j) {
        // the quotient by 2 pi in two doubles, so that a far position times its last bit is nothing yet (below 2^40 radians the two
        // are off by less than 2^-64 turns; NaN is refused too)
        if (!(std::fabs(inv_freq[j]) <= 0x1p40)) return bad("a frequency is not finite or above 2^40 radians per unit");
        constexpr double kTurn = 6.283185307179586, kTurnLow = 2.4492935982947064e-16;  // 2 pi
        const double f = std::fabs(inv_freq[j]), hi = f / kTurn;
        const double lo = (std::fma(-hi, kTurn, f) - hi * kTurnLow) / kTurn;
        const double whole = std::ldexp(hi - std::floor(hi), 32), top = std::floor(whole);  // exact
        const double rest = std::ldexp((whole - top) + std::ldexp(lo, 32), 32);
        const uint64_t turns = ((uint64_t)top << 32) + (uint64_t)(int64_t)std::nearbyint(rest);
        turns_out[j] = inv_freq[j] < 0 ? 0 - turns : turns;
    }
    return F3DC_OK;
}

extern "C" f3dc_status f3dc_kv_append_fp8(const f3dc_kv_cache *cache, const f3dc_kv_batch *batch,
                                          const f3dc_rotary *rotary, const void *k, int64_t ldk, const void *v,
                                          int64_t ldv, const void *q, int64_t ldq, void *q_out, int64_t ldqo,
                                          int32_t heads, const int32_t *positions, void *stream)
{
    const char *wrong = cache_shape(cache);
    if (!wrong) wrong = batch_shape(batch);
    if (wrong) return bad(wrong);
    const int64_t width = (int64_t)cache->kv_heads * cache->dh;
    if (!row_stride(ldk, width) || !row_stride(ldv, width)) return bad("ldk and ldv must be multiples of 8, at least kv_heads dh");
    if (q) {
        if (!rotary) return bad("queries are given to be rotated: q goes with rotary");
        if (heads < 1 || heads > 65536) return bad("heads must be 1 to 65536");
        if (!q_out) return bad("null q_out");
        if (!row_stride(ldq, (int64_t)heads * cache->dh) || !row_stride(ldqo, (int64_t)heads * cache->dh))
            return bad("ldq and ldqo must be multiples of 8, at least heads dh");
        if (q == q_out && ldq != ldqo) return bad("q_out in place of q needs ldqo = ldq");
    }
    if (rotary) {
        if (rotary->dims < 16 || rotary->dims % 16 || rotary->dims > cache->dh)
            return bad("rotary dims must be a multiple of 16, at most dh");
        if (rotary->interleaved != 0 && rotary->interleaved != 1) return bad("interleaved must be 0 or 1");
        if (rotary->axes < 1 || rotary->axes > 3) return bad("axes must be 1 to 3");
        if (rotary->axes > 1 && !positions) return bad("several axes need positions");
        if (!rotary->turns) return bad("null turns");
        if (misaligned(rotary->turns, 8)) return bad("turns must be 8-byte aligned");
    } else if (positions) {
        return bad("positions go with rotary");
    }
    if (misaligned(positions, 4)) return bad("positions must be 4-byte aligned");
    if (empty(batch)) return F3DC_OK;
    if ((wrong = cache_pointers(cache)) || (wrong = batch_pointers(batch))) return bad(wrong);
    if (!k || !v) return bad("null pointer");
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(q, 16) || (q && misaligned(q_out, 16)))
        return bad("pointers must be 16-byte aligned");
    if ((((int64_t)most_rows(batch) + cache->page_tokens - 2) / cache->page_tokens + 1) * batch->batch > INT32_MAX ||
        batch->max_length > INT32_MAX - 1024)
        return bad("the problem is too large");
    int sms = 0;
    cudaError_t e = sm_count(&sms);
    if (e != cudaSuccess) return fail(F3DC_ERR_CUDA, "device query", e);
    KvAppendArgs a = {};
    a.cache = cache_of(cache);
    a.batch = batch_of(batch);
    a.axes = 1;
    if (rotary) {
        a.dims = rotary->dims;
        a.interleaved = rotary->interleaved;
        a.axes = rotary->axes;
        a.turns = rotary->turns;
        a.positions = positions;
    }
    a.k = (const bf16 *)k;
    a.v = (const bf16 *)v;
    a.ldk = ldk;
    a.ldv = ldv;
    if (q) {
        a.q = (const bf16 *)q;
        a.ldq = ldq;
        a.q_out = (bf16 *)q_out;
        a.ldqo = ldqo;
        a.heads = heads;
    }
    // rows, lengths or pages out of range are recorded here (read by f3dc_gemm_status)
    a.err = gemm_status_word();
    if (!a.err) return fail(F3DC_ERR_CUDA, "cannot resolve the status word");
    e = launch_kv_append(a, sms, (cudaStream_t)stream);
    return e == cudaSuccess ? F3DC_OK : fail(F3DC_ERR_CUDA, "launch", e);
}

extern "C" size_t f3dc_kv_attention_workspace(const f3dc_kv_cache *cache, const f3dc_kv_batch *batch, int32_t heads)
{
    if (cache_shape(cache) || batch_shape(batch) || heads < 1 || heads % cache->kv_heads || heads > 65536 ||
        attention_too_large(cache, batch, heads))
        return 0;
    int sms = 0;
    if (sm_count(&sms) != cudaSuccess) return 0;
    bool cluster = false;
    const int n = splits(cache, batch, heads, sms, &cluster);
    return n > 1 && !cluster ? (size_t)(n * part_bytes(cache, batch, heads)) : 0;
}

extern "C" f3dc_status f3dc_kv_attention_fp8(const f3dc_kv_cache *cache, const f3dc_kv_batch *batch, const void *q,
                                             int64_t ldq, void *out, int64_t ldo, float *lse, int32_t heads,
                                             float scale, int32_t causal, void *workspace, size_t workspace_bytes,
                                             void *stream)
{
    const char *wrong = cache_shape(cache);
    if (!wrong) wrong = batch_shape(batch);
    if (wrong) return bad(wrong);
    if (heads < 1 || heads > 65536 || heads % cache->kv_heads) return bad("heads must be a multiple of kv_heads, at most 65536");
    if (!(scale > 0.f) || !std::isfinite(scale)) return bad("scale must be positive and finite");
    if (causal != 0 && causal != 1) return bad("causal must be 0 or 1");
    const int64_t width = (int64_t)heads * cache->dh;
    if (!row_stride(ldq, width) || !row_stride(ldo, width)) return bad("ldq and ldo must be multiples of 8, at least heads dh");
    if (empty(batch)) return F3DC_OK;
    if ((wrong = cache_pointers(cache)) || (wrong = batch_pointers(batch))) return bad(wrong);
    if (!q || !out) return bad("null pointer");
    if (misaligned(q, 16) || misaligned(out, 16) || misaligned(workspace, 16)) return bad("pointers must be 16-byte aligned");
    if (misaligned(lse, 4)) return bad("lse must be 4-byte aligned");
    if (attention_too_large(cache, batch, heads)) return bad("the problem is too large");
    int sms = 0;
    cudaError_t e = sm_count(&sms);
    if (e != cudaSuccess) return fail(F3DC_ERR_CUDA, "device query", e);
    KvAttnArgs a = {};
    a.cache = cache_of(cache);
    a.batch = batch_of(batch);
    a.q = (const bf16 *)q;
    a.ldq = ldq;
    a.out = (bf16 *)out;
    a.ldo = ldo;
    a.lse = lse;
    a.heads = heads;
    a.group = heads / cache->kv_heads;
    a.causal = causal;
    a.scale_log2 = (float)(scale * 1.4426950408889634);
    const bool many = kv_many_rows(most_rows(batch), heads, cache->kv_heads, cache->dh);
    bool cluster = false;
    a.splits = splits(cache, batch, heads, sms, &cluster);
    if (!cluster && a.splits > 1) {
        // without the whole workspace as many parts as fit it or, of few rows, as a cluster joins
        const int64_t fit = workspace ? (int64_t)(workspace_bytes / (size_t)part_bytes(cache, batch, heads)) : 0;
        const int least = many ? 1 : (a.splits < kMostCluster ? a.splits : kMostCluster);
        if (fit < a.splits) a.splits = fit > least ? (int)fit : least, cluster = !many && fit <= least;
    }
    a.cluster = cluster;
    a.part = (float *)workspace;
    // rows, lengths or pages out of range are recorded here (read by f3dc_gemm_status)
    a.err = gemm_status_word();
    if (!a.err) return fail(F3DC_ERR_CUDA, "cannot resolve the status word");
    e = many ? launch_kv_attn(a, (cudaStream_t)stream) : launch_kv_few(a, (cudaStream_t)stream);
    return e == cudaSuccess ? F3DC_OK : fail(F3DC_ERR_CUDA, "launch", e);
}
