// api_fp8.cu -- the C ABI of the 8-bit linear layers: f3dc_quantize_fp8, f3dc_gemm_fp8
// and f3dc_norm_residual.  Arguments are checked before any launch; nothing here
// allocates, synchronises or throws.
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

int blocks(int cols) { return (cols - 1) / kScaleBlock + 1; }

static_assert(noexcept(gemm_status_word()), "nothing may throw through these calls");

cudaError_t sm_count(int *sms)
{
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    return e != cudaSuccess ? e : cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
}

}  // namespace

extern "C" f3dc_status f3dc_quantize_fp8(const void *x, int32_t x_type, int64_t ldx, void *q, int64_t ldq,
                                         void *scales, int64_t lds, int32_t rows, int32_t cols, void *stream)
{
    if (rows < 0 || cols < 1) return bad("need rows >= 0 and cols >= 1");
    if (x_type != F3DC_TYPE_BF16 && x_type != F3DC_TYPE_F32) return bad("bad x_type");
    if (ldx < cols || ldq < cols || lds < blocks(cols)) return bad("a leading dimension is smaller than its row");
    if (rows == 0) return F3DC_OK;
    if (!x || !q || !scales) return bad("null pointer");
    if (misaligned(x, x_type == F3DC_TYPE_F32 ? 4 : 2)) return bad("x is not aligned to its elements");
    int sms = 0;
    cudaError_t e = sm_count(&sms);
    if (e != cudaSuccess) return fail(F3DC_ERR_CUDA, "device query", e);
    const QuantArgs a{x, ldx, (uint8_t *)q, ldq, (uint8_t *)scales, lds, rows, cols};
    e = launch_quantize(a, x_type == F3DC_TYPE_F32, sms, (cudaStream_t)stream);
    return e == cudaSuccess ? F3DC_OK : fail(F3DC_ERR_CUDA, "launch", e);
}

extern "C" f3dc_status f3dc_gemm_fp8(const void *A, int64_t lda, const void *a_scales, int64_t ldas, const void *B,
                                     int64_t ldb, const void *b_scales, int64_t ldbs, const void *bias,
                                     const float *gate, void *out, int64_t ldo, void *out_scales, int64_t ldos,
                                     int32_t M, int32_t N, int32_t K, int32_t epilogue, void *stream)
{
    if (M < 0 || N < 8 || N % 8 != 0 || K < 1) return bad("need M >= 0, N a positive multiple of 8, K >= 1");
    if (epilogue < F3DC_EPI_BIAS || epilogue > F3DC_EPI_RESID) return bad("bad epilogue");
    const bool out8 = out_scales != nullptr;
    if (out8 && epilogue == F3DC_EPI_RESID) return bad("the residual epilogue has no 8-bit output");
    if (gate && epilogue != F3DC_EPI_RESID) return bad("a gate goes with the residual epilogue");
    if (out8 && N % 16 != 0) return bad("8-bit output needs N a multiple of 16");
    if (lda < K || ldb < K || lda % 16 || ldb % 16) return bad("lda and ldb must be multiples of 16, at least K");
    if (ldas < blocks(K) || ldbs < blocks(K) || ldas % 4 || ldbs % 4)
        return bad("ldas and ldbs must be multiples of 4, at least ceil(K / 128)");
    if (lda >= (int64_t)1 << 40 || ldb >= (int64_t)1 << 40 || ldo >= (int64_t)1 << 36)
        return bad("a leading dimension is too large");
    const int esz = out8 ? 1 : (epilogue == F3DC_EPI_RESID ? 4 : 2);
    if (ldo < N || ldo * esz % 16) return bad("ldo must be at least N, and rows of out a multiple of 16 bytes");
    if (out8 && (ldos < blocks(N))) return bad("ldos is smaller than ceil(N / 128)");
    // (a tile of 2^26 K takes 0.15 s or so of the second that a wait for it may last)
    if (((int64_t)M + 255) / 256 * (((int64_t)N + 63) / 64) > (1 << 30) || M > INT32_MAX - 512 || N > INT32_MAX - 512 ||
        K > 1 << 26)
        return bad("the problem is too large");
    if (M == 0) return F3DC_OK;
    if (!A || !B || !a_scales || !b_scales || !out) return bad("null pointer");
    if (misaligned(A, 16) || misaligned(B, 16) || misaligned(out, 16) || misaligned(bias, 16) || misaligned(gate, 16))
        return bad("pointers must be 16-byte aligned");
    if (misaligned(a_scales, 4) || misaligned(b_scales, 4)) return bad("a_scales and b_scales must be 4-byte aligned");
    const int epi = epilogue == F3DC_EPI_BIAS ? kEpiBias : (epilogue == F3DC_EPI_GELU ? kEpiGelu : kEpiResid);
    if (gemm8_few_rows(M, N, K)) {
        const FewArgs g{M, N, K, (const uint8_t *)A, lda, (const uint8_t *)a_scales, ldas, (const uint8_t *)B, ldb,
                        (const uint8_t *)b_scales, ldbs, (const bf16 *)bias, gate, out, ldo, (uint8_t *)out_scales, ldos};
        int sms = 0;
        cudaError_t e = sm_count(&sms);
        if (e != cudaSuccess) return fail(F3DC_ERR_CUDA, "device query", e);
        e = launch_few8(g, epi, sms, (cudaStream_t)stream);
        return e == cudaSuccess ? F3DC_OK : fail(F3DC_ERR_CUDA, "launch", e);
    }
    Gemm8Params p;
    p.M = M;
    p.N = N;
    p.K = K;
    p.sa = (const uint8_t *)a_scales;
    p.sb = (const uint8_t *)b_scales;
    p.lda_s = ldas;
    p.ldb_s = ldbs;
    const uintptr_t align = (uintptr_t)a_scales | (uintptr_t)b_scales | (uintptr_t)ldas | (uintptr_t)ldbs;
    p.scale_sets = align % 16 == 0 ? 4 : (align % 8 == 0 ? 2 : 1);
    p.bias = (const bf16 *)bias;
    p.gate = gate;
    p.out_scales = (uint8_t *)out_scales;
    p.ldo_s = ldos;
    // a bounded wait that runs out is recorded here (read by f3dc_gemm_status)
    p.err = gemm_status_word();
    if (!p.err) return fail(F3DC_ERR_CUDA, "cannot resolve the status word");
    CUtensorMap ta, to;
    GemmPairB tb;
    const auto u8 = CU_TENSOR_MAP_DATA_TYPE_UINT8;
    bool ok = make_tmap_rows(&ta, u8, A, M, K, lda, 128, 128);
    for (int i = 0; i < 3; ++i) ok = ok && make_tmap_rows(&tb.rows[i], u8, B, N, K, ldb, 128 >> i, 128);
    ok = ok && make_tmap_rows(&to, out8 ? u8 : (esz == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16),
                              out, M, N, ldo * esz, 32, 128 / esz);
    if (!ok) return bad("cuTensorMapEncodeTiled rejected A, B or out");
    const cudaError_t e = launch_gemm8_pair(&ta, &tb, &to, p, epi, out8, (cudaStream_t)stream);
    return e == cudaSuccess ? F3DC_OK : fail(F3DC_ERR_CUDA, "launch", e);
}

extern "C" f3dc_status f3dc_norm_residual(const f3dc_norm_layer *l, const float *x, int64_t ldx, float *x_out,
                                          int64_t ldxo, const void *y, int64_t ldy, const float *gate,
                                          const float *scale, const float *shift, int64_t ldmod,
                                          const int32_t *group_of_row, int32_t groups, void *h, int64_t ldh,
                                          void *h_scales, int64_t ldhs, int32_t rows, void *stream)
{
    if (!l) return bad("null layer");
    const int W = l->width;
    if (rows < 0 || groups < 1) return bad("need rows >= 0 and groups >= 1");
    if (W < 8 || W > F3DC_NORM_MAX_WIDTH || W % 8) return bad("width must be a multiple of 8, at most 8192");
    if (l->post < F3DC_NORM_NONE || l->post > F3DC_NORM_RMS || l->pre < F3DC_NORM_NONE || l->pre > F3DC_NORM_RMS)
        return bad("bad norm kind");
    if (!(l->eps >= 0.f) || !std::isfinite(l->eps)) return bad("eps must be finite and not negative");
    if (!x_out && !h) return bad("nothing to write: x_out and h are both null");
    if (h_scales && !h) return bad("h_scales without h");
    if (gate && !y) return bad("a gate goes with y");
    if ((gate || scale || shift) && (ldmod < W || ldmod % 4)) return bad("ldmod must be a multiple of 4, at least the width");
    if (ldx < W || ldx % 4 || (x_out && (ldxo < W || ldxo % 4)) || (y && (ldy < W || ldy % 8)))
        return bad("rows of x, x_out and y must start 16 bytes aligned and hold the width");
    if (x && x_out == x && ldxo != ldx) return bad("x_out in place of x needs ldxo = ldx");
    if (h && (ldh < W || ldh % 8)) return bad("ldh must be a multiple of 8, at least the width");
    if (h_scales && ldhs < blocks(W)) return bad("ldhs is smaller than ceil(width / 128)");
    if (rows == 0) return F3DC_OK;
    if (!x) return bad("null x");
    const void *p16[] = {x, x_out, y, gate, scale, shift, h, l->post_g, l->post_b, l->pre_g, l->pre_b};
    for (const void *p : p16)
        if (misaligned(p, 16)) return bad("pointers must be 16-byte aligned");
    if (misaligned(group_of_row, 4)) return bad("group_of_row must be 4-byte aligned");
    int sms = 0;
    cudaError_t e = sm_count(&sms);
    if (e != cudaSuccess) return fail(F3DC_ERR_CUDA, "device query", e);
    NormArgs a;
    a.rows = rows;
    a.width = W;
    a.x = x;
    a.ldx = ldx;
    a.x_out = x_out;
    a.ldxo = ldxo;
    a.y = (const bf16 *)y;
    a.ldy = ldy;
    a.post = l->post;
    a.pre = l->pre;
    a.post_g = (const bf16 *)l->post_g;
    a.post_b = (const bf16 *)l->post_b;
    a.pre_g = (const bf16 *)l->pre_g;
    a.pre_b = (const bf16 *)l->pre_b;
    a.gate = gate;
    a.scale = scale;
    a.shift = shift;
    a.ldmod = ldmod;
    a.group = group_of_row;
    a.groups = groups;
    a.h = h;
    a.ldh = ldh;
    a.h_scales = (uint8_t *)h_scales;
    a.ldhs = ldhs;
    a.res_scale = l->res_scale;
    a.eps = l->eps;
    // a group outside its range is recorded here (read by f3dc_gemm_status)
    a.err = gemm_status_word();
    if (!a.err) return fail(F3DC_ERR_CUDA, "cannot resolve the status word");
    e = launch_norm_residual(a, sms, (cudaStream_t)stream);
    return e == cudaSuccess ? F3DC_OK : fail(F3DC_ERR_CUDA, "launch", e);
}
