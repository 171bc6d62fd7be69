// Host side of a quantised decoder layer's calls: argument validation.  As in dg_api.hip, everything is checked before anything is
// launched, and nothing synchronises.
#include "dg_decoder.h"

namespace {

bool known_type(dg_dtype t) { return t == DG_F32 || t == DG_F16 || t == DG_BF16; }

// The largest reduction that int32 holds: K * 128 * 128 < 2^31.
constexpr int64_t MOST_K = ((int64_t)1 << 17) - 1;
constexpr int64_t MOST_ROWS = ((int64_t)1 << 31) - 1;

int64_t codes_pitch(int64_t K) { return (K + 15) / 16 * 16; }

dg_status check_tokens(const char *what, const void *x, dg_dtype type, int64_t N, int64_t K, int64_t stride)
{
    if (N < 0 || K <= 0 || N > MOST_ROWS) return dg_fail(DG_ERR_SHAPE, "%s: N=%lld K=%lld", what, (long long)N, (long long)K);
    if (K > MOST_K) return dg_fail(DG_ERR_RANGE, "%s: K=%lld could overflow int32 (at most %lld)", what, (long long)K, (long long)MOST_K);
    if (!known_type(type)) return dg_fail(DG_ERR_UNSUPPORTED, "%s: unknown element type %d", what, (int)type);
    if (N > 0 && !x) return dg_fail(DG_ERR_NULL, "%s: NULL activations", what);
    if (stride < K) return dg_fail(DG_ERR_SHAPE, "%s: rows of %lld elements every %lld", what, (long long)K, (long long)stride);
    return DG_OK;
}

dg_status check_product(const char *what, const int8_t *W, int64_t stride_w, int64_t M, int64_t N, int64_t K, const float *scale_m,
                        const void *out, dg_dtype type, int64_t stride_out)
{
    if (M <= 0 || N < 0 || K <= 0 || M > MOST_ROWS || N > MOST_ROWS)
        return dg_fail(DG_ERR_SHAPE, "%s: M=%lld N=%lld K=%lld", what, (long long)M, (long long)N, (long long)K);
    if (K > MOST_K) return dg_fail(DG_ERR_RANGE, "%s: K=%lld could overflow int32 (at most %lld)", what, (long long)K, (long long)MOST_K);
    if ((M + 63) / 64 * ((N + 63) / 64) > MOST_ROWS) return dg_fail(DG_ERR_RANGE, "%s: M=%lld N=%lld is too large for one call", what, (long long)M, (long long)N);
    if (!known_type(type)) return dg_fail(DG_ERR_UNSUPPORTED, "%s: unknown element type %d", what, (int)type);
    if (!W || !scale_m || (N > 0 && !out)) return dg_fail(DG_ERR_NULL, "%s: NULL argument", what);
    if (stride_w < K) return dg_fail(DG_ERR_SHAPE, "%s: weight rows of %lld bytes every %lld", what, (long long)K, (long long)stride_w);
    if (stride_out < M) return dg_fail(DG_ERR_SHAPE, "%s: output rows of %lld elements every %lld", what, (long long)M, (long long)stride_out);
    return DG_OK;
}

dg_status check_cache(const char *what, const dg_cache_desc *d, const void *cache)
{
    if (!d || !cache) return dg_fail(DG_ERR_NULL, "%s: NULL cache", what);
    if (d->bits != 8 && d->bits != 4) return dg_fail(DG_ERR_UNSUPPORTED, "%s: %d-bit cache (8 or 4)", what, (int)d->bits);
    if (d->dim != 64 && d->dim != 128 && d->dim != 256)
        return dg_fail(DG_ERR_UNSUPPORTED, "%s: heads of %d channels (64, 128 or 256)", what, (int)d->dim);
    if (d->pages <= 0 || d->heads <= 0 || d->page_size <= 0 || d->page_size % 16 != 0)
        return dg_fail(DG_ERR_SHAPE, "%s: %d pages of %d tokens (a multiple of 16), %d heads", what, (int)d->pages, (int)d->page_size,
                       (int)d->heads);
    const int64_t head = d->page_size * (int64_t)(2 * d->dim * d->bits / 8 + (d->bits == 8 ? 8 : 16));       // a page's bytes for one head
    if ((int64_t)d->pages * d->page_size > MOST_ROWS || head > MOST_ROWS)
        return dg_fail(DG_ERR_RANGE, "%s: %d pages of %d tokens: slots, and a page's bytes for one head, are 32-bit numbers", what, (int)d->pages, (int)d->page_size);
    if (head * d->heads > INT64_MAX / d->pages)
        return dg_fail(DG_ERR_RANGE, "%s: %d pages of %d tokens, %d heads: the bytes are no 64-bit number", what, (int)d->pages, (int)d->page_size, (int)d->heads);
    if ((uintptr_t)cache % 16 != 0) return dg_fail(DG_ERR_BUFFER, "%s: the cache must be 16-byte aligned", what);
    return DG_OK;
}

// (token, head) rows; eight tokens' have to fit a launch, which a call has as many of as it takes
dg_status check_cache_tokens(const char *what, const dg_cache_desc *d, dg_dtype type, int64_t T, const int32_t *slots)
{
    if (!known_type(type)) return dg_fail(DG_ERR_UNSUPPORTED, "%s: unknown element type %d", what, (int)type);
    if (d->heads > 1 << 24) return dg_fail(DG_ERR_RANGE, "%s: %d heads (at most 2^24)", what, (int)d->heads);
    if (T < 0 || T > MOST_ROWS / d->heads) return dg_fail(DG_ERR_SHAPE, "%s: %lld tokens of %d heads", what, (long long)T, (int)d->heads);
    if (T > 0 && !slots) return dg_fail(DG_ERR_NULL, "%s: NULL slots", what);
    return DG_OK;
}

dg_status attention_of(const char *what, const dg_cache_desc *d, const void *cache, int64_t B, int64_t Hq, int64_t max_q, int64_t max_ctx,
                       DgAttention *a)
{
    const dg_status s = check_cache(what, d, cache);
    if (s) return s;
    if (B < 0 || Hq <= 0 || Hq % d->heads != 0 || max_q < 0 || max_ctx < 0)
        return dg_fail(DG_ERR_SHAPE, "%s: %lld sequences, %lld query heads on %d cached ones, up to %lld new tokens of %lld", what, (long long)B,
                       (long long)Hq, (int)d->heads, (long long)max_q, (long long)max_ctx);
    if (B > MOST_ROWS || Hq > 65535 || max_q > MOST_ROWS || max_ctx > MOST_ROWS - 65536 || max_q * Hq > MOST_ROWS - 65536 ||
        B * ((max_q * (Hq / d->heads) + 15) / 16) > MOST_ROWS / 256 / d->heads || B * max_q > MOST_ROWS / Hq)
        return dg_fail(DG_ERR_RANGE, "%s: %lld sequences of up to %lld new tokens are too many rows for one call", what, (long long)B,
                       (long long)max_q);
    *a = {};
    a->cache = dg_cache_of(d, const_cast<void *>(cache));
    a->B = (int32_t)B;
    a->Hq = (int32_t)Hq;
    a->max_q = (int32_t)max_q;
    a->max_ctx = (int32_t)max_ctx;
    return DG_OK;
}

}   // namespace

extern "C" {

dg_status dg_quantize_tokens(const void *x_dev, dg_dtype type, int64_t N, int64_t K, int64_t stride_n, int8_t *codes_dev,
                             int64_t stride_codes, float *scale_n_dev, void *hip_stream)
{
    const dg_status s = check_tokens("dg_quantize_tokens", x_dev, type, N, K, stride_n);
    if (s) return s;
    if (stride_codes < K) return dg_fail(DG_ERR_SHAPE, "dg_quantize_tokens: rows of %lld codes every %lld", (long long)K, (long long)stride_codes);
    if (N == 0) return DG_OK;
    if (!codes_dev || !scale_n_dev) return dg_fail(DG_ERR_NULL, "dg_quantize_tokens: NULL output");
    return dg_launch_quantize_tokens(x_dev, type, N, K, stride_n, codes_dev, stride_codes, K, scale_n_dev, (hipStream_t)hip_stream);
}

dg_status dg_gemm_i8(const int8_t *W_dev, int64_t stride_w, const int8_t *A_dev, int64_t stride_a, int64_t M, int64_t N, int64_t K,
                     const float *scale_m_dev, const float *scale_n_dev, const float *bias_m_dev, void *out_dev, dg_dtype out_type,
                     int64_t stride_out, void *hip_stream)
{
    const dg_status s = check_product("dg_gemm_i8", W_dev, stride_w, M, N, K, scale_m_dev, out_dev, out_type, stride_out);
    if (s) return s;
    if (stride_a < K) return dg_fail(DG_ERR_SHAPE, "dg_gemm_i8: token rows of %lld bytes every %lld", (long long)K, (long long)stride_a);
    if (N == 0) return DG_OK;
    if (!A_dev || !scale_n_dev) return dg_fail(DG_ERR_NULL, "dg_gemm_i8: NULL argument");
    const DgGemmI8 p = {W_dev, A_dev, stride_w, stride_a, (int32_t)M, (int32_t)N, (int32_t)K, scale_m_dev, scale_n_dev, bias_m_dev, out_dev, stride_out};
    return dg_launch_gemm_i8(p, out_type, (hipStream_t)hip_stream);
}

size_t dg_linear_i8_work_bytes(int64_t N, int64_t K) { return N <= 0 || K <= 0 || N > MOST_ROWS || K > MOST_K ? 0 : (size_t)(N * (codes_pitch(K) + 4)); }

dg_status dg_linear_i8(const int8_t *W_dev, int64_t stride_w, const void *x_dev, dg_dtype x_type, int64_t stride_x, int64_t M, int64_t N,
                       int64_t K, const float *scale_m_dev, const float *bias_m_dev, void *work_dev, size_t work_bytes, void *out_dev,
                       dg_dtype out_type, int64_t stride_out, void *hip_stream)
{
    dg_status s = check_product("dg_linear_i8", W_dev, stride_w, M, N, K, scale_m_dev, out_dev, out_type, stride_out);
    if (!s) s = check_tokens("dg_linear_i8", x_dev, x_type, N, K, stride_x);
    if (s || N == 0) return s;
    if (!work_dev) return dg_fail(DG_ERR_NULL, "dg_linear_i8: NULL work buffer");
    if (work_bytes < dg_linear_i8_work_bytes(N, K) || (uintptr_t)work_dev % 16 != 0)
        return dg_fail(DG_ERR_BUFFER, "dg_linear_i8: a work buffer of %zu bytes, 16-byte aligned, is needed (%zu given)",
                       dg_linear_i8_work_bytes(N, K), work_bytes);
    int8_t *codes = (int8_t *)work_dev;
    const int64_t pitch = codes_pitch(K);
    float *scale_n = (float *)(codes + N * pitch);
    const DgGemmI8 p = {W_dev, codes, stride_w, pitch, (int32_t)M, (int32_t)N, (int32_t)K, scale_m_dev, scale_n, bias_m_dev, out_dev, stride_out};
    if (dg_linear_i8_fuses(N, K)) return dg_launch_linear_i8_fused(p, x_dev, x_type, out_type, (hipStream_t)hip_stream);
    s = dg_launch_quantize_tokens(x_dev, x_type, N, K, stride_x, codes, pitch, pitch, scale_n, (hipStream_t)hip_stream);
    if (s) return s;
    return dg_launch_gemm_i8(p, out_type, (hipStream_t)hip_stream);
}

size_t dg_cache_bytes(const dg_cache_desc *desc)
{
    if (!desc || check_cache("dg_cache_bytes", desc, (const void *)16)) return 0;
    const DgCache c = dg_cache_of(desc, nullptr);
    return (size_t)c.page_bytes() * (size_t)c.pages;
}

dg_status dg_cache_write(const dg_cache_desc *desc, void *cache_dev, size_t cache_bytes, const void *k_dev, const void *v_dev, dg_dtype type,
                         int64_t T, int64_t stride_kt, int64_t stride_kh, int64_t stride_vt, int64_t stride_vh, const int32_t *slots_dev,
                         void *hip_stream)
{
    dg_status s = check_cache("dg_cache_write", desc, cache_dev);
    if (!s) s = check_cache_tokens("dg_cache_write", desc, type, T, slots_dev);
    if (s) return s;
    if (cache_bytes < dg_cache_bytes(desc))
        return dg_fail(DG_ERR_BUFFER, "dg_cache_write: a cache of %zu bytes is needed (%zu given)", dg_cache_bytes(desc), cache_bytes);
    if (T == 0) return DG_OK;
    if (!k_dev || !v_dev) return dg_fail(DG_ERR_NULL, "dg_cache_write: NULL keys or values");
    const int64_t strides[4] = {stride_kt, stride_kh, stride_vt, stride_vh};
    return dg_launch_cache_write(dg_cache_of(desc, cache_dev), k_dev, v_dev, type, T, strides, slots_dev, (hipStream_t)hip_stream);
}

dg_status dg_cache_read(const dg_cache_desc *desc, const void *cache_dev, size_t cache_bytes, const int32_t *slots_dev, int64_t T, void *k_dev,
                        void *v_dev, dg_dtype type, void *hip_stream)
{
    dg_status s = check_cache("dg_cache_read", desc, cache_dev);
    if (!s) s = check_cache_tokens("dg_cache_read", desc, type, T, slots_dev);
    if (s) return s;
    if (cache_bytes < dg_cache_bytes(desc))
        return dg_fail(DG_ERR_BUFFER, "dg_cache_read: a cache of %zu bytes is needed (%zu given)", dg_cache_bytes(desc), cache_bytes);
    if (T == 0 || (!k_dev && !v_dev)) return DG_OK;
    return dg_launch_cache_read(dg_cache_of(desc, const_cast<void *>(cache_dev)), slots_dev, T, k_dev, v_dev, type, (hipStream_t)hip_stream);
}

size_t dg_paged_attention_work_bytes(const dg_cache_desc *desc, int64_t B, int64_t Hq, int64_t max_q, int64_t max_ctx)
{
    DgAttention a;
    if (attention_of("dg_paged_attention_work_bytes", desc, (const void *)16, B, Hq, max_q, max_ctx, &a)) return 0;
    return B == 0 || max_q == 0 ? 0 : (size_t)dg_attention_work_bytes(a);
}

dg_status dg_paged_attention(const dg_cache_desc *desc, const void *cache_dev, size_t cache_bytes, const void *q_dev, dg_dtype type, int64_t T,
                             int64_t Hq, int64_t stride_qt, int64_t stride_qh, const int32_t *q_start_dev, const int32_t *ctx_len_dev,
                             const int32_t *table_dev, int64_t B, int64_t table_width, int64_t max_q, int64_t max_ctx, float scale,
                             int32_t causal, void *out_dev, int64_t stride_ot, int64_t stride_oh, void *work_dev, size_t work_bytes,
                             void *hip_stream)
{
    const char *what = "dg_paged_attention";
    DgAttention a;
    const dg_status s = attention_of(what, desc, cache_dev, B, Hq, max_q, max_ctx, &a);
    if (s) return s;
    if (type != DG_F16 && type != DG_BF16) return dg_fail(DG_ERR_UNSUPPORTED, "%s: queries of element type %d (binary16 or bfloat16)", what, (int)type);
    if (T < 0 || T > MOST_ROWS || table_width < 0 || table_width > MOST_ROWS)
        return dg_fail(DG_ERR_SHAPE, "%s: %lld tokens, tables of %lld pages", what, (long long)T, (long long)table_width);
    if (cache_bytes < dg_cache_bytes(desc))
        return dg_fail(DG_ERR_BUFFER, "%s: a cache of %zu bytes is needed (%zu given)", what, dg_cache_bytes(desc), cache_bytes);
    if (B == 0 || T == 0 || max_q == 0) return DG_OK;
    if (!q_dev || !q_start_dev || !ctx_len_dev || !out_dev || (table_width > 0 && !table_dev)) return dg_fail(DG_ERR_NULL, "%s: NULL argument", what);
    const size_t need = (size_t)dg_attention_work_bytes(a);
    if (need && !work_dev) return dg_fail(DG_ERR_NULL, "%s: NULL work buffer (%zu bytes are needed)", what, need);
    if (need && (work_bytes < need || (uintptr_t)work_dev % 16 != 0))
        return dg_fail(DG_ERR_BUFFER, "%s: a work buffer of %zu bytes, 16-byte aligned, is needed (%zu given)", what, need, work_bytes);
    a.q = q_dev;
    a.out = out_dev;
    a.q_token = stride_qt;
    a.q_head = stride_qh;
    a.out_token = stride_ot;
    a.out_head = stride_oh;
    a.q_start = q_start_dev;
    a.ctx_len = ctx_len_dev;
    a.table = table_dev;
    a.T = (int32_t)T;
    a.table_width = (int32_t)table_width;
    a.scale = scale;
    a.causal = causal != 0;
    a.work = work_dev;
    return dg_launch_attention(a, type, (hipStream_t)hip_stream);
}

}   // extern "C"
