// Host side of the calls around microscaled 4-bit floating point: argument validation.  As in dg_api.hip, everything is checked before anything is launched, and nothing
// synchronises.
#include "dg_decoder.h"
#include "dg_route_rule.h"

namespace {

constexpr int64_t MOST_K = (int64_t)1 << 24;
constexpr int64_t MOST_ROWS = ((int64_t)1 << 31) - 1;
constexpr int64_t MOST_STRIDE = (int64_t)1 << 26;        // 32 rows of a product lie within 2^31 bytes

bool known_type(dg_dtype t) { return t == DG_F32 || t == DG_F16 || t == DG_BF16; }

int64_t blocks_of(int64_t K) { return (K + 31) / 32; }
// Rows of tokens: long ones in whole cache lines (1024 x 7360 x 4096 28.0 us with rows of 3680 bytes, 26.3 with 3712; 355 x 7360 x 3456 20.4, 17.2).
int64_t codes_pitch(int64_t K) { return blocks_of(K) <= 64 ? 16 * blocks_of(K) : (blocks_of(K) + 7) / 8 * 128; }
int64_t scales_pitch(int64_t K) { return (blocks_of(K) + 3) / 4 * 4; }
bool aligned(const void *p, int64_t stride, int to) { return (uintptr_t)p % to == 0 && stride % to == 0; }

// Rows of `of` that are quantised: N may be 0, and then nothing of them is looked at.
dg_status check_rows(const char *what, const char *of, const void *codes, int64_t stride_codes, const void *scales, int64_t stride_scales, int64_t N, int64_t K)
{
    if (N == 0) return DG_OK;
    if (!codes || !scales) return dg_fail(DG_ERR_NULL, "%s: NULL %s", what, of);
    if (stride_codes < 16 * blocks_of(K) || stride_scales < blocks_of(K))
        return dg_fail(DG_ERR_SHAPE, "%s: %s of %lld elements, codes every %lld bytes, scales every %lld (%lld and %lld are needed)", what, of, (long long)K,
                       (long long)stride_codes, (long long)stride_scales, (long long)(16 * blocks_of(K)), (long long)blocks_of(K));
    if (stride_codes > MOST_STRIDE || stride_scales > MOST_STRIDE)
        return dg_fail(DG_ERR_RANGE, "%s: rows of %s lie %lld and %lld bytes apart (at most 2^26)", what, of, (long long)stride_codes, (long long)stride_scales);
    if (!aligned(codes, stride_codes, 16) || !aligned(scales, stride_scales, 4))
        return dg_fail(DG_ERR_BUFFER, "%s: %s: rows of codes begin on 16 bytes, rows of scales on 4", what, of);
    return DG_OK;
}

dg_status check_sizes(const char *what, dg_dtype type, int64_t N, int64_t K)
{
    if (N < 0 || K <= 0 || N > MOST_ROWS) return dg_fail(DG_ERR_SHAPE, "%s: N=%lld K=%lld", what, (long long)N, (long long)K);
    if (K > MOST_K) return dg_fail(DG_ERR_RANGE, "%s: K=%lld (at most 2^24)", what, (long long)K);
    if (!known_type(type)) return dg_fail(DG_ERR_UNSUPPORTED, "%s: unknown element type %d", what, (int)type);
    return DG_OK;
}

dg_status check_plain_rows(const char *what, const char *of, const void *x, int64_t N, int64_t K, int64_t stride)
{
    if (N > 0 && !x) return dg_fail(DG_ERR_NULL, "%s: NULL %s", what, of);
    if (stride < K) return dg_fail(DG_ERR_SHAPE, "%s: %s of %lld elements every %lld", what, of, (long long)K, (long long)stride);
    return DG_OK;
}

dg_status check_product(const char *what, const uint8_t *W, int64_t stride_w, const uint8_t *W_scales, int64_t stride_ws, int64_t M, int64_t N, int64_t K,
                        const void *out, dg_dtype type, int64_t stride_out)
{
    if (M <= 0 || M > MOST_ROWS) return dg_fail(DG_ERR_SHAPE, "%s: M=%lld N=%lld K=%lld", what, (long long)M, (long long)N, (long long)K);
    dg_status s = check_sizes(what, type, N, K);
    if (!s) s = check_rows(what, "weights", W, stride_w, W_scales, stride_ws, M, K);
    if (!s) s = check_plain_rows(what, "output rows", out, N, M, stride_out);
    if (!s && (M + 63) / 64 * ((N + 63) / 64) > MOST_ROWS)
        s = dg_fail(DG_ERR_RANGE, "%s: M=%lld N=%lld is too large for one call", what, (long long)M, (long long)N);
    return s;
}

dg_status check_work(const char *what, const void *work, size_t bytes, size_t need)
{
    if (!work) return dg_fail(DG_ERR_NULL, "%s: NULL work buffer (%zu bytes are needed)", what, need);
    if (bytes < need || (uintptr_t)work % 16 != 0)
        return dg_fail(DG_ERR_BUFFER, "%s: a work buffer of %zu bytes, 16-byte aligned, is needed (%zu given)", what, need, bytes);
    return DG_OK;
}

bool route_sizes(int64_t T, int64_t E) { return T > 0 && E > 0 && E <= 1024 && T <= MOST_ROWS / E; }
bool expert_sizes(int64_t T, int64_t top, int64_t hidden, int64_t inner)
{
    return T > 0 && T <= MOST_ROWS / 64 && top > 0 && top <= 64 && hidden > 0 && hidden <= 1 << 20 && inner > 0 && inner <= 1 << 20;
}

}   // namespace

extern "C" {

dg_status dg_quantize_mx4(const void *x_dev, dg_dtype type, int64_t N, int64_t K, int64_t stride_n, uint8_t *codes_dev, int64_t stride_codes,
                          uint8_t *scales_dev, int64_t stride_scales, void *hip_stream)
{
    const char *what = "dg_quantize_mx4";
    dg_status s = check_sizes(what, type, N, K);
    if (!s) s = check_plain_rows(what, "activations", x_dev, N, K, stride_n);
    if (!s) s = check_rows(what, "output rows", codes_dev, stride_codes, scales_dev, stride_scales, N, K);
    if (s || N == 0) return s;
    return dg_launch_quantize_mx4(x_dev, type, N, K, stride_n, codes_dev, stride_codes, scales_dev, stride_scales, (hipStream_t)hip_stream);
}

dg_status dg_dequantize_mx4(const uint8_t *codes_dev, int64_t stride_codes, const uint8_t *scales_dev, int64_t stride_scales, int64_t N, int64_t K,
                            void *out_dev, dg_dtype type, int64_t stride_out, void *hip_stream)
{
    const char *what = "dg_dequantize_mx4";
    dg_status s = check_sizes(what, type, N, K);
    if (!s) s = check_rows(what, "rows", codes_dev, stride_codes, scales_dev, stride_scales, N, K);
    if (!s) s = check_plain_rows(what, "output rows", out_dev, N, K, stride_out);
    if (s || N == 0) return s;
    return dg_launch_dequantize_mx4(codes_dev, stride_codes, scales_dev, stride_scales, N, K, out_dev, type, stride_out, (hipStream_t)hip_stream);
}

dg_status dg_gemm_mx4(const uint8_t *W_dev, int64_t stride_w, const uint8_t *W_scales_dev, int64_t stride_ws, const uint8_t *A_dev, int64_t stride_a,
                      const uint8_t *A_scales_dev, int64_t stride_as, int64_t M, int64_t N, int64_t K, const float *bias_m_dev, void *out_dev,
                      dg_dtype out_type, int64_t stride_out, void *hip_stream)
{
    const char *what = "dg_gemm_mx4";
    dg_status s = check_product(what, W_dev, stride_w, W_scales_dev, stride_ws, M, N, K, out_dev, out_type, stride_out);
    if (!s) s = check_rows(what, "tokens", A_dev, stride_a, A_scales_dev, stride_as, N, K);
    if (s || N == 0) return s;
    const DgGemmMx4 p = {W_dev, W_scales_dev, A_dev, A_scales_dev, stride_w, stride_ws, stride_a, stride_as, (int32_t)M, (int32_t)N,
                         (int32_t)blocks_of(K), bias_m_dev, out_dev, stride_out};
    return dg_launch_gemm_mx4(p, out_type, (hipStream_t)hip_stream);
}

size_t dg_linear_mx4_work_bytes(int64_t N, int64_t K)
{
    return N <= 0 || K <= 0 || N > MOST_ROWS || K > MOST_K ? 0 : (size_t)(N * (codes_pitch(K) + scales_pitch(K)));
}

dg_status dg_linear_mx4(const uint8_t *W_dev, int64_t stride_w, const uint8_t *W_scales_dev, int64_t stride_ws, const void *x_dev, dg_dtype x_type,
                        int64_t stride_x, int64_t M, int64_t N, int64_t K, const float *bias_m_dev, void *work_dev, size_t work_bytes, void *out_dev,
                        dg_dtype out_type, int64_t stride_out, void *hip_stream)
{
    const char *what = "dg_linear_mx4";
    dg_status s = check_product(what, W_dev, stride_w, W_scales_dev, stride_ws, M, N, K, out_dev, out_type, stride_out);
    if (!s) s = check_sizes(what, x_type, N, K);
    if (!s) s = check_plain_rows(what, "activations", x_dev, N, K, stride_x);
    if (s || N == 0) return s;
    s = check_work(what, work_dev, work_bytes, dg_linear_mx4_work_bytes(N, K));
    if (s) return s;
    uint8_t *codes = (uint8_t *)work_dev, *scales = codes + N * codes_pitch(K);
    const DgGemmMx4 p = {W_dev, W_scales_dev, codes, scales, stride_w, stride_ws, codes_pitch(K), scales_pitch(K), (int32_t)M, (int32_t)N,
                         (int32_t)blocks_of(K), bias_m_dev, out_dev, stride_out};
    if (dg_linear_mx4_fuses(N, x_dev)) return dg_launch_linear_mx4_fused(p, x_dev, x_type, K, out_type, (hipStream_t)hip_stream);
    s = dg_launch_quantize_mx4(x_dev, x_type, N, K, stride_x, codes, p.stride_a, scales, p.stride_as, (hipStream_t)hip_stream);
    if (s) return s;
    return dg_launch_gemm_mx4(p, out_type, (hipStream_t)hip_stream);
}

size_t dg_route_tokens_work_bytes(int64_t T, int64_t E) { return route_sizes(T, E) ? dg_route_work_bytes(T, E) : 0; }

dg_status dg_route_tokens(const void *x_dev, dg_dtype x_type, int64_t T, int64_t K, int64_t stride_x, const void *R_dev, dg_dtype r_type, int64_t E,
                          int64_t stride_r, const float *bias_e_dev, int64_t top, dg_route_mode mode, float factor, int32_t *ids_dev, float *weights_dev,
                          void *work_dev, size_t work_bytes, void *hip_stream)
{
    const char *what = "dg_route_tokens";
    if (T < 0 || K <= 0 || E <= 0 || top <= 0 || top > E)
        return dg_fail(DG_ERR_SHAPE, "%s: T=%lld K=%lld, %lld of %lld experts", what, (long long)T, (long long)K, (long long)top, (long long)E);
    if (E > 1024 || top > 64 || K > MOST_K || T > MOST_ROWS / E)
        return dg_fail(DG_ERR_RANGE, "%s: T=%lld K=%lld, %lld of %lld experts (at most 64 of 1024)", what, (long long)T, (long long)K, (long long)top, (long long)E);
    if (!known_type(x_type) || (r_type != x_type && r_type != DG_F32))
        return dg_fail(DG_ERR_UNSUPPORTED, "%s: element types %d and %d (the router's is the activations' or binary32)", what, (int)x_type, (int)r_type);
    if (mode != DG_ROUTE_SOFTMAX && mode != DG_ROUTE_SOFTMAX_ALL && mode != DG_ROUTE_SIGMOID) return dg_fail(DG_ERR_UNSUPPORTED, "%s: unknown mode %d", what, (int)mode);
    dg_status s = check_plain_rows(what, "activations", x_dev, T, K, stride_x);
    if (!s) s = check_plain_rows(what, "router", R_dev, E, K, stride_r);
    if (s || T == 0) return s;
    if (!ids_dev || !weights_dev) return dg_fail(DG_ERR_NULL, "%s: NULL output", what);
    s = check_work(what, work_dev, work_bytes, dg_route_tokens_work_bytes(T, E));
    if (s) return s;
    const DgRoute p = {x_dev, R_dev, stride_x, stride_r, (int32_t)T, (int32_t)K, (int32_t)E, (int32_t)top, bias_e_dev, mode, factor, ids_dev, weights_dev, {(float *)work_dev}};
    return dg_launch_route(p, x_type, r_type, (hipStream_t)hip_stream);
}

size_t dg_experts_mx4_work_bytes(int64_t T, int64_t top, int64_t hidden, int64_t inner)
{
    return expert_sizes(T, top, hidden, inner) ? (size_t)dg_experts_work_bytes(T, top, hidden, inner) : 0;
}

dg_status dg_experts_mx4(const dg_experts_desc *desc, const void *x_dev, dg_dtype type, int64_t T, int64_t stride_x, const int32_t *ids_dev,
                         const float *weights_dev, int64_t top, void *work_dev, size_t work_bytes, void *out_dev, int64_t stride_out, void *hip_stream)
{
    const char *what = "dg_experts_mx4";
    if (!desc) return dg_fail(DG_ERR_NULL, "%s: NULL experts", what);
    const dg_experts_desc &d = *desc;
    if (d.experts <= 0 || d.hidden <= 0 || d.inner <= 0 || T < 0 || top <= 0)
        return dg_fail(DG_ERR_SHAPE, "%s: %d experts of %d channels and %d, %lld tokens to %lld each", what, (int)d.experts, (int)d.hidden, (int)d.inner, (long long)T,
                       (long long)top);
    if (d.experts > 1 << 16 || (T > 0 && !expert_sizes(T, top, d.hidden, d.inner)) || top > 64)
        return dg_fail(DG_ERR_RANGE, "%s: %d experts of %d channels and %d, %lld tokens to %lld each", what, (int)d.experts, (int)d.hidden, (int)d.inner, (long long)T,
                       (long long)top);
    if ((type != DG_F16 && type != DG_BF16) || d.reserved != 0) return dg_fail(DG_ERR_UNSUPPORTED, "%s: activations of element type %d (binary16 or bfloat16)", what, (int)type);
    dg_status s = check_rows(what, "up", d.up, d.up_row, d.up_scales, d.up_scales_row, 2 * (int64_t)d.inner, d.hidden);
    if (!s) s = check_rows(what, "down", d.down, d.down_row, d.down_scales, d.down_scales_row, d.hidden, d.inner);
    if (!s && (d.up_expert < 0 || d.down_expert < 0 || d.up_scales_expert < 0 || d.down_scales_expert < 0))
        s = dg_fail(DG_ERR_SHAPE, "%s: experts lie backwards", what);
    if (!s && (d.up_expert % 16 || d.down_expert % 16 || d.up_scales_expert % 4 || d.down_scales_expert % 4))
        s = dg_fail(DG_ERR_BUFFER, "%s: rows of codes begin on 16 bytes, rows of scales on 4", what);
    if (!s) s = check_plain_rows(what, "activations", x_dev, T, d.hidden, stride_x);
    if (!s) s = check_plain_rows(what, "output rows", out_dev, T, d.hidden, stride_out);
    if (s || T == 0) return s;
    if (!ids_dev || !weights_dev) return dg_fail(DG_ERR_NULL, "%s: NULL ids or weights", what);
    s = check_work(what, work_dev, work_bytes, dg_experts_mx4_work_bytes(T, top, d.hidden, d.inner));
    if (s) return s;
    const DgExperts p = {d, x_dev, out_dev, stride_x, stride_out, ids_dev, weights_dev, (int32_t)T, (int32_t)top, work_dev};
    return dg_launch_experts(p, type, (hipStream_t)hip_stream);
}

}   // extern "C"
