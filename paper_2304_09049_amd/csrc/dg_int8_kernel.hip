// Tokens quantised to 8 bits, and products of 8-bit codes with a scale for each token and each channel.
#include "dg_decoder.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

// ---- quantising tokens: one workgroup per token, two passes over its row (the second finds it in the caches) --------------

template <class T>
__global__ __launch_bounds__(256) void quantize_tokens_kernel(const T *x, int32_t K, int64_t stride_n, int8_t *codes, int64_t stride_codes,
                                                               float *scale)
{
    __shared__ float part[4];
    __shared__ int whole[4];
    const T *row = x + (int64_t)blockIdx.x * stride_n;
    int8_t *out = codes + (int64_t)blockIdx.x * stride_codes;
    float most = 0.0f;
    bool finite = true;
    for (int k = threadIdx.x; k < K; k += 256) {
        const float f = fabsf(dg_to_float(row[k]));
        most = fmaxf(most, f);
        finite = finite && f < __builtin_inff();
    }
#pragma unroll
    for (int i = 32; i; i >>= 1) most = fmaxf(most, __shfl_xor(most, i));
    finite = __all(finite);
    if ((threadIdx.x & 63) == 0) {
        part[threadIdx.x >> 6] = most;
        whole[threadIdx.x >> 6] = finite;
    }
    __syncthreads();
    most = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    const float s = whole[0] && whole[1] && whole[2] && whole[3] ? dg_scale8(most) : __builtin_nanf("");
    if (threadIdx.x == 0) scale[blockIdx.x] = s;
    for (int k = threadIdx.x; k < K; k += 256) out[k] = (int8_t)dg_code8(dg_to_float(row[k]), s);
}

// ---- the product ------------------------------------------------------------------------------------------------------

// 16 codes from position k of a row of K; those at K and beyond count as 0 and are not read.
__device__ __forceinline__ v4i codes16(const int8_t *row, int32_t k, int32_t K)
{
    v4i v = {0, 0, 0, 0};
    if (k + 16 <= K)
        __builtin_memcpy(&v, row + k, 16);
    else
        for (int i = 0; k + i < K; ++i) v[i >> 2] |= (int)(uint8_t)row[k + i] << (8 * (i & 3));
    return v;
}

// 16 channels x 16 TOKENS tokens by a workgroup whose eight wavefronts share K; their sums meet in LDS.
template <class T, int TOKENS>
__global__ __launch_bounds__(512) void gemm_i8_few_kernel(DgGemmI8 p)
{
    __shared__ v4i sums[7][TOKENS][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int32_t m0 = blockIdx.x * 16, n0 = blockIdx.y * (16 * TOKENS);
    const int8_t *w = p.W + (int64_t)min(m0 + r, p.M - 1) * p.stride_w;
    const int8_t *a[TOKENS];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) a[t] = p.A + (int64_t)min(n0 + 16 * t + r, p.N - 1) * p.stride_a;
    v4i acc[TOKENS] = {};
    for (int32_t k = 64 * wave; k < p.K; k += 512) {
        const v4i wk = codes16(w, k + 16 * g, p.K);
#pragma unroll
        for (int t = 0; t < TOKENS; ++t)
            acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wk, codes16(a[t], k + 16 * g, p.K), acc[t], 0, 0, 0);
    }
    if (wave)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) sums[wave - 1][t][lane] = acc[t];
    __syncthreads();
    // wavefront w finishes token blocks w, w + 8, ... (its own sums are among the ones in LDS unless it is the first)
    if (wave) return;
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        v4i s = acc[t];
#pragma unroll
        for (int i = 0; i < 7; ++i) s += sums[i][t][lane];
        const int32_t n = n0 + 16 * t + r;
        if (n >= p.N) continue;
        const float sn = p.scale_n[n];
        T *out = (T *)p.out + (int64_t)n * p.stride_out;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t m = m0 + 4 * g + i;
            if (m >= p.M) continue;
            const float y = (float)s[i] * p.scale_m[m] * sn;
            out[m] = dg_from_float<T>(p.bias ? y + p.bias[m] : y);
        }
    }
}

}   // namespace

dg_status dg_launch_quantize_tokens(const void *x, dg_dtype type, int64_t N, int64_t K, int64_t stride_n, int8_t *codes,
                                    int64_t stride_codes, float *scale, hipStream_t stream)
{
    dg_with_type(type, [&](auto t) {
        quantize_tokens_kernel<<<(uint32_t)N, 256, 0, stream>>>((const decltype(t) *)x, (int32_t)K, stride_n, codes, stride_codes, scale);
        return 0;
    });
    return dg_check_launch("dg_quantize_tokens");
}

dg_status dg_launch_gemm_i8(const DgGemmI8 &p, dg_dtype type, hipStream_t stream)
{
    dg_with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const uint32_t rows = (uint32_t)((p.M + 15) / 16);
        if (p.N <= 16) gemm_i8_few_kernel<T, 1><<<dim3(rows, 1), 512, 0, stream>>>(p);
        else gemm_i8_few_kernel<T, 4><<<dim3(rows, (uint32_t)((p.N + 63) / 64)), 512, 0, stream>>>(p);
        return 0;
    });
    return dg_check_launch("dg_gemm_i8");
}
