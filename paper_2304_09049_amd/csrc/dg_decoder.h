// What the kernels of a quantised decoder layer share (8-bit and 4-bit products, the paged cache, the attention on it, experts): element types, the
// cache's layout and the launchers.  Internal; the public ABI is include/deepgemm_hip.h.
#pragma once

#include <algorithm>

#include "dg_common.h"

// ---- element types -----------------------------------------------------------------------------------------------------

template <class T>
__device__ __forceinline__ float dg_to_float(T x) { return (float)x; }
// One rounding to nearest even (none for binary32).
template <class T>
__device__ __forceinline__ T dg_from_float(float x) { return (T)x; }

// COUNT neighbouring elements; the address needs the element's alignment only (the hardware takes vector accesses at any).
template <class T, int COUNT>
struct DgVec {
    T e[COUNT];
};
template <class T, int COUNT>
__device__ __forceinline__ DgVec<T, COUNT> dg_load_vec(const T *p)
{
    DgVec<T, COUNT> v;
    __builtin_memcpy(&v, p, sizeof(v));
    return v;
}
template <class T, int COUNT>
__device__ __forceinline__ void dg_store_vec(T *p, const DgVec<T, COUNT> &v)
{
    __builtin_memcpy(p, &v, sizeof(v));
}

// Elements k ... k + 7 of a row; those at K and beyond are 0 and are not read.
template <class T>
__device__ __forceinline__ DgVec<T, 8> dg_eight(const T *row, int32_t k, int32_t K)
{
    if (k + 8 <= K) return dg_load_vec<T, 8>(row + k);
    DgVec<T, 8> v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v.e[i] = k + i < K ? row[k + i] : T(0.0f);
    return v;
}

// f(element type) for a dg_dtype that the API layer has checked.
template <class F>
auto dg_with_type(dg_dtype type, F f)
{
    if (type == DG_F32) return f(float{});
    if (type == DG_F16) return f((_Float16){});
    return f((__bf16){});
}
inline int64_t dg_type_size(dg_dtype type) { return type == DG_F32 ? 4 : 2; }

// ---- one number out of a wavefront's, by register moves (a shuffle by way of LDS is some 130 cycles, and six of them make a kernel of 2 us 0.3 longer) ----

template <int CONTROL>
__device__ __forceinline__ float dg_other_lane(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CONTROL, 0xF, 0xF, false));
}
// f over neighbouring lanes, the same in each: 8 or 16 of them, the four that are 16 apart, all 64.
template <int LANES, class F>
__device__ __forceinline__ float dg_over_lanes(float v, F f)
{
    static_assert(LANES == 8 || LANES == 16, "within a row of lanes");
    if (LANES == 16) v = f(v, dg_other_lane<0x140>(v));        // row_mirror
    v = f(v, dg_other_lane<0xB1>(v));          // quad_perm 1, 0, 3, 2
    v = f(v, dg_other_lane<0x4E>(v));          // quad_perm 2, 3, 0, 1
    return f(v, dg_other_lane<0x141>(v));      // row_half_mirror
}
template <class F>
__device__ __forceinline__ float dg_over_rows(float v, F f)
{
    const auto near = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(near[0]), __uint_as_float(near[1]));
    const auto far = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(far[0]), __uint_as_float(far[1]));
}
template <class F>
__device__ __forceinline__ float dg_over_wave(float v, F f) { return dg_over_rows(dg_over_lanes<16>(v, f), f); }
struct DgMax {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct DgMin {
    __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); }
};
struct DgAdd {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

// ---- quantisers (binary32, operation by operation) -----------------------------------------------------------------------

// Division by one s for many x, correctly rounded and without a branch: x times the rounded reciprocal, then twice the remainder, which a fused
// multiply-add gives exactly, times the reciprocal added on (Markstein's theorem: a quotient within one unit of the last place and a correctly
// rounded reciprocal give the correctly rounded quotient; the first correction brings it within one unit).  Nine instructions a code where the
// divide takes about twenty; and short code counts as well: a kernel of a few microseconds waits for its instructions to arrive, 17 us for 256 tokens of
// 4096 with eight divides written out for 4 with these.  `up`: a power of two that keeps remainders and reciprocal in range; x comes times it.
struct DgDivisor {
    float s, inverse, up;
    uint32_t keep;            // 0 where codes are 0 by definition: s is 0 or NaN
};
__device__ __forceinline__ DgDivisor dg_divisor(float s)
{
    DgDivisor d;
    d.up = s < 0x1p-60f ? 0x1p64f : s > 0x1p60f ? 0x1p-64f : 1.0f;
    d.s = s > 0.0f ? s * d.up : 0.0f;
    d.inverse = s > 0.0f ? 1.0f / d.s : 0.0f;
    d.keep = s > 0.0f ? 0xFFFFFFFFu : 0u;
    return d;
}
__device__ __forceinline__ float dg_quotient(float x, const DgDivisor &d)
{
    float q = x * d.inverse;
    q = __builtin_fmaf(__builtin_fmaf(-q, d.s, x), d.inverse, q);
    return __builtin_fmaf(__builtin_fmaf(-q, d.s, x), d.inverse, q);
}
// A code, before `keep`: of the symmetric 8-bit quantiser (s = max|x| / 127), of the 4-bit one (x is about s * code + z).
__device__ __forceinline__ int dg_code8(float x, const DgDivisor &d)
{
    return (int)__builtin_amdgcn_fmed3f(rintf(dg_quotient(x * d.up, d)), -127.0f, 127.0f);
}
__device__ __forceinline__ int dg_code4(float x, float z, const DgDivisor &d)
{
    return (int)__builtin_amdgcn_fmed3f(rintf(dg_quotient(x * d.up - z * d.up, d)), 0.0f, 15.0f);
}
// Four codes as bytes, the first lowest.
__device__ __forceinline__ uint32_t dg_bytes(const int *code)
{
    const uint32_t a = __builtin_amdgcn_perm((uint32_t)code[1], (uint32_t)code[0], 0x0C0C0400u);
    return __builtin_amdgcn_perm((uint32_t)code[3], (uint32_t)code[2], 0x04000C0Cu) | a;
}
// The scale for a row whose largest magnitude is `most`; a row with an infinity or a NaN (`most` not finite) gets a NaN, so that
// whatever is computed from it shows it.
__device__ __forceinline__ float dg_scale8(float most) { return most < __builtin_inff() ? most / 127.0f : __builtin_nanf(""); }

// ---- the cache ---------------------------------------------------------------------------------------------------------

// A cache as the kernels take it.  A page holds `heads` blocks of `head` bytes: keys' codes (`part` bytes), values' codes (`part`),
// then `page_size` binary32 numbers each of key scale, value scale and, 4 bits, key z and value z.  `head` is below 2^31 (the API layer has seen to it),
// so places within a head are 32-bit numbers; a token's bytes are whole, so that no product here is larger than what it stands for.
struct DgCache {
    uint8_t *base;
    int32_t pages, page_size, heads, dim, bits;
    int32_t part, head;
    DgFastDiv by_page;                  // token number / page_size
    __host__ __device__ int64_t page_bytes() const { return (int64_t)head * heads; }
};

inline DgCache dg_cache_of(const dg_cache_desc *d, void *base)
{
    DgCache c;
    c.base = (uint8_t *)base;
    c.pages = d->pages;
    c.page_size = d->page_size;
    c.heads = d->heads;
    c.dim = d->dim;
    c.bits = d->bits;
    c.part = d->page_size * (d->dim * d->bits / 8);
    c.head = 2 * c.part + d->page_size * (d->bits == 8 ? 8 : 16);
    c.by_page = dg_make_div((uint32_t)d->page_size);
    return c;
}

// Where the byte of channel d (4 bits: of channels d and d + 1, d even) of a page's token t lies in the keys' or the values' codes.
template <int BITS>
__device__ __forceinline__ uint32_t dg_key_byte(uint32_t t, uint32_t d, uint32_t dim)
{
    return (t >> 4) * (2 * BITS * dim) + (d >> 4) * (32 * BITS) + (t & 15) * (2 * BITS) + (d & 15) * BITS / 8;
}
template <int BITS>
__device__ __forceinline__ uint32_t dg_value_byte(uint32_t t, uint32_t d, uint32_t dim)
{
    return (t >> 2) * (BITS * dim / 2) + (d * BITS / 8) * 4 + (t & 3);
}

// ---- launchers (each validates nothing: the API layer has done that) ---------------------------------------------------

// f(first, count) for `total` rows, `most` a launch: HIP counts a grid's threads in 32 bits, and the kernels count rows in them.
template <class F>
dg_status dg_in_turns(int64_t total, int64_t most, F f)
{
    for (int64_t first = 0; first < total; first += most) {
        const dg_status s = f(first, std::min(most, total - first));
        if (s) return s;
    }
    return DG_OK;
}

// pad: K, or up to where a row's codes are cleared
dg_status dg_launch_quantize_tokens(const void *x, dg_dtype type, int64_t N, int64_t K, int64_t stride_n, int8_t *codes,
                                    int64_t stride_codes, int64_t pad, float *scale, hipStream_t stream);

struct DgGemmI8 {
    const int8_t *W, *A;
    int64_t stride_w, stride_a;          // bytes from row to row
    int32_t M, N, K;
    const float *scale_m, *scale_n, *bias;
    void *out;
    int64_t stride_out;                  // elements from token to token
};
dg_status dg_launch_gemm_i8(const DgGemmI8 &p, dg_dtype type, hipStream_t stream);
// The product's kernel for few tokens quantising one itself (p.A and p.scale_n are not used), and whether it does.
bool dg_linear_i8_fuses(int64_t N, int64_t K);
dg_status dg_launch_linear_i8_fused(const DgGemmI8 &p, const void *x, dg_dtype x_type, dg_dtype type, hipStream_t stream);

dg_status dg_launch_cache_write(const DgCache &c, const void *k, const void *v, dg_dtype type, int64_t T, const int64_t strides[4],
                                const int32_t *slots, hipStream_t stream);
dg_status dg_launch_cache_read(const DgCache &c, const int32_t *slots, int64_t T, void *k, void *v, dg_dtype type, hipStream_t stream);

struct DgAttention {
    DgCache cache;
    const void *q;
    void *out;
    int64_t q_token, q_head, out_token, out_head;        // element strides
    const int32_t *q_start, *ctx_len, *table;
    int32_t T, Hq, B, table_width, max_q, max_ctx;
    float scale;
    int32_t causal;
    void *work;
};
int64_t dg_attention_work_bytes(const DgAttention &p);
dg_status dg_launch_attention(const DgAttention &p, dg_dtype type, hipStream_t stream);

// ---- microscaled 4-bit floating point ------------------------------------------------------------------------------------

// A scale's byte as a binary32 number: 2^(byte - 127), NaN for 255.
__device__ __forceinline__ float dg_mx_scale(uint32_t byte)
{
    const uint32_t bits = byte == 0 ? 0x00400000u : byte << 23;
    return __uint_as_float(byte == 255 ? 0x7FC00000u : bits);
}

dg_status dg_launch_quantize_mx4(const void *x, dg_dtype type, int64_t N, int64_t K, int64_t stride_n, uint8_t *codes, int64_t stride_codes,
                                 uint8_t *scales, int64_t stride_scales, hipStream_t stream);
dg_status dg_launch_dequantize_mx4(const uint8_t *codes, int64_t stride_codes, const uint8_t *scales, int64_t stride_scales, int64_t N, int64_t K,
                                   void *out, dg_dtype type, int64_t stride_out, hipStream_t stream);
struct DgGemmMx4 {
    const uint8_t *W, *W_scales, *A, *A_scales;
    int64_t stride_w, stride_ws, stride_a, stride_as;    // bytes from row to row
    int32_t M, N, blocks;                                // blocks of 32 in a row
    const float *bias;
    void *out;
    int64_t stride_out;                                  // elements from token to token
};
dg_status dg_launch_gemm_mx4(const DgGemmMx4 &p, dg_dtype type, hipStream_t stream);
// The product's kernel for few tokens quantising one itself (p.A and p.A_scales are not used), and whether it does.
bool dg_linear_mx4_fuses(int64_t N, const void *x);
dg_status dg_launch_linear_mx4_fused(const DgGemmMx4 &p, const void *x, dg_dtype x_type, int64_t K, dg_dtype type, hipStream_t stream);

struct DgRoute {
    const void *x, *R;
    int64_t stride_x, stride_r;                          // elements
    int32_t T, K, E, top;
    const float *bias;
    dg_route_mode mode;
    float factor;
    int32_t *ids;
    float *weights;
    union {                                              // (the work buffer)
        float *logits;                                   // [T][E]
        double *sums;                                    // of parts of K: [parts][T][E]
    };
};
dg_status dg_launch_route(const DgRoute &p, dg_dtype x_type, dg_dtype r_type, hipStream_t stream);

struct DgExperts {
    dg_experts_desc d;
    const void *x;
    void *out;
    int64_t stride_x, stride_out;                        // elements
    const int32_t *ids;
    const float *weights;
    int32_t T, top;
    void *work;
};
int64_t dg_experts_work_bytes(int64_t T, int64_t top, int64_t hidden, int64_t inner);
dg_status dg_launch_experts(const DgExperts &p, dg_dtype type, hipStream_t stream);
