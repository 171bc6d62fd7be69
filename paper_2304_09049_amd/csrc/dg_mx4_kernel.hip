// Rows quantised to microscaled 4-bit floating point and read back, and products of such rows.
#include "dg_decoder.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));

// ---- quantising and reading back -----------------------------------------------------------------------------------------
//
// A lane has 8 elements of a block, four neighbouring lanes a block of 32; rows lie behind one another in the lanes' numbers, blocks not cut.  The largest magnitude is found on the
// numbers' bits, which order as they do and put infinities and NaN above all, and its exponent is the scale: no division, and the conversion takes the scale itself.

constexpr int THREADS = 256;

struct MxRows {
    int64_t stride_x, stride_codes, stride_scales;       // elements, bytes, bytes
    int32_t K;
    uint32_t total;                                      // lanes' pieces of 8 elements
    DgFastDiv by_row;                                    // a row's pieces
};

__device__ __forceinline__ uint32_t most_of_four(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));        // quad_perm 1, 0, 3, 2
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));     // quad_perm 2, 3, 0, 1
}

// The scale's byte for a block whose largest magnitude has these bits.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most)
{
    const uint32_t exponent = most >> 23;
    return exponent == 255 ? 255u : max(exponent, 2u) - 2u;
}

__device__ __forceinline__ uint32_t codes_of(const float (&f)[8], uint32_t byte)
{
    const float s = dg_mx_scale(byte);
    int word = 0;
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, f[0], f[1], s, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, f[2], f[3], s, 1);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, f[4], f[5], s, 2);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, f[6], f[7], s, 3);
    return byte == 255 ? 0u : (uint32_t)word;
}

template <class T, int HELD>
__global__ __launch_bounds__(THREADS) void quantize_mx4_kernel(const T *x, MxRows r, uint8_t *codes, uint8_t *scales)
{
    const uint32_t first = blockIdx.x * (THREADS * HELD) + threadIdx.x;
    DgVec<T, 8> held[HELD];
    uint32_t row[HELD], piece[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const uint32_t at = min(first + i * THREADS, r.total - 1);
        row[i] = dg_fdiv(at, r.by_row);
        piece[i] = at - row[i] * r.by_row.d;
        held[i] = dg_eight<T>(x + row[i] * r.stride_x, 8 * piece[i], r.K);
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        float f[8];
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = dg_to_float(held[i].e[j]);
            most = max(most, __float_as_uint(f[j]) & 0x7FFFFFFFu);
        }
        const uint32_t byte = scale_byte(most_of_four(most));
        if (first + i * THREADS < r.total) {
            *(uint32_t *)(codes + row[i] * r.stride_codes + 4 * piece[i]) = codes_of(f, byte);
            if (piece[i] % 4 == 0) scales[row[i] * r.stride_scales + piece[i] / 4] = (uint8_t)byte;
        }
    }
}

template <class T, int HELD>
__global__ __launch_bounds__(THREADS) void dequantize_mx4_kernel(const uint8_t *codes, const uint8_t *scales, MxRows r, T *out)
{
    const uint32_t first = blockIdx.x * (THREADS * HELD) + threadIdx.x;
    uint32_t word[HELD], byte[HELD], row[HELD], piece[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const uint32_t at = min(first + i * THREADS, r.total - 1);
        row[i] = dg_fdiv(at, r.by_row);
        piece[i] = at - row[i] * r.by_row.d;
        word[i] = *(const uint32_t *)(codes + row[i] * r.stride_codes + 4 * piece[i]);
        byte[i] = scales[row[i] * r.stride_scales + piece[i] / 4];
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        if (first + i * THREADS >= r.total) break;
        const float s = dg_mx_scale(byte[i]);
        const v2f f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], s, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], s, 3)};
        DgVec<T, 8> v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v.e[j] = dg_from_float<T>(byte[i] == 255 ? s : f[j / 2][j % 2]);
        T *to = out + row[i] * r.stride_x + 8 * piece[i];
        const int32_t left = r.K - 8 * (int32_t)piece[i];
        if (left >= 8) dg_store_vec<T, 8>(to, v);
        else
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < left) to[j] = v.e[j];
    }
}

// f(the pieces of a launch, its first row): pieces' numbers are 31-bit, and a launch's rows as many as that allows.
template <class F>
void in_launches(int64_t N, int64_t K, int64_t stride_x, int64_t stride_codes, int64_t stride_scales, F f)
{
    const int64_t pieces = (K + 31) / 32 * 4;
    dg_in_turns(N, std::max<int64_t>(1, ((int64_t)1 << 30) / pieces), [&](int64_t n, int64_t rows) {
        const MxRows r = {stride_x, stride_codes, stride_scales, (int32_t)K, (uint32_t)(rows * pieces), dg_make_div((uint32_t)pieces)};
        f(r, n);
        return DG_OK;
    });
}

// ---- the product: few tokens ---------------------------------------------------------------------------------------------
//
// v_mfma_scale_f32_16x16x128_f8f6f4: lane (r, g) holds block g of four of row r, 16 bytes as they lie, and the block's scale in the lowest byte of a register.
// Sums come out with four neighbouring channels of one token in a lane.
// A workgroup computes 16 ROWS channels x 16 TOKENS tokens; its wavefronts share K in pieces of 256 positions, a cache line of a row, and their sums meet in LDS,
// in the wavefronts' order.

__device__ __forceinline__ v4f multiply(const v4i &w, const v4i &a, const v4f &c, int ws, int as)
{
    const v8i x = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, y = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, ws, 0, as);
}

// Four neighbouring channels of token n.
template <class T>
__device__ __forceinline__ void store4(const DgGemmMx4 &p, int32_t m, int32_t n, const v4f &sum)
{
    T *out = (T *)p.out + (int64_t)n * p.stride_out + m;
    DgVec<T, 4> y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y.e[i] = dg_from_float<T>(p.bias && m + i < p.M ? sum[i] + p.bias[m + i] : sum[i]);
    if (m + 4 <= p.M) dg_store_vec<T, 4>(out, y);
    else
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (m + i < p.M) out[i] = y.e[i];
}

// Block b of a row of `blocks`, and its scale's byte; past them zeros.
__device__ __forceinline__ v4i block_or_zero(const uint8_t *row, int32_t b, int32_t blocks) { return b < blocks ? *(const v4i *)(row + 16 * (int64_t)b) : v4i{}; }
__device__ __forceinline__ int scale_or_zero(const uint8_t *row, int32_t b, int32_t blocks) { return b < blocks ? row[b] : 0; }

template <class T, int WAVES, int ROWS, int TOKENS>
__global__ __launch_bounds__(64 * WAVES) void gemm_mx4_few_kernel(DgGemmMx4 p)
{
    __shared__ v4f sums[WAVES][ROWS][TOKENS][64];
    // (a matrix instruction runs whatever the lanes' mask: what it stands under has to be a scalar branch)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t m0 = blockIdx.x * (16 * ROWS), n0 = blockIdx.y * (16 * TOKENS);
    const uint8_t *w[ROWS], *ws[ROWS], *a[TOKENS], *as[TOKENS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t row = min(m0 + 16 * i + r, p.M - 1);
        w[i] = p.W + row * p.stride_w;
        ws[i] = p.W_scales + row * p.stride_ws;
    }
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        const int64_t row = min(n0 + 16 * t + r, p.N - 1);
        a[t] = p.A + row * p.stride_a;
        as[t] = p.A_scales + row * p.stride_as;
    }
    v4f acc[ROWS][TOKENS] = {};
    const int32_t pieces = p.blocks / 8;
    for (int32_t piece = wave; piece < pieces; piece += WAVES) {
        v4i wk[ROWS][2], ak[TOKENS][2];
        uint2 wsk[ROWS], ask[TOKENS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) wk[i][h] = *(const v4i *)(w[i] + 128 * (int64_t)piece + 64 * h + 16 * g);
            wsk[i] = dg_load_vec<uint2, 1>((const uint2 *)(ws[i] + 8 * (int64_t)piece)).e[0];
        }
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) {
#pragma unroll
            for (int h = 0; h < 2; ++h) ak[t][h] = *(const v4i *)(a[t] + 128 * (int64_t)piece + 64 * h + 16 * g);
            ask[t] = dg_load_vec<uint2, 1>((const uint2 *)(as[t] + 8 * (int64_t)piece)).e[0];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < TOKENS; ++t)
#pragma unroll
                for (int i = 0; i < ROWS; ++i)
                    acc[i][t] = multiply(wk[i][h], ak[t][h], acc[i][t], (int)((h ? wsk[i].y : wsk[i].x) >> (8 * g)), (int)((h ? ask[t].y : ask[t].x) >> (8 * g)));
    }
    if (8 * pieces < p.blocks && pieces % WAVES == wave)               // the rest of the row
        for (int32_t b = 8 * pieces; b < p.blocks; b += 4)
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
                const v4i at = block_or_zero(a[t], b + g, p.blocks);
                const int scale = scale_or_zero(as[t], b + g, p.blocks);
#pragma unroll
                for (int i = 0; i < ROWS; ++i)
                    acc[i][t] = multiply(block_or_zero(w[i], b + g, p.blocks), at, acc[i][t], scale_or_zero(ws[i], b + g, p.blocks), scale);
            }
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) sums[wave][i][t][lane] = acc[i][t];
    __syncthreads();
    // the blocks of 16 x 16 are dealt out to the wavefronts
#pragma unroll
    for (int block = 0; block < ROWS * TOKENS; ++block) {
        if (block % WAVES != wave) continue;
        const int i = block % ROWS, t = block / ROWS;
        v4f s = sums[0][i][t][lane];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) s += sums[k][i][t][lane];
        const int32_t n = n0 + 16 * t + r;
        if (n < p.N) store4<T>(p, m0 + 16 * i + 4 * g, n, s);
    }
}

template <class T>
void launch_few(const DgGemmMx4 &p, hipStream_t stream)
{
    gemm_mx4_few_kernel<T, 8, 1, 1><<<dim3((p.M + 15) / 16, (p.N + 15) / 16), 512, 0, stream>>>(p);
}

}   // namespace

dg_status dg_launch_quantize_mx4(const void *x, dg_dtype type, int64_t N, int64_t K, int64_t stride_n, uint8_t *codes, int64_t stride_codes,
                                 uint8_t *scales, int64_t stride_scales, hipStream_t stream)
{
    in_launches(N, K, stride_n, stride_codes, stride_scales, [&](const MxRows &r, int64_t n) {
        dg_with_type(type, [&](auto t) {
            typedef decltype(t) T;
            quantize_mx4_kernel<T, 1><<<(r.total + THREADS - 1) / THREADS, THREADS, 0, stream>>>((const T *)x + n * stride_n, r, codes + n * stride_codes,
                                                                                                 scales + n * stride_scales);
            return 0;
        });
    });
    return dg_check_launch("dg_quantize_mx4");
}

dg_status dg_launch_dequantize_mx4(const uint8_t *codes, int64_t stride_codes, const uint8_t *scales, int64_t stride_scales, int64_t N, int64_t K,
                                   void *out, dg_dtype type, int64_t stride_out, hipStream_t stream)
{
    in_launches(N, K, stride_out, stride_codes, stride_scales, [&](const MxRows &r, int64_t n) {
        dg_with_type(type, [&](auto t) {
            typedef decltype(t) T;
            dequantize_mx4_kernel<T, 1><<<(r.total + THREADS - 1) / THREADS, THREADS, 0, stream>>>(codes + n * stride_codes, scales + n * stride_scales, r,
                                                                                                   (T *)out + n * stride_out);
            return 0;
        });
    });
    return dg_check_launch("dg_dequantize_mx4");
}

dg_status dg_launch_gemm_mx4(const DgGemmMx4 &all, dg_dtype type, hipStream_t stream)
{
    // channels and tokens whose workgroups are a grid
    dg_in_turns(all.M, 1 << 24, [&](int64_t m, int64_t channels) {
        return dg_in_turns(all.N, std::min<int64_t>(1 << 19, ((int64_t)1 << 34) / channels), [&](int64_t n, int64_t tokens) {
            DgGemmMx4 p = all;
            p.W += m * p.stride_w;
            p.W_scales += m * p.stride_ws;
            p.bias = p.bias ? p.bias + m : nullptr;
            p.A += n * p.stride_a;
            p.A_scales += n * p.stride_as;
            p.out = (uint8_t *)p.out + (n * p.stride_out + m) * dg_type_size(type);
            p.M = (int32_t)channels;
            p.N = (int32_t)tokens;
            dg_with_type(type, [&](auto t) {
                launch_few<decltype(t)>(p, stream);
                return 0;
            });
            return DG_OK;
        });
    });
    return dg_check_launch("dg_gemm_mx4");
}
