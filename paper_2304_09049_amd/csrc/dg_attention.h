// What the two kernels of dg_paged_attention share: codes to binary16, a query row as an operand, a sequence's lengths.
#pragma once

#include <type_traits>

#include "dg_decoder.h"
#include "dg_lds_dma.h"

// A row's share of the work (one workgroup's piece of the context): sums relative to 2^m.
struct DgAttentionShares {
    float *o;         // [piece][sequence][its new token][query head][dim]
    float *m, *l;     // the same without the last
};

struct DgAttentionArgs {
    DgAttention a;
    int32_t group, row_blocks, pieces, piece_tokens;
    DgFastDiv by_group;
    DgAttentionShares shares;
};

// The kernel for chunks (dg_attention_chunk_kernel.hip), CHUNK_ROWS rows a workgroup; `args` with its cut of the context.
constexpr int CHUNK_ROWS = 128, CHUNK_STEP = 64;
void dg_launch_attention_chunk(const DgAttentionArgs &args, dg_dtype type, hipStream_t stream);

namespace {

typedef DgAttentionArgs Args;

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

constexpr float WEIGHT_UNIT = 1024.0f, RAISE = 4.0f;

__device__ __forceinline__ v2h as_halves(uint32_t w) { return __builtin_bit_cast(v2h, w); }

// Codes become binary16 below the bits of a power of two, without their bias taken off: that is done on the matrix pipe, which has time to spare
// where the vector pipe has none (32 packed additions a tile against 8 matrix instructions).  Scores start from minus the bias times the sum of the
// query; outputs get minus the bias times the tile's weights by a product of its own, so that what cancels are sums over one tile, and what that rounds
// off is 2^-24 of these.

// Four 8-bit codes in storage order: 1024 + byte, in pairs of neighbours.
constexpr float BIAS8 = 1024.0f + 128.0f;
__device__ __forceinline__ void halves8(uint32_t w, v2h &a, v2h &b)
{
    a = as_halves(__builtin_amdgcn_perm(w, 0x64646464u, 0x00050004u));
    b = as_halves(__builtin_amdgcn_perm(w, 0x64646464u, 0x00070006u));
}
// Eight 4-bit codes, nibbles 0 ... 7, in pairs of nibbles (0, 4), (1, 5), (2, 6), (3, 7).  Values: 1024 + code in the even pairs, 64 + code in the odd
// ones, which are other channels; they count as code - 8, the 8 s joining z.  Keys: 64 + code throughout.
constexpr float BIAS4_EVEN = 1024.0f + 8.0f, BIAS4_ODD = 64.0f + 8.0f, BIAS4_KEYS = 64.0f;
__device__ __forceinline__ void halves4(uint32_t w, v2h (&o)[4])
{
    const uint32_t x = w >> 8;
    o[0] = as_halves((w & 0x000F000Fu) | 0x64006400u);
    o[1] = as_halves((w & 0x00F000F0u) | 0x54005400u);
    o[2] = as_halves((x & 0x000F000Fu) | 0x64006400u);
    o[3] = as_halves((x & 0x00F000F0u) | 0x54005400u);
}
__device__ __forceinline__ void halves4_keys(uint32_t w, v2h *o)
{
    o[0] = as_halves((w << 4 & 0x00F000F0u) | 0x54005400u);
    o[1] = as_halves((w & 0x00F000F0u) | 0x54005400u);
    o[2] = as_halves((w >> 4 & 0x00F000F0u) | 0x54005400u);
    o[3] = as_halves((w >> 8 & 0x00F000F0u) | 0x54005400u);
}
__device__ __forceinline__ v8h join(v2h a, v2h b, v2h c, v2h d)
{
    return (v8h){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight neighbouring channels of a query row as the product's operand: pairs of neighbours for 8-bit keys, of the first and the last four
// for 4-bit ones (as halves4 gives them).
template <int BITS>
__device__ __forceinline__ v8h query_operand(const float (&x)[8], float up)
{
    v8h q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        q[2 * i] = (_Float16)(x[BITS == 8 ? 2 * i : i] * up);
        q[2 * i + 1] = (_Float16)(x[BITS == 8 ? 2 * i + 1 : i + 4] * up);
    }
    return q;
}

// max / sum over the four lanes that hold a row (l, l ^ 16, l ^ 32, l ^ 48)
__device__ __forceinline__ float row_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float row_sum(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}
// In a block that few tiles come to: keeps it a branch of its own, where the compiler would select value by value in every tile.
__device__ __forceinline__ void branch() { asm volatile(""); }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// A lane's channels of a query row, and the row's largest magnitude (an infinity if it holds an infinity or a NaN).
template <class T, int DIM>
__device__ __forceinline__ float load_query(const T *row, int g, float (&x)[DIM / 32][8])
{
    float most = 0.0f;
    bool finite = true;
#pragma unroll
    for (int s = 0; s < DIM / 32; ++s) {
        const DgVec<T, 8> v = dg_load_vec<T, 8>(row + 64 * (s / 2) + 16 * g + 8 * (s & 1));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[s][e] = dg_to_float(v.e[e]);
            most = fmaxf(most, fabsf(x[s][e]));
            finite = finite && fabsf(x[s][e]) < __builtin_inff();
        }
    }
    return row_max(finite ? most : __builtin_inff());
}
// The same as operands, times a power of two that takes `most` (finite) into [2^13, 2^14), at most 2^126; `f` takes a score to the base-2 logit.  The
// sum of the operands' numbers over the row.
template <int BITS, int DIM>
__device__ __forceinline__ float query_operands(const float (&x)[DIM / 32][8], float most, float scale, v8h (&q)[DIM / 32], float &f)
{
    const uint32_t up_bits = min(267u - min(__float_as_uint(most) >> 23, 254u), 253u);
    const float up = __uint_as_float(up_bits << 23), down = __uint_as_float((254u - up_bits) << 23);
    f = scale * 1.4426950408889634f * down;
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < DIM / 32; ++s) {
        q[s] = query_operand<BITS>(x[s], up);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += (float)q[s][e];
    }
    return row_sum(sum);
}

// The power of two above a value scale, from 2^-100 to 2^126, by its exponent's bits.
__device__ __forceinline__ uint32_t above_scale(float most) { return min(max((__float_as_uint(most) >> 23) + 1, 27u), 253u); }

// What a sequence's new tokens are, with everything that lies in device memory held to what the buffers have.
struct Sequence {
    int32_t first, count, ctx, past;      // past: the context before its new tokens (negative if these are more than the context)
};
// (b is the same in every lane of a wavefront)
__device__ __forceinline__ Sequence sequence(const DgAttention &a, int b)
{
    typedef const __attribute__((address_space(4))) int32_t *Scalars;
    b = __builtin_amdgcn_readfirstlane(b);
    Sequence s;
    const int start = ((Scalars)a.q_start)[b], stop = ((Scalars)a.q_start)[b + 1], ctx = ((Scalars)a.ctx_len)[b];
    s.first = min(max(start, 0), a.T);
    s.count = min(max(stop, s.first), a.T) - s.first;
    s.ctx = (int32_t)min((int64_t)max(ctx, 0), (int64_t)a.table_width * a.cache.page_size);
    s.past = s.ctx - s.count;
    s.count = min(s.count, a.max_q);
    return s;
}

// f(element type, bits, channels), the last two as constants
template <class F>
void with_form(const DgAttention &a, dg_dtype type, F f)
{
    const auto by_dim = [&](auto t, auto bits) {
        switch (a.cache.dim) {
        case 64: f(t, bits, std::integral_constant<int, 64>{}); break;
        case 128: f(t, bits, std::integral_constant<int, 128>{}); break;
        default: f(t, bits, std::integral_constant<int, 256>{}); break;
        }
    };
    const auto by_bits = [&](auto t) {
        if (a.cache.bits == 8) by_dim(t, std::integral_constant<int, 8>{});
        else by_dim(t, std::integral_constant<int, 4>{});
    };
    if (type == DG_F16) by_bits((_Float16){});
    else by_bits((__bf16){});
}

}   // namespace
