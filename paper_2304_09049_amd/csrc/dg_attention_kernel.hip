// Attention of new tokens over the paged cache.
//
// A row is one query head of one new token; the rows of a sequence that read the same cached head -- (token, head of the group), the
// token outermost -- are taken 16 at a time.  Scores come out transposed, S^T = K Q^T (tokens x rows): a lane then holds four tokens of
// one row in the order in which the second product, O^T = V^T P^T, takes its operand, so that the weights never leave the lane.  Keys and
// values lie in the cache as the two products' first operands: 16 contiguous bytes a lane, neighbouring lanes side by side.
//
// Numbers: codes become binary16 exactly (8 bits: code - 128; 4 bits: code - 8, the 8 s joining z).  A query row is scaled by a power of
// two to a largest magnitude in [2^13, 2^14), so that bfloat16's range fits binary16 and nothing above 2^-28 of the row's largest loses a
// bit.  Scores, maxima, sums and outputs are binary32.  A weight is rounded once, to binary16, as p * (value scale / R) * 2^10, where R is
// a power of two no smaller than any value scale met so far: what is 2^-34 of the largest is still counted.  The maximum is
// raised only when a score passes it by 2^4, so that p <= 16 and the weights stay below 2^15.
#include <algorithm>
#include <type_traits>

#include "dg_decoder.h"

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

constexpr float WEIGHT_UNIT = 1024.0f, RAISE = 4.0f;

__device__ __forceinline__ v2h as_halves(uint32_t w) { return __builtin_bit_cast(v2h, w); }

// Four 8-bit codes in storage order -> code - 128 as binary16: a byte below 0x64 is 1024 + byte.
__device__ __forceinline__ void halves8(uint32_t w, v2h &a, v2h &b)
{
    const v2h bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    a = as_halves(__builtin_amdgcn_perm(w, 0x64646464u, 0x00050004u)) - bias;
    b = as_halves(__builtin_amdgcn_perm(w, 0x64646464u, 0x00070006u)) - bias;
}
// Eight 4-bit codes, in nibbles 0 ... 7 -> code - 8 as binary16, in pairs of nibbles (0, 4), (1, 5), (2, 6), (3, 7): a nibble at bit 0 below
// 0x6400 is 1024 + code, at bit 4 below 0x5400 64 + code.
__device__ __forceinline__ void halves4(uint32_t w, v2h (&o)[4])
{
    const v2h b0 = {(_Float16)1032.0f, (_Float16)1032.0f}, b1 = {(_Float16)72.0f, (_Float16)72.0f};
    const uint32_t x = w >> 8;
    o[0] = as_halves((w & 0x000F000Fu) | 0x64006400u) - b0;
    o[1] = as_halves((w & 0x00F000F0u) | 0x54005400u) - b1;
    o[2] = as_halves((x & 0x000F000Fu) | 0x64006400u) - b0;
    o[3] = as_halves((x & 0x00F000F0u) | 0x54005400u) - b1;
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
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// A row's share of the work (one workgroup's piece of the context): sums relative to 2^m.
struct Shares {
    float *o;         // [piece][sequence][its new token][query head][dim]
    float *m, *l;     // the same without the last
};

struct Args {
    DgAttention a;
    int32_t group, row_blocks, pieces, piece_tokens;
    DgFastDiv by_group;
    Shares shares;
};

// What a sequence's new tokens are, with everything that lies in device memory held to what the buffers have.
struct Sequence {
    int32_t first, count, ctx, past;      // past: the context before its new tokens (negative if these are more than the context)
};
__device__ __forceinline__ Sequence sequence(const DgAttention &a, int b)
{
    Sequence s;
    s.first = min(max(a.q_start[b], 0), a.T);
    s.count = min(max(a.q_start[b + 1], s.first), a.T) - s.first;
    s.ctx = (int32_t)min((int64_t)max(a.ctx_len[b], 0), (int64_t)a.table_width * a.cache.page_size);
    s.past = s.ctx - s.count;
    s.count = min(s.count, a.max_q);
    return s;
}

constexpr int WAVES = 4, TILE = 32;      // tokens per step of a wavefront

template <class T, int BITS, int DIM>
__global__ __launch_bounds__(256) void attention_kernel(Args args)
{
    constexpr int STEPS = DIM / 32;                       // products of 32 channels
    constexpr int BLOCKS = DIM / 16;                      // accumulators of 16 channels
    constexpr int VALUE_WORDS = DIM * BITS / 128;         // words of 4 tokens that a lane takes of a unit
    const DgAttention &a = args.a;
    // (a matrix instruction runs whatever the lanes' mask: what it stands under has to be a scalar branch)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int piece = blockIdx.x % args.pieces, rows = blockIdx.x / args.pieces;
    const int row_block = rows % args.row_blocks, bh = rows / args.row_blocks;
    const int h = bh % a.cache.heads, b = bh / a.cache.heads;
    const Sequence seq = sequence(a, b);
    const int row = row_block * 16 + r;
    const int i = (int)dg_fdiv((uint32_t)row, args.by_group), j = row - i * args.group;     // new token, head of the group
    const bool there = i < seq.count;
    if (row_block * 16 >= seq.count * args.group) return;                                   // (no row of the block is there)
    const int last_i = min((row_block * 16 + 15) / args.group, seq.count - 1);
    const int past = seq.past;
    // tokens that the row sees: those before `end`; any row of the block: before `block_end`; every row: before `all_end`
    const int end = !there ? 0 : a.causal ? max(past + i + 1, 0) : seq.ctx;
    const int block_end = a.causal ? max(past + last_i + 1, 0) : seq.ctx;
    const int all_end = row_block * 16 + 15 >= seq.count * args.group ? 0 : a.causal ? max(past + (int)dg_fdiv((uint32_t)row_block * 16, args.by_group) + 1, 0) : seq.ctx;
    const int from = piece * args.piece_tokens;
    const int to = piece == args.pieces - 1 ? block_end : min(block_end, from + args.piece_tokens);

    // the row's query
    v8h q[STEPS];
    float f, q_sum = 0.0f;
    {
        float x[STEPS][8], most = 0.0f;
        const T *src = (const T *)a.q + (int64_t)(seq.first + (there ? i : 0)) * a.q_token + (int64_t)(h * args.group + (there ? j : 0)) * a.q_head;
        bool finite = true;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const DgVec<T, 8> v = dg_load_vec<T, 8>(src + 64 * (s / 2) + 16 * g + 8 * (s & 1));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[s][e] = dg_to_float(v.e[e]);
                most = fmaxf(most, fabsf(x[s][e]));
                finite = finite && fabsf(x[s][e]) < __builtin_inff();
            }
        }
        most = row_max(finite ? most : __builtin_inff());
        // up = 2^(13 - floor(log2 most)), at most 2^126
        const uint32_t biased = __float_as_uint(most) >> 23;
        const uint32_t up_bits = min(267u - min(biased, 254u), 253u);
        const float up = __uint_as_float(up_bits << 23), down = __uint_as_float((254u - up_bits) << 23);
        f = most < __builtin_inff() ? a.scale * 1.4426950408889634f * down : __builtin_nanf("");
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            q[s] = query_operand<BITS>(x[s], up);
            if (BITS == 4)
#pragma unroll
                for (int e = 0; e < 8; ++e) q_sum += (float)q[s][e];
        }
        if (BITS == 4) q_sum = row_sum(q_sum);
    }

    v4f o[BLOCKS] = {};
    float m = -__builtin_inff(), shift = 0.0f, l = 0.0f, oz = 0.0f, R = 0.0f, per_R = 0.0f;
    const uint8_t *const heads = a.cache.base + (int64_t)h * a.cache.head;
    const int32_t *const table = a.table + (int64_t)b * a.table_width;

    for (int t0 = from + TILE * wave; t0 < to; t0 += TILE * WAVES) {
        // the two units' places; a unit past the context, or whose page is none of the cache's, is not read: its tokens count as unseen
        const uint8_t *unit[2];
        uint32_t in_page[2];
        int unit_end[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int t = t0 + 16 * u;
            const bool in = t < seq.ctx;
            const uint32_t entry = in ? dg_fdiv((uint32_t)t, a.cache.by_page) : 0;
            const int32_t page = in ? table[entry] : -1;
            const bool ok = (uint32_t)page < (uint32_t)a.cache.pages;
            in_page[u] = ok ? (uint32_t)t - entry * a.cache.page_size : 0;
            unit[u] = heads + (ok ? (int64_t)page : 0) * a.cache.page_bytes();
            unit_end[u] = ok ? end : 0;
        }
        const bool all_seen = t0 + TILE <= all_end && unit_end[0] && unit_end[1];
        v4f score[2], ks[2], vs[2], kz[2], vz[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float *numbers = (const float *)(unit[u] + 2 * a.cache.part) + in_page[u] + 4 * g;
            ks[u] = *(const v4f *)numbers;
            vs[u] = *(const v4f *)(numbers + a.cache.page_size);
            if (BITS == 4) {
                kz[u] = *(const v4f *)(numbers + 2 * a.cache.page_size);
                vz[u] = *(const v4f *)(numbers + 3 * a.cache.page_size);
            }
        }
        // scores
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint8_t *keys = unit[u] + in_page[u] * (DIM * BITS / 8);
            v4f acc = {};
#pragma unroll
            for (int s = 0; s < STEPS; s += 2) {
                v8h k0, k1;
                if constexpr (BITS == 8) {
                    const v4u w = *(const v4u *)(keys + 512 * s + 16 * lane);
                    v2h c[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) halves8(w[e], c[2 * e], c[2 * e + 1]);
                    k0 = join(c[0], c[1], c[2], c[3]);
                    k1 = join(c[4], c[5], c[6], c[7]);
                } else {
                    const v2u w = *(const v2u *)(keys + 256 * s + 8 * lane);
                    v2h c[4];
                    halves4(w[0], c);
                    k0 = join(c[0], c[1], c[2], c[3]);
                    halves4(w[1], c);
                    k1 = join(c[0], c[1], c[2], c[3]);
                }
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[s], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[s + 1], acc, 0, 0, 0);
            }
            score[u] = acc;
        }
        float top = -__builtin_inff(), most_vs = 0.0f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = score[u][e] * ks[u][e];
                if (BITS == 4) x = __builtin_fmaf(q_sum, __builtin_fmaf(8.0f, ks[u][e], kz[u][e]), x);
                x *= f;
                const int t = t0 + 16 * u + 4 * g + e;
                if (!all_seen) {
                    x = t < unit_end[u] ? x : -__builtin_inff();
                    vs[u][e] = t < unit_end[u] ? vs[u][e] : 0.0f;
                    if (BITS == 4) vz[u][e] = t < unit_end[u] ? vz[u][e] : 0.0f;
                }
                top = fmaxf(top, x);
                most_vs = fmaxf(most_vs, fabsf(vs[u][e]));
                score[u][e] = x;
            }
        if (__any(top > m + RAISE)) {
            const float next = fmaxf(m, row_max(top));
            const float next_shift = next == -__builtin_inff() ? 0.0f : next;
            const float keep = exp2_(m - next_shift);
            m = next;
            shift = next_shift;
            l *= keep;
            oz *= keep;
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k) o[k] *= keep;
        }
        if (__any(most_vs > R)) {
#pragma unroll
            for (int k = 32; k; k >>= 1) most_vs = fmaxf(most_vs, __shfl_xor(most_vs, k));
            // the next power of two above it, from 2^-100 to 2^127
            const uint32_t bits = min(max((__float_as_uint(most_vs) >> 23) + 1, 27u), 254u);
            const float next = __uint_as_float(bits << 23);
            const float keep = R / next;
            R = next;
            per_R = __uint_as_float((254u - bits) << 23) * WEIGHT_UNIT;
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k) o[k] *= keep;
        }
        v2h w[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float p[4], x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[e] = exp2_(score[u][e] - shift);
                l += p[e];
                if (BITS == 4) oz = __builtin_fmaf(p[e], __builtin_fmaf(8.0f, vs[u][e], vz[u][e]), oz);
                x[e] = p[e] * (vs[u][e] * per_R);
            }
            if constexpr (BITS == 8) {
                w[u][0] = (v2h){(_Float16)x[0], (_Float16)x[1]};
                w[u][1] = (v2h){(_Float16)x[2], (_Float16)x[3]};
            } else {
                w[u][0] = (v2h){(_Float16)x[0], (_Float16)x[2]};
                w[u][1] = (v2h){(_Float16)x[1], (_Float16)x[3]};
            }
        }
        const v8h weights = join(w[0][0], w[0][1], w[1][0], w[1][1]);
        // values
        uint32_t words[2][VALUE_WORDS];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint8_t *values = unit[u] + a.cache.part + in_page[u] * (DIM * BITS / 8) + g * (DIM * BITS / 2);
            if constexpr (VALUE_WORDS == 2) {
                const v2u x = *(const v2u *)(values + 8 * r);
                words[u][0] = x[0];
                words[u][1] = x[1];
            } else {
#pragma unroll
                for (int k = 0; k < VALUE_WORDS / 4; ++k) {
                    const v4u x = *(const v4u *)(values + 256 * k + 16 * r);
#pragma unroll
                    for (int e = 0; e < 4; ++e) words[u][4 * k + e] = x[e];
                }
            }
        }
#pragma unroll
        for (int k = 0; k < VALUE_WORDS; ++k) {
            if constexpr (BITS == 8) {
                v2h c[4];
                halves8(words[0][k], c[0], c[1]);
                halves8(words[1][k], c[2], c[3]);
                o[k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join(c[0], c[1], c[2], c[3]), weights, o[k], 0, 0, 0);
            } else {
                v2h c[4], d[4];      // (tokens 0 and 2, 1 and 3; even and odd channels)
                halves4(words[0][k], c);
                halves4(words[1][k], d);
                o[2 * k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join(c[0], c[2], d[0], d[2]), weights, o[2 * k], 0, 0, 0);
                o[2 * k + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join(c[1], c[3], d[1], d[3]), weights, o[2 * k + 1], 0, 0, 0);
            }
        }
    }

    // the wavefronts' shares meet: a lane holds channel `channel(k, e)` of row r in o[k][e]
    __shared__ float sum_o[16][DIM + 4];
    __shared__ float wave_m[WAVES][16], wave_l[WAVES][16];
    l = row_sum(l);
    oz = row_sum(oz);
    if (g == 0) wave_m[wave][r] = m;
    __syncthreads();
    float most = wave_m[0][r];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) most = fmaxf(most, wave_m[k][r]);
    const float mine = m == -__builtin_inff() && l == 0.0f ? 0.0f : exp2_(m - most);       // (a NaN stays one)
    if (g == 0) wave_l[wave][r] = l * mine;
    const float unit_o = R * (1.0f / WEIGHT_UNIT) * mine;
    auto channel = [&](int k, int e) {
        if (BITS == 8) return 64 * (k / 4) + 16 * g + 4 * e + k % 4;
        return DIM == 64 ? 16 * g + 4 * e + k : 128 * (k / 8) + 32 * g + 8 * e + k % 8;
    };
    for (int turn = 0; turn < WAVES; ++turn) {
        if (wave == turn)
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = R == 0.0f ? o[k][e] : o[k][e] * unit_o;                // (nothing met: 0, or the NaN of a NaN)
                    const float y = BITS == 4 ? __builtin_fmaf(oz, mine, x) : x;
                    float &s = sum_o[r][channel(k, e)];
                    s = turn ? s + y : y;
                }
        __syncthreads();
    }
    // 16 threads a row
    const int my_row = threadIdx.x >> 4, part = threadIdx.x & 15;
    const int out_row = row_block * 16 + my_row;
    if (out_row >= seq.count * args.group) return;
    const float total = wave_l[0][my_row] + wave_l[1][my_row] + wave_l[2][my_row] + wave_l[3][my_row];
    const int oi = (int)dg_fdiv((uint32_t)out_row, args.by_group), oj = out_row - oi * args.group;
    if (args.pieces == 1) {
        T *out = (T *)a.out + (int64_t)(seq.first + oi) * a.out_token + (int64_t)(h * args.group + oj) * a.out_head;
        const float by = total == 0.0f ? 0.0f : 1.0f / total;
        DgVec<T, DIM / 16> v;
#pragma unroll
        for (int k = 0; k < DIM / 16; ++k) v.e[k] = dg_from_float<T>(sum_o[my_row][part * (DIM / 16) + k] * by);
        dg_store_vec<T, DIM / 16>(out + part * (DIM / 16), v);
    } else {
        const int64_t at = (((int64_t)piece * a.B + b) * a.max_q + oi) * a.Hq + h * args.group + oj;
        DgVec<float, DIM / 16> v;
#pragma unroll
        for (int k = 0; k < DIM / 16; ++k) v.e[k] = sum_o[my_row][part * (DIM / 16) + k];
        dg_store_vec<float, DIM / 16>(args.shares.o + at * DIM + part * (DIM / 16), v);
        if (part == 0) {
            float x = wave_m[0][my_row];
            for (int k = 1; k < WAVES; ++k) x = fmaxf(x, wave_m[k][my_row]);
            args.shares.m[at] = x;
            args.shares.l[at] = total;
        }
    }
}

// The pieces' shares of a row joined, in the pieces' order: a wavefront a row.
template <class T, int DIM>
__global__ __launch_bounds__(256) void attention_join_kernel(Args args)
{
    const DgAttention &a = args.a;
    const int lane = threadIdx.x & 63;
    const int64_t rows = (int64_t)a.B * a.max_q * a.Hq, at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= rows) return;
    const int64_t token = at / a.Hq, head = at % a.Hq;
    const int b = (int)(token / a.max_q), i = (int)(token % a.max_q);
    const Sequence seq = sequence(a, b);
    if (i >= seq.count) return;
    float most = -__builtin_inff();
    for (int k = 0; k < args.pieces; ++k) most = fmaxf(most, args.shares.m[k * rows + at]);
    constexpr int PER = DIM / 64;
    float total = 0.0f, o[PER] = {};
    for (int k = 0; k < args.pieces; ++k) {
        const float m = args.shares.m[k * rows + at], l = args.shares.l[k * rows + at];
        const float w = m == -__builtin_inff() && l == 0.0f ? 0.0f : exp2_(m - most);
        const DgVec<float, PER> v = dg_load_vec<float, PER>(args.shares.o + (k * rows + at) * DIM + PER * lane);
        total += l * w;
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] += v.e[e] * w;
    }
    const float by = total == 0.0f ? 0.0f : 1.0f / total;
    DgVec<T, PER> v;
#pragma unroll
    for (int e = 0; e < PER; ++e) v.e[e] = dg_from_float<T>(o[e] * by);
    dg_store_vec<T, PER>((T *)a.out + (int64_t)(seq.first + i) * a.out_token + head * a.out_head + PER * lane, v);
}

// How the context is cut: enough workgroups for the chip, pieces of at least 256 tokens.
struct Plan {
    int32_t row_blocks, pieces, piece_tokens;
};
Plan plan_of(const DgAttention &a)
{
    const int32_t group = a.Hq / a.cache.heads;
    Plan p;
    p.row_blocks = (int32_t)(((int64_t)a.max_q * group + 15) / 16);
    const int64_t blocks = (int64_t)p.row_blocks * a.B * a.cache.heads, wanted = dg_simd_count();
    const int64_t most = (a.max_ctx + 255) / 256;
    p.pieces = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(wanted / blocks, most), 256));
    const int32_t step = WAVES * TILE;
    p.piece_tokens = (int32_t)(((a.max_ctx + (int64_t)p.pieces * step - 1) / ((int64_t)p.pieces * step)) * step);
    return p;
}

}   // namespace

int64_t dg_attention_work_bytes(const DgAttention &a)
{
    const Plan p = plan_of(a);
    if (p.pieces == 1) return 0;
    return (int64_t)p.pieces * a.B * a.max_q * a.Hq * (a.cache.dim + 2) * 4;
}

dg_status dg_launch_attention(const DgAttention &a, dg_dtype type, hipStream_t stream)
{
    const Plan p = plan_of(a);
    Args args = {a, a.Hq / a.cache.heads, p.row_blocks, p.pieces, p.piece_tokens, dg_make_div((uint32_t)(a.Hq / a.cache.heads)), {}};
    const int64_t rows = (int64_t)a.B * a.max_q * a.Hq;
    args.shares.o = (float *)a.work;
    args.shares.m = args.shares.o + (int64_t)p.pieces * rows * a.cache.dim;
    args.shares.l = args.shares.m + (int64_t)p.pieces * rows;
    const uint32_t blocks = (uint32_t)((int64_t)p.row_blocks * a.B * a.cache.heads * p.pieces);
    auto launch = [&](auto t, auto bits, auto dim) {
        typedef decltype(t) T;
        constexpr int BITS = decltype(bits)::value, DIM = decltype(dim)::value;
        attention_kernel<T, BITS, DIM><<<blocks, 256, 0, stream>>>(args);
        if (p.pieces > 1) attention_join_kernel<T, DIM><<<(uint32_t)((rows + 3) / 4), 256, 0, stream>>>(args);
    };
    auto by_dim = [&](auto t, auto bits) {
        switch (a.cache.dim) {
        case 64: launch(t, bits, std::integral_constant<int, 64>{}); break;
        case 128: launch(t, bits, std::integral_constant<int, 128>{}); break;
        default: launch(t, bits, std::integral_constant<int, 256>{}); break;
        }
    };
    auto by_bits = [&](auto t) {
        if (a.cache.bits == 8) by_dim(t, std::integral_constant<int, 8>{});
        else by_dim(t, std::integral_constant<int, 4>{});
    };
    if (type == DG_F16) by_bits((_Float16){});
    else by_bits((__bf16){});
    return dg_check_launch("dg_paged_attention");
}
