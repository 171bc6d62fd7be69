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
    DgFastDiv by_group, by_heads, by_sequences, by_blocks, by_pieces, by_Hq, by_max_q;       // (divisions by numbers as they come are 100 to 200 instructions each)
    DgAttentionShares shares;
};

// The kernel for many rows (dg_attention_chunk_kernel.hip), CHUNK_ROWS rows a workgroup; `args` with its cut of the context.
constexpr int CHUNK_ROWS = 128, CHUNK_STEP = 64;
void dg_launch_attention_chunk(const DgAttentionArgs &args, dg_dtype type, hipStream_t stream);

namespace {

typedef DgAttentionArgs Args;

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

// A token's weight, the second product's operand, is its power 2^(logit - shift) times its value scale.  A row's shift is its own, by what the row sees and how
// much of the output that is: the first tile's largest weight becomes 2^FIRST_WEIGHT, and the shift is raised, to that again, when a weight passes MOST_WEIGHT.
// Binary16 then holds weights down to 2^-18 of the largest in full, and counts them down to 2^-28.  (Begun at 2^10 the shift is raised often: 300 x 12 queries on
// 3000 tokens in 4 bits took 57 us, 2048 on 32768 1550, where 2^4 took 48 and 1490; 2^0 is as 2^4.)
// Where value scales are so small that the powers would leave binary32, the shift goes by these: 2^FIRST_POWER, and a lane's sum at most MOST_SUM (four lanes,
// four wavefronts and 256 pieces of it are a number).  A row that has seen nothing raises it whatever they are.
constexpr float FIRST_WEIGHT = 4.0f, MOST_WEIGHT = 0x1p14f, FIRST_POWER = 104.0f, MOST_SUM = 0x1p110f, NOT_BEGUN = -1.0f;
// 4 bits: what a lane adds up of power * z stays in binary32, the shift counting 2^-6 of it as a weight (values that are all alike have no scale).
constexpr float MOST_Z = 0x1p100f;

__device__ __forceinline__ v2h as_halves(uint32_t w) { return __builtin_bit_cast(v2h, w); }

// Codes become binary16 below the bits of a power of two, without their bias taken off: that is done on the matrix pipe, which has time to spare
// where the vector pipe has none (32 packed additions a tile against 8 matrix instructions).  Scores start from minus the bias times the sum of the
// query; outputs get minus the bias times the tile's weights by a product of its own where that does not show (Rows::add), so that what cancels are sums
// over one tile, and what that rounds off is 2^-24 of these.

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
__device__ __forceinline__ uint32_t two_halves(float a, float b)       // rounded to nearest even
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){a, b}, v2h));
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
__device__ __forceinline__ float row_max(float v) { return dg_over_rows(v, DgMax()); }
__device__ __forceinline__ float row_sum(float v) { return dg_over_rows(v, DgAdd()); }
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
// The same as operands, times a power of two that takes `most` into [2^13, 2^14), at most 2^126; `f` takes a score to the base-2 logit.  The
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

// Half of the factor that takes sums relative to 2^m to 2^top.  Squared, it is for outputs; for the sum of weights it is multiplied twice, because that one counts
// where the factor is below binary32: 2^m goes by the values' sizes too.
__device__ __forceinline__ float half_factor(float m, float l, float top)
{
    return m == -__builtin_inff() && l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(0.5f * (m - top));       // (a NaN stays one)
}

// at / by, and at becomes the rest.
__device__ __forceinline__ uint32_t taken(uint32_t &at, const DgFastDiv &by)
{
    const uint32_t n = dg_fdiv(at, by);
    at -= n * by.d;
    return n;
}

// A context's longest: a place a few stages past its end is still a 32-bit number (a table may name a page as often as it likes, so the cache's size
// does not see to that).
constexpr int32_t MOST_CONTEXT = INT32_MAX - 65536;

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
    s.ctx = (int32_t)min((int64_t)min(max(ctx, 0), MOST_CONTEXT), (int64_t)a.table_width * a.cache.page_size);
    s.past = s.ctx - s.count;
    s.count = min(s.count, a.max_q);
    return s;
}

// ---- a unit in LDS --------------------------------------------------------------------------------------------------------

// 16 tokens: keys, values, and 64 numbers (key scale, value scale and, with 4 bits, key z and value z, of 16 tokens each).
template <int BITS, int DIM>
struct Unit {
    static constexpr int PART = 2 * DIM * BITS, BYTES = 2 * PART + 256;
    static constexpr int LOADS = (2 * PART + 1023) / 1024 + 1;
};

// The wavefront's loads of the unit from token t of a sequence, to LDS byte `lds`.  `heads`: the head's place in page 0.  A page that is none of the
// cache's (false is returned): the first page is read instead, and its tokens are to count as unseen.
template <int BITS, int DIM>
__device__ __forceinline__ bool fetch_unit(const DgCache &c, const uint8_t *heads, int t, int page, uint32_t lds, int lane)
{
    constexpr int PART = Unit<BITS, DIM>::PART;
    const bool is = (uint32_t)page < (uint32_t)c.pages;
    const uint32_t in_page = is ? (uint32_t)t - dg_fdiv((uint32_t)t, c.by_page) * c.page_size : 0;
    const uint8_t *const block = heads + (is ? (int64_t)page : 0) * c.page_bytes(), *const keys = block + in_page * (DIM * BITS / 8);
    if constexpr (PART >= 1024) {
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int n = 0; n < PART / 1024; ++n) dg_load16_to_lds(keys + which * c.part, 1024 * n + 16 * lane, lds + which * PART + 1024 * n);
    } else {
        dg_load16_to_lds(keys, (lane < 32 ? 0 : c.part) + 16 * (lane & 31), lds);
    }
    const int number = BITS == 8 ? lane >> 4 & 1 : lane >> 4;
    dg_load4_to_lds(block + 2 * c.part, 4 * (int)(in_page + number * c.page_size + (lane & 15)), lds + 2 * PART);
    return is;
}

// ---- a wavefront's rows: N blocks of 16, a lane's row r = lane % 16 of each, its channels and tokens by g = lane / 16 --------------------------------

template <class T, int BITS, int DIM, int N>
struct Rows {
    static constexpr int STEPS = DIM / 32;                    // products of 32 channels
    static constexpr int BLOCKS = DIM / 16;                   // accumulators of 16 channels
    static constexpr int WORDS = DIM * BITS / 128;            // words of 4 tokens' values that a lane takes of a unit
    // Binary16 outputs show a weight's rounding beside their own (the error against 64 bits was 1.4 times a binary32 computation's): there what the rounding
    // left off goes through the matrix instructions as well.
    static constexpr bool TWICE = std::is_same<T, _Float16>::value;

    v8h q[N][STEPS];
    v4f o[N][BLOCKS];                                         // sums of weight * code
    float f[N], per_z[N], from_bias[N];                       // what takes a score, and what takes a key's z, to the base-2 logit; where scores start
    float shift[N], above[N], l[N], oz[N];                    // sums are relative to 2^shift: of powers 2^(logit - shift), and of powers * z
    int end[N];                                               // a row sees the tokens before this
    int all_end, any_end;                                     // tokens that every row sees, and that any sees

    // Rows first ... first + have - 1 of a sequence's cached head h (rows that are not there are computed as its first one).  Each row is scaled by a power of
    // two of its own: a softmax is relative to its row, so what a row gives must not go by how large others are.
    __device__ __forceinline__ void begin(const Args &args, const Sequence &seq, int h, int first, int have, int r, int g)
    {
        const DgAttention &a = args.a;
        const int first_i = (int)dg_fdiv((uint32_t)first, args.by_group), last_i = (int)dg_fdiv((uint32_t)(first + max(have, 1) - 1), args.by_group);
        all_end = a.causal ? max(seq.past + first_i + 1, 0) : seq.ctx;
        any_end = have <= 0 ? 0 : a.causal ? max(seq.past + last_i + 1, 0) : seq.ctx;
        float x[N][STEPS][8], most[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int at = 16 * n + r;
            const bool there = at < have;
            const int i = there ? (int)dg_fdiv((uint32_t)(first + at), args.by_group) : 0, j = there ? first + at - i * args.group : 0;
            most[n] = load_query<T, DIM>((const T *)a.q + (int64_t)(seq.first + i) * a.q_token + (int64_t)(h * args.group + j) * a.q_head, g, x[n]);
            end[n] = there && a.causal ? max(seq.past + i + 1, 0) : all_end;
            shift[n] = 0.0f;
            above[n] = NOT_BEGUN;
            l[n] = oz[n] = 0.0f;
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k) o[n][k] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float sum = query_operands<BITS, DIM>(x[n], most[n], a.scale, q[n], f[n]);
            from_bias[n] = most[n] < __builtin_inff() ? -(BITS == 8 ? BIAS8 : BIAS4_KEYS) * sum : __builtin_nanf("");
            per_z[n] = __builtin_amdgcn_fmed3f(sum * f[n], -__FLT_MAX__, __FLT_MAX__);         // (finite: a z of 0 adds nothing)
        }
    }

    // The 32 tokens from t0 on, two units one after another in LDS; is0, is1: whether their pages are the cache's.
    __device__ __forceinline__ void step(const uint8_t *pair, int t0, bool is0, bool is1, int lane)
    {
        typedef Unit<BITS, DIM> U;
        const int r = lane & 15, g = lane >> 4;
        const bool all_seen = t0 + 32 <= all_end && is0 && is1;
        v4f score[N][2], ks[2], vs[2], kz[2], vz[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint8_t *const unit = pair + u * U::BYTES;
            const v4f *const numbers = (const v4f *)(unit + 2 * U::PART) + g;
            ks[u] = numbers[0];
            vs[u] = numbers[4];
            if (BITS == 4) {
                kz[u] = numbers[8];
                vz[u] = numbers[12];
            }
#pragma unroll
            for (int n = 0; n < N; ++n) score[n][u] = (v4f){from_bias[n], from_bias[n], from_bias[n], from_bias[n]};
#pragma unroll
            for (int s = 0; s < STEPS / 2; ++s) {
                v2h c[8];
                if constexpr (BITS == 8) {
                    const v4u w = *(const v4u *)(unit + 1024 * s + 16 * lane);
#pragma unroll
                    for (int e = 0; e < 4; ++e) halves8(w[e], c[2 * e], c[2 * e + 1]);
                } else {
                    const v2u w = *(const v2u *)(unit + 512 * s + 8 * lane);
                    halves4_keys(w[0], c);
                    halves4_keys(w[1], c + 4);
                }
                const v8h k0 = join(c[0], c[1], c[2], c[3]), k1 = join(c[4], c[5], c[6], c[7]);
#pragma unroll
                for (int n = 0; n < N; ++n) score[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[n][2 * s], score[n][u], 0, 0, 0);
#pragma unroll
                for (int n = 0; n < N; ++n) score[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[n][2 * s + 1], score[n][u], 0, 0, 0);
            }
        }
        // Logits relative to the shift.
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    score[n][u][e] = __builtin_fmaf(score[n][u][e], ks[u][e] * f[n],
                                                    BITS == 8 ? -shift[n] : __builtin_fmaf(per_z[n], kz[u][e], -shift[n]));
        // A token's powers, the weights, and what to the outputs comes from z (a code counts as code - 8).
        float p[N][2][4], x[N][8], xz[N][2][4], y[2][4], sum[N], z[N];
        if (BITS == 4)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[u][e] = __builtin_fmaf(8.0f, vs[u][e], vz[u][e]);
        const auto weigh = [&](int n, float by) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[n][u][e] = exp2_(score[n][u][e] - by);
                    x[n][place(u, e)] = p[n][u][e] * vs[u][e];
                    if (BITS == 4) xz[n][u][e] = p[n][u][e] * y[u][e];
                }
        };
        // What a row does not see is selected away, whatever it is.
        const auto hide = [&](int n) {
            int first = t0 + 4 * g;
            asm volatile("" : "+v"(first));                                            // (or the places are worked out for every tile)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool seen = ((u ? is1 : is0) ? first + 16 * u + e : INT32_MAX) < end[n];
                    score[n][u][e] = seen ? score[n][u][e] : -__builtin_inff();
                    p[n][u][e] = seen ? p[n][u][e] : 0.0f;
                    x[n][place(u, e)] = seen ? x[n][place(u, e)] : 0.0f;
                    if (BITS == 4) xz[n][u][e] = seen ? xz[n][u][e] : 0.0f;
                }
        };
        const auto add_up = [&](int n) {
            sum[n] = p[n][0][0];
            z[n] = BITS == 4 ? xz[n][0][0] : 0.0f;
#pragma unroll
            for (int k = 1; k < 8; ++k) {
                sum[n] += p[n][k / 4][k % 4];
                if (BITS == 4) z[n] += xz[n][k / 4][k % 4];
            }
        };
#pragma unroll
        for (int n = 0; n < N; ++n) weigh(n, 0.0f);
        if (!all_seen) {
            branch();
#pragma unroll
            for (int n = 0; n < N; ++n) hide(n);
        }
        bool raise[N], any_raise = false;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            add_up(n);
            float most = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) most = fmaxf(most, fabsf(x[n][k]));
            raise[n] = (most > MOST_WEIGHT) | (l[n] + sum[n] > above[n]);                        // (| : || would be branches of its own)
            if (BITS == 4) raise[n] |= !(fabsf(oz[n] + z[n]) <= MOST_Z);
            any_raise |= raise[n];
        }
        if (__any(any_raise)) {
            float size[2][4];                                                          // log2 of what a weight is its power times
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) size[u][e] = __builtin_amdgcn_logf(BITS == 8 ? fabsf(vs[u][e]) : fmaxf(fabsf(vs[u][e]), fabsf(y[u][e]) * 0x1p-6f));
#pragma unroll
            for (int n = 0; n < N; ++n) {
                // (only the rows that ask for it: a row's bits do not go by its neighbours)
                const bool mine = row_max(raise[n] ? 1.0f : 0.0f) > 0.0f, full = row_max(l[n] + sum[n]) > MOST_SUM;
                float high = -__builtin_inff(), power = -__builtin_inff();
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        power = fmaxf(power, score[n][u][e]);
                        high = fmaxf(high, score[n][u][e] + size[u][e]);
                    }
                power = row_max(power);
                high = fmaxf(row_max(high) - FIRST_WEIGHT, power - FIRST_POWER);
                const bool begun = above[n] == MOST_SUM, nothing = high == -__builtin_inff();
                const float by = !mine || nothing ? 0.0f : begun ? fmaxf(high, full ? 8.0f : 0.0f) : high;
                const float half = begun ? exp2_(-0.5f * by) : 0.0f, keep = half * half;          // (nothing is summed before)
                shift[n] += by;
                above[n] = begun || (mine && !nothing) ? MOST_SUM : NOT_BEGUN;
                l[n] = l[n] * half * half;
                oz[n] *= keep;
                weigh(n, by);
                if (!all_seen) hide(n);
                add_up(n);
#pragma unroll
                for (int k = 0; k < BLOCKS; ++k) o[n][k] *= keep;
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            l[n] += sum[n];
            oz[n] += z[n];
        }
        // The weights as the second product's operand.
        v8h weights[N], rests[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v4u w, rest = {};
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = two_halves(x[n][2 * k], x[n][2 * k + 1]);
            weights[n] = __builtin_bit_cast(v8h, w);
            if (TWICE)
#pragma unroll
                for (int k = 0; k < 4; ++k) rest[k] = two_halves(x[n][2 * k] - (float)weights[n][2 * k], x[n][2 * k + 1] - (float)weights[n][2 * k + 1]);
            rests[n] = __builtin_bit_cast(v8h, rest);
        }
        uint32_t words[2][WORDS];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint8_t *const values = pair + u * U::BYTES + U::PART + g * (DIM * BITS / 2);
            if constexpr (WORDS == 2) {
                const v2u w = *(const v2u *)(values + 8 * r);
                words[u][0] = w[0];
                words[u][1] = w[1];
            } else {
#pragma unroll
                for (int k = 0; k < WORDS / 4; ++k) {
                    const v4u w = *(const v4u *)(values + 256 * k + 16 * r);
#pragma unroll
                    for (int e = 0; e < 4; ++e) words[u][4 * k + e] = w[e];
                }
            }
        }
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            v2h c[4], d[4];
            if constexpr (BITS == 8) {
                halves8(words[0][k], c[0], c[1]);
                halves8(words[1][k], c[2], c[3]);
                add(k, join(c[0], c[1], c[2], c[3]), BIAS8, weights, rests);
            } else {
                halves4(words[0][k], c);          // (tokens 0 and 2, 1 and 3; even and odd channels)
                halves4(words[1][k], d);
                add(2 * k, join(c[0], c[2], d[0], d[2]), BIAS4_EVEN, weights, rests);
                add(2 * k + 1, join(c[1], c[3], d[1], d[3]), BIAS4_ODD, weights, rests);
            }
        }
    }

    // Where unit u's token 4 g + e stands in a lane's operand (4 bits: tokens 0, 2, 1, 3, as halves4 has them).
    static constexpr __device__ int place(int u, int e) { return 4 * u + (BITS == 8 ? e : (e & 1) * 2 + (e >> 1)); }

    // o[.][k] += values * weights.  The values' bias comes off in a product of its own for one block of rows and bfloat16 outputs, where the matrix pipe has time to
    // spare: what is rounded off then is 2^-24 of one tile's sums with the bias.  Before the products for two blocks, which share it, and for binary16 outputs,
    // which show that rounding: over 60000 tokens the error against 64 bits was 1.54 times the outputs' own rounding with 4 bits, 1.03 with 8, and is 1.000;
    // bfloat16's, eight times as coarse, is 1.01 at most, and taking the bias off first there makes 64 contexts of up to 8192 in 4 bits 85 us for 82.
    __device__ __forceinline__ void add(int k, v8h values, float bias, const v8h (&weights)[N], const v8h (&rests)[N])
    {
        const _Float16 b = (_Float16)-bias;
        const v8h off = {b, b, b, b, b, b, b, b};
        constexpr bool APART = N == 1 && !TWICE;
        if (!APART) values += off;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (APART) o[n][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(off, weights[n], o[n][k], 0, 0, 0);
            o[n][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(values, weights[n], o[n][k], 0, 0, 0);
            if (TWICE) o[n][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(values, rests[n], o[n][k], 0, 0, 0);
        }
    }

    __device__ __forceinline__ float most(int n) const { return above[n] == MOST_SUM ? shift[n] : -__builtin_inff(); }

    // Channels channel(k, e, g) ... + 3 of the lane's row of block n, times `by`; z: `by` times the row's sum of weight * z.
    static constexpr __device__ int channel(int k, int e, int g)
    {
        return BITS == 8 ? 64 * k + 16 * g + 4 * e : DIM == 64 ? 16 * g + 4 * e : 128 * (k / 2) + 32 * g + 8 * e + 4 * (k % 2);
    }
    __device__ __forceinline__ v4f channels(int n, int k, int e, float by, float z) const
    {
        v4f x;
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = BITS == 4 ? __builtin_fmaf(o[n][4 * k + c][e], by, z) : o[n][4 * k + c][e] * by;
        return x;
    }
};

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
