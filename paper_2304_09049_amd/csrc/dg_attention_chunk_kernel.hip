// Attention of chunks of new tokens over the paged cache: the products of dg_attention_kernel.hip, for many rows.
//
// A workgroup takes 128 rows of a cached head, 32 a wavefront: two blocks of 16, so that a code is turned into binary16 once for two products.  The
// tokens go by in stages of 64, four units, one loaded by each wavefront into a ring in LDS that all four read.
#include "dg_attention.h"

namespace {

constexpr int WAVES = 4, BLOCKS_Q = CHUNK_ROWS / (16 * WAVES);

// What a lane's eight weights of a tile may add up to before the shift is raised: p <= 16, so that weights stay below 2^14.  A row that has seen nothing
// raises it whatever they are.
constexpr float MOST_SUM = 16.0f, NOT_BEGUN = -1.0f;

__device__ __forceinline__ uint32_t two_halves(float a, float b)       // rounded to nearest even
{
    uint32_t w;
    asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(w) : "v"(a), "v"(b));
    return w;
}

// A stage in LDS: four units, each keys, values and 64 numbers (key scale, value scale and, 4 bits, key z and value z of 16 tokens).
template <int BITS, int DIM>
struct Stage {
    static constexpr int PART = 2 * DIM * BITS, UNIT = 2 * PART + 256, BYTES = 4 * UNIT;
    static constexpr int LOADS = (2 * PART + 1023) / 1024 + 1;       // a wavefront's, of its unit
    static constexpr int RING = DIM == 256 && BITS == 8 ? 2 : 3;
};

template <class T, int BITS, int DIM>
__global__ __launch_bounds__(64 * WAVES, DIM == 256 ? 1 : 2) void attention_chunk_kernel(Args args)
{
    typedef Stage<BITS, DIM> Kept;
    constexpr int STEPS = DIM / 32, BLOCKS = DIM / 16, VALUE_WORDS = DIM * BITS / 128, RING = Kept::RING;
    constexpr bool TWICE = std::is_same<T, _Float16>::value;
    __shared__ __align__(1024) uint8_t ring[RING * Kept::BYTES];
    __shared__ int is_there[RING][4];
    const DgAttention &a = args.a;
    // (a matrix instruction runs whatever the lanes' mask: what it stands under has to be a scalar branch)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    // heads innermost: a head's workgroups follow each other at a distance of `heads`, so with eight of them each die has its own; the last rows, which see
    // most, first
    int rest = blockIdx.x;
    const int h = rest % a.cache.heads;
    rest /= a.cache.heads;
    const int piece = rest % args.pieces;
    rest /= args.pieces;
    const int row_block = args.row_blocks - 1 - rest % args.row_blocks, b = rest / args.row_blocks;
    const Sequence seq = sequence(a, b);
    const int first_row = row_block * CHUNK_ROWS, have = min(seq.count * args.group - first_row, CHUNK_ROWS);
    if (have <= 0) return;
    const int mine = min(have - 16 * BLOCKS_Q * wave, 16 * BLOCKS_Q);                         // the wavefront's rows (0 or fewer: none)
    const int wave_row = first_row + 16 * BLOCKS_Q * wave;
    const int wave_i = (int)dg_fdiv((uint32_t)wave_row, args.by_group), wave_last_i = (int)dg_fdiv((uint32_t)(wave_row + max(mine, 1) - 1), args.by_group);
    const int block_end = a.causal ? max(seq.past + (int)dg_fdiv((uint32_t)(first_row + have - 1), args.by_group) + 1, 0) : seq.ctx;
    // tokens that the wavefront's rows see: every one those before all_end, any those before wave_end
    const int all_end = a.causal ? max(seq.past + wave_i + 1, 0) : seq.ctx;
    const int wave_end = mine <= 0 ? 0 : a.causal ? max(seq.past + wave_last_i + 1, 0) : seq.ctx;
    const int from = piece * args.piece_tokens;
    const int to = piece == args.pieces - 1 ? block_end : min(block_end, from + args.piece_tokens);

    const uint8_t *const heads = a.cache.base + (int64_t)h * a.cache.head;
    const auto table = (const __attribute__((address_space(4))) int32_t *)(a.table + (int64_t)b * a.table_width);
    const uint32_t ring_lds = dg_lds_address(ring) + wave * Kept::UNIT;
    const auto page_of = [&](int t) { return t < seq.ctx ? table[dg_fdiv((uint32_t)t, a.cache.by_page)] : -1; };
    // This wavefront's unit of the stage from token t0.  One past the context, or whose page is none of the cache's, is read from the first page instead
    // and its tokens count as unseen.
    const auto fetch = [&](int t0, int page, int slot) {
        const uint32_t t = (uint32_t)(t0 + 16 * wave);
        const bool is = (uint32_t)page < (uint32_t)a.cache.pages;
        const uint32_t in_page = is ? t - dg_fdiv(t, a.cache.by_page) * a.cache.page_size : 0, lds = ring_lds + slot * Kept::BYTES;
        const uint8_t *const block = heads + (is ? (int64_t)page : 0) * a.cache.page_bytes(), *const keys = block + in_page * (DIM * BITS / 8);
        if constexpr (Kept::PART >= 1024) {
#pragma unroll
            for (int which = 0; which < 2; ++which)
#pragma unroll
                for (int n = 0; n < Kept::PART / 1024; ++n)
                    dg_load16_to_lds(keys + which * a.cache.part, 1024 * n + 16 * lane, lds + which * Kept::PART + 1024 * n);
        } else {
            dg_load16_to_lds(keys, (lane < 32 ? 0 : a.cache.part) + 16 * (lane & 31), lds);
        }
        const uint32_t number = BITS == 8 ? lane >> 4 & 1 : lane >> 4;
        dg_load4_to_lds(block + 2 * a.cache.part + 4 * (in_page + number * a.cache.page_size + (lane & 15)), lds + 2 * Kept::PART);
        if (lane == 0) is_there[slot][wave] = is;
    };
    int ahead = from;                                   // the stage whose page was asked for last
    int page = page_of(ahead + 16 * wave);
#pragma unroll
    for (int n = 0; n < RING - 1; ++n) {
        fetch(ahead, page, n);
        ahead += CHUNK_STEP;
        page = page_of(ahead + 16 * wave);
    }

    // The wavefront's rows are scaled by one power of two, the one for its largest query: a score's factor is then the token's alone.  (A row whose
    // queries are 2^-10 of another's keeps 18 bits of them, for logits that are as much smaller.)
    v8h q[BLOCKS_Q][STEPS];
    float f, q_sum[BLOCKS_Q], from_bias[BLOCKS_Q], shift[BLOCKS_Q], above[BLOCKS_Q], l[BLOCKS_Q], oz[BLOCKS_Q];
    int end[BLOCKS_Q];
    {
        float x[BLOCKS_Q][STEPS][8], most[BLOCKS_Q], largest = 0.0f;
#pragma unroll
        for (int n = 0; n < BLOCKS_Q; ++n) {
            const int at = 16 * n + r, row = wave_row + at;
            const bool there = at < mine;
            const int i = there ? (int)dg_fdiv((uint32_t)row, args.by_group) : 0, j = there ? row - i * args.group : 0;
            most[n] = load_query<T, DIM>((const T *)a.q + (int64_t)(seq.first + i) * a.q_token + (int64_t)(h * args.group + j) * a.q_head, g, x[n]);
            largest = fmaxf(largest, there && most[n] < __builtin_inff() ? most[n] : 0.0f);
            end[n] = there && a.causal ? max(seq.past + i + 1, 0) : all_end;
            shift[n] = 0.0f;
            above[n] = NOT_BEGUN;
            l[n] = oz[n] = 0.0f;
        }
#pragma unroll
        for (int k = 8; k; k >>= 1) largest = fmaxf(largest, __shfl_xor(largest, k));
#pragma unroll
        for (int n = 0; n < BLOCKS_Q; ++n) {
            q_sum[n] = query_operands<BITS, DIM>(x[n], largest, a.scale, q[n], f);
            from_bias[n] = most[n] < __builtin_inff() ? -(BITS == 8 ? BIAS8 : BIAS4_KEYS) * q_sum[n] : __builtin_nanf("");
        }
    }
    v4f o[BLOCKS_Q][BLOCKS] = {};
    float R = 0.0f, per_R = 0.0f;
    int slot = 0, next_slot = RING - 1;
#pragma unroll 1
    for (int t0 = from; t0 < to; t0 += CHUNK_STEP) {
        dg_wait_for_loads<(RING - 2) * Kept::LOADS>();
        __syncthreads();
        // (past the end there is nothing to load; the waits count on loads, so they go on, from the first page)
        fetch(ahead, ahead < to ? page : -1, next_slot);
        ahead += CHUNK_STEP;
        page = page_of(ahead + 16 * wave);
        const uint8_t *const stage = ring + slot * Kept::BYTES;
        int is[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) is[u] = __builtin_amdgcn_readfirstlane(is_there[slot][u]);
        slot = slot + 1 == RING ? 0 : slot + 1;
        next_slot = next_slot + 1 == RING ? 0 : next_slot + 1;
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            const int t1 = t0 + 32 * half;
            if (t1 >= wave_end) break;
            const int is0 = half ? is[2] : is[0], is1 = half ? is[3] : is[1];
            const bool all_seen = t1 + 32 <= all_end && is0 && is1;
            const uint8_t *const pair = stage + half * (2 * Kept::UNIT);
            v4f score[BLOCKS_Q][2], ks[2], vs[2], kz[2], vz[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint8_t *const unit = pair + u * Kept::UNIT;
                const v4f *const numbers = (const v4f *)(unit + 2 * Kept::PART) + g;
                ks[u] = numbers[0];
                vs[u] = numbers[4];
                if (BITS == 4) {
                    kz[u] = numbers[8];
                    vz[u] = numbers[12];
                }
#pragma unroll
                for (int n = 0; n < BLOCKS_Q; ++n) score[n][u] = (v4f){from_bias[n], from_bias[n], from_bias[n], from_bias[n]};
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
                    for (int n = 0; n < BLOCKS_Q; ++n) score[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[n][2 * s], score[n][u], 0, 0, 0);
#pragma unroll
                    for (int n = 0; n < BLOCKS_Q; ++n) score[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[n][2 * s + 1], score[n][u], 0, 0, 0);
                }
            }
            // Logits, and their exponentials relative to 2^shift.  That these have grown too large is seen from their sum, which is needed anyway.
            float p[BLOCKS_Q][2][4], sum[BLOCKS_Q];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                ks[u] *= f;
                if (BITS == 4) kz[u] *= f;
            }
#pragma unroll
            for (int n = 0; n < BLOCKS_Q; ++n)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        score[n][u][e] = __builtin_fmaf(score[n][u][e], ks[u][e], BITS == 8 ? -shift[n] : __builtin_fmaf(q_sum[n], kz[u][e], -shift[n]));
            if (!all_seen) {
                branch();
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int t = (u ? is1 : is0) ? t1 + 16 * u + 4 * g + e : INT32_MAX;
#pragma unroll
                        for (int n = 0; n < BLOCKS_Q; ++n) score[n][u][e] = t < end[n] ? score[n][u][e] : -__builtin_inff();
                        // (a row that does not see a token that others see: its weight is 0 times this, which may be a NaN; see below)
                        vs[u][e] = t < wave_end ? vs[u][e] : 0.0f;
                        if (BITS == 4) vz[u][e] = t < wave_end ? vz[u][e] : 0.0f;
                    }
            }
#pragma unroll
            for (int n = 0; n < BLOCKS_Q; ++n)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[n][u][e] = exp2_(score[n][u][e]);
                        sum[n] = u + e == 0 ? p[n][0][0] : sum[n] + p[n][u][e];
                    }
            bool raise = false;
#pragma unroll
            for (int n = 0; n < BLOCKS_Q; ++n) raise = raise || sum[n] > above[n];
            if (__any(raise)) {
#pragma unroll
                for (int n = 0; n < BLOCKS_Q; ++n) {
                    float high = -__builtin_inff();
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 4; ++e) high = fmaxf(high, score[n][u][e]);
                    high = row_max(high);
                    const bool begun = above[n] == MOST_SUM;
                    const float by = begun ? fmaxf(high, 0.0f) : high == -__builtin_inff() ? 0.0f : high;
                    const float keep = begun ? exp2_(-by) : 0.0f;                          // (nothing is summed before)
                    shift[n] += by;
                    above[n] = begun || high > -__builtin_inff() ? MOST_SUM : NOT_BEGUN;
                    l[n] *= keep;
                    oz[n] *= keep;
                    sum[n] = 0.0f;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            p[n][u][e] = exp2_(score[n][u][e] - by);
                            sum[n] += p[n][u][e];
                        }
#pragma unroll
                    for (int k = 0; k < BLOCKS; ++k) o[n][k] *= keep;
                }
            }
#pragma unroll
            for (int n = 0; n < BLOCKS_Q; ++n) l[n] += sum[n];
            float most_vs = 0.0f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) most_vs = fmaxf(most_vs, fabsf(vs[u][e]));
            if (__any(most_vs > R)) {
#pragma unroll
                for (int k = 32; k; k >>= 1) most_vs = fmaxf(most_vs, __shfl_xor(most_vs, k));
                const uint32_t bits = above_scale(most_vs);
                const float inverse = __uint_as_float((254u - bits) << 23), keep = R * inverse;
                R = __uint_as_float(bits << 23);
                per_R = inverse * WEIGHT_UNIT;
#pragma unroll
                for (int n = 0; n < BLOCKS_Q; ++n)
#pragma unroll
                    for (int k = 0; k < BLOCKS; ++k) o[n][k] *= keep;
            }
            v8h weights[BLOCKS_Q], rests[TWICE ? BLOCKS_Q : 1];
            float x[BLOCKS_Q][8], xz[BITS == 4 ? BLOCKS_Q : 1][8];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float by = vs[u][e] * per_R, z = BITS == 4 ? __builtin_fmaf(8.0f, vs[u][e], vz[u][e]) : 0.0f;
                    const int at = 4 * u + (BITS == 8 ? e : (e & 1) * 2 + (e >> 1));          // (4 bits: tokens 0, 2, 1, 3)
#pragma unroll
                    for (int n = 0; n < BLOCKS_Q; ++n) {
                        x[n][at] = p[n][u][e] * by;
                        if (BITS == 4) xz[n][at] = p[n][u][e] * z;
                    }
                }
            if (!all_seen) {
                branch();
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int n = 0; n < BLOCKS_Q; ++n) {
                            const int at = 4 * u + (BITS == 8 ? e : (e & 1) * 2 + (e >> 1));
                            const bool seen = t1 + 16 * u + 4 * g + e < end[n];
                            x[n][at] = seen ? x[n][at] : 0.0f;
                            if (BITS == 4) xz[n][at] = seen ? xz[n][at] : 0.0f;
                        }
            }
            if (BITS == 4)
#pragma unroll
                for (int n = 0; n < BLOCKS_Q; ++n)
#pragma unroll
                    for (int k = 0; k < 8; ++k) oz[n] += xz[n][k];
#pragma unroll
            for (int n = 0; n < BLOCKS_Q; ++n) {
                v4u w, rest = {};
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = two_halves(x[n][2 * k], x[n][2 * k + 1]);
                weights[n] = __builtin_bit_cast(v8h, w);
                if (TWICE) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        rest[k] = two_halves(x[n][2 * k] - (float)weights[n][2 * k], x[n][2 * k + 1] - (float)weights[n][2 * k + 1]);
                    rests[n] = __builtin_bit_cast(v8h, rest);
                }
            }
            uint32_t words[2][VALUE_WORDS];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint8_t *const values = pair + u * Kept::UNIT + Kept::PART + g * (DIM * BITS / 2);
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
            const auto add = [&](int k, v8h values) {
#pragma unroll
                for (int n = 0; n < BLOCKS_Q; ++n) {
                    o[n][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(values, weights[n], o[n][k], 0, 0, 0);
                    if (TWICE) o[n][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(values, rests[n], o[n][k], 0, 0, 0);
                }
            };
            const auto off = [](v2h (&c)[4], float even, float odd) {
                const v2h x = {(_Float16)even, (_Float16)even}, y = {(_Float16)odd, (_Float16)odd};
                c[0] -= x;
                c[1] -= y;
                c[2] -= x;
                c[3] -= y;
            };
#pragma unroll
            for (int k = 0; k < VALUE_WORDS; ++k) {
                v2h c[4], d[4];
                if constexpr (BITS == 8) {
                    halves8(words[0][k], c[0], c[1]);
                    halves8(words[1][k], c[2], c[3]);
                    off(c, BIAS8, BIAS8);
                    add(k, join(c[0], c[1], c[2], c[3]));
                } else {
                    halves4(words[0][k], c);      // (tokens 0 and 2, 1 and 3; even and odd channels)
                    halves4(words[1][k], d);
                    off(c, BIAS4_EVEN, BIAS4_ODD);
                    off(d, BIAS4_EVEN, BIAS4_ODD);
                    add(2 * k, join(c[0], c[2], d[0], d[2]));
                    add(2 * k + 1, join(c[1], c[3], d[1], d[3]));
                }
            }
        }
    }
    dg_wait_for_loads<0>();
    // A lane holds channels channel(4 k, e) ... + 3 of a row in o[n][4 k ... 4 k + 3][e].
#pragma unroll
    for (int n = 0; n < BLOCKS_Q; ++n) {
        const float total = row_sum(l[n]), z = row_sum(oz[n]);
        const int at = 16 * n + r, row = wave_row + at;
        if (at >= mine) continue;
        const int i = (int)dg_fdiv((uint32_t)row, args.by_group), head = h * args.group + row - i * args.group;
        const bool alone = args.pieces == 1;
        const float by = !alone ? 1.0f : total == 0.0f ? 0.0f : 1.0f / total, unit = R == 0.0f ? 1.0f : R * (1.0f / WEIGHT_UNIT);
        const int64_t share = (((int64_t)piece * a.B + b) * a.max_q + i) * a.Hq + head;
        T *const out = (T *)a.out + (int64_t)(seq.first + i) * a.out_token + (int64_t)head * a.out_head;
#pragma unroll
        for (int k = 0; k < BLOCKS / 4; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int channel = BITS == 8 ? 64 * k + 16 * g + 4 * e : DIM == 64 ? 16 * g + 4 * e : 128 * (k / 2) + 32 * g + 8 * e + 4 * (k % 2);
                v4f x;
                DgVec<T, 4> y;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    x[c] = (BITS == 4 ? __builtin_fmaf(o[n][4 * k + c][e], unit, z) : o[n][4 * k + c][e] * unit) * by;
                    y.e[c] = dg_from_float<T>(x[c]);
                }
                if (alone) dg_store_vec<T, 4>(out + channel, y);
                else *(v4f *)(args.shares.o + share * DIM + channel) = x;
            }
        if (!alone && g == 0) {
            args.shares.m[share] = above[n] == MOST_SUM ? shift[n] : -__builtin_inff();
            args.shares.l[share] = total;
        }
    }
}

}   // namespace

void dg_launch_attention_chunk(const DgAttentionArgs &args, dg_dtype type, hipStream_t stream)
{
    const DgAttention &a = args.a;
    with_form(a, type, [&](auto t, auto bits, auto dim) {
        attention_chunk_kernel<decltype(t), decltype(bits)::value, decltype(dim)::value>
            <<<(uint32_t)((int64_t)args.row_blocks * a.B * a.cache.heads * args.pieces), 64 * WAVES, 0, stream>>>(args);
    });
}
