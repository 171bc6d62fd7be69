// Attention of new tokens over the paged cache.
//
// A row is one query head of one new token; the rows of a sequence that read the same cached head -- (token, head of the group), the
// token outermost -- are taken 16 at a time.  Scores come out transposed, S^T = K Q^T (tokens x rows): a lane then holds four tokens of
// one row in the order in which the second product, O^T = V^T P^T, takes its operand, so that the weights never leave the lane.  Keys and
// values lie in the cache as the two products' first operands: 16 contiguous bytes a lane, neighbouring lanes side by side.
//
// Numbers: codes become binary16 exactly.  A query row is scaled by a power of
// two to a largest magnitude in [2^13, 2^14), so that bfloat16's range fits binary16 and nothing above 2^-28 of the row's largest loses a
// bit.  Scores, maxima, sums and outputs are binary32.  A weight is rounded once, to binary16, as p * (value scale / R) * 2^10, where R is
// a power of two no smaller than any value scale met so far: what is 2^-34 of the largest is still counted.  The maximum is
// raised only when a score passes it by 2^4, so that p <= 16 and the weights stay below 2^15.
#include <algorithm>

#include "dg_attention.h"

namespace {

constexpr int TILE = 32;      // tokens per step of a wavefront

// A tile -- two units of 16 tokens -- as a wavefront keeps it in LDS: keys, values, and 64 numbers (unit 0's key and value scales, unit 1's), with 4
// bits 64 more (z).  A wavefront has DEPTH tiles of its own on the way, by loads that write LDS, so that they take no registers: what hides HBM's one or
// two microseconds is wavefronts, four to a SIMD at 128 registers and 40 KB a workgroup (64 contexts of up to 8192, 4 bits: two wavefronts with three
// tiles each 131 us, four with two 100; 131071 tokens, 8 bits: two with two 74, four with one 64).
template <int BITS, int DIM>
struct Tile {
    static constexpr int PART = 4 * DIM * BITS, NUMBERS = BITS == 8 ? 256 : 512, BYTES = 2 * PART + NUMBERS;
    static constexpr int LOADS = 2 * PART / 1024 + NUMBERS / 256;
    static constexpr int DEPTH = 4 * 2 * BYTES <= 40960 ? 2 : 1, WAVES_PER_SIMD = DIM == 256 ? 1 : DIM == 128 && BITS == 4 ? 3 : 4;
};

template <class T, int BITS, int DIM, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (Tile<BITS, DIM>::WAVES_PER_SIMD)) void attention_kernel(Args args)
{
    constexpr int STEPS = DIM / 32;                       // products of 32 channels
    constexpr int BLOCKS = DIM / 16;                      // accumulators of 16 channels
    constexpr int VALUE_WORDS = DIM * BITS / 128;         // words of 4 tokens that a lane takes of a unit
    constexpr bool TWICE = std::is_same<T, _Float16>::value;        // weights in two halves, see below
    const DgAttention &a = args.a;
    // (a matrix instruction runs whatever the lanes' mask: what it stands under has to be a scalar branch)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    // Heads innermost and pieces outermost: neighbouring workgroups go to different dies (eight), and a context's last pieces, which shorter ones do not
    // have, are not to be all of one die (64 contexts of up to 8192 in 4 pieces, pieces innermost: 104 us for 81).
    int rest = blockIdx.x;
    const int h = rest % a.cache.heads;
    rest /= a.cache.heads;
    const int b = rest % a.B;
    rest /= a.B;
    const int row_block = rest % args.row_blocks, piece = rest / args.row_blocks;
    const Sequence seq = sequence(a, b);
    const int have = min(seq.count * args.group - row_block * 16, 16);                      // rows of the block that are there
    if (have <= 0) return;
    const int row = row_block * 16 + r;
    const int i = (int)dg_fdiv((uint32_t)row, args.by_group), j = row - i * args.group;     // new token, head of the group
    const bool there = r < have;
    const int first_i = (int)dg_fdiv((uint32_t)row_block * 16, args.by_group), last_i = (int)dg_fdiv((uint32_t)(row_block * 16 + have - 1), args.by_group);
    // tokens that the row sees: those before `end`; any row of the block: before `block_end`; every row: before `all_end` (rows that are not there
    // are computed as the block's first)
    const int block_end = a.causal ? max(seq.past + last_i + 1, 0) : seq.ctx;
    const int all_end = a.causal ? max(seq.past + first_i + 1, 0) : seq.ctx;
    const int end = a.causal && there ? max(seq.past + i + 1, 0) : all_end;
    const int from = piece * args.piece_tokens;
    const int to = piece == args.pieces - 1 ? block_end : min(block_end, from + args.piece_tokens);

    const uint8_t *const heads = a.cache.base + (int64_t)h * a.cache.head;
    // (through the scalar cache: a vector load would be waited for together with the tiles on the way)
    const auto table = (const __attribute__((address_space(4))) int32_t *)(a.table + (int64_t)b * a.table_width);
    typedef Tile<BITS, DIM> Kept;
    constexpr int SHARES = WAVES * 16 * (DIM + 4) * 4, RINGS = WAVES * Kept::DEPTH * Kept::BYTES;
    __shared__ __align__(1024) uint8_t room[SHARES > RINGS ? SHARES : RINGS];
    const uint8_t *const ring = room + wave * (Kept::DEPTH * Kept::BYTES);
    const uint32_t ring_lds = dg_lds_address(ring);
    // A unit past the context, or whose page is none of the cache's, is read from the first page instead and its tokens count as unseen.
    const auto page_of = [&](int t) { return t < seq.ctx ? table[dg_fdiv((uint32_t)t, a.cache.by_page)] : -1; };
    const auto is_page = [&](int page) { return (uint32_t)page < (uint32_t)a.cache.pages; };
    const auto fetch = [&](int t0, const int (&page)[2], int slot) {
        const uint8_t *block[2];
        uint32_t in_page[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t t = (uint32_t)(t0 + 16 * u);
            in_page[u] = is_page(page[u]) ? t - dg_fdiv(t, a.cache.by_page) * a.cache.page_size : 0;
            block[u] = heads + (is_page(page[u]) ? (int64_t)page[u] : 0) * a.cache.page_bytes();
        }
        const uint32_t lds = ring_lds + slot * Kept::BYTES;
        constexpr int CHUNKS = DIM * BITS / 8;                  // of 16 bytes, of a unit's keys or values
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int n = 0; n < Kept::PART / 1024; ++n) {
                const uint32_t to = lds + which * Kept::PART + 1024 * n;
                if constexpr (CHUNKS >= 64) {
                    const int u = 64 * n / CHUNKS;
                    dg_load16_to_lds(block[u] + which * a.cache.part + in_page[u] * (DIM * BITS / 8), 1024 * (n % (CHUNKS / 64)) + 16 * lane, to);
                } else {
                    const bool u = lane >= 32;
                    dg_load16_to_lds((u ? block[1] : block[0]) + which * a.cache.part + (u ? in_page[1] : in_page[0]) * (DIM * BITS / 8) + 16 * (lane & 31), to);
                }
            }
        const bool u = lane >= 32;
        const uint8_t *numbers = (u ? block[1] : block[0]) + 2 * a.cache.part + 4 * ((u ? in_page[1] : in_page[0]) + (lane & 16 ? a.cache.page_size : 0) + (lane & 15));
#pragma unroll
        for (int n = 0; n < Kept::NUMBERS / 256; ++n) dg_load4_to_lds(numbers + 8 * n * a.cache.page_size, lds + 2 * Kept::PART + 256 * n);
    };
    // the pages of the DEPTH tiles on the way; those of the one after are asked for a tile ahead
    constexpr int DEPTH = Kept::DEPTH, STRIDE = TILE * WAVES;
    int t0 = from + TILE * wave;
    int page[DEPTH + 1][2];
#pragma unroll
    for (int n = 0; n <= DEPTH; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) page[n][u] = page_of(t0 + n * STRIDE + 16 * u);
#pragma unroll
    for (int n = 0; n < DEPTH; ++n)
        if (t0 + n * STRIDE < to) fetch(t0 + n * STRIDE, page[n], n);
    int slot = 0;

    // the row's query
    v8h q[STEPS];
    float f, x[STEPS][8];
    const float most_q = load_query<T, DIM>((const T *)a.q + (int64_t)(seq.first + (there ? i : first_i)) * a.q_token +
                                                (int64_t)(h * args.group + (there ? j : 0)) * a.q_head, g, x);
    const float q_sum = query_operands<BITS, DIM>(x, most_q, a.scale, q, f);
    if (!(most_q < __builtin_inff())) f = __builtin_nanf("");
    const float from_bias = -(BITS == 8 ? BIAS8 : BIAS4_KEYS) * q_sum, f_sum = f * q_sum;

    v4f o[BLOCKS] = {};
    // sums are relative to 2^shift; a row's begin when it sees its first token, and `above` is what a score has to pass for the shift to be raised
    float shift = 0.0f, above = -__builtin_inff(), l = 0.0f, oz = 0.0f, R = 0.0f, per_R = 0.0f;
#pragma unroll 1
    for (; t0 < to; t0 += STRIDE) {
        if (t0 + (DEPTH - 1) * STRIDE < to) dg_wait_for_loads<(DEPTH - 1) * Kept::LOADS>();
        else dg_wait_for_loads<0>();
        const uint8_t *const tile = ring + slot * Kept::BYTES;
        const bool is[2] = {is_page(page[0][0]), is_page(page[0][1])};
        const int unit_end[2] = {is[0] ? end : 0, is[1] ? end : 0};
        const bool all_seen = t0 + TILE <= all_end && is[0] && is[1];
        // scores
        v4f score[2], ks[2], kz[2], vs[2], vz[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const v4f *numbers = (const v4f *)(tile + 2 * Kept::PART + 128 * u) + g;
            ks[u] = numbers[0];
            vs[u] = numbers[4];
            if (BITS == 4) {
                kz[u] = numbers[16];
                vz[u] = numbers[20];
            }
            v4f acc = {from_bias, from_bias, from_bias, from_bias};
#pragma unroll
            for (int s = 0; s < STEPS / 2; ++s) {
                const uint8_t *keys = tile + u * (Kept::PART / 2) + s * (128 * BITS);
                v2h c[8];
                if constexpr (BITS == 8) {
                    const v4u w = *(const v4u *)(keys + 16 * lane);
#pragma unroll
                    for (int e = 0; e < 4; ++e) halves8(w[e], c[2 * e], c[2 * e + 1]);
                } else {
                    const v2u w = *(const v2u *)(keys + 8 * lane);
                    halves4_keys(w[0], c);
                    halves4_keys(w[1], c + 4);
                }
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(join(c[0], c[1], c[2], c[3]), q[2 * s], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(join(c[4], c[5], c[6], c[7]), q[2 * s + 1], acc, 0, 0, 0);
            }
            score[u] = acc;
        }
        float top = -__builtin_inff(), most_vs = 0.0f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // (relative to the maximum that the sums go by)
                float x = BITS == 8 ? __builtin_fmaf(score[u][e], ks[u][e] * f, -shift)
                                    : __builtin_fmaf(score[u][e] * f, ks[u][e], __builtin_fmaf(f_sum, kz[u][e], -shift));
                score[u][e] = x;
            }
        if (!all_seen) {
            branch();
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool seen = t0 + 16 * u + 4 * g + e < unit_end[u];
                    score[u][e] = seen ? score[u][e] : -__builtin_inff();
                    vs[u][e] = seen ? vs[u][e] : 0.0f;
                    if (BITS == 4) vz[u][e] = seen ? vz[u][e] : 0.0f;
                }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                top = fmaxf(top, score[u][e]);
                most_vs = fmaxf(most_vs, fabsf(vs[u][e]));
            }
        if (__any(top > above)) {
            top = row_max(top);
            const bool begun = above == RAISE;
            const float by = begun ? fmaxf(top, 0.0f) : top == -__builtin_inff() ? 0.0f : top;
            const float keep = begun ? exp2_(-by) : 0.0f;                          // (nothing is summed before)
            shift += by;
            above = begun || top > -__builtin_inff() ? RAISE : above;
            l *= keep;
            oz *= keep;
#pragma unroll
            for (int u = 0; u < 2; ++u) score[u] -= by;
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k) o[k] *= keep;
        }
        if (__any(most_vs > R)) {
#pragma unroll
            for (int k = 32; k; k >>= 1) most_vs = fmaxf(most_vs, __shfl_xor(most_vs, k));
            const uint32_t bits = above_scale(most_vs);
            const float inverse = __uint_as_float((254u - bits) << 23), keep = R * inverse;
            R = __uint_as_float(bits << 23);
            per_R = inverse * WEIGHT_UNIT;
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k) o[k] *= keep;
        }
        // The weights as the second product's operand.  Binary16 outputs show a weight's rounding beside their own (the error against 64 bits was 1.4
        // times a binary32 computation's): there what the rounding left off goes through the matrix instructions as well.
        _Float16 w[8], rest[8] = {};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = exp2_(score[u][e]);
                l += p;
                if (BITS == 4) oz = __builtin_fmaf(p, __builtin_fmaf(8.0f, vs[u][e], vz[u][e]), oz);
                const float x = p * (vs[u][e] * per_R);
                const int at = 4 * u + (BITS == 8 ? e : (e & 1) * 2 + (e >> 1));          // (4 bits: tokens 0, 2, 1, 3)
                w[at] = (_Float16)x;
                if (TWICE) rest[at] = (_Float16)(x - (float)w[at]);
            }
        const v8h weights = {w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]};
        const v8h rests = {rest[0], rest[1], rest[2], rest[3], rest[4], rest[5], rest[6], rest[7]};
        const auto add = [&](v4f &acc, v8h values, float bias) {
            const _Float16 x = (_Float16)-bias;
            const v8h off = {x, x, x, x, x, x, x, x};
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(off, weights, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(values, weights, acc, 0, 0, 0);
            if (TWICE) {
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(off, rests, acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(values, rests, acc, 0, 0, 0);
            }
        };
        uint32_t words[2][VALUE_WORDS];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint8_t *values = tile + Kept::PART + u * (Kept::PART / 2) + g * (DIM * BITS / 2);
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
                add(o[k], join(c[0], c[1], c[2], c[3]), BIAS8);
            } else {
                v2h c[4], d[4];      // (tokens 0 and 2, 1 and 3; even and odd channels)
                halves4(words[0][k], c);
                halves4(words[1][k], d);
                add(o[2 * k], join(c[0], c[2], d[0], d[2]), BIAS4_EVEN);
                add(o[2 * k + 1], join(c[1], c[3], d[1], d[3]), BIAS4_ODD);
            }
        }
        // the tile has been read: its place is the next one's
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (t0 + DEPTH * STRIDE < to) fetch(t0 + DEPTH * STRIDE, page[DEPTH], slot);
        slot = slot + 1 == DEPTH ? 0 : slot + 1;
#pragma unroll
        for (int n = 0; n < DEPTH; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u) page[n][u] = page[n + 1][u];
#pragma unroll
        for (int u = 0; u < 2; ++u) page[DEPTH][u] = page_of(t0 + (DEPTH + 1) * STRIDE + 16 * u);
    }

    // The wavefronts' shares meet.  A lane holds channels channel(4 k, e) ... + 3 of row r in o[4 k ... 4 k + 3][e].
    float (*const all_o)[16][DIM + 4] = (float(*)[16][DIM + 4])room;       // (once every wavefront is done with its tiles)
    __shared__ float wave_m[WAVES][16], wave_l[WAVES][16];
    l = row_sum(l);
    oz = row_sum(oz);
    const float m = above == RAISE ? shift : -__builtin_inff();
    if (g == 0) wave_m[wave][r] = m;
    __syncthreads();
    float most = wave_m[0][r];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) most = fmaxf(most, wave_m[k][r]);
    const float mine = m == -__builtin_inff() && l == 0.0f ? 0.0f : exp2_(m - most);       // (a NaN stays one)
    if (g == 0) wave_l[wave][r] = l * mine;
    const float unit_o = R == 0.0f ? 1.0f : R * (1.0f / WEIGHT_UNIT) * mine;               // (nothing met: 0, or the NaN of a NaN)
    const float add_z = oz * mine;
    if (there)
#pragma unroll
        for (int k = 0; k < BLOCKS / 4; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int channel = BITS == 8 ? 64 * k + 16 * g + 4 * e : DIM == 64 ? 16 * g + 4 * e : 128 * (k / 2) + 32 * g + 8 * e + 4 * (k % 2);
                v4f x;
#pragma unroll
                for (int n = 0; n < 4; ++n) x[n] = BITS == 4 ? __builtin_fmaf(o[4 * k + n][e], unit_o, add_z) : o[4 * k + n][e] * unit_o;
                *(v4f *)&all_o[wave][r][channel] = x;
            }
    __syncthreads();
#pragma unroll 1
    for (int at = threadIdx.x; at < have * (DIM / 4); at += 64 * WAVES) {
        const int my_row = at / (DIM / 4), d = 4 * (at % (DIM / 4));
        v4f sum = *(const v4f *)&all_o[0][my_row][d];
        float total = wave_l[0][my_row], top = wave_m[0][my_row];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) {
            sum += *(const v4f *)&all_o[k][my_row][d];
            total += wave_l[k][my_row];
            top = fmaxf(top, wave_m[k][my_row]);
        }
        const int out_row = row_block * 16 + my_row;
        const int oi = (int)dg_fdiv((uint32_t)out_row, args.by_group), head = h * args.group + out_row - oi * args.group;
        if (args.pieces == 1) {
            const float by = total == 0.0f ? 0.0f : 1.0f / total;
            DgVec<T, 4> v;
#pragma unroll
            for (int k = 0; k < 4; ++k) v.e[k] = dg_from_float<T>(sum[k] * by);
            dg_store_vec<T, 4>((T *)a.out + (int64_t)(seq.first + oi) * a.out_token + (int64_t)head * a.out_head + d, v);
        } else {
            const int64_t to_row = (((int64_t)piece * a.B + b) * a.max_q + oi) * a.Hq + head;
            *(v4f *)(args.shares.o + to_row * DIM + d) = sum;
            if (d == 0) {
                args.shares.m[to_row] = top;
                args.shares.l[to_row] = total;
            }
        }
    }
}

// The pieces' shares of a row joined, a workgroup a row: the pieces' weights first, then groups of DIM / 4 threads take every GROUPS-th piece; the
// groups' sums are added in their order, so that the same call gives the same bits.
constexpr int MOST_PIECES = 256;

template <class T, int DIM>
__global__ __launch_bounds__(256) void attention_join_kernel(Args args)
{
    constexpr int LANES = DIM / 4, GROUPS = 256 / LANES;
    __shared__ float weight[MOST_PIECES], wave_max[4], wave_sum[4];
    __shared__ v4f sums[GROUPS][LANES];
    const DgAttention &a = args.a;
    const int64_t rows = (int64_t)a.B * a.max_q * a.Hq, at = blockIdx.x;
    const int64_t token = at / a.Hq, head = at % a.Hq;
    const int b = (int)(token / a.max_q), i = (int)(token % a.max_q);
    const Sequence seq = sequence(a, b);
    if (i >= seq.count) return;
    // (a thread a piece)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = threadIdx.x / LANES, part = threadIdx.x % LANES;
    const bool mine = (int)threadIdx.x < args.pieces;
    const float m = mine ? args.shares.m[threadIdx.x * rows + at] : -__builtin_inff(), l = mine ? args.shares.l[threadIdx.x * rows + at] : 0.0f;
    float most = m;
#pragma unroll
    for (int k = 32; k; k >>= 1) most = fmaxf(most, __shfl_xor(most, k));
    if (lane == 0) wave_max[wave] = most;
    __syncthreads();
    most = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
    const float w = m == -__builtin_inff() && l == 0.0f ? 0.0f : exp2_(m - most);
    weight[threadIdx.x] = w;
    float total = l * w;
#pragma unroll
    for (int k = 32; k; k >>= 1) total += __shfl_xor(total, k);
    if (lane == 0) wave_sum[wave] = total;
    __syncthreads();
    v4f o = {};
    const float *from = args.shares.o + at * DIM + 4 * part;
#pragma unroll 4
    for (int k = group; k < args.pieces; k += GROUPS) o += *(const v4f *)(from + k * rows * DIM) * weight[k];
    sums[group][part] = o;
    __syncthreads();
    if (group) return;
    for (int k = 1; k < GROUPS; ++k) o += sums[k][part];
    total = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
    const float by = total == 0.0f ? 0.0f : 1.0f / total;
    DgVec<T, 4> v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v.e[e] = dg_from_float<T>(o[e] * by);
    dg_store_vec<T, 4>((T *)a.out + (int64_t)(seq.first + i) * a.out_token + head * a.out_head + 4 * part, v);
}

// How the rows and the context are cut.
struct Plan {
    bool chunk;
    int32_t row_blocks, pieces, piece_tokens;
};
// One workgroup a SIMD (more: 64 contexts of up to 8192, 4 bits, 92 us with one or two, 107 with eight), pieces of 512 tokens at least; where that leaves
// compute units without a workgroup, pieces of 256 (one context of 1000 9.7 us for 11.3, of 4096 10.9 for 12.7; four of 8192 23.0 for 19.4).
Plan plan_of(const DgAttention &a)
{
    const int64_t rows = (int64_t)a.max_q * (a.Hq / a.cache.heads), simds = dg_simd_count(), units = simds / 4;
    Plan p;
    p.chunk = rows > 16;
    const int32_t block = p.chunk ? CHUNK_ROWS : 16, step = p.chunk ? CHUNK_STEP : TILE * 4;
    p.row_blocks = (int32_t)((rows + block - 1) / block);
    const int64_t blocks = (int64_t)p.row_blocks * a.B * a.cache.heads;
    const auto cut = [&](int64_t most, int64_t least) { return std::max<int64_t>(1, std::min({most / blocks, (a.max_ctx + least - 1) / least, (int64_t)MOST_PIECES})); };
    int64_t pieces = cut(p.chunk ? 2 * units : simds, 512);
    if (blocks * pieces < units) pieces = cut(units, 256);
    p.pieces = (int32_t)pieces;
    p.piece_tokens = (int32_t)((a.max_ctx + pieces * step - 1) / (pieces * step) * step);
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
    if (p.chunk) dg_launch_attention_chunk(args, type, stream);
    with_form(a, type, [&](auto t, auto bits, auto dim) {
        typedef decltype(t) T;
        constexpr int BITS = decltype(bits)::value, DIM = decltype(dim)::value;
        const uint32_t blocks = (uint32_t)((int64_t)p.row_blocks * a.B * a.cache.heads * p.pieces);
        if (!p.chunk) attention_kernel<T, BITS, DIM, 4><<<blocks, 256, 0, stream>>>(args);
        if (p.pieces > 1) attention_join_kernel<T, DIM><<<(uint32_t)rows, 256, 0, stream>>>(args);
    });
    return dg_check_launch("dg_paged_attention");
}
