// Attention of new tokens over the paged cache.
//
// A row is one query head of one new token; the rows of a sequence that read the same cached head -- (token, head of the group), the
// token outermost -- are taken 16 at a time (two such blocks a wavefront where there are many).  Scores come out transposed, S^T = K Q^T (tokens x rows): a lane then holds four tokens of
// one row in the order in which the second product, O^T = V^T P^T, takes its operand, so that the weights never leave the lane.  Keys and
// values lie in the cache as the two products' first operands: 16 contiguous bytes a lane, neighbouring lanes side by side.
//
// Numbers: codes become binary16 exactly.  A query row is scaled by a power of
// two to a largest magnitude in [2^13, 2^14), so that bfloat16's range fits binary16 and nothing above 2^-28 of the row's largest loses a
// bit.  Scores, shifts, sums and outputs are binary32.  A weight is rounded once, to binary16 (twice, with what that left off, for binary16 outputs), as
// 2^(logit - shift) times the token's value scale, the row's largest being kept between 2^4 and 2^14: what is 2^-28 of it is still counted.  Nothing of this
// goes by other rows, or by what a row does not see: a row's bits are the same whatever stands beside it.
//
// What bounds it: for single tokens the cache's bytes, read once (one context of 131071 tokens, 32 heads on 8 of 128 channels, 8 bits: 56 us, 4.9 TB/s; 64 contexts of
// up to 8192, 4 bits: 80 us, 3.9 TB/s: there the vector unit is as busy, 16 columns of a product for the 4 rows that there are), or, for short contexts, two launches
// and one tile's chain of latencies (one context of 1000: 8.2 us; of 250, one launch, 6.1); for many rows the vector unit (chunk kernel).
#include <algorithm>
#include <cstring>

#include "dg_attention.h"

namespace {

constexpr int TILE = 32, WAVES = 4;      // tokens per step of a wavefront; wavefronts that share a piece of the context

// A wavefront has DEPTH tiles of two units of its own on the way, by loads that write LDS, so that they take no registers: what hides HBM's one or two
// microseconds is wavefronts, four to a SIMD at 128 registers and 40 KB a workgroup (64 contexts of up to 8192, 4 bits: two wavefronts with three tiles each
// 131 us, four with two 100; 131071 tokens, 8 bits: two with two 74, four with one 64).
template <int BITS, int DIM, int N>
struct Kept {
    static constexpr int TILE_BYTES = 2 * Unit<BITS, DIM>::BYTES, LOADS = 2 * Unit<BITS, DIM>::LOADS;
    static constexpr int DEPTH = WAVES * 2 * TILE_BYTES <= 40960 ? 2 : 1, RINGS = WAVES * DEPTH * TILE_BYTES;
    static constexpr int SHARES = WAVES * 16 * (DIM + 4) * 4;
    // Two blocks of rows of 64 channels: three, at 168 registers (300 x 12 queries on 3000 tokens in 4 bits 45.7 us, by two 49.7).  256 channels: what the registers
    // give, two for one block (one token on 8192, 32 heads on 8, 8 bits 16.0 us, 2.1 TB/s; 16 on up to 4096, 4 bits 37.6; 500 on 4000, 16 heads on 4, 8 bits 83).
    static constexpr int WAVES_PER_SIMD = DIM == 256 ? 1 : N == 2 ? (DIM == 64 ? 3 : 2) : DIM == 128 && BITS == 4 ? 3 : 4;
};

// 16 N rows of a cached head and a piece of the context by a workgroup, whose wavefronts take a tile in turn.
template <class T, int BITS, int DIM, int N>
__global__ __launch_bounds__(64 * WAVES, (Kept<BITS, DIM, N>::WAVES_PER_SIMD)) void attention_kernel(Args args)
{
    typedef Kept<BITS, DIM, N> K;
    constexpr int DEPTH = K::DEPTH, STRIDE = TILE * WAVES, ROWS = 16 * N;
    __shared__ __align__(1024) uint8_t room[K::SHARES > K::RINGS ? K::SHARES : K::RINGS];
    __shared__ float wave_m[WAVES][16], wave_l[WAVES][16];
    const DgAttention &a = args.a;
    // (a matrix instruction runs whatever the lanes' mask: what it stands under has to be a scalar branch)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    // Heads innermost and pieces outermost: neighbouring workgroups go to different dies (eight), and a context's last pieces, which shorter ones do not
    // have, are not to be all of one die (64 contexts of up to 8192 in 4 pieces, pieces innermost: 104 us for 92).
    uint32_t in_heads = blockIdx.x, in_sequences = taken(in_heads, args.by_heads), in_blocks = taken(in_sequences, args.by_sequences);
    const int piece = taken(in_blocks, args.by_blocks), h = in_heads, b = in_sequences, row_block = in_blocks;
    const Sequence seq = sequence(a, b);
    const int have = min(seq.count * args.group - row_block * ROWS, ROWS);                  // rows of the block that are there
    if (have <= 0) return;
    // tokens that any row of the block sees
    const int block_end = a.causal ? max(seq.past + (int)dg_fdiv((uint32_t)(row_block * ROWS + have - 1), args.by_group) + 1, 0) : seq.ctx;
    const int from = piece * args.piece_tokens;
    const int to = piece == args.pieces - 1 ? block_end : min(block_end, from + args.piece_tokens);

    const uint8_t *const heads = a.cache.base + (int64_t)h * a.cache.head;
    // (through the scalar cache: a vector load would be waited for together with the tiles on the way)
    const auto table = (const __attribute__((address_space(4))) int32_t *)(a.table + (int64_t)b * a.table_width);
    const uint8_t *const ring = room + wave * (DEPTH * K::TILE_BYTES);
    const uint32_t ring_lds = dg_lds_address(ring);
    const auto page_of = [&](int t) { return t < seq.ctx ? table[dg_fdiv((uint32_t)t, a.cache.by_page)] : -1; };
    const auto fetch = [&](int t0, const int (&page)[2], int slot) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            fetch_unit<BITS, DIM>(a.cache, heads, t0 + 16 * u, page[u], ring_lds + slot * K::TILE_BYTES + u * Unit<BITS, DIM>::BYTES, lane);
    };
    // the pages of the DEPTH tiles on the way; those of the one after are asked for a tile ahead
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
    Rows<T, BITS, DIM, N> rows;
    rows.begin(args, seq, h, row_block * ROWS, have, r, g);
#pragma unroll 1
    for (; t0 < to; t0 += STRIDE) {
        if (t0 + (DEPTH - 1) * STRIDE < to) dg_wait_for_loads<(DEPTH - 1) * K::LOADS>();
        else dg_wait_for_loads<0>();
        const auto is_page = [&](int p) { return (uint32_t)p < (uint32_t)a.cache.pages; };
        rows.step(ring + slot * K::TILE_BYTES, t0, is_page(page[0][0]), is_page(page[0][1]), lane);
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

    // The wavefronts' shares meet in LDS, 16 rows at a time.
    float (*const all_o)[16][DIM + 4] = (float(*)[16][DIM + 4])room;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        __syncthreads();                                     // (every wavefront is done with its tiles, or with the rows before)
        const float l = row_sum(rows.l[n]), oz = row_sum(rows.oz[n]), m = rows.most(n);
        if (g == 0) wave_m[wave][r] = m;
        __syncthreads();
        float most = wave_m[0][r];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) most = fmaxf(most, wave_m[k][r]);
        const float half = half_factor(m, l, most), mine = half * half;
        if (g == 0) wave_l[wave][r] = l * half * half;
        if (16 * n + r < have)
#pragma unroll
            for (int k = 0; k < DIM / 64; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) *(v4f *)&all_o[wave][r][rows.channel(k, e, g)] = rows.channels(n, k, e, mine, oz * mine);
        __syncthreads();
#pragma unroll 1
        for (int at = threadIdx.x; at < min(have - 16 * n, 16) * (DIM / 4); at += 64 * WAVES) {
            const int my_row = at / (DIM / 4), d = 4 * (at % (DIM / 4));
            v4f sum = *(const v4f *)&all_o[0][my_row][d];
            float total = wave_l[0][my_row], top = wave_m[0][my_row];
#pragma unroll
            for (int k = 1; k < WAVES; ++k) {
                sum += *(const v4f *)&all_o[k][my_row][d];
                total += wave_l[k][my_row];
                top = fmaxf(top, wave_m[k][my_row]);
            }
            const int out_row = row_block * ROWS + 16 * n + my_row;
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
    uint32_t in_token = (uint32_t)at, in_sequence = taken(in_token, args.by_Hq);
    const int b = taken(in_sequence, args.by_max_q), i = in_sequence, head = in_token;
    const Sequence seq = sequence(a, b);
    if (i >= seq.count) return;
    // (a thread a piece)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = threadIdx.x / LANES, part = threadIdx.x % LANES;
    const bool mine = (int)threadIdx.x < args.pieces;
    const float m = mine ? args.shares.m[threadIdx.x * rows + at] : -__builtin_inff(), l = mine ? args.shares.l[threadIdx.x * rows + at] : 0.0f;
    float most = dg_over_wave(m, DgMax());
    if (lane == 0) wave_max[wave] = most;
    __syncthreads();
    most = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
    const float half = half_factor(m, l, most);
    weight[threadIdx.x] = half * half;
    float total = dg_over_wave(l * half * half, DgAdd());
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

// The same, a wavefront a row, for many rows of few pieces (64 at most): 16000 rows of two pieces 19 us by workgroups, 7 by wavefronts.
template <class T, int DIM>
__global__ __launch_bounds__(256) void attention_join_rows_kernel(Args args)
{
    constexpr int PER = DIM / 64;
    const DgAttention &a = args.a;
    const int64_t rows = (int64_t)a.B * a.max_q * a.Hq, at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= rows) return;
    const int lane = threadIdx.x & 63;
    uint32_t in_token = (uint32_t)at, in_sequence = taken(in_token, args.by_Hq);
    const int b = taken(in_sequence, args.by_max_q), i = in_sequence, head = in_token;
    const Sequence seq = sequence(a, b);
    if (i >= seq.count) return;
    const bool mine = lane < args.pieces;
    const float m = mine ? args.shares.m[lane * rows + at] : -__builtin_inff(), l = mine ? args.shares.l[lane * rows + at] : 0.0f;
    const float most = dg_over_wave(m, DgMax());
    const float half = half_factor(m, l, most), w = half * half;
    float total = dg_over_wave(l * half * half, DgAdd());
    float o[PER] = {};
    const float *from = args.shares.o + at * DIM + PER * lane;
    for (int k = 0; k < args.pieces; ++k) {
        const DgVec<float, PER> x = dg_load_vec<float, PER>(from + k * rows * DIM);
        const float by = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), k));
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] += x.e[e] * by;
    }
    const float by = total == 0.0f ? 0.0f : 1.0f / total;
    DgVec<T, PER> v;
#pragma unroll
    for (int e = 0; e < PER; ++e) v.e[e] = dg_from_float<T>(o[e] * by);
    dg_store_vec<T, PER>((T *)a.out + (int64_t)(seq.first + i) * a.out_token + head * a.out_head + PER * lane, v);
}

// How the rows and the context are cut.
struct Plan {
    int32_t rows;                       // of a workgroup: 16 or 32, or CHUNK_ROWS
    int32_t row_blocks, pieces, piece_tokens;
};

// Rows: 16 a workgroup, whose wavefronts share its piece of the context, give most workgroups; 32 turn each code into binary16 once for two products; 128,
// 32 a wavefront, load a token once for all of them and have nothing to join at the end, but wait for one another at every stage.  us with 16, 32, 128
// (queries x sequences on contexts, heads / cached heads x channels; several sequences have lengths spread evenly up to these), the rule's choice marked:
//     8 x 32 on 2048, 64/8 x 128       *23    28    55        256 on 8192, 32/8 x 128, 4 bits        92   *80    87
//     64 on 16384, 32/8 x 128          *48    44    58        300 x 12 on 3000, 16/16 x 64, 4 bits   51   *50    99
//     1000 on 1000, 16/16 x 64         *16    16    28        512 x 4 on 4096, 32/8 x 128           106  *113   133
//     2048 x 2 on 2048, 32/8 x 128     172   179  *121        2048 on 32768, 32/8 x 128            1856  1437 *1378
// and where its lines are, 32/8 x 128 but for the last:
//     512 on 32768      502  *381   372        1024 on 8192    239  *196   199        2048 on 4096                 206  *166   156
//     1024 on 32768     969  *740   721        2048 on 8192    437   344  *330        3000 on 3000                 169  *147   119
//     1536 on 32768    1414 *1089  1370        1024 on 32768, 4 bits 1093 *924 950    4096 on 8192, 16/16 x 64     302   233  *265
// So the lines are near where the sides meet for long contexts; a prompt of its own (3000 on 3000) and narrow heads lose 14 to 24 % on the wrong side of them.
// Pieces: one workgroup a SIMD (half as many of 32 rows; more: 64 contexts of up to 8192, 4 bits, 92 us with one or two a SIMD, 107 with eight), pieces of 512
// tokens at least; where that leaves compute units without a workgroup, pieces of 128, a tile a wavefront (one context of 1000 8.1 us, 8.9 by pieces of
// 256; of 4000 8.8, 9.9; but four of 8192 by pieces of 256 23.0 for 19.4), or one piece, which needs no joining, of up to four tiles a wavefront (two with
// 256 channels, whose tiles take twice as long): 250 tokens 6.1 for 8.0, 500 7.8 for 8.1, 600 8.6 for 8.1.
Plan plan_of(const DgAttention &a)
{
    const int64_t rows = (int64_t)a.max_q * (a.Hq / a.cache.heads), simds = dg_simd_count(), units = simds / 4;
    const auto blocks_of = [&](int64_t n) { return (rows + n - 1) / n * a.B * a.cache.heads; };
    Plan p;
    const int64_t chunks = blocks_of(CHUNK_ROWS);
    if (rows > 16 && (chunks >= 4 * units || (chunks >= 2 * units && a.max_ctx >= 8192))) p.rows = CHUNK_ROWS;
    else p.rows = rows > 16 && blocks_of(16) * a.max_ctx >= 3500000 ? 32 : 16;
    if (const char *forced = dg_override("DG_ATTENTION_ROWS")) p.rows = !strcmp(forced, "16") ? 16 : !strcmp(forced, "32") ? 32 : !strcmp(forced, "128") ? CHUNK_ROWS : p.rows;
    const int32_t step = p.rows == CHUNK_ROWS ? CHUNK_STEP : TILE * WAVES;
    p.row_blocks = (int32_t)((rows + p.rows - 1) / p.rows);
    const int64_t blocks = blocks_of(p.rows);
    const auto cut = [&](int64_t most, int64_t least) { return std::max<int64_t>(1, std::min({most / blocks, (a.max_ctx + least - 1) / least, (int64_t)MOST_PIECES})); };
    int64_t pieces = cut(p.rows == 16 ? simds : simds / 2, 512);
    if (blocks * pieces < units) pieces = a.max_ctx <= (a.cache.dim == 256 ? 256 : 512) ? 1 : cut(units, 128);
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
    Args args = {a, a.Hq / a.cache.heads, p.row_blocks, p.pieces, p.piece_tokens, dg_make_div((uint32_t)(a.Hq / a.cache.heads)), dg_make_div(a.cache.heads), dg_make_div(a.B),
                 dg_make_div(p.row_blocks), dg_make_div(p.pieces), dg_make_div(a.Hq), dg_make_div(a.max_q), {}};
    const int64_t rows = (int64_t)a.B * a.max_q * a.Hq;
    args.shares.o = (float *)a.work;
    args.shares.m = args.shares.o + (int64_t)p.pieces * rows * a.cache.dim;
    args.shares.l = args.shares.m + (int64_t)p.pieces * rows;
    if (p.rows == CHUNK_ROWS) dg_launch_attention_chunk(args, type, stream);
    with_form(a, type, [&](auto t, auto bits, auto dim) {
        typedef decltype(t) T;
        constexpr int BITS = decltype(bits)::value, DIM = decltype(dim)::value;
        const uint32_t blocks = (uint32_t)((int64_t)p.row_blocks * a.B * a.cache.heads * p.pieces);
        if (p.rows == 16) attention_kernel<T, BITS, DIM, 1><<<blocks, 64 * WAVES, 0, stream>>>(args);
        if (p.rows == 32) attention_kernel<T, BITS, DIM, 2><<<blocks, 64 * WAVES, 0, stream>>>(args);
        if (p.pieces > 1 && p.pieces <= 64 && rows >= 1024) attention_join_rows_kernel<T, DIM><<<(uint32_t)((rows + 3) / 4), 256, 0, stream>>>(args);
        else if (p.pieces > 1) attention_join_kernel<T, DIM><<<(uint32_t)rows, 256, 0, stream>>>(args);
    });
    return dg_check_launch("dg_paged_attention");
}
