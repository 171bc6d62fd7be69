// Attention of chunks of new tokens over the paged cache: the products of dg_attention_kernel.hip, for many rows.
//
// A workgroup takes 128 rows of a cached head, 32 a wavefront: two blocks of 16, so that a code is turned into binary16 once for two products.  The
// tokens go by in stages of 64, four units, one loaded by each wavefront into a ring in LDS that all four read.
//
// What bounds it is the vector unit: 32 tokens are 285 of its instructions for a wavefront (16 exponentials, 4 more for each weight of a lane, 96 for codes to binary16) beside
// 32 matrix instructions, which it hardly overlaps (the one 71 % of the cycles, the other 31 %).  2048 queries of 32 heads on 8 of 128 channels against 32768 tokens,
// 8 bits: 1.39 ms, 770 TFLOP/s.  Slower, when it took 1.4 to 1.48 ms: four blocks of rows a wavefront (half the conversions, but one wavefront a SIMD: 2.3 ms); operands made once for all
// four wavefronts and handed on through LDS (226 instructions, but a barrier every 32 tokens and four times the bytes from LDS: 1.56 ms).
#include "dg_attention.h"

namespace {

constexpr int WAVES = 4, N = CHUNK_ROWS / (16 * WAVES);

template <class T, int BITS, int DIM>
__global__ __launch_bounds__(64 * WAVES, DIM == 256 ? 1 : DIM == 64 ? 3 : 2) void attention_chunk_kernel(Args args)
{
    typedef Unit<BITS, DIM> U;
    constexpr int RING = DIM == 256 && BITS == 8 ? 2 : 3, STAGE = 4 * U::BYTES;
    __shared__ __align__(1024) uint8_t ring[RING * STAGE];
    __shared__ int is_there[RING][4];
    const DgAttention &a = args.a;
    // (a matrix instruction runs whatever the lanes' mask: what it stands under has to be a scalar branch)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    // heads innermost: a head's workgroups follow each other at a distance of `heads`, so with eight of them each die has its own; the last rows, which see
    // most, first
    uint32_t in_heads = blockIdx.x, in_pieces = taken(in_heads, args.by_heads), in_blocks = taken(in_pieces, args.by_pieces);
    const int b = taken(in_blocks, args.by_blocks), row_block = args.row_blocks - 1 - (int)in_blocks, piece = in_pieces, h = in_heads;
    const Sequence seq = sequence(a, b);
    const int first_row = row_block * CHUNK_ROWS, have = min(seq.count * args.group - first_row, CHUNK_ROWS);
    if (have <= 0) return;
    const int block_end = a.causal ? max(seq.past + (int)dg_fdiv((uint32_t)(first_row + have - 1), args.by_group) + 1, 0) : seq.ctx;
    const int from = piece * args.piece_tokens;
    const int to = piece == args.pieces - 1 ? block_end : min(block_end, from + args.piece_tokens);

    const uint8_t *const heads = a.cache.base + (int64_t)h * a.cache.head;
    const auto table = (const __attribute__((address_space(4))) int32_t *)(a.table + (int64_t)b * a.table_width);
    const uint32_t ring_lds = dg_lds_address(ring) + wave * U::BYTES;
    const auto page_of = [&](int t) { return t < seq.ctx ? table[dg_fdiv((uint32_t)t, a.cache.by_page)] : -1; };
    // this wavefront's unit of the stage from token t0
    const auto fetch = [&](int t0, int page, int slot) {
        const bool is = fetch_unit<BITS, DIM>(a.cache, heads, t0 + 16 * wave, page, ring_lds + slot * STAGE, lane);
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

    const int wave_row = 16 * N * wave, mine = min(have - wave_row, 16 * N);                  // the wavefront's rows (0 or fewer: none)
    Rows<T, BITS, DIM, N> rows;
    rows.begin(args, seq, h, first_row + wave_row, mine, r, g);
    int slot = 0, next_slot = RING - 1;
#pragma unroll 1
    for (int t0 = from; t0 < to; t0 += CHUNK_STEP) {
        dg_wait_for_loads<(RING - 2) * U::LOADS>();
        __syncthreads();
        // (past the end there is nothing to load; the waits count on loads, so they go on, from the first page)
        fetch(ahead, ahead < to ? page : -1, next_slot);
        ahead += CHUNK_STEP;
        page = page_of(ahead + 16 * wave);
        const uint8_t *const stage = ring + slot * STAGE;
        int is[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) is[u] = __builtin_amdgcn_readfirstlane(is_there[slot][u]);
        slot = slot + 1 == RING ? 0 : slot + 1;
        next_slot = next_slot + 1 == RING ? 0 : next_slot + 1;
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            if (t0 + 32 * half >= rows.any_end) break;
            rows.step(stage + half * (2 * U::BYTES), t0 + 32 * half, half ? is[2] : is[0], half ? is[3] : is[1], lane);
        }
    }
    dg_wait_for_loads<0>();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const float total = row_sum(rows.l[n]), z = row_sum(rows.oz[n]);
        const int at = 16 * n + r, row = first_row + wave_row + at;
        if (at >= mine) continue;
        const int i = (int)dg_fdiv((uint32_t)row, args.by_group), head = h * args.group + row - i * args.group;
        const bool alone = args.pieces == 1;
        const float by = !alone ? 1.0f : total == 0.0f ? 0.0f : 1.0f / total;
        const int64_t share = (((int64_t)piece * a.B + b) * a.max_q + i) * a.Hq + head;
        T *const out = (T *)a.out + (int64_t)(seq.first + i) * a.out_token + (int64_t)head * a.out_head;
#pragma unroll
        for (int k = 0; k < DIM / 64; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const v4f x = rows.channels(n, k, e, by, z * by);
                DgVec<T, 4> y;
#pragma unroll
                for (int c = 0; c < 4; ++c) y.e[c] = dg_from_float<T>(x[c]);
                if (alone) dg_store_vec<T, 4>(out + rows.channel(k, e, g), y);
                else *(v4f *)(args.shares.o + share * DIM + rows.channel(k, e, g)) = x;
            }
        if (!alone && g == 0) {
            args.shares.m[share] = rows.most(n);
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
