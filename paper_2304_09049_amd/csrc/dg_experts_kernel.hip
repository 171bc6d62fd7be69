// The gated feed-forward of chosen experts, weights in microscaled 4-bit floating point, for few tokens.
//
// Two products with what each expert's tokens have of x, and of h between them.  A (token, choice) is a pair; an expert's pairs are the columns of its products.  Few tokens: the
// experts' weights are read once for all their pairs, and that is what bounds it, so activations stay as they are: weights become bfloat16 on their way into the matrix
// instruction (exactly: two bits and a power of two), x is bfloat16 or two of them (binary16's eleven bits), h is held as two, 2^-17 off at most.  (As three, all of its 24 bits, 0.05 % instead of 0.25 % of bfloat16 results
// differ by a unit from those of binary32 throughout, errors against 64 bits stay as they are to six digits, and what it takes is more: one token to 4 of 64, 2048 x 1024, 11.6 us for 10.9, 64 to 6 of 64, 4096 x 1024, 92 for 84,
// 256 to 2 of 8, 4096 x 4096, 210 for 155.)
//
// v_mfma_f32_16x16x32_bf16: lane (r, g) holds eight numbers of row (or column) r; which eight of the 32 positions is free as long as both operands take the same.  A lane takes a block of
// 32 weights, 16 bytes and a scale, and uses eight after eight: word i of block 4 h + g of a stage.  Everything comes by way of LDS (neighbouring lanes load neighbouring bytes), in stages
// of 256 positions: 128 bytes of a row of weights, 512 of a row of activations.
#include "dg_mx4.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

constexpr int MOST_PAIRS = 4096;         // of a turn: their numbers are 16-bit
constexpr int MOST_TOKENS = 256;
constexpr int FEW_PAIRS = 16;            // each pair by itself

// Rows of activations as the products take them: PLANES of bfloat16 whose sum is the number, rows that begin on 4 bytes, `pitch` elements from the next, `size` of them counting; from there to the next multiple
// of 8 they are 0.
struct Rows {
    const __bf16 *x;
    int32_t pitch, plane, size;          // elements
    uint32_t bytes;                      // of all of it; a turn's are below 2^31
};
struct Work {
    __bf16 *x;               // [planes][T][pitch_x], where x is not taken as it is
    __bf16 *h;               // [2][pairs][pitch_h]; zeros from inner on
    float *y;                // [pairs][pitch_y]
    int32_t pitch_x, pitch_h, pitch_y;
};

// ---- what the products share ---------------------------------------------------------------------------------------------

// The eight weights of word i of a block: 16 bytes and its scale's byte.  (255 << 23 is an infinity; the conversion makes NaNs by it.)
__device__ __forceinline__ v8b weights_of(const v4i &codes, uint32_t byte, int i)
{
    const float s = __uint_as_float(byte ? byte << 23 : 0x00400000u);
    const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 1);
    const v2b c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 3);
    return (v8b){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ v4f multiply(const v8b &w, const v8b &x, const v4f &c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0); }

// The number as two: what bfloat16 holds of it, and what bfloat16 holds of the rest.
__device__ __forceinline__ void split(float f, __bf16 &high, __bf16 &low)
{
    high = (__bf16)f;
    low = fabsf((float)high) < __builtin_inff() ? (__bf16)(f - (float)high) : (__bf16)0.0f;
}

__device__ __forceinline__ float gated(float gate, float other) { return gate / (1.0f + expf(-gate)) * other; }

// h of four neighbouring channels of a pair, 0 from `inner` on.
__device__ __forceinline__ void store_h(const DgExperts &p, const Work &work, int32_t pair, int32_t f, const v4f &gate, const v4f &other)
{
    DgVec<__bf16, 4> high, low;
#pragma unroll
    for (int e = 0; e < 4; ++e) split(f + e < p.d.inner ? gated(gate[e], other[e]) : 0.0f, high.e[e], low.e[e]);
    __bf16 *to = work.h + (int64_t)pair * work.pitch_h + f;
    dg_store_vec<__bf16, 4>(to, high);
    dg_store_vec<__bf16, 4>(to + (int64_t)p.T * p.top * work.pitch_h, low);
}

// A block of 16 rows of an expert's weights, from `row` on: none past `last`.
struct Weights {
    dg_v4i codes, scales;
    int32_t have, row, scales_row;
};
__device__ __forceinline__ Weights weights_at(const uint8_t *codes, int64_t row_bytes, const uint8_t *scales, int64_t scales_row_bytes, int64_t row, int32_t rows, int32_t blocks)
{
    const int32_t have = max(1, min(16, rows));                      // (a block past the end: one row of it is read, and nothing becomes of it)
    return {dg_rows_buffer(codes, row, row_bytes, have, 16 * blocks), dg_rows_buffer(scales, row, scales_row_bytes, have, (blocks + 3) / 4 * 4), have, (int32_t)row_bytes, (int32_t)scales_row_bytes};
}
// A lane's offsets: in load i (0, 1) of a stage's 8 rows each, and in one of 16 rows' scales, `each` bytes of a row and 16 a lane.
__device__ __forceinline__ uint32_t codes_offset(const Weights &w, int i)
{
    const int lane = threadIdx.x & 63, row = 8 * i + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
    return row < w.have ? row * (uint32_t)w.row + 16 * piece : DG_NOWHERE;
}
__device__ __forceinline__ bool codes_past(int i, int32_t b, int32_t blocks)
{
    const int lane = threadIdx.x & 63, row = 8 * i + (lane >> 3);
    return b + ((lane & 7) ^ ((row >> 1) & 7)) >= blocks;
}

// ONCE: codes that nothing of this call reads again are not kept in the caches (us, kept and not: 64 tokens to 6 of 64 experts, 4096 x 1024, 100 and 92; one to 4 of 64, 2048 x 1024, 11.7 and
// 11.0; but 256 to 2 of 8, 4096 x 4096, where they are read again for the next pairs, 184 and 188).
template <bool ONCE>
__device__ __forceinline__ void load_codes(const Weights &w, uint32_t offset, uint32_t lds)
{
    if (ONCE) dg_load16_once_to_lds(w.codes, offset, lds);
    else dg_load16_to_lds(w.codes, offset, lds);
}

// The stage's products for a lane's row blocks and columns: `w` where the 16 rows' codes lie, their scales' bytes, `x` where its column's activations lie (element 0; planes PLANE bytes apart).
template <int BLOCKS, int COLUMNS, int PLANES>
__device__ __forceinline__ void stage_products(const uint8_t *const (&w)[BLOCKS], const uint32_t (&byte)[BLOCKS][2], const uint8_t *const (&x)[COLUMNS], int plane, int twist, v4f (&acc)[BLOCKS][COLUMNS])
{
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        v4i codes[BLOCKS];
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) codes[i] = *(const v4i *)(w[i] + r * 128 + (((4 * h + g) ^ ((r >> 1) & 7)) << 4));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v8b xk[COLUMNS][PLANES];
#pragma unroll
            for (int c = 0; c < COLUMNS; ++c)
#pragma unroll
                for (int k = 0; k < PLANES; ++k) xk[c][k] = *(const v8b *)(x[c] + k * plane + (((16 * h + 4 * g + q) ^ twist) << 4));
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                const v8b wk = weights_of(codes[i], byte[i][h], q);
#pragma unroll
                for (int c = 0; c < COLUMNS; ++c)
#pragma unroll
                    for (int k = 0; k < PLANES; ++k) acc[i][c] = multiply(wk, xk[c][k], acc[i][c]);
            }
        }
    }
}

// ---- activations that are not taken as they are ---------------------------------------------------------------------------

template <class T>
__global__ __launch_bounds__(256) void experts_rows_kernel(DgExperts p, Work work)
{
    constexpr bool TWO = !std::is_same<T, __bf16>::value;
    const int32_t k = (blockIdx.x * 256 + threadIdx.x) * 8, t = blockIdx.y;
    if (k >= work.pitch_x) return;
    const DgVec<T, 8> at = dg_eight<T>((const T *)p.x + t * p.stride_x, k, p.d.hidden);
    DgVec<__bf16, 8> high, low;
#pragma unroll
    for (int i = 0; i < 8; ++i) split(dg_to_float(at.e[i]), high.e[i], low.e[i]);
    __bf16 *to = work.x + (int64_t)t * work.pitch_x + k;
    dg_store_vec<__bf16, 8>(to, high);
    if (TWO) dg_store_vec<__bf16, 8>(to + (int64_t)p.T * work.pitch_x, low);
}

// ---- few pairs: each by itself ---------------------------------------------------------------------------------------------
//
// up: a workgroup has 16 channels (their gates' rows and the others') of a pair; four wavefronts share K in chunks of 512 positions and work alone, each with a ring of stages, until their sums meet.
// down: a workgroup has 16 channels of every token; eight wavefronts take pair after pair, and the pairs' results meet in LDS, so that the choices are added up here, in their order.
// One token to 4 of 64, 2048 x 1024: two launches of 6 us, each a chain of latencies (ids, rows, a few loads one behind another, sums).

template <int PLANES, bool ONCE>
__global__ __launch_bounds__(256) void experts_few_up_kernel(DgExperts p, Rows rows, Work work)
{
    constexpr int WAVES = 4, RING = 3, LOADS = 5, STAGE = LOADS * 1024, SCALES = 512, MINE = RING * STAGE + 2 * SCALES;
    __shared__ __align__(1024) uint8_t room[WAVES * MINE];
    __shared__ v4f sums[WAVES][2][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t pair = blockIdx.y, f0 = blockIdx.x * 16, blocks = (p.d.hidden + 31) / 32, expert = p.ids[pair];
    if ((uint32_t)expert >= (uint32_t)p.d.experts) return;
    Weights w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = weights_at(p.d.up + expert * p.d.up_expert, p.d.up_row, p.d.up_scales + expert * p.d.up_scales_expert, p.d.up_scales_row, min(f0, p.d.inner - 1) + (int64_t)i * p.d.inner,
                          p.d.inner - f0, blocks);
    // (planes: the lanes from 32 on load the second one's)
    const dg_v4i x = dg_buffer((const uint8_t *)rows.x, rows.bytes);
    const uint32_t x_first = 2u * (uint32_t)(pair / p.top * rows.pitch), x_offset = lane < 32 ? x_first + 16 * lane : PLANES == 2 ? x_first + 2u * rows.plane + 16 * (lane - 32) : DG_NOWHERE;
    uint8_t *const mine = room + wave * MINE, *const scale_room = mine + RING * STAGE;
    const uint32_t lds = dg_lds_address(mine), scale_lds = lds + RING * STAGE;
    uint32_t offset[2][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) offset[i / 2][i % 2] = codes_offset(w[i / 2], i % 2);
    const auto fetch = [&](int32_t s) __attribute__((always_inline)) {
        const int32_t chunk = wave + WAVES * (s / 2), b = 16 * chunk + 8 * (s % 2);
        if (s % 2 == 0) {
            const int row = lane & 15;
            const uint32_t to = scale_lds + s / 2 % 2 * SCALES;
            // (two loads of 16 lanes: a lane's 16 bytes lie at its place whether the others load or not)
            if (lane < 16) dg_load16_to_lds(w[0].scales, row < w[0].have && 16 * chunk < blocks ? row * (uint32_t)w[0].scales_row + 16 * chunk : DG_NOWHERE, to);
            if (lane >= 16 && lane < 32) dg_load16_to_lds(w[1].scales, row < w[1].have && 16 * chunk < blocks ? row * (uint32_t)w[1].scales_row + 16 * chunk : DG_NOWHERE, to);
        }
        const uint32_t to = lds + s % RING * STAGE;
#pragma unroll
        for (int i = 0; i < 4; ++i) load_codes<ONCE>(w[i / 2], codes_past(i % 2, b, blocks) ? DG_NOWHERE : offset[i / 2][i % 2] + 16 * b, to + 1024 * i);
        dg_load16_to_lds(x, (PLANES == 2 || lane < 32) && 32 * b + 8 * (lane & 31) < rows.size ? x_offset + 64 * b : DG_NOWHERE, to + 4096);
    };
    const int32_t chunks = (blocks + 15) / 16, stages = chunks > wave ? (chunks - wave + WAVES - 1) / WAVES * 2 : 0;
    v4f acc[2][1] = {};
    if (stages) {
#pragma unroll
        for (int s = 0; s < RING; ++s) fetch(s);
    }
#pragma unroll 1
    for (int32_t s = 0; s < stages; ++s) {
        const int32_t b = 16 * (wave + WAVES * (s / 2)) + 8 * (s % 2);
        dg_wait_for_loads<(RING - 1) * LOADS>();
        const uint8_t *stage = mine + s % RING * STAGE, *const wk[2] = {stage, stage + 2048}, *const xk[1] = {stage + 4096};
        uint32_t byte[2][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) byte[i / 2][i % 2] = scale_room[s / 2 % 2 * SCALES + 256 * (i / 2) + 16 * r + 8 * (s % 2) + 4 * (i % 2) + g];
        if (b + 8 > blocks) {
            // scales past the row: its codes are 0, and 0 by whatever lies there might be no number
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (b + 4 * (i % 2) + g >= blocks) byte[i / 2][i % 2] = 127;
        }
        stage_products<2, 1, PLANES>(wk, byte, xk, 512, 0, acc);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        fetch(s + RING);
    }
    dg_wait_for_loads<0>();
#pragma unroll
    for (int i = 0; i < 2; ++i) sums[wave][i][lane] = acc[i][0];
    __syncthreads();
    if (wave == 0 && r == 0) {
        v4f gate = sums[0][0][lane], other = sums[0][1][lane];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) {
            gate += sums[k][0][lane];
            other += sums[k][1][lane];
        }
        store_h(p, work, pair, f0 + 4 * g, gate, other);
    }
}

template <class T, bool ONCE>
__global__ __launch_bounds__(512) void experts_few_down_kernel(DgExperts p, Rows rows)
{
    constexpr int WAVES = 8, RING = 4, LOADS = 3, STAGE = LOADS * 1024, SCALES = 512, MINE = RING * STAGE + 2 * SCALES;
    __shared__ __align__(1024) uint8_t room[WAVES * MINE];
    __shared__ float results[FEW_PAIRS][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t m0 = blockIdx.x * 16, blocks = (p.d.inner + 31) / 32, pairs = p.T * p.top, all_stages = (blocks + 7) / 8;
    uint8_t *const mine = room + wave * MINE, *const scale_room = mine + RING * STAGE;
    const uint32_t lds = dg_lds_address(mine), scale_lds = lds + RING * STAGE;
    // (fewer pairs than wavefronts: parts of inner as well, their sums added up in order; one token to 1 of 8, 4096 x 4096, 17.4 us without and 12.8, to 2 21.8 and 18.7)
    const int32_t parts = pairs == 1 ? 8 : pairs == 2 ? 4 : pairs <= 4 ? 2 : 1, each = (all_stages + parts - 1) / parts;
    for (int32_t task = wave; task < pairs * parts; task += WAVES) {
        const int32_t pair = task / parts, from = task % parts * each, stages = min(all_stages - from, each), end = min(blocks, 8 * (from + stages));
        const int32_t expert = __builtin_amdgcn_readfirstlane(p.ids[pair]);
        if ((uint32_t)expert >= (uint32_t)p.d.experts) continue;
        const Weights w = weights_at(p.d.down + expert * p.d.down_expert, p.d.down_row, p.d.down_scales + expert * p.d.down_scales_expert, p.d.down_scales_row, m0, p.d.hidden - m0, blocks);
        const dg_v4i h = dg_buffer((const uint8_t *)rows.x, rows.bytes);
        const uint32_t h_offset = 2u * (uint32_t)(pair * rows.pitch) + (lane < 32 ? 16 * lane : 2u * rows.plane + 16 * (lane - 32));
        const uint32_t offset[2] = {codes_offset(w, 0), codes_offset(w, 1)};
        const auto fetch = [&](int32_t s) __attribute__((always_inline)) {
            const int32_t b = 8 * (from + s);
            if (s % 4 == 0) {
                const int row = lane >> 1;
                const int32_t k = b + 16 * (lane & 1);
                if (lane < 32) dg_load16_to_lds(w.scales, row < w.have && k < blocks && b < end ? row * (uint32_t)w.scales_row + k : DG_NOWHERE, scale_lds + s / 4 % 2 * SCALES);
            }
            const uint32_t to = lds + s % RING * STAGE;
#pragma unroll
            for (int i = 0; i < 2; ++i) load_codes<ONCE>(w, codes_past(i, b, end) ? DG_NOWHERE : offset[i] + 16 * b, to + 1024 * i);
            dg_load16_to_lds(h, b < end && 32 * b + 8 * (lane & 31) < rows.size ? h_offset + 64 * b : DG_NOWHERE, to + 2048);
        };
        v4f acc[1][1] = {};
#pragma unroll
        for (int s = 0; s < RING; ++s) fetch(s);
#pragma unroll 1
        for (int32_t s = 0; s < stages; ++s) {
            dg_wait_for_loads<(RING - 1) * LOADS>();
            const uint8_t *stage = mine + s % RING * STAGE, *const wk[1] = {stage}, *const xk[1] = {stage + 2048};
            uint32_t byte[1][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                byte[0][i] = scale_room[s / 4 % 2 * SCALES + 32 * r + 8 * (s % 4) + 4 * i + g];
                if (8 * (from + s) + 4 * i + g >= blocks) byte[0][i] = 127;
            }
            stage_products<1, 1, 2>(wk, byte, xk, 512, 0, acc);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch(s + RING);
        }
        dg_wait_for_loads<0>();
        if (r == 0) *(v4f *)&results[task][4 * g] = acc[0][0];
    }
    __syncthreads();
    // a token's choices together, in their order
    for (int32_t at = threadIdx.x; at < 16 * p.T; at += 64 * WAVES) {
        const int32_t t = at / 16, c = at % 16;
        float sum = 0.0f;
        for (int32_t j = 0; j < p.top; ++j)
            if ((uint32_t)p.ids[t * p.top + j] < (uint32_t)p.d.experts) {
                const int32_t task = (t * p.top + j) * parts;
                float y = results[task][c];
                for (int32_t i = 1; i < parts; ++i) y += results[task + i][c];
                sum += p.weights[t * p.top + j] * y;
            }
        if (m0 + c < p.d.hidden) ((T *)p.out)[t * p.stride_out + m0 + c] = dg_from_float<T>(sum);
    }
}

// ---- more pairs: an expert's together --------------------------------------------------------------------------------------
//
// A wavefront has 16 channels of `up` (gates and others) or 32 of `down`, a workgroup PAIRS of the expert's pairs at a time.  A wavefront's rows come into a ring of its own, the pairs' activations into one that
// all of the workgroup's read (64 tokens to 6 of 64, 4096 x 1024: up 50 to 55 us, 5.2 TB/s; down 34, 4.1; the matrix pipe busy 12 and 17 % of the cycles, vector instructions 31 and 25).  With fewer pairs than experts a workgroup's slot is a pair, whose expert it takes unless an earlier pair names it too, otherwise an expert.

template <bool UP, int WAVES, int PAIRS, int PLANES, int RING>
__global__ __launch_bounds__(64 * WAVES) void experts_kernel(DgExperts p, Rows rows, Work work)
{
    constexpr int COLUMNS = PAIRS / 16, LOADS_X = PAIRS * PLANES / (2 * WAVES), LOADS = 4 + LOADS_X, STAGE_W = 4096, STAGE_X = PAIRS * PLANES * 512, SCALES = 1024;
    static_assert(PAIRS * PLANES % (2 * WAVES) == 0 && PAIRS % 16 == 0, "whole loads");
    __shared__ __align__(1024) uint8_t room[RING * (WAVES * STAGE_W + STAGE_X) + WAVES * 2 * SCALES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t pairs = p.T * p.top, slot = blockIdx.y, blocks = ((UP ? p.d.hidden : p.d.inner) + 31) / 32;
    const bool by_pair = pairs < p.d.experts;
    const int32_t expert = by_pair ? __builtin_amdgcn_readfirstlane(p.ids[slot]) : slot;
    if ((uint32_t)expert >= (uint32_t)p.d.experts) return;
    uint8_t *const mine = room + wave * (RING * STAGE_W), *const shared = room + WAVES * RING * STAGE_W, *const scale_room = shared + RING * STAGE_X + wave * (2 * SCALES);
    // which pairs are its: every wavefront looks for itself; numbers `from` ... of them into `list` (its own place, before anything is loaded there)
    uint16_t *const list = (uint16_t *)mine;
    const auto find = [&](int32_t from) __attribute__((always_inline)) {
        int32_t n = 0;
        for (int32_t first = 0; first < pairs; first += 512) {
            int32_t ids[8];                                          // (asked for together: one after another each would be a wait)
#pragma unroll
            for (int i = 0; i < 8; ++i) ids[i] = first + 64 * i + lane < pairs ? p.ids[first + 64 * i + lane] : -1;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool is = ids[i] == expert;
                const uint64_t which = __ballot(is);
                if (!which) continue;
                if (by_pair && n == 0 && first + 64 * i + __builtin_ctzll(which) != slot) return 0;
                const int32_t number = n + __builtin_popcountll(which & ((1ull << lane) - 1)) - from;
                if (is && number >= 0 && number < PAIRS) list[number] = (uint16_t)(first + 64 * i + lane);
                n += __builtin_popcountll(which);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        return n;
    };
    const int32_t first_column = PAIRS * blockIdx.z, count = find(first_column);
    if (count <= first_column) return;
    const int32_t all = UP ? p.d.inner : p.d.hidden, each = UP ? 16 : 32, tiles = ((UP ? work.pitch_h : p.d.hidden) + WAVES * each - 1) / (WAVES * each), stages = (blocks + 7) / 8;
    // its rows of the tile that is being loaded
    Weights w[2];
    uint32_t offset[2][2];
    const auto begin = [&](int32_t tile) __attribute__((always_inline)) {
        const int32_t m = (tile * WAVES + wave) * each;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (UP)
                w[i] = weights_at(p.d.up + expert * p.d.up_expert, p.d.up_row, p.d.up_scales + expert * p.d.up_scales_expert, p.d.up_scales_row, min(m, all - 1) + (int64_t)i * all, all - m, blocks);
            else
                w[i] = weights_at(p.d.down + expert * p.d.down_expert, p.d.down_row, p.d.down_scales + expert * p.d.down_scales_expert, p.d.down_scales_row, min(m + 16 * i, all - 1),
                                  all - m - 16 * i, blocks);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) offset[i / 2][i % 2] = codes_offset(w[i / 2], i % 2);
    };
    const dg_v4i x = dg_buffer((const uint8_t *)rows.x, rows.bytes);
    const uint32_t lds = dg_lds_address(mine), x_lds = dg_lds_address(shared), scale_lds = dg_lds_address(scale_room);
    for (int32_t column = first_column; column < count; column += PAIRS * gridDim.z) {
        if (column != first_column) {
            __syncthreads();
            find(column);
        }
        const int32_t here = min(count - column, PAIRS);
        // load i of a wavefront's share of the activations: rows 2 q and 2 q + 1 of the planes behind one another, q = wave + WAVES i; place l of a row holds piece l ^ (row % 16)
        const auto piece = [&](int i) { return (lane & 31) ^ ((2 * (wave + WAVES * i) + (lane >> 5)) % 16); };
        int32_t pair[COLUMNS];
        uint32_t from[LOADS_X];
#pragma unroll
        for (int c = 0; c < COLUMNS; ++c) pair[c] = list[min(16 * c + r, here - 1)];
#pragma unroll
        for (int i = 0; i < LOADS_X; ++i) {
            const int row = (2 * (wave + WAVES * i) + (lane >> 5)) % PAIRS, plane = 2 * WAVES * i / PAIRS;
            const int32_t its = list[min(row, here - 1)];
            from[i] = row < here ? 2u * (uint32_t)(plane * rows.plane + (UP ? its / p.top : its) * rows.pitch) + 16 * piece(i) : DG_NOWHERE;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        // Loads: stage `ahead` of tile `loading`, and on into the next one's.  (Scales before codes: the waits below count a stage's other loads, and what was asked for before them is in with them.  Behind the last
        // tile there is nothing to load; the waits count on loads, so they go on, from nowhere: zeros.)
        int32_t loading = blockIdx.x, ahead = 0, to = 0, scale_to = 0;
        const auto fetch = [&]() __attribute__((always_inline)) {
            const int32_t b = 8 * ahead;
            if (ahead % 4 == 0) {
                // (this place's last scales are read: the fifth stage of a tile of five has the other place, and the next tile's first comes here two stages ahead)
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                const uint32_t at = scale_lds + scale_to * SCALES;
                const int row = (lane & 31) >> 1;
                const int32_t k = b + 16 * (lane & 1);
                if (lane < 32) dg_load16_to_lds(w[0].scales, row < w[0].have && k < blocks ? row * (uint32_t)w[0].scales_row + k : DG_NOWHERE, at);
                else dg_load16_to_lds(w[1].scales, row < w[1].have && k < blocks ? row * (uint32_t)w[1].scales_row + k : DG_NOWHERE, at);
                scale_to ^= 1;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) load_codes<PAIRS == 16>(w[i / 2], codes_past(i % 2, b, blocks) ? DG_NOWHERE : offset[i / 2][i % 2] + 16 * b, lds + to * STAGE_W + 1024 * i);
#pragma unroll
            for (int i = 0; i < LOADS_X; ++i) {
                const bool past = 32 * b + 8 * piece(i) >= rows.size;
                dg_load16_to_lds(x, past ? DG_NOWHERE : from[i] + 64 * b, x_lds + to * STAGE_X + 1024 * (wave + WAVES * i));
            }
            to = to + 1 == RING ? 0 : to + 1;
            if (++ahead == stages && loading + (int32_t)gridDim.x < tiles) {
                loading += gridDim.x;
                ahead = 0;
                begin(loading);
            }
        };
        // A stage's loads are waited for when its turn comes; the barrier after that says that every wavefront's are in, and that all are done with the stage before, whose place the
        // loads of RING - 1 ahead then take.
        begin(loading);
        for (int i = 0; i < RING - 1; ++i) fetch();
        int now = 0, scale_now = 1;
#pragma unroll 1
        for (int32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
            v4f acc[2][COLUMNS] = {};
#pragma unroll 1
            for (int32_t s = 0; s < stages; ++s) {
                dg_wait_for_loads<(RING - 2) * LOADS>();
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (nothing of the stage before is still being read)
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                // (its scales before the loads, which may bring others to their place)
                if (s % 4 == 0) scale_now ^= 1;
                uint32_t byte[2][2];
#pragma unroll
                for (int i = 0; i < 4; ++i) byte[i / 2][i % 2] = scale_room[scale_now * SCALES + 512 * (i / 2) + 32 * r + 8 * (s % 4) + 4 * (i % 2) + g];
                fetch();
                if (8 * s + 8 > blocks) {
                    // scales past the row: its codes are 0, and 0 by whatever lies there might be no number
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (8 * s + 4 * (i % 2) + g >= blocks) byte[i / 2][i % 2] = 127;
                }
                const uint8_t *stage = mine + now * STAGE_W, *const wk[2] = {stage, stage + 2048}, *xk[COLUMNS];
#pragma unroll
                for (int c = 0; c < COLUMNS; ++c) xk[c] = shared + now * STAGE_X + (16 * c + r) * 512;
                stage_products<2, COLUMNS, PLANES>(wk, byte, xk, PAIRS * 512, r, acc);
                now = now + 1 == RING ? 0 : now + 1;
            }
            const int32_t m = (tile * WAVES + wave) * each;
#pragma unroll
            for (int c = 0; c < COLUMNS; ++c) {
                if (16 * c + r >= here) continue;
                if (UP) {
                    if (m < work.pitch_h) store_h(p, work, pair[c], m + 4 * g, acc[0][c], acc[1][c]);
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        if (m + 16 * i + 4 * g < p.d.hidden) *(v4f *)(work.y + (int64_t)pair[c] * work.pitch_y + m + 16 * i + 4 * g) = acc[i][c];
                }
            }
        }
        dg_wait_for_loads<0>();
    }
}

// A token's choices together, in their order.
template <class T>
__global__ __launch_bounds__(256) void experts_join_kernel(DgExperts p, Work work)
{
    const int32_t m = (blockIdx.x * 256 + threadIdx.x) * 4, t = blockIdx.y, have = min(p.d.hidden - m, 4);
    if (have <= 0) return;
    v4f sum = {};
    constexpr int AT_ONCE = 8;                                       // (all asked for together: what an id that is no expert has in y is loaded and left)
    for (int32_t first = 0; first < p.top; first += AT_ONCE) {
        int32_t id[AT_ONCE];
        float weight[AT_ONCE];
        v4f y[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int32_t pair = t * p.top + min(first + j, p.top - 1);
            id[j] = first + j < p.top ? p.ids[pair] : -1;
            weight[j] = p.weights[pair];
            y[j] = *(const v4f *)(work.y + (int64_t)pair * work.pitch_y + m);
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
            if ((uint32_t)id[j] < (uint32_t)p.d.experts) sum += weight[j] * y[j];
    }
    T *out = (T *)p.out + t * p.stride_out + m;
    DgVec<T, 4> y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y.e[e] = dg_from_float<T>(sum[e]);
    if (have == 4) dg_store_vec<T, 4>(out, y);
    else
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < have) out[e] = y.e[e];
}

int64_t up_to(int64_t n, int64_t multiple) { return (n + multiple - 1) / multiple * multiple; }
// Tokens that are worked through together: their pairs have 16-bit numbers, and what they have of h lies within 2^31 bytes.
int64_t turn_of(int64_t T, int64_t top, int64_t inner) { return std::min({T, (int64_t)MOST_TOKENS, std::min<int64_t>(MOST_PAIRS, ((int64_t)1 << 28) / up_to(inner, 128)) / top}); }

struct Sizes {
    int64_t x, h, y, pitch_x, pitch_h, pitch_y;          // bytes; elements
};
Sizes sizes_of(int64_t T, int64_t top, int64_t hidden, int64_t inner)
{
    Sizes s = {0, 0, 0, up_to(hidden, 8), up_to(inner, 128), up_to(hidden, 4)};
    s.x = up_to(4 * T * s.pitch_x, 16);
    s.h = 4 * T * top * s.pitch_h;
    s.y = 4 * T * top * s.pitch_y;
    return s;
}

template <int PLANES>
void launch(const DgExperts &p, const Rows &x, const Work &work, dg_dtype type, hipStream_t stream)
{
    const int32_t pairs = p.T * p.top;
    const Rows h = {work.h, work.pitch_h, pairs * work.pitch_h, work.pitch_h, (uint32_t)(4 * pairs) * (uint32_t)work.pitch_h};
    // (us, each by itself and together, 2048 x 1024: 64 experts, 4 pairs 11.8, 20.2; 12 19.9, 21.7; 16 22.9, 22.1; 32 40, 28; 4096 x 4096, 4 experts, 4 pairs 30.7, 37.9; 8 48, 43)
    if (pairs <= std::min(FEW_PAIRS, p.d.experts)) {
        const auto both = [&](auto once) {                           // (a token's choices are different experts as a rule, several tokens' may be the same)
            constexpr bool ONCE = decltype(once)::value;
            experts_few_up_kernel<PLANES, ONCE><<<dim3(work.pitch_h / 16, pairs), 256, 0, stream>>>(p, x, work);
            if (type == DG_F16) experts_few_down_kernel<_Float16, ONCE><<<(p.d.hidden + 15) / 16, 512, 0, stream>>>(p, h);
            else experts_few_down_kernel<__bf16, ONCE><<<(p.d.hidden + 15) / 16, 512, 0, stream>>>(p, h);
        };
        if (p.T == 1) both(std::true_type());
        else both(std::false_type());
        return;
    }
    const uint32_t slots = std::min(pairs, p.d.experts);
    const auto grid = [&](int32_t channels, int each, int32_t size) {
        // (tiles behind one another in a workgroup, as many as leave two workgroups a compute unit, the nearest number; us by that and with one tile each: 64 tokens to 6 of 64 experts, 4096 x 1024, 91 and 96,
        // 256 to 8 221 and 231, 24 to 4 of 60, 2048 x 1408, 60 and 66; the next larger number instead: 9 to 4 of 64, 2048 x 1024, 40 for 30; with a stage of its own a tile would need a third place for its scales)
        const uint32_t tiles = (channels + each - 1) / each, room = dg_simd_count() / 2, behind = std::max(1u, (tiles * slots + room / 2) / room);
        return dim3(size <= 256 ? tiles : (tiles + behind - 1) / behind, slots);
    };
    // (us, 16 and 32 pairs at a time: 64 tokens to 6 of 64 experts, 4096 x 1024, 92 and 105; 128 tokens 144, 131; 64 to 2 of 8, 4096 x 4096, 91, 76: what an expert has of a batch varies, and a pass behind the first costs as much)
    // (16 columns leave a compute unit room for two workgroups; 64 tokens to 6 of 64 experts, 4096 x 1024: down with three stages, one workgroup, 59 us for 40, by eight wavefronts 43)
    if (pairs <= 8 * p.d.experts) {
        experts_kernel<true, 4, 16, PLANES, PLANES == 1 ? 3 : 2><<<grid(work.pitch_h, 64, p.d.hidden), 256, 0, stream>>>(p, x, work);
        experts_kernel<false, 4, 16, 2, 2><<<grid(p.d.hidden, 128, p.d.inner), 256, 0, stream>>>(p, h, work);
    } else {
        // (what an expert has is dealt out in 32s to as many workgroups as fit beside one another, to twice the mean: 256 tokens to 2 of 4, 2048 x 2048, 152 us without and 53, 123 to 6 of 8, 352 x 480, 65 and 25,
        // 256 to 2 of 8, 4096 x 4096, 185 and 160)
        const auto dealt = [&](dim3 g) {
            const uint32_t mean = (pairs + 32 * slots - 1) / (32 * slots), fit = dg_simd_count() / 4 / (g.x * g.y);
            g.z = std::max(1u, std::min(2 * mean, fit));
            return g;
        };
        experts_kernel<true, 8, 32, PLANES, PLANES == 1 ? 3 : 2><<<dealt(grid(work.pitch_h, 128, p.d.hidden)), 512, 0, stream>>>(p, x, work);
        experts_kernel<false, 8, 32, 2, 2><<<dealt(grid(p.d.hidden, 256, p.d.inner)), 512, 0, stream>>>(p, h, work);
    }
    const dim3 join((p.d.hidden + 1023) / 1024, p.T);
    if (type == DG_F16) experts_join_kernel<_Float16><<<join, 256, 0, stream>>>(p, work);
    else experts_join_kernel<__bf16><<<join, 256, 0, stream>>>(p, work);
}

}   // namespace

int64_t dg_experts_work_bytes(int64_t T, int64_t top, int64_t hidden, int64_t inner)
{
    const Sizes s = sizes_of(turn_of(T, top, inner), top, hidden, inner);
    return s.x + s.h + s.y;
}

dg_status dg_launch_experts(const DgExperts &all, dg_dtype type, hipStream_t stream)
{
    dg_in_turns(all.T, turn_of(all.T, all.top, all.d.inner), [&](int64_t t, int64_t count) {
        DgExperts p = all;
        p.x = (const uint8_t *)p.x + 2 * t * p.stride_x;
        p.out = (uint8_t *)p.out + 2 * t * p.stride_out;
        p.ids += t * p.top;
        p.weights += t * p.top;
        p.T = (int32_t)count;
        const Sizes s = sizes_of(count, p.top, p.d.hidden, p.d.inner);
        uint8_t *at = (uint8_t *)p.work;
        const Work work = {(__bf16 *)at, (__bf16 *)(at + s.x), (float *)(at + s.x + s.h), (int32_t)s.pitch_x, (int32_t)s.pitch_h, (int32_t)s.pitch_y};
        // bfloat16 rows of whole pieces of 8 that begin on words are taken as they are
        if (type == DG_BF16 && p.d.hidden % 8 == 0 && (uintptr_t)p.x % 4 == 0 && p.stride_x % 2 == 0 && count * p.stride_x < (int64_t)1 << 30) {
            const Rows x = {(const __bf16 *)p.x, (int32_t)p.stride_x, 0, p.d.hidden, (uint32_t)(2 * ((count - 1) * p.stride_x + p.d.hidden))};
            launch<1>(p, x, work, type, stream);
            return DG_OK;
        }
        const dim3 grid((uint32_t)((s.pitch_x + 2047) / 2048), (uint32_t)count);
        const int planes = type == DG_BF16 ? 1 : 2;
        const Rows x = {work.x, work.pitch_x, p.T * work.pitch_x, p.d.hidden, (uint32_t)(2 * planes * p.T) * (uint32_t)work.pitch_x};
        if (type == DG_BF16) {
            experts_rows_kernel<__bf16><<<grid, 256, 0, stream>>>(p, work);
            launch<1>(p, x, work, type, stream);
        } else {
            experts_rows_kernel<_Float16><<<grid, 256, 0, stream>>>(p, work);
            launch<2>(p, x, work, type, stream);
        }
        return DG_OK;
    });
    return dg_check_launch("dg_experts_mx4");
}
