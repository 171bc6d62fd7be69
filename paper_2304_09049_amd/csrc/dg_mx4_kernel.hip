// Rows quantised to microscaled 4-bit floating point and read back, and products of such rows.
#include <cstring>

#include "dg_mx4.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v2f __attribute__((ext_vector_type(2)));

// ---- quantising and reading back -----------------------------------------------------------------------------------------
//
// A lane has 8 elements of a block, four neighbouring lanes a block of 32; rows lie behind one another in the lanes' numbers, blocks not cut.  The largest magnitude is found on the
// numbers' bits, which order as they do and put infinities and NaN above all, and its exponent is the scale: no division, and the conversion takes the scale itself.  Bytes bound both ways:
// 16384 x 8192 from bfloat16 60 us (5.7 TB/s), back 48 to 53 (6.4 to 7); more than 8 elements a lane, or codes past the caches, which the next launch reads, were no faster (60 and 54, but 120 for 106 with
// reading back behind it).

constexpr int THREADS = 256;

struct MxRows {
    int64_t stride_x, stride_codes, stride_scales;       // elements, bytes, bytes
    int32_t K;
    uint32_t total;                                      // lanes' pieces
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

template <class T>
__global__ __launch_bounds__(THREADS) void quantize_mx4_kernel(const T *x, MxRows r, uint8_t *codes, uint8_t *scales)
{
    const uint32_t number = blockIdx.x * THREADS + threadIdx.x, at = min(number, r.total - 1), row = dg_fdiv(at, r.by_row), piece = at - row * r.by_row.d;
    const DgVec<T, 8> v = dg_eight<T>(x + row * r.stride_x, 8 * piece, r.K);
    float f[8];
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        f[j] = dg_to_float(v.e[j]);
        most = max(most, __float_as_uint(f[j]) & 0x7FFFFFFFu);
    }
    const uint32_t byte = scale_byte(most_of_four(most));
    if (number >= r.total) return;
    *(uint32_t *)(codes + row * r.stride_codes + 4 * piece) = codes_of(f, byte);
    if (piece % 4 == 0) scales[row * r.stride_scales + piece / 4] = (uint8_t)byte;
}

// A lane has 16 bytes of the output, so that a store instruction writes whole lines, and they bypass the caches: kept there they cost twice the time (16384 x 8192 to bfloat16 92 us, 48,
// and with a copy of the output behind it 205 and 167).
template <class T>
__global__ __launch_bounds__(THREADS) void dequantize_mx4_kernel(const uint8_t *codes, const uint8_t *scales, MxRows r, T *out)
{
    constexpr int COUNT = 16 / sizeof(T);
    const uint32_t at = blockIdx.x * THREADS + threadIdx.x, row = dg_fdiv(at, r.by_row), piece = at - row * r.by_row.d;
    if (at >= r.total) return;
    const uint8_t *from = codes + row * r.stride_codes + COUNT / 2 * piece;
    const uint32_t word = COUNT == 8 ? *(const uint32_t *)from : *(const uint16_t *)from, byte = scales[row * r.stride_scales + piece / (32 / COUNT)];
    const float s = dg_mx_scale(byte);
    const v2f f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 3)};
    DgVec<T, COUNT> v;
#pragma unroll
    for (int j = 0; j < COUNT; ++j) v.e[j] = dg_from_float<T>(byte == 255 ? s : f[j / 2][j % 2]);
    T *to = out + row * r.stride_x + COUNT * piece;
    const int32_t left = r.K - COUNT * (int32_t)piece;
    if (left >= COUNT) dg_store_past(to, v);
    else
#pragma unroll
        for (int j = 0; j < COUNT - 1; ++j)
            if (j < left) to[j] = v.e[j];
}

// f(the pieces of `per` elements of a launch, its first row): pieces' numbers are 31-bit, and a launch's rows as many as that allows.
template <class F>
void in_launches(int64_t N, int64_t K, int per, int64_t stride_x, int64_t stride_codes, int64_t stride_scales, F f)
{
    const int64_t pieces = (K + 31) / 32 * (32 / per);
    dg_in_turns(N, std::max<int64_t>(1, ((int64_t)1 << 30) / pieces), [&](int64_t n, int64_t rows) {
        const MxRows r = {stride_x, stride_codes, stride_scales, (int32_t)K, (uint32_t)(rows * pieces), dg_make_div((uint32_t)pieces)};
        f(r, n);
        return DG_OK;
    });
}

// ---- the product -----------------------------------------------------------------------------------------------------------
//
// A lane's operand is a block of 32, 16 bytes as they lie, and its scale a byte of a register.  But neighbouring lanes have different rows, and a compute unit's address unit takes 16 bytes each from 64
// places in some 100 cycles, neighbouring lanes on neighbouring bytes in 16 (operands straight from memory: 25 bytes/ns a compute unit, however many wavefronts).  So everything goes by way of
// LDS, by loads that write it themselves: eight lanes a row's 128 bytes, 256 positions.  Such a row's blocks lie exchanged, block c of row r at place c ^ (r / 2 % 8), so that the 16 lanes that an
// LDS read serves together find 16 different places.

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

// ---- few tokens ----
//
// v_mfma_scale_f32_16x16x128_f8f6f4: lane (r, g) holds block g of four of row r; sums come out with four neighbouring channels of one token in a lane.
// A workgroup computes 16 ROWS channels x 8 EIGHTS tokens.  Its wavefronts share K in chunks of 1024 positions and work alone, each with a ring of four stages of 256 positions in LDS, until
// their sums meet, in the wavefronts' order.
// X: a single token that is not quantised yet; a wavefront quantises what it multiplies of it, and no launch is needed for that.
// A launch and a chain of latencies bound it where weights are small (1 x 4096 x 4096 4.2 us, 16 x 4096 x 4096 4.7), their bytes where they are not (16 x 8192 x 8192 9.8 to 10.9 us, 3.5 TB/s; 16 x 4096 x 28672
// 16 us, 4 TB/s).  Weights past the caches: 4.7 -> 4.8, 5.8 -> 7.4 at 64 tokens.

template <class X>
constexpr int bytes_of = sizeof(X);
template <>
constexpr int bytes_of<void> = 0;

template <class T, class X, int WAVES, int ROWS, int EIGHTS>
__global__ __launch_bounds__(64 * WAVES) void gemm_mx4_few_kernel(DgGemmMx4 p, const X *x, int32_t K)
{
    constexpr bool QUANTIZE = bytes_of<X> != 0;
    constexpr int TOKENS = (EIGHTS + 1) / 2, LOADS_W = 2 * ROWS, LOADS = LOADS_W + (QUANTIZE ? 0 : EIGHTS), STAGE = LOADS * 1024, RING = 4;
    static_assert(ROWS <= 2 && EIGHTS <= 4, "a load of scales has 32 rows");
    // LDS: the ring; twice a chunk's scales of either operand; twice a chunk of the token, as it comes, and its codes and scales
    constexpr int SCALES = QUANTIZE ? 1024 : 2048, RAW = 1024 * bytes_of<X>, MINE = RING * STAGE + 2 * SCALES + 2 * RAW + (QUANTIZE ? 1024 : 0);
    static_assert(MINE >= ROWS * TOKENS * 1024, "the sums' place");
    __shared__ __align__(1024) uint8_t room[WAVES * MINE];
    // (a matrix instruction runs whatever the lanes' mask: what it stands under has to be a scalar branch)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t m0 = blockIdx.x * (16 * ROWS), n0 = blockIdx.y * (8 * EIGHTS), have_w = min(p.M - m0, 16 * ROWS), have_a = min(p.N - n0, 8 * EIGHTS);
    const int32_t scale_bytes = (p.blocks + 3) / 4 * 4;
    const dg_v4i buffer_w = dg_rows_buffer(p.W, m0, p.stride_w, have_w, 16 * p.blocks), buffer_ws = dg_rows_buffer(p.W_scales, m0, p.stride_ws, have_w, scale_bytes);
    dg_v4i buffer_a, buffer_as = buffer_ws;
    if constexpr (QUANTIZE) {
        buffer_a = dg_buffer((const uint8_t *)x, (uint32_t)(K * bytes_of<X> + 3) / 4 * 4);
    } else {
        buffer_a = dg_rows_buffer(p.A, n0, p.stride_a, have_a, 16 * p.blocks);
        buffer_as = dg_rows_buffer(p.A_scales, n0, p.stride_as, have_a, scale_bytes);
    }
    uint8_t *const mine = room + wave * MINE, *const scale_room = mine + RING * STAGE, *const raw = scale_room + 2 * SCALES, *const made = raw + 2 * RAW;
    const uint32_t lds = dg_lds_address(mine), scale_lds = lds + RING * STAGE, raw_lds = scale_lds + 2 * SCALES;

    // load i of a stage: row 8 i + lane / 8 of an operand
    uint32_t offset[LOADS], scale_offset[2];
    const int piece[2] = {(lane & 7) ^ (lane >> 4), (lane & 7) ^ (4 + (lane >> 4))};
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const bool weights = i < LOADS_W;
        const int row = 8 * (weights ? i : i - LOADS_W) + (lane >> 3);
        offset[i] = row < (weights ? have_w : have_a) ? row * (uint32_t)(weights ? p.stride_w : p.stride_a) + 16 * piece[i & 1] : DG_NOWHERE;
    }
    scale_offset[0] = (lane >> 1) < have_w ? (lane >> 1) * (uint32_t)p.stride_ws + 16 * (lane & 1) : DG_NOWHERE;
    scale_offset[1] = (lane >> 1) < have_a ? (lane >> 1) * (uint32_t)p.stride_as + 16 * (lane & 1) : DG_NOWHERE;
    // The wavefront's stage s: stage s % 4 of chunk wave + WAVES (s / 4) of the row.  (A chunk's scales and elements before its codes: the waits below count a stage's loads of codes, and what
    // was asked for before them is in with them.  Past the row there is nothing to load; the waits count on loads, so they go on, from nowhere: zeros.)
    const auto fetch = [&](int32_t s) __attribute__((always_inline)) {
        const int32_t chunk = wave + WAVES * (s / 4), b = 32 * chunk + 8 * (s % 4);
        if (s % 4 == 0) {
            const bool past = 32 * chunk + 16 * (lane & 1) >= scale_bytes;
            const uint32_t to = scale_lds + s / 4 % 2 * SCALES;
            dg_load16_to_lds(buffer_ws, past ? DG_NOWHERE : scale_offset[0] + 32 * chunk, to);
            if constexpr (!QUANTIZE) dg_load16_to_lds(buffer_as, past ? DG_NOWHERE : scale_offset[1] + 32 * chunk, to + 1024);
#pragma unroll
            for (int i = 0; i < bytes_of<X>; ++i)
                dg_load16_to_lds(buffer_a, 32 * chunk >= p.blocks ? DG_NOWHERE : (uint32_t)chunk * RAW + 1024 * i + 16 * lane, raw_lds + s / 4 % 2 * RAW + 1024 * i);
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            dg_load16_to_lds(i < LOADS_W ? buffer_w : buffer_a, b + piece[i & 1] < p.blocks ? offset[i] + 16 * b : DG_NOWHERE, lds + s % RING * STAGE + i * 1024);
    };
    const int32_t chunks = (p.blocks + 31) / 32, stages = chunks > wave ? (chunks - wave + WAVES - 1) / WAVES * 4 : 0;
    const uint32_t first = r * 128 + ((g ^ ((r >> 1) & 7)) << 4);
    v4f acc[ROWS][TOKENS] = {};
    if (stages) {
#pragma unroll
        for (int s = 0; s < RING; ++s) fetch(s);
    }
#pragma unroll 1
    for (int32_t s = 0; s < stages; ++s) {
        const int32_t chunk = wave + WAVES * (s / 4), b = 32 * chunk + 8 * (s % 4);
        dg_wait_for_loads<(RING - 1) * LOADS>();
        if constexpr (QUANTIZE) {
            if (s % 4 == 0) {
                // 16 elements a lane, two lanes a block
                typedef std::conditional_t<QUANTIZE, X, float> E;
                float f[2][8];
                uint32_t most = 0;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    DgVec<E, 8> e;
                    __builtin_memcpy(&e, raw + s / 4 % 2 * RAW + (16 * lane + 8 * i) * sizeof(E), sizeof(e));
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        f[i][j] = 1024 * chunk + 16 * lane + 8 * i + j < K ? dg_to_float(e.e[j]) : 0.0f;
                        most = max(most, __float_as_uint(f[i][j]) & 0x7FFFFFFFu);
                    }
                }
                most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xB1, 0xF, 0xF, false));         // quad_perm 1, 0, 3, 2
                const uint32_t byte = scale_byte(most);
                const uint2 codes = make_uint2(codes_of(f[0], byte), codes_of(f[1], byte));
                *(uint2 *)(made + 8 * lane) = codes;
                made[512 + lane / 2] = (uint8_t)byte;
                asm volatile("" ::: "memory");                       // (other lanes read them: to LDS a wavefront's order is that of its instructions)
            }
        }
        v4i w[ROWS][2], a[TOKENS][2];
        int ws[ROWS][2], as[TOKENS][2];
        const uint8_t *stage = mine + s % RING * STAGE, *scales = scale_room + s / 4 % 2 * SCALES + 8 * (s % 4) + g;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                w[i][h] = *(const v4i *)(stage + 2048 * i + (first ^ (64 * h)));
                ws[i][h] = scales[32 * (16 * i + r) + 4 * h];
            }
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
                if constexpr (QUANTIZE) {
                    a[t][h] = *(const v4i *)(made + 16 * (8 * (s % 4) + 4 * h + g));
                    as[t][h] = made[512 + 8 * (s % 4) + 4 * h + g];
                } else {
                    // (with eight tokens the others' rows are the next stage's, or scales: results that are not stored)
                    a[t][h] = *(const v4i *)(stage + 1024 * LOADS_W + 2048 * t + (first ^ (64 * h)));
                    as[t][h] = scales[1024 + 32 * (16 * t + r) + 4 * h];
                }
            }
        }
        if (b + 8 > p.blocks) {
            // scales past the row: its codes are 0, and 0 by whatever lies there might be no number
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool past = b + 4 * h + g >= p.blocks;
#pragma unroll
                for (int i = 0; i < ROWS; ++i) ws[i][h] = past ? 0 : ws[i][h];
#pragma unroll
                for (int t = 0; t < TOKENS; ++t) as[t][h] = past ? 0 : as[t][h];
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        fetch(s + RING);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < ROWS; ++i)
#pragma unroll
                for (int t = 0; t < TOKENS; ++t) {
                    const v8i X8 = {w[i][h][0], w[i][h][1], w[i][h][2], w[i][h][3], 0, 0, 0, 0}, Y8 = {a[t][h][0], a[t][h][1], a[t][h][2], a[t][h][3], 0, 0, 0, 0};
                    acc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(X8, Y8, acc[i][t], 4, 4, 0, ws[i][h], 0, as[t][h]);
                }
    }
    dg_wait_for_loads<0>();
    __syncthreads();
    v4f *const sums = (v4f *)room;                                   // [wavefront][row block][token block][lane]
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) sums[((wave * ROWS + i) * TOKENS + t) * 64 + lane] = acc[i][t];
    __syncthreads();
    // the blocks of 16 x 16 are dealt out to the wavefronts
#pragma unroll
    for (int block = 0; block < ROWS * TOKENS; ++block) {
        if (block % WAVES != wave) continue;
        v4f s = sums[block * 64 + lane];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) s += sums[(k * ROWS * TOKENS + block) * 64 + lane];
        const int32_t t = block % TOKENS, n = 16 * t + r;
        if (n < have_a) store4<T>(p, m0 + 16 * (block / TOKENS) + 4 * g, n0 + n, s);
    }
}

template <class T, class X, int WAVES, int ROWS, int EIGHTS>
void launch_few(const DgGemmMx4 &p, const X *x, int32_t K, hipStream_t stream)
{
    gemm_mx4_few_kernel<T, X, WAVES, ROWS, EIGHTS><<<dim3((p.M + 16 * ROWS - 1) / (16 * ROWS), (p.N + 8 * EIGHTS - 1) / (8 * EIGHTS)), 64 * WAVES, 0, stream>>>(p, x, K);
}

// A single token, quantised before or here: 16 channels a workgroup by four wavefronts, or 32 by two where that leaves more than one and a half workgroups of 16 a compute unit.  One rule for both, so that a token's sums
// have one order whichever call makes them.  (us, 16 and 32, quantised here: 5120 x 4096 4.7 and 5.5, 6144 x 4096 5.4 and 5.6, 6144 x 8192 8.6 and 7.9, 7168 x 8192 9.5 and 8.4, 16384 x 4096 9.8 and 8.3; 4096 x 14336 8.4 and 11.5, 6144 x 14336
// 10.8 and 11.6; quantised before: 5120 x 4096 4.5 and 4.8, 6144 x 4096 5.3 and 4.8, 6144 x 8192 8.1 and 7.3.  Tiles of 128 x 64 take 11.8 for 12.9 at 28672 x 4096, and 30 for 28 at 28672 x 8192.)
bool many_channels(const DgGemmMx4 &p) { return p.M >= 6 * dg_simd_count(); }

// ---- many tokens: tiles --------------------------------------------------------------------------------------------------
//
// KS groups of WM x WN wavefronts compute 32 WM TM channels x 32 WN TN tokens, TM x TN blocks of 32 x 32 a wavefront; a group takes 256 positions of K, 128 bytes of a row, of a
// round's 256 KS, and the groups' sums meet in LDS at the end, in the groups' order.  The rounds are a ring in LDS: the next ones' loads, which write LDS themselves, are in
// flight while one is multiplied.  A row's 128 bytes lie as eight blocks of 16, block c of row r at place c ^ (r / 2 % 8), so that the 16 lanes that an LDS read serves together find
// 16 different ones.  v_mfma_scale_f32_32x32x64_f8f6f4: lane (r, g) holds block g of two of row r, and names the byte of a register that is its scale: the four steps' are the four bytes.
// Scales come 16 bytes of a row at a time, 512 positions, by loads of 64 rows.  The results leave by way of LDS in whole lines and past the caches (1024 x 4096 x 4096 19.1 us kept there, 17.8;
// 1024 x 2048 x 8192 20.1, 17.1).  Start, rounds and end bound it where tiles are few (333 x 2000 x 1537 5.8 us), the address units' loads and the waits at a round's barrier in between: 1024 x 4096 x 4096
// 1.9 POP/s, the matrix pipe busy 15 % of the cycles.

struct TileArgs {
    DgGemmMx4 p;
    int32_t tiles_m, tiles_n;
    DgFastDiv by_group, by_rest;         // tile order: groups of GROUP rows of tiles
    int32_t rest;                        // rows of the last group
};
constexpr int GROUP = 4;

// Where tile `number` lies.  Neighbouring workgroups go to different dies (eight): each die takes a run of tiles of its own, and walks it in groups of GROUP rows
// of tiles, so that what it reads twice is in its own cache.
template <int BM, int BN>
__device__ __forceinline__ void place_of(const TileArgs &args, uint32_t number, int32_t &m0, int32_t &n0)
{
    const uint32_t tiles = (uint32_t)args.tiles_m * args.tiles_n, die = number & 7, in_die = number >> 3;
    const uint32_t tile = die * (tiles >> 3) + min(die, tiles & 7) + in_die;
    const uint32_t group = dg_fdiv(tile, args.by_group), left = tile - group * (GROUP * args.tiles_n);
    const bool last = (int32_t)(group * GROUP) + GROUP > args.tiles_m;
    const uint32_t column = last ? dg_fdiv(left, args.by_rest) : left / GROUP;
    m0 = (int32_t)(group * GROUP + left - column * (last ? args.rest : GROUP)) * BM;
    n0 = (int32_t)column * BN;
}

template <int STEP>
__device__ __forceinline__ v16f multiply(const v4i &w, const v4i &a, const v16f &c, int ws, int as)
{
    const v8i x = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, y = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, STEP, ws, STEP, as);
}

template <class T, int WM, int WN, int TM, int TN, int KS, int RING>
__global__ __launch_bounds__(64 * WM * WN * KS) void gemm_mx4_tile_kernel(TileArgs args)
{
    constexpr int WAVES = WM * WN, BM = 32 * WM * TM, BN = 32 * WN * TN, STAGE = (BM + BN) * 128;
    constexpr int LOADS_M = BM / (8 * WAVES), LOADS = (BM + BN) / (8 * WAVES);       // loads of 8 rows a wavefront makes of its group's stage
    static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && WAVES % 2 == 0, "whole loads, and the same places in each");
    // Scales: what one load brings of 64 rows, the weights' first; CHUNKS of 512 positions in a round, or (KS = 1) one in two rounds.
    constexpr int SCALES_M = (BM + 63) / 64, SCALES_N = (BN + 63) / 64, CHUNK = (SCALES_M + SCALES_N) * 1024, CHUNKS = KS > 1 ? KS / 2 : 1;
    constexpr int CHUNK_RING = KS > 1 ? RING : RING <= 3 ? 2 : 4, SCALE_LOADS = (SCALES_M + SCALES_N) * CHUNKS;
    constexpr int RESULTS = WAVES * 32 * (32 * TM + 4) * 4, ROOM = RING * STAGE * KS > RESULTS ? RING * STAGE * KS : RESULTS;
    static_assert(ROOM + CHUNK * CHUNKS * CHUNK_RING <= 160 * 1024, "a compute unit's LDS");
    __shared__ __align__(1024) uint8_t room[ROOM];
    __shared__ __align__(1024) uint8_t scale_room[CHUNK * CHUNKS * CHUNK_RING];
    const DgGemmMx4 &p = args.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % WAVES);
    const int share = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) / WAVES), of_all = wave + WAVES * share;
    uint8_t (*const stages)[STAGE] = (uint8_t(*)[STAGE])room + share * RING;          // (each group has a ring of its own)

    int32_t m0, n0;
    place_of<BM, BN>(args, blockIdx.x, m0, n0);

    // what this lane loads: block (lane % 8) ^ ... of row 8 q + lane / 8
    const int piece = (lane & 7) ^ ((((wave & 1) << 2) + (lane >> 4)) & 7);
    const int32_t have_w = min(p.M - m0, BM), have_a = min(p.N - n0, BN);
    uint32_t offset[LOADS];
    const auto row_of = [&](int i) { return (wave + WAVES * (i < LOADS_M ? i : i - LOADS_M)) * 8 + (lane >> 3); };
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const uint32_t stride = (uint32_t)(i < LOADS_M ? p.stride_w : p.stride_a);
        offset[i] = row_of(i) < (i < LOADS_M ? have_w : have_a) ? row_of(i) * stride + 16 * piece : DG_NOWHERE;
    }
    const int32_t scale_bytes = (p.blocks + 3) / 4 * 4;
    const dg_v4i buffer_w = dg_rows_buffer(p.W, m0, p.stride_w, have_w, 16 * p.blocks), buffer_a = dg_rows_buffer(p.A, n0, p.stride_a, have_a, 16 * p.blocks);
    const dg_v4i buffer_ws = dg_rows_buffer(p.W_scales, m0, p.stride_ws, have_w, scale_bytes), buffer_as = dg_rows_buffer(p.A_scales, n0, p.stride_as, have_a, scale_bytes);
    const uint32_t lds = dg_lds_address(room) + share * (RING * STAGE) + 1024 * wave, scale_lds = dg_lds_address(scale_room);

    const auto fetch = [&](int32_t round, int to) {
        // (the scales before the codes: the waits below count a round's loads of codes, and what was asked for before them is in with them)
        if (KS > 1 || round % 2 == 0) {
            const int32_t chunk = KS > 1 ? round * CHUNKS : round / 2, ring = KS > 1 ? to : chunk % CHUNK_RING;
#pragma unroll
            for (int i = 0; i < (SCALE_LOADS + WAVES * KS - 1) / (WAVES * KS); ++i) {
                const int load = of_all + i * (WAVES * KS), c = load / (SCALES_M + SCALES_N), block = load % (SCALES_M + SCALES_N);
                if (load >= SCALE_LOADS) break;
                const bool weights = block < SCALES_M;
                const int row = 64 * (weights ? block : block - SCALES_M) + lane;
                const int32_t k = 16 * (chunk + c);
                const uint32_t at = row < (weights ? have_w : have_a) && k < scale_bytes ? row * (uint32_t)(weights ? p.stride_ws : p.stride_as) + k : DG_NOWHERE;
                dg_load16_to_lds(weights ? buffer_ws : buffer_as, at, scale_lds + ring * (CHUNK * CHUNKS) + load * 1024);
            }
        }
        const int32_t b = 8 * (round * KS + share);
        const bool past = b + piece >= p.blocks;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t at = past ? DG_NOWHERE : offset[i] + 16 * b;
            dg_load16_to_lds(i < LOADS_M ? buffer_w : buffer_a, at, lds + to * STAGE + i * (1024 * WAVES));
        }
    };
    const int r = lane & 31, g = lane >> 5, wm = wave % WM, wn = wave / WM;
    const uint32_t first = r * 128 + ((g ^ ((r >> 1) & 7)) << 4);
    v16f acc[TM][TN] = {};
    // 64 positions at a time; the operands of the next ones are read before these are multiplied
    v4i wk[2][TM], ak[2][TN];
    int ws[TM], as[TN];
    const auto read = [&](int now, int s) {
        const uint8_t *w = stages[now] + wm * (TM * 4096) + (first ^ (s * 32)), *a = stages[now] + BM * 128 + wn * (TN * 4096) + (first ^ (s * 32));
#pragma unroll
        for (int i = 0; i < TM; ++i) wk[s & 1][i] = *(const v4i *)(w + i * 4096);
#pragma unroll
        for (int j = 0; j < TN; ++j) ak[s & 1][j] = *(const v4i *)(a + j * 4096);
    };
    // a lane's four of a row's eight scales; those past the row are 0 (its codes are, and 0 by whatever lies there might be no number)
    const auto read_scales = [&](int32_t round, int now) {
        const int32_t ring = KS > 1 ? now : (round / 2) % CHUNK_RING, have = p.blocks - 8 * (round * KS + share);
        const uint8_t *at = scale_room + ring * (CHUNK * CHUNKS) + (share / 2) * CHUNK + 8 * (KS > 1 ? share & 1 : round & 1) + 16 * r;
        const uint32_t which = g ? 0x07050301u : 0x06040200u;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const uint2 s = *(const uint2 *)(at + 512 * (wm * TM + i));
            ws[i] = (int)__builtin_amdgcn_perm(s.y, s.x, which);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const uint2 s = *(const uint2 *)(at + 1024 * SCALES_M + 512 * (wn * TN + j));
            as[j] = (int)__builtin_amdgcn_perm(s.y, s.x, which);
        }
        if (have < 8) {
            const int count = have > g ? (have - g + 1) / 2 : 0;                      // blocks g, g + 2 ... below `have`
            const int mask = count >= 4 ? -1 : (int)((1u << (8 * count)) - 1u);
#pragma unroll
            for (int i = 0; i < TM; ++i) ws[i] &= mask;
#pragma unroll
            for (int j = 0; j < TN; ++j) as[j] &= mask;
        }
    };
    const auto step = [&](int now, auto s_) {
        constexpr int s = decltype(s_)::value;
        if (s < 3) read(now, s + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = multiply<s>(wk[s & 1][i], ak[s & 1][j], acc[i][j], ws[i], as[j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // A round's loads are waited for when its turn comes; the barrier after that says that every wavefront's are in, and that all are done with
    // the round before, whose place the loads of RING - 1 ahead then take.  (Past the end of K there is nothing to load; the waits count on
    // loads, so they go on, from outside the buffers: zeros, which nothing reads.)
    const int32_t rounds = (p.blocks + 8 * KS - 1) / (8 * KS);
    for (int i = 0; i < RING - 1; ++i) fetch(i, i);
    int now = 0, to = RING - 1;
    for (int32_t round = 0; round < rounds; ++round) {
        dg_wait_for_loads<(RING - 2) * LOADS>();
        __syncthreads();
        read_scales(round, now);
        read(now, 0);
        fetch(round + RING - 1, to);
        step(now, std::integral_constant<int, 0>{});
        step(now, std::integral_constant<int, 1>{});
        step(now, std::integral_constant<int, 2>{});
        step(now, std::integral_constant<int, 3>{});
        now = now + 1 == RING ? 0 : now + 1;
        to = to + 1 == RING ? 0 : to + 1;
    }
    dg_wait_for_loads<0>();
    // The results go by way of LDS, a wavefront's 32 tokens at a time: rows of channels leave side by side.
    constexpr int PITCH = 32 * TM + 4, LANES = 8 * TM, ROWS = 64 / LANES;
    __syncthreads();
    float *mine = (float *)room + wave * (32 * PITCH);
    if constexpr (KS > 1) {
        // the other groups' sums, one group after another
        static_assert(TM * TN * 4096 * WAVES <= ROOM, "a group's sums fit");
        float4 *const sums = (float4 *)room + wave * (TM * TN * 256) + lane;
#pragma unroll 1
        for (int from = 1; from < KS; ++from) {
            if (share == from)
#pragma unroll
                for (int i = 0; i < TM * TN; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const v16f &c = acc[i / TN][i % TN];
                        sums[(4 * i + e) * 64] = make_float4(c[4 * e], c[4 * e + 1], c[4 * e + 2], c[4 * e + 3]);
                    }
            __syncthreads();
            if (share == 0)
#pragma unroll
                for (int i = 0; i < TM * TN; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float4 x = sums[(4 * i + e) * 64];
                        v16f &c = acc[i / TN][i % TN];
                        c[4 * e] += x.x;
                        c[4 * e + 1] += x.y;
                        c[4 * e + 2] += x.z;
                        c[4 * e + 3] += x.w;
                    }
            __syncthreads();
        }
        if (share) return;
    }
    const int32_t m = m0 + wm * (32 * TM) + 4 * (lane % LANES), have = min(p.M - m, 4);
    float bias[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) bias[e] = p.bias && e < have ? p.bias[m + e] : 0.0f;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *(v4f *)(mine + r * PITCH + 32 * i + 8 * e + 4 * g) = (v4f){acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
        const int32_t first_n = n0 + (wn * TN + j) * 32, end = min(p.N - first_n, 32);
#pragma unroll 1
        for (int t = lane / LANES; t < end; t += ROWS) {
            const v4f sum = *(const v4f *)(mine + t * PITCH + 4 * (lane % LANES));
            T *out = (T *)p.out + (int64_t)(first_n + t) * p.stride_out + m;
            DgVec<T, 4> y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y.e[e] = dg_from_float<T>(p.bias ? sum[e] + bias[e] : sum[e]);
            if (have >= 4) dg_store_past(out, y);
            else
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < have) out[e] = y.e[e];
        }
    }
}

// ---- many tokens: wide tiles, one behind another ---------------------------------------------------------------------------
//
// WM x WN wavefronts of TM x TN blocks of 32 x 32, stages of 256 positions as above, two of them: one is multiplied in four steps, the other on its way.
// A compute unit's address unit takes a load's 64 lanes in 16 cycles and more, and a wavefront that asks for more waits with its products: the loads of a stage are spread between the
// products of two steps.  The last step has its operands in registers: before it the next stage's loads are waited for, and after the barrier, which says that every wavefront's are in and that
// all have read this stage, the next one's first operands are read and this place is loaded anew.
// Such tiles leave room for one workgroup a compute unit, which would have nothing to multiply while a tile's results leave and the next one's first stages arrive: a workgroup takes tile
// after tile, and its loads run on into the next tile's stages.
// 8192 x 8192 x 8192 to bfloat16 274 to 289 us (3.8 to 4.0 POP/s; results kept in the caches 311): the matrix pipe is busy for 143 us of it, at a clock that falls to 1.84 GHz, and a third of the wavefronts' cycles are waits: two places,
// and all loads waited for at each stage.  Without the loads the loop took 206 to 235, the loads alone 137 to 195.

template <int N>
using Int = std::integral_constant<int, N>;

template <class T, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN) void gemm_mx4_stream_kernel(TileArgs args)
{
    constexpr int WAVES = WM * WN, BM = 32 * WM * TM, BN = 32 * WN * TN, STAGE = (BM + BN) * 128;
    constexpr int LOADS_M = BM / (8 * WAVES), LOADS = (BM + BN) / (8 * WAVES);                               // of 8 rows
    constexpr int SCALES_M = BM / 64, SCALE_LOADS = (BM + BN) / 64, CHUNK = SCALE_LOADS * 1024;              // of 64 rows, 512 positions
    static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && WAVES % 2 == 0 && BM % 64 == 0 && BN % 64 == 0 && TM % 2 == 0, "whole loads, whole lines of results");
    // results leave 16 tokens at a time, a line of 128 bytes of each; a store is eight of them
    constexpr int LINE = 128 / sizeof(T), STORES = TM * TN * (int)sizeof(T);
    __shared__ __align__(1024) uint8_t room[2 * STAGE];
    __shared__ __align__(1024) uint8_t scale_room[2 * CHUNK];
    __shared__ __align__(1024) uint8_t way_out[WAVES][2048];
    const DgGemmMx4 &p = args.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5, wm = wave % WM, wn = wave / WM;
    const uint32_t tiles = (uint32_t)args.tiles_m * args.tiles_n, grid = gridDim.x;
    const int32_t stages = (p.blocks + 7) / 8, scale_bytes = (p.blocks + 3) / 4 * 4;

    // ---- loads: of tile `loading`, stage `ahead`, into place `to` ----
    const int piece = (lane & 7) ^ ((((wave & 1) << 2) + (lane >> 4)) & 7);
    const uint32_t lds = dg_lds_address(room) + 1024 * wave, scale_lds = dg_lds_address(scale_room);
    uint32_t loading = blockIdx.x, offset[LOADS];
    int32_t ahead = 0, load_w, load_a, to = 0, scale_to = 0;
    dg_v4i buffer_w, buffer_a, buffer_ws, buffer_as;
    const auto begin_loading = [&] {
        int32_t m, n;
        place_of<BM, BN>(args, loading, m, n);
        load_w = min(p.M - m, BM);
        load_a = min(p.N - n, BN);
        buffer_w = dg_rows_buffer(p.W, m, p.stride_w, load_w, 16 * p.blocks);
        buffer_a = dg_rows_buffer(p.A, n, p.stride_a, load_a, 16 * p.blocks);
        buffer_ws = dg_rows_buffer(p.W_scales, m, p.stride_ws, load_w, scale_bytes);
        buffer_as = dg_rows_buffer(p.A_scales, n, p.stride_as, load_a, scale_bytes);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const bool weights = i < LOADS_M;
            const int row = (wave + WAVES * (weights ? i : i - LOADS_M)) * 8 + (lane >> 3);
            offset[i] = row < (weights ? load_w : load_a) ? row * (uint32_t)(weights ? p.stride_w : p.stride_a) + 16 * piece : DG_NOWHERE;
        }
    };
    const auto load_scales = [&] {
        if (ahead % 2 != 0) return;
#pragma unroll
        for (int i = 0; i < (SCALE_LOADS + WAVES - 1) / WAVES; ++i) {
            const int load = wave + i * WAVES;
            if (load >= SCALE_LOADS) break;
            const bool weights = load < SCALES_M;
            const int row = 64 * (weights ? load : load - SCALES_M) + lane;
            const uint32_t at = row < (weights ? load_w : load_a) && 8 * ahead < scale_bytes ? row * (uint32_t)(weights ? p.stride_ws : p.stride_as) + 8 * ahead : DG_NOWHERE;
            dg_load16_to_lds(weights ? buffer_ws : buffer_as, at, scale_lds + scale_to * CHUNK + load * 1024);
        }
        scale_to ^= 1;
    };
    const auto load_codes = [&](int i) {
        const uint32_t at = 8 * ahead + piece >= p.blocks ? DG_NOWHERE : offset[i] + 128 * ahead;
        dg_load16_to_lds(i < LOADS_M ? buffer_w : buffer_a, at, lds + to * STAGE + i * (1024 * WAVES));
    };
    const auto next_loads = [&] {
        to ^= 1;
        if (++ahead == stages && loading + grid < tiles) {      // (behind the last tile there is nothing to load: from nowhere come zeros, which nothing reads)
            loading += grid;
            ahead = 0;
            begin_loading();
        }
    };

    // ---- operands ----
    const uint32_t first = r * 128 + ((g ^ ((r >> 1) & 7)) << 4);
    v16f acc[TM][TN] = {};
    v4i wk[2][TM], ak[2][TN];
    uint2 ws_next[TM], as_next[TN];                                  // (a stage's scales are read before the stage before is done with its own)
    int ws[TM], as[TN];
    const auto read = [&](int now, int s) {
        const uint8_t *w = room + now * STAGE + wm * (TM * 4096) + (first ^ (s * 32)), *a = room + now * STAGE + BM * 128 + wn * (TN * 4096) + (first ^ (s * 32));
#pragma unroll
        for (int i = 0; i < TM; ++i) wk[s & 1][i] = *(const v4i *)(w + i * 4096);
#pragma unroll
        for (int j = 0; j < TN; ++j) ak[s & 1][j] = *(const v4i *)(a + j * 4096);
    };
    const auto read_scales = [&](int32_t t, int ring) {
        const uint8_t *at = scale_room + ring * CHUNK + 8 * (t % 2) + 16 * r;
#pragma unroll
        for (int i = 0; i < TM; ++i) ws_next[i] = *(const uint2 *)(at + 512 * (wm * TM + i));
#pragma unroll
        for (int j = 0; j < TN; ++j) as_next[j] = *(const uint2 *)(at + 16 * BM + 512 * (wn * TN + j));
    };
    const auto take_scales = [&](int32_t t) {
        const uint32_t which = g ? 0x07050301u : 0x06040200u;
        const int32_t have = p.blocks - 8 * t, count = have > g ? (have - g + 1) / 2 : 0;                   // blocks g, g + 2 ... below `have`
        const int mask = count >= 4 ? -1 : (int)((1u << (8 * count)) - 1u);
#pragma unroll
        for (int i = 0; i < TM; ++i) ws[i] = (int)__builtin_amdgcn_perm(ws_next[i].y, ws_next[i].x, which) & mask;
#pragma unroll
        for (int j = 0; j < TN; ++j) as[j] = (int)__builtin_amdgcn_perm(as_next[j].y, as_next[j].x, which) & mask;
    };
    // Step s.  Between the products of step 3 half of a stage's loads, and with `more` the others as well; between those of step 0, with `more`, the others.  (Products know no order but
    // that of their operands: without the asm line all of a stage's are put behind its barrier.)
    const auto step = [&](auto s_, bool more) __attribute__((always_inline)) {
        constexpr int s = decltype(s_)::value, HALF = LOADS / 2;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TM * TN; ++i) {
            acc[i / TN][i % TN] = multiply<s>(wk[s & 1][i / TN], ak[s & 1][i % TN], acc[i / TN][i % TN], ws[i / TN], as[i % TN]);
            asm volatile("" : "+v"(acc[i / TN][i % TN]));
            if constexpr (s == 3) {
#pragma unroll
                for (int l = i * HALF / (TM * TN); l < (i + 1) * HALF / (TM * TN); ++l) load_codes(l);
            }
            if constexpr (s == 0 || s == 3) {
                if (more)
#pragma unroll
                    for (int l = i * (LOADS - HALF) / (TM * TN); l < (i + 1) * (LOADS - HALF) / (TM * TN); ++l) load_codes(HALF + l);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    begin_loading();
#pragma unroll 1
    for (int t = 0; t < 2; ++t) {
        load_scales();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load_codes(i);
        if (t == 0) next_loads();
    }
    dg_wait_for_loads<LOADS>();
    __syncthreads();
    int now = 0, scales_now = 0;
    bool asked = true, stored = false;                               // the stage behind this has been asked for whole; stores of the last tile are under way
    read_scales(0, 0);
    read(0, 0);
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += grid) {
#pragma unroll 1
        for (int32_t t = 0; t < stages; ++t) {
            const bool over = t + 1 == stages;
            take_scales(t);
            read(now, 1);
            step(Int<0>{}, !asked);
            read(now, 2);
            step(Int<1>{}, false);
            read(now, 3);
            step(Int<2>{}, false);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (stored) dg_wait_for_loads<STORES>();                 // (the stage was asked for before they were)
            else dg_wait_for_loads<0>();
            stored = false;
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            next_loads();
            if (over || t % 2 == 1) scales_now ^= 1;
            read_scales(over ? 0 : t + 1, scales_now);
            read(now ^ 1, 0);
            __builtin_amdgcn_sched_barrier(0);
            load_scales();
            asked = over;
            step(Int<3>{}, over);
            now ^= 1;
        }
        int32_t m0, n0;
        place_of<BM, BN>(args, tile, m0, n0);
        if (p.bias) {
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                float bias[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) bias[e] = p.bias[min(m0 + 32 * (TM * wm + i) + 8 * (e / 4) + 4 * g + e % 4, p.M - 1)];
#pragma unroll
                for (int e = 0; e < 16; ++e)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j][e] += bias[e];
            }
        }
        uint8_t *const mine = way_out[wave];
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int c = 0; c < 32 * TM / LINE; ++c) {               // lines of channels
                constexpr int BLOCKS = LINE / 32;                    // of 32 channels in one
                const int32_t m = m0 + 32 * TM * wm + LINE * c;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (r / 16 == h) {
#pragma unroll
                        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const v16f &sum = acc[BLOCKS * c + b][j];
                                const int32_t at = 32 * b + 8 * e + 4 * g;
                                DgVec<T, 4> y;
#pragma unroll
                                for (int k = 0; k < 4; ++k) y.e[k] = dg_from_float<T>(sum[4 * e + k]);
                                const uint32_t byte = at * sizeof(T), row = r % 16;
                                __builtin_memcpy(mine + row * 128 + ((byte / 16 ^ (row / 2 & 7)) * 16 + byte % 16), &y, sizeof(y));
                            }
                    }
                    asm volatile("" ::: "memory");                   // (what other lanes of the wavefront wrote: to LDS their order is that of the instructions)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        constexpr int COUNT = 16 / sizeof(T);
                        const uint32_t row = 8 * q + lane / 8;
                        DgVec<T, COUNT> y;
                        __builtin_memcpy(&y, mine + row * 128 + (((lane & 7) ^ (row / 2 & 7)) * 16), 16);
                        const int32_t n = n0 + 32 * (TN * wn + j) + 16 * h + row, channel = m + COUNT * (lane & 7);
                        T *out = (T *)p.out + (int64_t)n * p.stride_out + channel;
                        if (n < p.N && channel + COUNT <= p.M) {
                            dg_store_past(out, y);
                        } else if (n < p.N) {
#pragma unroll
                            for (int e = 0; e < COUNT - 1; ++e)
                                if (channel + e < p.M) out[e] = y.e[e];
                        }
                    }
                    asm volatile("" ::: "memory");
                }
            }
        stored = m0 + BM <= p.M && n0 + BN <= p.N;
#pragma unroll
        for (int i = 0; i < TM * TN; ++i) acc[i / TN][i % TN] = v16f{};
    }
    dg_wait_for_loads<0>();
}

TileArgs tiles_of(const DgGemmMx4 &p, int32_t bm, int32_t bn)
{
    TileArgs a = {p, (p.M + bm - 1) / bm, (p.N + bn - 1) / bn, {}, {}, 0};
    a.by_group = dg_make_div((uint32_t)GROUP * a.tiles_n);
    a.rest = a.tiles_m % GROUP ? a.tiles_m % GROUP : GROUP;
    a.by_rest = dg_make_div((uint32_t)a.rest);
    return a;
}

template <class T, int WM, int WN, int TM, int TN, int KS, int RING>
void launch_tiles(const DgGemmMx4 &p, hipStream_t stream)
{
    const TileArgs a = tiles_of(p, 32 * WM * TM, 32 * WN * TN);
    gemm_mx4_tile_kernel<T, WM, WN, TM, TN, KS, RING><<<(uint32_t)a.tiles_m * a.tiles_n, 64 * WM * WN * KS, 0, stream>>>(a);
}

template <class T, int WM, int WN, int TM, int TN>
void launch_stream(const DgGemmMx4 &p, hipStream_t stream)
{
    const TileArgs a = tiles_of(p, 32 * WM * TM, 32 * WN * TN);
    const uint32_t tiles = (uint32_t)a.tiles_m * a.tiles_n, units = (uint32_t)dg_simd_count() / 4;
    // (tiles are places of eight dies; and with a stage of its own a tile would need a third place for its scales)
    gemm_mx4_stream_kernel<T, WM, WN, TM, TN><<<p.blocks > 8 && units % 8 == 0 ? std::min(tiles, units) : tiles, 64 * WM * WN, 0, stream>>>(a);
}

enum class Form { Few16x16, Few16x32, Few32x16, Few32x32, Tile32x64, Tile64x64, Tile128x64, Tile128x128, Tile256x128, Tile256x256 };

// The form (channels x tokens a workgroup) whose rounds over the compute units cost least (a single token's: many_channels).  `cost`: of a round with a workgroup on each; `both`: with two, where two fit.
// A round by form, us for K = 2048 and 8192, launch included: 16x16 3.6 (two 4.3), 5.3 (7.4); 16x32 4.2, 6.0; 32x16 4.2 (4.8), 6.9 (7.8); 32x32 4.9 (5.9), 8.3 (10.1); 32x64 5.7, 9.3 (13, where the weights come from
// memory); 64x64 6.0, 11 (16); 128x64 7.5, 16 (22); 128x128 10, 27; 256x128 16, 43; 256x256 20, 57.  Of 239 products drawn (2 to
// 4096 tokens, weights from memory) this is within 3 % of the fastest form on 209; the farthest from it: 94 x 288 x 4112 tokens, positions, channels 1.19 times its time, 4 x 1216 x 18816 1.16, 498 x 384 x 784 1.15.
Form form_of(const DgGemmMx4 &p)
{
    static const struct {
        Form form;
        int32_t m, n, cost, both;
        const char *name;
    } forms[] = {{Form::Few16x16, 16, 16, 13, 21, "16x16"}, {Form::Few16x32, 16, 32, 16, 0, "16x32"}, {Form::Few32x16, 32, 16, 19, 22, "32x16"}, {Form::Few32x32, 32, 32, 25, 31, "32x32"},
                 {Form::Tile32x64, 32, 64, 28, 0, "32x64"}, {Form::Tile64x64, 64, 64, 33, 0, "64x64"}, {Form::Tile128x64, 128, 64, 43, 0, "128x64"},
                 {Form::Tile128x128, 128, 128, 57, 0, "128x128"}, {Form::Tile256x128, 256, 128, 92, 0, "256x128"}, {Form::Tile256x256, 256, 256, 120, 0, "256x256"}};
    const char *forced = dg_override("DG_GEMM_MX4_TILE");
    if (!forced && p.N == 1) return many_channels(p) ? Form::Few32x16 : Form::Few16x16;
    const int64_t units = dg_simd_count() / 4;
    Form best = Form::Few16x16;
    int64_t least = INT64_MAX;
    for (const auto &f : forms) {
        if (std::max({p.stride_w, p.stride_a, p.stride_ws, p.stride_as}) * std::max(f.m, f.n) > (int64_t)1 << 31) break;     // (a workgroup's rows lie within 2^31 bytes)
        if (forced && !strcmp(forced, f.name)) return f.form;
        const int64_t count = ((p.M + f.m - 1) / f.m) * (int64_t)((p.N + f.n - 1) / f.n);
        const int64_t cost = f.both && count > units ? (count + 2 * units - 1) / (2 * units) * f.both : (count + units - 1) / units * f.cost;
        if (cost < least) {
            least = cost;
            best = f.form;
        }
    }
    return best;
}

}   // namespace

dg_status dg_launch_quantize_mx4(const void *x, dg_dtype type, int64_t N, int64_t K, int64_t stride_n, uint8_t *codes, int64_t stride_codes,
                                 uint8_t *scales, int64_t stride_scales, hipStream_t stream)
{
    in_launches(N, K, 8, stride_n, stride_codes, stride_scales, [&](const MxRows &r, int64_t n) {
        dg_with_type(type, [&](auto t) {
            typedef decltype(t) T;
            quantize_mx4_kernel<T><<<(r.total + THREADS - 1) / THREADS, THREADS, 0, stream>>>((const T *)x + n * stride_n, r, codes + n * stride_codes, scales + n * stride_scales);
            return 0;
        });
    });
    return dg_check_launch("dg_quantize_mx4");
}

dg_status dg_launch_dequantize_mx4(const uint8_t *codes, int64_t stride_codes, const uint8_t *scales, int64_t stride_scales, int64_t N, int64_t K,
                                   void *out, dg_dtype type, int64_t stride_out, hipStream_t stream)
{
    in_launches(N, K, 16 / (int)dg_type_size(type), stride_out, stride_codes, stride_scales, [&](const MxRows &r, int64_t n) {
        dg_with_type(type, [&](auto t) {
            typedef decltype(t) T;
            dequantize_mx4_kernel<T><<<(r.total + THREADS - 1) / THREADS, THREADS, 0, stream>>>(codes + n * stride_codes, scales + n * stride_scales, r, (T *)out + n * stride_out);
            return 0;
        });
    });
    return dg_check_launch("dg_dequantize_mx4");
}

// f(a part of the product): channels and tokens whose workgroups are a grid.
template <class F>
static void in_parts(const DgGemmMx4 &all, dg_dtype type, F f)
{
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
            f(p);
            return DG_OK;
        });
    });
}

// (its elements are loaded by words of four bytes)
bool dg_linear_mx4_fuses(int64_t N, const void *x) { return N == 1 && (uintptr_t)x % 4 == 0; }

dg_status dg_launch_linear_mx4_fused(const DgGemmMx4 &all, const void *x, dg_dtype x_type, int64_t K, dg_dtype type, hipStream_t stream)
{
    in_parts(all, type, [&](const DgGemmMx4 &p) {
        dg_with_type(type, [&](auto t) {
            dg_with_type(x_type, [&](auto s) {
                typedef decltype(t) T;
                typedef decltype(s) X;
                if (many_channels(p)) launch_few<T, X, 2, 2, 1>(p, (const X *)x, (int32_t)K, stream);
                else launch_few<T, X, 4, 1, 1>(p, (const X *)x, (int32_t)K, stream);
                return 0;
            });
            return 0;
        });
    });
    return dg_check_launch("dg_linear_mx4");
}

dg_status dg_launch_gemm_mx4(const DgGemmMx4 &all, dg_dtype type, hipStream_t stream)
{
    in_parts(all, type, [&](const DgGemmMx4 &p) {
        dg_with_type(type, [&](auto t) {
            typedef decltype(t) T;
            switch (form_of(p)) {
            case Form::Few16x16:
                if (p.N <= 8) launch_few<T, void, 4, 1, 1>(p, nullptr, 0, stream);
                else launch_few<T, void, 4, 1, 2>(p, nullptr, 0, stream);
                break;
            case Form::Few16x32: launch_few<T, void, 4, 1, 4>(p, nullptr, 0, stream); break;
            case Form::Few32x16:
                if (p.N <= 8) launch_few<T, void, 2, 2, 1>(p, nullptr, 0, stream);
                else launch_few<T, void, 2, 2, 2>(p, nullptr, 0, stream);
                break;
            case Form::Few32x32: launch_few<T, void, 2, 2, 4>(p, nullptr, 0, stream); break;
            case Form::Tile32x64: launch_tiles<T, 1, 2, 1, 1, 4, 3>(p, stream); break;
            case Form::Tile64x64: launch_tiles<T, 2, 2, 1, 1, 2, 4>(p, stream); break;
            case Form::Tile128x64: launch_tiles<T, 2, 2, 2, 1, 2, 3>(p, stream); break;
            case Form::Tile128x128: launch_tiles<T, 2, 2, 2, 2, 1, 4>(p, stream); break;
            case Form::Tile256x128: launch_tiles<T, 2, 2, 4, 2, 1, 3>(p, stream); break;
            case Form::Tile256x256: launch_stream<T, 2, 4, 4, 2>(p, stream); break;
            }
            return 0;
        });
    });
    return dg_check_launch("dg_gemm_mx4");
}
