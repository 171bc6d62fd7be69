// Tokens quantised to 8 bits, and products of 8-bit codes with a scale for each token and each channel.
#include <cstring>

#include "dg_decoder.h"
#include "dg_lds_dma.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

// ---- quantising tokens ---------------------------------------------------------------------------------------------------
//
// s = max|x| / 127, code = rint(x / s).  A workgroup a token.  Its row is read once, into registers, 16 bytes a lane and load (HELD loads), where it fits; a longer one is read twice,
// the second time from the caches.  Bytes from K to PAD (a multiple of 16, or K) are cleared.  Few tokens are a launch and two waits (16 of 8192 2.9 us), many their
// bytes (8192 x 8192, bfloat16, 37 us, 5.5 TB/s).

// The largest magnitude over a workgroup; an infinity if any value was an infinity or a NaN (a NaN compares false, so it is counted apart).
template <int WAVES>
__device__ __forceinline__ float workgroup_most(float most, bool finite, float *part)
{
    most = dg_over_wave(finite ? most : __builtin_inff(), DgMax());
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
    __syncthreads();
    most = part[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) most = fmaxf(most, part[i]);
    return most;
}

template <class T, int COUNT>
__device__ __forceinline__ void look_at(const DgVec<T, COUNT> &v, float &most, bool &finite)
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const float f = fabsf(dg_to_float(v.e[i]));
        most = fmaxf(most, f);
        finite = finite && f < __builtin_inff();
    }
}

// COUNT elements from position k of a row of K; those at K and beyond are 0 and are not read.
template <class T, int COUNT>
__device__ __forceinline__ DgVec<T, COUNT> elements(const T *row, int32_t k, int32_t K)
{
    if (k + COUNT <= K) return dg_load_vec<T, COUNT>(row + k);
    uint64_t word[2] = {0, 0};
    for (int i = 0; k + i < K; ++i) {                   // (a loop: code that is short arrives soon, and few lanes come here)
        uint64_t bits = 0;
        __builtin_memcpy(&bits, row + k + i, sizeof(T));
        (i * (int)sizeof(T) < 8 ? word[0] : word[1]) |= bits << (8 * sizeof(T) * i & 63);
    }
    DgVec<T, COUNT> v;
    static_assert(sizeof(v) == sizeof(word), "16 bytes");
    __builtin_memcpy(&v, word, sizeof(v));
    return v;
}

// The codes of COUNT elements to position k of a row whose bytes up to `end` are this kernel's.
template <class T, int COUNT>
__device__ __forceinline__ void store_codes(int8_t *row, int32_t k, int32_t end, const DgVec<T, COUNT> &v, const DgDivisor &d)
{
    int code[COUNT];
    uint32_t words[COUNT / 4];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) code[i] = dg_code8(dg_to_float(v.e[i]), d);
#pragma unroll
    for (int i = 0; i < COUNT / 4; ++i) words[i] = dg_bytes(code + 4 * i) & d.keep;
    if (k + COUNT <= end) {
        __builtin_memcpy(row + k, words, COUNT);
    } else {
        uint64_t all = 0;
        __builtin_memcpy(&all, words, COUNT);
        for (; k < end; ++k, all >>= 8) row[k] = (int8_t)all;
    }
}

template <class T, int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void quantize_tokens_kernel(const T *x, int32_t K, int32_t pad, int64_t stride_n, int8_t *codes,
                                                                  int64_t stride_codes, float *scale)
{
    constexpr int COUNT = 16 / sizeof(T), STEP = THREADS * COUNT;
    __shared__ float part[THREADS / 64];
    const T *row = x + (int64_t)blockIdx.x * stride_n;
    int8_t *out = codes + (int64_t)blockIdx.x * stride_codes;
    const int32_t mine = threadIdx.x * COUNT;
    DgVec<T, COUNT> held[HELD ? HELD : 1];
    float most = 0.0f;
    bool finite = true;
    if constexpr (HELD) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) held[i] = elements<T, COUNT>(row, mine + i * STEP, K);
#pragma unroll
        for (int i = 0; i < HELD; ++i) look_at(held[i], most, finite);
    } else {
        for (int32_t k = mine; k < K; k += STEP) look_at(elements<T, COUNT>(row, k, K), most, finite);
    }
    const float s = dg_scale8(workgroup_most<THREADS / 64>(most, finite, part));
    const DgDivisor by = dg_divisor(s);
    if (threadIdx.x == 0) scale[blockIdx.x] = s;
    if constexpr (HELD) {
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (mine + i * STEP < pad) store_codes(out, mine + i * STEP, pad, held[i], by);
    } else {
        for (int32_t k = mine; k < pad; k += STEP) store_codes(out, k, pad, elements<T, COUNT>(row, k, K), by);
    }
}

// ---- the product ------------------------------------------------------------------------------------------------------

// 16 codes from position k of a row of K; those at K and beyond count as 0 and are not read.
__device__ __forceinline__ v4i codes16(const int8_t *row, int32_t k, int32_t K)
{
    v4i v;
    if (k + 16 <= K) {
        __builtin_memcpy(&v, row + k, 16);
        return v;
    }
    uint64_t word[2] = {0, 0};
    for (int i = 0; k + i < K; ++i) (i < 8 ? word[0] : word[1]) |= (uint64_t)(uint8_t)row[k + i] << (8 * i & 63);
    __builtin_memcpy(&v, word, 16);
    return v;
}

// y of one output channel and token, rounded once: the sum is converted, multiplied by the two scales, and the bias added.
template <class T>
__device__ __forceinline__ T finished(int sum, float sm, float sn, const float *bias, int32_t m)
{
    const float y = (float)sum * sm * sn;
    return dg_from_float<T>(bias ? y + bias[m] : y);
}

// Four neighbouring channels of token n.
template <class T>
__device__ __forceinline__ void store4(const DgGemmI8 &p, int32_t m, int32_t n, float sn, const int (&sum)[4])
{
    T *out = (T *)p.out + (int64_t)n * p.stride_out + m;
    if (m + 4 <= p.M) {
        const DgVec<float, 4> sm = dg_load_vec<float, 4>(p.scale_m + m);
        DgVec<T, 4> y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y.e[i] = finished<T>(sum[i], sm.e[i], sn, p.bias, m + i);
        dg_store_vec<T, 4>(out, y);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (m + i < p.M) out[i] = finished<T>(sum[i], p.scale_m[m + i], sn, p.bias, m + i);
    }
}

// ---- few tokens ---------------------------------------------------------------------------------------------------------
//
// A workgroup computes 16 ROWS channels x 16 TOKENS tokens; its wavefronts share K in pieces of 128 positions, a cache line of a row, and
// their sums meet in LDS.  The weights are read once, straight into the matrix instructions' operands, a piece on its way while the one before is
// multiplied.  That reading bounds it (16 x 8192 x 8192 17.2 us, 3.9 TB/s with the launch; one token 13.7, 4.9 TB/s): two or three pieces asked for at once
// and then multiplied 18.3, pieces two or three at a time in this way 17.6 and 17.8.
// FUSED: a single token is quantised here too, by every workgroup for itself, into LDS, while the first weights are on their way (4096 x 4096
// 6.5 us for 8.1 as two launches; four tokens 11.3 for 8.5).

constexpr int FUSED_BYTES = 32768;       // codes that FUSED holds in LDS

template <class X>
struct Fused {
    const X *x;
    int32_t pitch;                       // its codes' bytes in LDS: K rounded up to 128
};

template <class T, class X, int WAVES, int ROWS, int TOKENS, bool FUSED>
__global__ __launch_bounds__(64 * WAVES) void gemm_i8_few_kernel(DgGemmI8 p, Fused<X> f)
{
    __shared__ v4i sums[WAVES][ROWS][TOKENS][64];
    extern __shared__ int8_t quantized[];
    __shared__ float part[WAVES];
    float own_scale = 0.0f;
    // (a matrix instruction runs whatever the lanes' mask: what it stands under has to be a scalar branch)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t m0 = blockIdx.x * (16 * ROWS), last = p.N - 1;
    const int8_t *w[ROWS], *a[TOKENS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) w[i] = p.W + (int64_t)min(m0 + 16 * i + r, p.M - 1) * p.stride_w;
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) a[t] = FUSED ? quantized : p.A + (int64_t)min(16 * t + r, last) * p.stride_a;
    // a piece: two instructions of 64 positions, 16 a lane
    const int32_t pieces = p.K / 128;
    v4i wk[2][ROWS][2], ak[2][TOKENS][2], acc[ROWS][TOKENS] = {};
    const auto fetch_tokens = [&](int to, int32_t piece) {
#pragma unroll
        for (int t = 0; t < TOKENS; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) __builtin_memcpy(&ak[to][t][h], a[t] + 128 * piece + 64 * h + 16 * g, 16);
    };
    const auto fetch = [&](int to, int32_t piece) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) __builtin_memcpy(&wk[to][i][h], w[i] + 128 * piece + 64 * h + 16 * g, 16);
        if (!FUSED) fetch_tokens(to, piece);
    };
    const auto multiply = [&](int from, int32_t piece) {
        __builtin_amdgcn_sched_barrier(0);                  // (or the compiler moves the next piece's loads behind these products)
        if (FUSED) fetch_tokens(from, piece);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < TOKENS; ++t)
#pragma unroll
                for (int i = 0; i < ROWS; ++i) acc[i][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wk[from][i][h], ak[from][t][h], acc[i][t], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    if (wave < pieces) fetch(0, wave);
    if constexpr (FUSED) {
        constexpr int COUNT = 16 / sizeof(X), STEP = 64 * WAVES * COUNT;
        float most = 0.0f;
        bool finite = true;
        for (int32_t at = threadIdx.x * COUNT; at < p.K; at += STEP) look_at(elements<X, COUNT>(f.x, at, p.K), most, finite);
        own_scale = dg_scale8(workgroup_most<WAVES>(most, finite, part));
        const DgDivisor by = dg_divisor(own_scale);
        for (int32_t at = threadIdx.x * COUNT; at < f.pitch; at += STEP)
            store_codes(quantized, at, f.pitch, elements<X, COUNT>(f.x, at, p.K), by);
        __syncthreads();
    }
    int32_t at = wave;
#pragma unroll 1
    for (; at + 2 * WAVES < pieces; at += 2 * WAVES) {
        fetch(1, at + WAVES);
        multiply(0, at);
        fetch(0, at + 2 * WAVES);
        multiply(1, at + WAVES);
    }
    if (at + WAVES < pieces) {
        fetch(1, at + WAVES);
        multiply(0, at);
        multiply(1, at + WAVES);
    } else if (at < pieces) {
        multiply(0, at);
    }
    if (128 * pieces < p.K && pieces % WAVES == wave)               // the rest of the row
#pragma unroll 1
        for (int32_t k = 128 * pieces; k < p.K; k += 64)
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
                const v4i at = codes16(a[t], k + 16 * g, p.K);
#pragma unroll
                for (int i = 0; i < ROWS; ++i) acc[i][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(codes16(w[i], k + 16 * g, p.K), at, acc[i][t], 0, 0, 0);
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
        v4i s = sums[0][i][t][lane];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) s += sums[k][i][t][lane];
        const int32_t n = 16 * t + r;
        if (n <= last) store4<T>(p, m0 + 16 * i + 4 * g, n, FUSED ? own_scale : p.scale_n[n], {s[0], s[1], s[2], s[3]});
    }
}

// Whether 16 channels a workgroup are one workgroup a compute unit at most: then twice the wavefronts (one token x 4096 x 4096 5.2 us for 5.5, quantised here
// as well 6.9 for 7.3; but not where each would have one piece at most: 2048 x 2048 3.1 for 3.0).
bool few_channels(const DgGemmI8 &p, int units) { return p.M <= 16 * units && p.K > 2048; }

template <class T, int TOKENS>
void launch_few(const DgGemmI8 &p, hipStream_t stream)
{
    const Fused<float> none = {nullptr, 0};
    const int units = dg_simd_count() / 4;
    // 32 channels a workgroup share the tokens' loads (16 x 8192 x 8192 17.2 us for 19.9); with too few channels for that, or tokens that cost
    // little to load, 16 (one token 13.7 for 15.4, four 15.1 for 16.5)
    if (p.N > 4 && p.M >= 32 * units) gemm_i8_few_kernel<T, float, 8, 2, TOKENS, false><<<(p.M + 31) / 32, 512, 0, stream>>>(p, none);
    else if (!few_channels(p, units)) gemm_i8_few_kernel<T, float, 8, 1, TOKENS, false><<<(p.M + 15) / 16, 512, 0, stream>>>(p, none);
    else gemm_i8_few_kernel<T, float, 16, 1, TOKENS, false><<<(p.M + 15) / 16, 1024, 0, stream>>>(p, none);
}

// ---- many tokens: tiles ------------------------------------------------------------------------------------------------
//
// KS groups of WM x WN wavefronts compute 32 WM TM channels x 32 WN TN tokens, TM x TN blocks of 32 x 32 a wavefront; a group takes 128
// positions of K of a stage's 128 KS, and the groups' sums meet in LDS at the end.  The stages are a ring in LDS: the next ones' loads are in flight while one
// is multiplied.  256 x 256 by eight wavefronts of 128 x 64: six kilobytes read from LDS for eight products, and the pipe busy 55 % of the cycles at the 1.83 GHz
// that the card holds meanwhile; 8192 x 8192 x 8192 takes 490 to 510 us, 2.2 POP/s, where the library's product of the same codes reaches 2.07; small products are start, end and a round of tiles that does not fill the
// card (333 x 1537 x 2000: 8.7 us, 150 tiles of 64 x 64).  A row's 128 bytes lie in LDS as eight pieces of 16, piece c of row r at place c ^ (r / 2 % 8), so that the 16 lanes that an LDS read serves together find 16 different ones.
// DIRECT: rows begin on 16 bytes and K is whole pieces: the loads write LDS themselves.  Otherwise they go through registers.

typedef int v16i __attribute__((ext_vector_type(16)));

struct TileArgs {
    DgGemmI8 p;
    int32_t tiles_m, tiles_n;
    DgFastDiv by_group, by_rest;         // tile order: groups of GROUP rows of tiles
    int32_t rest;                        // rows of the last group
};
constexpr int GROUP = 4;

template <class T, int WM, int WN, int TM, int TN, int KS, int RING, bool DIRECT>
__global__ __launch_bounds__(64 * WM * WN * KS) void gemm_i8_tile_kernel(TileArgs args)
{
    constexpr int WAVES = WM * WN, BM = 32 * WM * TM, BN = 32 * WN * TN, STAGE = (BM + BN) * 128, STAGES = DIRECT ? RING : 2;
    constexpr int LOADS_M = BM / (8 * WAVES), LOADS = (BM + BN) / (8 * WAVES);       // loads of 8 rows a wavefront makes of its group's stage
    static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && WAVES % 2 == 0, "whole loads, and the same places in each");
    constexpr int RESULTS = WAVES * 32 * (32 * TM + 4) * 4;
    __shared__ __align__(1024) uint8_t room[STAGES * STAGE * KS > RESULTS ? STAGES * STAGE * KS : RESULTS];
    const DgGemmI8 &p = args.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % WAVES);
    const int share = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) / WAVES);
    uint8_t (*const stages)[STAGE] = (uint8_t(*)[STAGE])room + share * STAGES;        // (each group has a ring of its own)

    // Neighbouring workgroups go to different dies (eight): each die takes a run of tiles of its own, and walks it in groups of GROUP rows
    // of tiles, so that what it reads twice is in its own cache.
    const uint32_t tiles = (uint32_t)args.tiles_m * args.tiles_n, die = blockIdx.x & 7, in_die = blockIdx.x >> 3;
    const uint32_t tile = die * (tiles >> 3) + min(die, tiles & 7) + in_die;
    const uint32_t group = dg_fdiv(tile, args.by_group), left = tile - group * (GROUP * args.tiles_n);
    const bool last = (int32_t)(group * GROUP) + GROUP > args.tiles_m;
    const uint32_t column = last ? dg_fdiv(left, args.by_rest) : left / GROUP;
    const int32_t m0 = (int32_t)(group * GROUP + left - column * (last ? args.rest : GROUP)) * BM, n0 = (int32_t)column * BN;

    // what this lane loads: piece (lane % 8) ^ ... of row 8 q + lane / 8
    const int piece = (lane & 7) ^ ((((wave & 1) << 2) + (lane >> 4)) & 7);
    const int8_t *rows_w = p.W + (int64_t)m0 * p.stride_w, *rows_a = p.A + (int64_t)n0 * p.stride_a;
    const int32_t have_w = min(p.M - m0, BM), have_a = min(p.N - n0, BN);
    uint32_t offset[LOADS];
    const auto row_of = [&](int i) { return (wave + WAVES * (i < LOADS_M ? i : i - LOADS_M)) * 8 + (lane >> 3); };
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const uint32_t stride = (uint32_t)(i < LOADS_M ? p.stride_w : p.stride_a);
        offset[i] = row_of(i) < (i < LOADS_M ? have_w : have_a) ? row_of(i) * stride + 16 * piece : 0xF0000000u;
    }
    const dg_v4i buffer_w = dg_buffer((const uint8_t *)rows_w, DIRECT ? (uint32_t)((have_w - 1) * (uint32_t)p.stride_w + p.K) : 0u);
    const dg_v4i buffer_a = dg_buffer((const uint8_t *)rows_a, DIRECT ? (uint32_t)((have_a - 1) * (uint32_t)p.stride_a + p.K) : 0u);
    const uint32_t lds = dg_lds_address(room) + share * (STAGES * STAGE) + 1024 * wave;
    // Through registers, two stages on their way where a stage is few of them (300 x 4000 x 5001 37.8 us, one 39.5).  What bounds this form is the loads themselves,
    // which the hardware serves at a fraction of its rate where they do not begin on 16 bytes (300 x 4000 x 4992 16.5).
    constexpr int AHEAD = LOADS <= 6 ? 2 : 1;
    v4i held[DIRECT ? 1 : AHEAD][LOADS];
    const auto address = [&](int i, int32_t k) {
        int row = min(row_of(i), (i < LOADS_M ? have_w : have_a) - 1);                       // (what a row past the end gives is not stored)
        if (AHEAD == 1) asm volatile("" : "+v"(row));                                        // (its address is not worth two registers)
        return (i < LOADS_M ? rows_w : rows_a) + row * (i < LOADS_M ? p.stride_w : p.stride_a) + k;
    };

    auto fetch = [&](int32_t k, int to) {
        if constexpr (DIRECT) {
            const bool past = k + 16 * piece >= p.K;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const uint32_t at = past ? 0xF0000000u : offset[i] + k;
                dg_load16_to_lds(i < LOADS_M ? buffer_w : buffer_a, at, lds + to * STAGE + i * (1024 * WAVES));
            }
        } else if (k + 128 <= p.K) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) __builtin_memcpy(&held[to][i], address(i, k) + 16 * piece, 16);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) held[to][i] = codes16(address(i, 0), k + 16 * piece, p.K);
        }
    };
    const int r = lane & 31, g = lane >> 5, wm = wave % WM, wn = wave / WM;
    const uint32_t first = r * 128 + ((g ^ ((r >> 1) & 7)) << 4);
    v16i acc[TM][TN] = {};
    // 32 positions at a time; the operands of the next ones are read before these are multiplied (left to itself the compiler reads each just
    // before its use, and a wavefront waits for LDS four times a stage)
    v4i wk[2][TM], ak[2][TN];
    const auto read = [&](int now, int s) {
        const uint8_t *w = stages[now] + wm * (TM * 4096) + (first ^ (s * 32)), *a = stages[now] + BM * 128 + wn * (TN * 4096) + (first ^ (s * 32));
#pragma unroll
        for (int i = 0; i < TM; ++i) wk[s & 1][i] = *(const v4i *)(w + i * 4096);
#pragma unroll
        for (int j = 0; j < TN; ++j) ak[s & 1][j] = *(const v4i *)(a + j * 4096);
    };
    const auto multiply = [&](int now) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s < 3) read(now, s + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wk[s & 1][i], ak[s & 1][j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if constexpr (DIRECT) {
        // A stage's loads are waited for when its turn comes; the barrier after that says that every wavefront's are in, and that all are done with
        // the stage before, whose place the loads of STAGES - 1 ahead then take.  (Past the end of K there is nothing to load; the waits count on
        // loads, so they go on, from outside the buffers: zeros, which nothing reads.)
        for (int i = 0; i < STAGES - 1; ++i) fetch(128 * (KS * i + share), i);
        int now = 0, to = STAGES - 1;
        for (int32_t k = 0; k < p.K; k += 128 * KS) {
            dg_wait_for_loads<(STAGES - 2) * LOADS>();
            __syncthreads();
            read(now, 0);
            fetch(k + 128 * (KS * (STAGES - 1) + share), to);
            multiply(now);
            now = now + 1 == STAGES ? 0 : now + 1;
            to = to + 1 == STAGES ? 0 : to + 1;
        }
        dg_wait_for_loads<0>();
    } else {
        const auto put = [&](int from, int to) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) *(v4i *)(stages[to] + 1024 * (wave + WAVES * i) + 16 * lane) = held[from][i];
            __syncthreads();
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fetch(128 * (KS * i + share), i);
        put(0, 0);
        for (int32_t k = 0, now = 0; k < p.K;) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (i && k >= p.K) break;
                const bool more = k + 128 * KS < p.K;
                if (k + 128 * KS * AHEAD < p.K) fetch(k + 128 * (KS * AHEAD + share), i);
                read(now, 0);
                multiply(now);
                if (more) put((i + 1) % AHEAD, now ^ 1);
                k += 128 * KS;
                now ^= 1;
            }
        }
    }
    // The results go by way of LDS, a wavefront's 32 tokens at a time: rows of channels leave side by side, and a loop does it (written out
    // it was 20 KB of instructions, which a small product waited for as they arrived).
    constexpr int PITCH = 32 * TM + 4, LANES = 8 * TM, ROWS = 64 / LANES;
    __syncthreads();
    int *mine = (int *)room + wave * (32 * PITCH);
    if constexpr (KS > 1) {
        // the other groups' sums, one group after another
        static_assert(TM * TN * 4096 * WAVES <= STAGES * STAGE * KS, "a group's sums fit");
        int4 *const sums = (int4 *)room + wave * (TM * TN * 256) + lane;
#pragma unroll 1
        for (int from = 1; from < KS; ++from) {
            if (share == from)
#pragma unroll
                for (int i = 0; i < TM * TN; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const v16i &c = acc[i / TN][i % TN];
                        sums[(4 * i + e) * 64] = make_int4(c[4 * e], c[4 * e + 1], c[4 * e + 2], c[4 * e + 3]);
                    }
            __syncthreads();
            if (share == 0)
#pragma unroll
                for (int i = 0; i < TM * TN; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int4 x = sums[(4 * i + e) * 64];
                        v16i &c = acc[i / TN][i % TN];
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
    float sm[4], bias[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        sm[e] = e < have ? p.scale_m[m + e] : 0.0f;
        bias[e] = p.bias && e < have ? p.bias[m + e] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *(v4i *)(mine + r * PITCH + 32 * i + 8 * e + 4 * g) = (v4i){acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
        const int32_t first_n = n0 + (wn * TN + j) * 32, end = min(p.N - first_n, 32);
#pragma unroll 1
        for (int t = lane / LANES; t < end; t += ROWS) {
            const v4i sum = *(const v4i *)(mine + t * PITCH + 4 * (lane % LANES));
            const float sn = p.scale_n[first_n + t];
            T *out = (T *)p.out + (int64_t)(first_n + t) * p.stride_out + m;
            DgVec<T, 4> y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = (float)sum[e] * sm[e] * sn;
                y.e[e] = dg_from_float<T>(p.bias ? x + bias[e] : x);
            }
            if (have == 4) dg_store_vec<T, 4>(out, y);
            else
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < have) out[e] = y.e[e];
        }
    }
}

template <class T, int WM, int WN, int TM, int TN, int KS, int RING>
void launch_tiles(const DgGemmI8 &p, hipStream_t stream)
{
    TileArgs a = {p, (p.M + 32 * WM * TM - 1) / (32 * WM * TM), (p.N + 32 * WN * TN - 1) / (32 * WN * TN), {}, {}, 0};
    a.by_group = dg_make_div((uint32_t)GROUP * a.tiles_n);
    a.rest = a.tiles_m % GROUP ? a.tiles_m % GROUP : GROUP;
    a.by_rest = dg_make_div((uint32_t)a.rest);
    const uint32_t tiles = (uint32_t)a.tiles_m * a.tiles_n;
    const bool direct = p.K % 16 == 0 && p.stride_w % 16 == 0 && p.stride_a % 16 == 0 && (uintptr_t)p.W % 16 == 0 && (uintptr_t)p.A % 16 == 0 &&
                        p.stride_w < (1 << 22) && p.stride_a < (1 << 22);          // (a tile's rows lie within 2^30 bytes)
    if (direct) gemm_i8_tile_kernel<T, WM, WN, TM, TN, KS, RING, true><<<tiles, 64 * WM * WN * KS, 0, stream>>>(a);
    else gemm_i8_tile_kernel<T, WM, WN, TM, TN, KS, 2, false><<<tiles, 64 * WM * WN * KS, 0, stream>>>(a);
}

enum class Form { Few, Tile32x64, Tile64x64, Tile128x64, Tile128x128, Tile256x128, Tile256x256 };
constexpr int FEW_TOKENS = 32;

// The kernel for up to 32 tokens (16 x 4096 x 4096 6.6 us, 32 x 64 tiles 7.7; 32 tokens 8.5, 8.1; 32 x 1000 x 1000 6.0, 10.4; 32 x 12288 x 1024 6.9, 9.8; but
// long sums of 24 and 32 tokens are faster in tiles: 24 x 8192 x 8192 19.1, 17.0; 32 x 8192 x 8192 20.0, 17.5; 32 x 2048 x 8192 13.1, 11.0), or the tile (channels x tokens) whose
// rounds over the compute units, one workgroup each, cost least.  A round's cost by tile, us for K = 4096 and 8192: 32 x 64 8, 18; 64 x 64 10, 24; 128 x 64 15, 34;
// 128 x 128 23, 46; 256 x 128 39, 72; 256 x 256 54, 104.  Of 60 products, 33 to 2048 tokens, this is within 3 % of the fastest tile on 58, 6 % on two (64 x 2048 x 8192
// 11.7 us by 32 x 64, 15.0 by 64 x 64; 128 x 8192 x 8192 33.8, 24.1).
Form form_of(const DgGemmI8 &p)
{
    static const struct {
        Form form;
        int32_t m, n, cost;
        const char *name;
    } tiles[] = {{Form::Tile32x64, 32, 64, 22, "32x64"}, {Form::Tile64x64, 64, 64, 28, "64x64"}, {Form::Tile128x64, 128, 64, 40, "128x64"}, {Form::Tile128x128, 128, 128, 54, "128x128"},
                 {Form::Tile256x128, 256, 128, 85, "256x128"}, {Form::Tile256x256, 256, 256, 124, "256x256"}};
    const char *forced = dg_override("DG_GEMM_I8_TILE");
    const int64_t units = dg_simd_count() / 4;
    Form best = Form::Few;
    int64_t least = INT64_MAX;
    if (!forced && p.N <= FEW_TOKENS) return best;
    for (const auto &t : tiles) {
        if (forced && !strcmp(forced, t.name)) return t.form;
        const int64_t count = ((p.M + t.m - 1) / t.m) * (int64_t)((p.N + t.n - 1) / t.n), cost = (count + units - 1) / units * t.cost;
        if (cost < least) {
            least = cost;
            best = t.form;
        }
    }
    return p.N <= FEW_TOKENS ? Form::Few : best;
}

}   // namespace

dg_status dg_launch_quantize_tokens(const void *x, dg_dtype type, int64_t N, int64_t K, int64_t stride_n, int8_t *codes,
                                    int64_t stride_codes, int64_t pad, float *scale, hipStream_t stream)
{
    dg_with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const auto launch = [&](auto threads, auto held) {
            constexpr int THREADS = decltype(threads)::value;
            dg_in_turns(N, 1 << 21, [&](int64_t n, int64_t count) {
                quantize_tokens_kernel<T, THREADS, decltype(held)::value><<<(uint32_t)count, THREADS, 0, stream>>>((const T *)x + n * stride_n, (int32_t)K, (int32_t)pad,
                                                                                                               stride_n, codes + n * stride_codes, stride_codes, scale + n);
                return DG_OK;
            });
        };
        const auto by_length = [&](auto threads) {
            const int64_t step = decltype(threads)::value * (16 / sizeof(T));
            if (K <= step) launch(threads, std::integral_constant<int, 1>{});
            else if (K <= 2 * step) launch(threads, std::integral_constant<int, 2>{});
            else if (K <= 4 * step) launch(threads, std::integral_constant<int, 4>{});
            else if (K <= 8 * step) launch(threads, std::integral_constant<int, 8>{});
            else launch(threads, std::integral_constant<int, 0>{});
        };
        // few tokens: as many threads as there are, so that each has little to do (256 x 8192 3.6 us, 256 threads 4.1); many: workgroups that others can stand
        // beside (512 x 4096 3.6, 1024 threads 4.0; 8192 x 8192 37, 45)
        if (N <= 256) by_length(std::integral_constant<int, 1024>{});
        else by_length(std::integral_constant<int, 256>{});
        return 0;
    });
    return dg_check_launch("dg_quantize_tokens");
}

bool dg_linear_i8_fuses(int64_t N, int64_t K) { return N == 1 && K <= FUSED_BYTES; }

// f(a part of the product): channels and tokens whose workgroups, tiles of 2^16 results where there are many of both, are a grid.
template <class F>
static dg_status in_parts(const DgGemmI8 &p, dg_dtype type, F f)
{
    return dg_in_turns(p.M, 1 << 24, [&](int64_t m, int64_t channels) {
        return dg_in_turns(p.N, std::min<int64_t>(1 << 24, ((int64_t)1 << 38) / channels), [&](int64_t n, int64_t tokens) {
            DgGemmI8 part = p;
            part.W += m * p.stride_w;
            part.scale_m += m;
            part.bias = p.bias ? p.bias + m : nullptr;
            part.A += n * p.stride_a;
            part.scale_n += n;
            part.out = (uint8_t *)p.out + (n * p.stride_out + m) * dg_type_size(type);
            part.M = (int32_t)channels;
            part.N = (int32_t)tokens;
            f(part);
            return DG_OK;
        });
    });
}

dg_status dg_launch_linear_i8_fused(const DgGemmI8 &all, const void *x, dg_dtype x_type, dg_dtype type, hipStream_t stream)
{
    in_parts(all, type, [&](const DgGemmI8 &p) {
        dg_with_type(type, [&](auto t) {
            dg_with_type(x_type, [&](auto s) {
                const Fused<decltype(s)> f = {(const decltype(s) *)x, (p.K + 127) / 128 * 128};
                const uint32_t blocks = (p.M + 15) / 16, room = f.pitch;
                if (few_channels(p, dg_simd_count() / 4)) gemm_i8_few_kernel<decltype(t), decltype(s), 16, 1, 1, true><<<blocks, 1024, room, stream>>>(p, f);
                else gemm_i8_few_kernel<decltype(t), decltype(s), 8, 1, 1, true><<<blocks, 512, room, stream>>>(p, f);
                return 0;
            });
            return 0;
        });
    });
    return dg_check_launch("dg_linear_i8");
}

dg_status dg_launch_gemm_i8(const DgGemmI8 &all, dg_dtype type, hipStream_t stream)
{
    in_parts(all, type, [&](const DgGemmI8 &p) {
        dg_with_type(type, [&](auto t) {
            typedef decltype(t) T;
            switch (form_of(p)) {
            case Form::Few:
                if (p.N <= 16) launch_few<T, 1>(p, stream);
                else launch_few<T, 2>(p, stream);
                break;
            case Form::Tile32x64: launch_tiles<T, 1, 2, 1, 1, 4, 3>(p, stream); break;
            case Form::Tile64x64: launch_tiles<T, 2, 2, 1, 1, 2, 4>(p, stream); break;
            case Form::Tile128x64: launch_tiles<T, 2, 2, 2, 1, 2, 3>(p, stream); break;
            case Form::Tile128x128: launch_tiles<T, 2, 2, 2, 2, 1, 4>(p, stream); break;
            case Form::Tile256x128: launch_tiles<T, 2, 2, 4, 2, 1, 3>(p, stream); break;
            case Form::Tile256x256: launch_tiles<T, 2, 4, 4, 2, 1, 2>(p, stream); break;
            }
            return 0;
        });
    });
    return dg_check_launch("dg_gemm_i8");
}
