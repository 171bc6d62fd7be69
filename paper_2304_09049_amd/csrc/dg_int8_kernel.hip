// Tokens quantised to 8 bits, and products of 8-bit codes with a scale for each token and each channel.
#include "dg_decoder.h"
#include "dg_lds_dma.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

// ---- quantising tokens: one workgroup per token, two passes over its row (the second finds it in the caches) --------------

template <class T>
__global__ __launch_bounds__(256) void quantize_tokens_kernel(const T *x, int32_t K, int64_t stride_n, int8_t *codes, int64_t stride_codes,
                                                               float *scale)
{
    __shared__ float part[4];
    __shared__ int whole[4];
    const T *row = x + (int64_t)blockIdx.x * stride_n;
    int8_t *out = codes + (int64_t)blockIdx.x * stride_codes;
    float most = 0.0f;
    bool finite = true;
    for (int k = threadIdx.x; k < K; k += 256) {
        const float f = fabsf(dg_to_float(row[k]));
        most = fmaxf(most, f);
        finite = finite && f < __builtin_inff();
    }
#pragma unroll
    for (int i = 32; i; i >>= 1) most = fmaxf(most, __shfl_xor(most, i));
    finite = __all(finite);
    if ((threadIdx.x & 63) == 0) {
        part[threadIdx.x >> 6] = most;
        whole[threadIdx.x >> 6] = finite;
    }
    __syncthreads();
    most = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    const float s = whole[0] && whole[1] && whole[2] && whole[3] ? dg_scale8(most) : __builtin_nanf("");
    if (threadIdx.x == 0) scale[blockIdx.x] = s;
    for (int k = threadIdx.x; k < K; k += 256) out[k] = (int8_t)dg_code8(dg_to_float(row[k]), s);
}

// ---- the product ------------------------------------------------------------------------------------------------------

// 16 codes from position k of a row of K; those at K and beyond count as 0 and are not read.
__device__ __forceinline__ v4i codes16(const int8_t *row, int32_t k, int32_t K)
{
    v4i v = {0, 0, 0, 0};
    if (k + 16 <= K)
        __builtin_memcpy(&v, row + k, 16);
    else
        for (int i = 0; k + i < K; ++i) v[i >> 2] |= (int)(uint8_t)row[k + i] << (8 * (i & 3));
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

// 16 channels x 16 TOKENS tokens by a workgroup whose eight wavefronts share K; their sums meet in LDS.
template <class T, int TOKENS>
__global__ __launch_bounds__(512) void gemm_i8_few_kernel(DgGemmI8 p)
{
    __shared__ v4i sums[7][TOKENS][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int32_t m0 = blockIdx.x * 16, n0 = blockIdx.y * (16 * TOKENS);
    const int8_t *w = p.W + (int64_t)min(m0 + r, p.M - 1) * p.stride_w + 16 * g;
    const int8_t *a[TOKENS];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) a[t] = p.A + (int64_t)min(n0 + 16 * t + r, p.N - 1) * p.stride_a + 16 * g;
    v4i acc[TOKENS] = {};
    constexpr int AHEAD = TOKENS == 1 ? 4 : 2;              // steps whose loads are in flight together
    int32_t k = 64 * wave;
    for (; k + 512 * (AHEAD - 1) + 64 <= p.K; k += 512 * AHEAD) {
        v4i wk[AHEAD], ak[AHEAD][TOKENS];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            __builtin_memcpy(&wk[u], w + k + 512 * u, 16);
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) __builtin_memcpy(&ak[u][t], a[t] + k + 512 * u, 16);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wk[u], ak[u][t], acc[t], 0, 0, 0);
    }
    for (; k < p.K; k += 512) {
        const v4i wk = codes16(w - 16 * g, k + 16 * g, p.K);
#pragma unroll
        for (int t = 0; t < TOKENS; ++t)
            acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wk, codes16(a[t] - 16 * g, k + 16 * g, p.K), acc[t], 0, 0, 0);
    }
    if (wave)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) sums[wave - 1][t][lane] = acc[t];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        v4i s = acc[t];
#pragma unroll
        for (int i = 0; i < 7; ++i) s += sums[i][t][lane];
        const int32_t n = n0 + 16 * t + r;
        if (n < p.N) store4<T>(p, m0 + 4 * g, n, p.scale_n[n], {s[0], s[1], s[2], s[3]});
    }
}

// ---- many tokens: tiles ------------------------------------------------------------------------------------------------
//
// A workgroup of WM x WN wavefronts computes 32 WM TM channels x 32 WN TN tokens, TM x TN blocks of 32 x 32 a wavefront, 128 positions of
// K at a time, in two LDS stages: the next stage's loads are in flight while this one is multiplied.  A row's 128 bytes lie in LDS as eight pieces
// of 16, piece c of row r at place c ^ (r / 2 % 8), so that the 16 lanes that an LDS read serves together find 16 different ones.
// DIRECT: rows begin on 16 bytes and K is whole pieces: the loads write LDS themselves.  Otherwise they go through registers.

typedef int v16i __attribute__((ext_vector_type(16)));

struct TileArgs {
    DgGemmI8 p;
    int32_t tiles_m, tiles_n;
    DgFastDiv by_group, by_rest;         // tile order: groups of GROUP rows of tiles
    int32_t rest;                        // rows of the last group
};
constexpr int GROUP = 4;

template <class T, int WM, int WN, int TM, int TN, bool DIRECT>
__global__ __launch_bounds__(64 * WM * WN) void gemm_i8_tile_kernel(TileArgs args)
{
    constexpr int WAVES = WM * WN, BM = 32 * WM * TM, BN = 32 * WN * TN, STAGE = (BM + BN) * 128;
    constexpr int LOADS_M = BM / (8 * WAVES), LOADS = (BM + BN) / (8 * WAVES);       // loads of 8 rows a wavefront makes of a stage
    static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && WAVES % 2 == 0, "whole loads, and the same places in each");
    __shared__ __align__(1024) uint8_t stages[2][STAGE];
    const DgGemmI8 &p = args.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

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
    bool there[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int row = (wave + WAVES * (i < LOADS_M ? i : i - LOADS_M)) * 8 + (lane >> 3);
        there[i] = row < (i < LOADS_M ? have_w : have_a);
        const uint32_t stride = (uint32_t)(i < LOADS_M ? p.stride_w : p.stride_a);
        offset[i] = there[i] ? row * stride + 16 * piece : DIRECT ? 0xF0000000u : 0u;
    }
    const dg_v4i buffer_w = dg_buffer((const uint8_t *)rows_w, DIRECT ? (uint32_t)((have_w - 1) * (uint32_t)p.stride_w + p.K) : 0u);
    const dg_v4i buffer_a = dg_buffer((const uint8_t *)rows_a, DIRECT ? (uint32_t)((have_a - 1) * (uint32_t)p.stride_a + p.K) : 0u);
    const uint32_t lds = dg_lds_address(stages) + 1024 * wave;
    v4i held[DIRECT ? 1 : LOADS];

    auto fetch = [&](int32_t k, int to) {
        if constexpr (DIRECT) {
            const bool past = k + 16 * piece >= p.K;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const uint32_t at = past ? 0xF0000000u : offset[i] + k;
                dg_load16_to_lds(i < LOADS_M ? buffer_w : buffer_a, at, lds + to * STAGE + i * (1024 * WAVES));
            }
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int8_t *row = (i < LOADS_M ? rows_w : rows_a) + (int64_t)((wave + WAVES * (i < LOADS_M ? i : i - LOADS_M)) * 8 + (lane >> 3)) *
                                                                          (i < LOADS_M ? p.stride_w : p.stride_a);
                held[i] = there[i] ? codes16(row, k + 16 * piece, p.K) : (v4i){0, 0, 0, 0};
            }
        }
    };
    auto arrive = [&](int to) {
        if constexpr (DIRECT) {
            dg_wait_for_loads<0>();
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) *(v4i *)(stages[to] + 1024 * (wave + WAVES * i) + 16 * lane) = held[i];
        }
        __syncthreads();
    };

    const int r = lane & 31, g = lane >> 5, wm = wave % WM, wn = wave / WM;
    const uint32_t first = r * 128 + ((g ^ ((r >> 1) & 7)) << 4);
    v16i acc[TM][TN] = {};
    fetch(0, 0);
    arrive(0);
    for (int32_t k = 0, now = 0; k < p.K; k += 128, now ^= 1) {
        const bool more = k + 128 < p.K;
        if (more) fetch(k + 128, now ^ 1);
        const uint8_t *w = stages[now] + wm * (TM * 4096), *a = stages[now] + BM * 128 + wn * (TN * 4096);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const uint32_t at = first ^ (s * 32);
            v4i wk[TM], ak[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) wk[i] = *(const v4i *)(w + i * 4096 + at);
#pragma unroll
            for (int j = 0; j < TN; ++j) ak[j] = *(const v4i *)(a + j * 4096 + at);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wk[i], ak[j], acc[i][j], 0, 0, 0);
        }
        if (more) arrive(now ^ 1);
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int32_t n = n0 + (wn * TN + j) * 32 + r;
        if (n >= p.N) continue;
        const float sn = p.scale_n[n];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t m = m0 + (wm * TM + i) * 32 + 8 * e + 4 * g;
                store4<T>(p, m, n, sn, {acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]});
            }
    }
}

template <class T, int WM, int WN, int TM, int TN>
void launch_tiles(const DgGemmI8 &p, hipStream_t stream)
{
    TileArgs a = {p, (p.M + 32 * WM * TM - 1) / (32 * WM * TM), (p.N + 32 * WN * TN - 1) / (32 * WN * TN), {}, {}, 0};
    a.by_group = dg_make_div((uint32_t)GROUP * a.tiles_n);
    a.rest = a.tiles_m % GROUP ? a.tiles_m % GROUP : GROUP;
    a.by_rest = dg_make_div((uint32_t)a.rest);
    const uint32_t tiles = (uint32_t)a.tiles_m * a.tiles_n;
    const bool direct = p.K % 16 == 0 && p.stride_w % 16 == 0 && p.stride_a % 16 == 0 && (uintptr_t)p.W % 16 == 0 && (uintptr_t)p.A % 16 == 0 &&
                        p.stride_w < (1 << 22) && p.stride_a < (1 << 22);          // (a tile's rows lie within 2^30 bytes)
    if (direct) gemm_i8_tile_kernel<T, WM, WN, TM, TN, true><<<tiles, 64 * WM * WN, 0, stream>>>(a);
    else gemm_i8_tile_kernel<T, WM, WN, TM, TN, false><<<tiles, 64 * WM * WN, 0, stream>>>(a);
}

}   // namespace

dg_status dg_launch_quantize_tokens(const void *x, dg_dtype type, int64_t N, int64_t K, int64_t stride_n, int8_t *codes,
                                    int64_t stride_codes, float *scale, hipStream_t stream)
{
    dg_with_type(type, [&](auto t) {
        quantize_tokens_kernel<<<(uint32_t)N, 256, 0, stream>>>((const decltype(t) *)x, (int32_t)K, stride_n, codes, stride_codes, scale);
        return 0;
    });
    return dg_check_launch("dg_quantize_tokens");
}

dg_status dg_launch_gemm_i8(const DgGemmI8 &p, dg_dtype type, hipStream_t stream)
{
    dg_with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const uint32_t rows = (uint32_t)((p.M + 15) / 16);
        const auto tiles = [&](int64_t side) { return ((p.M + side - 1) / side) * ((p.N + side - 1) / side); };
        if (p.N <= 16) gemm_i8_few_kernel<T, 1><<<rows, 512, 0, stream>>>(p);
        else if (p.N <= 64) gemm_i8_few_kernel<T, 4><<<rows, 512, 0, stream>>>(p);
        else if (tiles(256) >= 192) launch_tiles<T, 2, 4, 4, 2>(p, stream);
        else if (tiles(128) >= 192) launch_tiles<T, 2, 2, 2, 2>(p, stream);
        else launch_tiles<T, 2, 2, 1, 1>(p, stream);
        return 0;
    });
    return dg_check_launch("dg_gemm_i8");
}
