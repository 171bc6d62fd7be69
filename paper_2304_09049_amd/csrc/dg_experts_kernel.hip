// The gated feed-forward of chosen experts, weights in microscaled 4-bit floating point, for few tokens.
//
// Two products with what each expert's tokens have of x, and of h between them.  A (token, choice) is a pair; an expert's pairs are the columns of its products.  Few tokens: the
// experts' weights are read once for all their pairs, and that is what bounds it, so activations stay as they are: weights become bfloat16 on their way into the matrix
// instruction (exactly: two bits and a power of two), x is bfloat16 or two of them (binary16's eleven bits), h is held as two, 2^-17 off at most.
#include "dg_decoder.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

constexpr int MOST_PAIRS = 4096;         // of a turn: their numbers lie in LDS
constexpr int MOST_TOKENS = 256;

// ---- what both products share --------------------------------------------------------------------------------------------

// One block of 32 weights as a lane holds it: 16 bytes and a scale; the eight weights of word i as an operand.
struct Block {
    v4i codes;
    uint32_t byte;
};
__device__ __forceinline__ v8b weights_of(const Block &w, int i)
{
    const float s = dg_mx_scale(w.byte);
    const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w.codes[i], s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w.codes[i], s, 1);
    const v2b c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w.codes[i], s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w.codes[i], s, 3);
    return (v8b){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Block b of a row of `blocks`; past them zeros.
__device__ __forceinline__ Block block_or_zero(const uint8_t *codes, const uint8_t *scales, int32_t b, int32_t blocks)
{
    Block w = {{}, 0};
    if (b < blocks) {
        w.codes = *(const v4i *)(codes + 16 * b);
        w.byte = scales[b];
    }
    return w;
}

__device__ __forceinline__ v4f multiply(const v8b &w, const v8b &x, const v4f &c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0); }

// The number as two: what bfloat16 holds of it, and what bfloat16 holds of the rest.
__device__ __forceinline__ void split(float f, __bf16 &high, __bf16 &low)
{
    high = (__bf16)f;
    low = fabsf((float)high) < __builtin_inff() ? (__bf16)(f - (float)high) : (__bf16)0.0f;
}

// An expert's pairs, in order, and how many; `pairs` numbers in LDS.  A workgroup has slot `slot`: with fewer pairs than experts that is a pair, whose expert it takes unless an
// earlier pair names it too, otherwise an expert.  -1: nothing to do.
template <int WAVES>
__device__ __forceinline__ int32_t find_pairs(const DgExperts &p, int32_t slot, uint16_t *list, int32_t &count)
{
    __shared__ int32_t counted;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t pairs = p.T * p.top;
    const bool by_pair = pairs < p.d.experts;
    const int32_t expert = by_pair ? p.ids[slot] : slot;
    if ((uint32_t)expert >= (uint32_t)p.d.experts) return -1;
    if (wave == 0) {
        int32_t n = 0;
        bool first = true;
        for (int32_t at = 0; at < pairs; at += 64) {
            const uint64_t which = __ballot(at + lane < pairs && p.ids[at + lane] == expert);
            if (which >> lane & 1) list[n + __builtin_popcountll(which & ((1ull << lane) - 1))] = (uint16_t)(at + lane);
            if (by_pair && n == 0 && which) first = at + __builtin_ctzll(which) == slot;
            n += __builtin_popcountll(which);
        }
        if (lane == 0) counted = first ? n : 0;
    }
    __syncthreads();
    count = counted;
    return count ? expert : -1;
}

struct Work {
    __bf16 *h;               // [2][pairs][pitch]
    float *y;                // [pairs][hidden]
    int32_t pitch;           // inner rounded up to 128; zeros from inner on
};

// ---- gate and other, and what becomes of them ----------------------------------------------------------------------------

template <class T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void experts_up_kernel(DgExperts p, Work work)
{
    __shared__ uint16_t list[MOST_PAIRS];
    __shared__ v4f sums[WAVES][2][64];
    int32_t count;
    const int32_t expert = find_pairs<WAVES>(p, blockIdx.y, list, count);
    if (expert < 0) return;
    constexpr bool TWO = !std::is_same<T, __bf16>::value;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t f0 = blockIdx.x * 16, K = p.d.hidden, blocks = (K + 31) / 32, last = p.d.inner - 1, pairs = p.T * p.top;
    const uint8_t *codes[2], *scales[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t row = min(f0 + r, last) + i * p.d.inner;
        codes[i] = p.d.up + expert * p.d.up_expert + row * p.d.up_row;
        scales[i] = p.d.up_scales + expert * p.d.up_scales_expert + row * p.d.up_scales_row;
    }
    for (int32_t column = 0; column < count; column += 16) {
        const int32_t pair = list[min(column + r, count - 1)];
        const T *x = (const T *)p.x + (pair / p.top) * p.stride_x;
        v4f acc[2] = {};
        for (int32_t b = 4 * wave; b < blocks; b += 4 * WAVES) {
            Block w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] = block_or_zero(codes[i], scales[i], b + g, blocks);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const DgVec<T, 8> at = dg_eight<T>(x, 32 * (b + g) + 8 * j, K);
                v8b high, low;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    __bf16 a, c;
                    split(dg_to_float(at.e[e]), a, c);
                    high[e] = a;
                    low[e] = c;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const v8b wk = weights_of(w[i], j);
                    acc[i] = multiply(wk, high, acc[i]);
                    if (TWO) acc[i] = multiply(wk, low, acc[i]);
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) sums[wave][i][lane] = acc[i];
        __syncthreads();
        if (wave == 0 && column + r < count) {
            v4f gate = sums[0][0][lane], other = sums[0][1][lane];
#pragma unroll
            for (int k = 1; k < WAVES; ++k) {
                gate += sums[k][0][lane];
                other += sums[k][1][lane];
            }
            DgVec<__bf16, 4> high, low;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float h = gate[e] / (1.0f + expf(-gate[e])) * other[e];
                split(f0 + 4 * g + e <= last ? h : 0.0f, high.e[e], low.e[e]);
            }
            __bf16 *to = work.h + (int64_t)pair * work.pitch + f0 + 4 * g;
            dg_store_vec<__bf16, 4>(to, high);
            dg_store_vec<__bf16, 4>(to + (int64_t)pairs * work.pitch, low);
        }
    }
}

// ---- down ----------------------------------------------------------------------------------------------------------------

template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void experts_down_kernel(DgExperts p, Work work)
{
    __shared__ uint16_t list[MOST_PAIRS];
    __shared__ v4f sums[WAVES][64];
    int32_t count;
    const int32_t expert = find_pairs<WAVES>(p, blockIdx.y, list, count);
    if (expert < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t m0 = blockIdx.x * 16, blocks = (p.d.inner + 31) / 32, last = p.d.hidden - 1, pairs = p.T * p.top;
    const int64_t row = min(m0 + r, last);
    const uint8_t *codes = p.d.down + expert * p.d.down_expert + row * p.d.down_row;
    const uint8_t *scales = p.d.down_scales + expert * p.d.down_scales_expert + row * p.d.down_scales_row;
    for (int32_t column = 0; column < count; column += 16) {
        const int32_t pair = list[min(column + r, count - 1)];
        const __bf16 *h = work.h + (int64_t)pair * work.pitch;
        v4f acc = {};
        for (int32_t b = 4 * wave; b < blocks; b += 4 * WAVES) {
            const Block w = block_or_zero(codes, scales, b + g, blocks);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v8b high, low;
                __builtin_memcpy(&high, h + 32 * (b + g) + 8 * j, 16);
                __builtin_memcpy(&low, h + (int64_t)pairs * work.pitch + 32 * (b + g) + 8 * j, 16);
                const v8b wk = weights_of(w, j);
                acc = multiply(wk, high, acc);
                acc = multiply(wk, low, acc);
            }
        }
        __syncthreads();
        sums[wave][lane] = acc;
        __syncthreads();
        if (wave == 0 && column + r < count) {
            v4f s = sums[0][lane];
#pragma unroll
            for (int k = 1; k < WAVES; ++k) s += sums[k][lane];
            float *to = work.y + (int64_t)pair * p.d.hidden + m0 + 4 * g;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (m0 + 4 * g + e <= last) to[e] = s[e];
        }
    }
}

// ---- a token's choices together, in their order ----------------------------------------------------------------------------

template <class T>
__global__ __launch_bounds__(256) void experts_join_kernel(DgExperts p, Work work)
{
    const int32_t m = (blockIdx.x * 256 + threadIdx.x) * 4, t = blockIdx.y, have = min(p.d.hidden - m, 4);
    if (have <= 0) return;
    float sum[4] = {};
    for (int32_t j = 0; j < p.top; ++j) {
        const int32_t pair = t * p.top + j;
        if ((uint32_t)p.ids[pair] >= (uint32_t)p.d.experts) continue;
        const float w = p.weights[pair], *y = work.y + (int64_t)pair * p.d.hidden + m;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) sum[e] += w * y[e];
    }
    T *out = (T *)p.out + t * p.stride_out + m;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < have) out[e] = dg_from_float<T>(sum[e]);
}

int64_t turn_of(int64_t T, int64_t top) { return std::min({T, (int64_t)MOST_TOKENS, MOST_PAIRS / top}); }
int64_t pitch_of(int64_t inner) { return (inner + 127) / 128 * 128; }

template <class T>
void launch(const DgExperts &p, hipStream_t stream)
{
    const int64_t pairs = (int64_t)p.T * p.top;
    const int32_t pitch = (int32_t)pitch_of(p.d.inner);
    const Work work = {(__bf16 *)p.work, (float *)((__bf16 *)p.work + 2 * pairs * pitch), pitch};
    const uint32_t slots = (uint32_t)std::min<int64_t>(pairs, p.d.experts);
    experts_up_kernel<T, 8><<<dim3(pitch / 16, slots), 512, 0, stream>>>(p, work);
    experts_down_kernel<8><<<dim3((p.d.hidden + 15) / 16, slots), 512, 0, stream>>>(p, work);
    experts_join_kernel<T><<<dim3((p.d.hidden + 1023) / 1024, p.T), 256, 0, stream>>>(p, work);
}

}   // namespace

int64_t dg_experts_work_bytes(int64_t T, int64_t top, int64_t hidden, int64_t inner) { return turn_of(T, top) * top * (4 * pitch_of(inner) + 4 * ((hidden + 3) / 4 * 4)); }

dg_status dg_launch_experts(const DgExperts &all, dg_dtype type, hipStream_t stream)
{
    dg_in_turns(all.T, turn_of(all.T, all.top), [&](int64_t t, int64_t count) {
        DgExperts p = all;
        p.x = (const uint8_t *)p.x + 2 * t * p.stride_x;
        p.out = (uint8_t *)p.out + 2 * t * p.stride_out;
        p.ids += t * p.top;
        p.weights += t * p.top;
        p.T = (int32_t)count;
        if (type == DG_F16) launch<_Float16>(p, stream);
        else launch<__bf16>(p, stream);
        return DG_OK;
    });
    return dg_check_launch("dg_experts_mx4");
}
