// A router: logits in binary64, each token's largest choices, their weights.
#include "dg_decoder.h"

namespace {

typedef double v4d __attribute__((ext_vector_type(4)));

// ---- logits --------------------------------------------------------------------------------------------------------------
//
// Which experts a token goes to is decided by comparing sums that may lie as close as their rounding errors, and a choice that changes with the order of summation is
// another result, not one a little off.  In binary64 the products of 16- and 32-bit numbers are exact, and sums of thousands of them are good to 2^-50: rounded once to binary32
// they are the same whatever the order, but for sums within that of a border.
// v_mfma_f64_16x16x4f64: lane (r, g) holds number g of four of row r; sums 4 e + g (of 16 experts) of token r come out in a lane.  A lane loads eight neighbours, and number i of
// each lane's go into one instruction: any four positions may, as long as both operands take the same.

template <class X, class R, int WAVES, int BLOCKS>
__global__ __launch_bounds__(64 * WAVES) void route_logits_kernel(DgRoute p)
{
    __shared__ v4d sums[WAVES][BLOCKS][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t e0 = blockIdx.x * (16 * BLOCKS), t0 = blockIdx.y * 16;
    const X *x = (const X *)p.x + (int64_t)min(t0 + r, p.T - 1) * p.stride_x;
    const R *w[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) w[b] = (const R *)p.R + (int64_t)min(e0 + 16 * b + r, p.E - 1) * p.stride_r;
    v4d acc[BLOCKS] = {};
    for (int32_t k = 32 * wave; k < p.K; k += 32 * WAVES) {
        const DgVec<X, 8> xk = dg_eight<X>(x, k + 8 * g, p.K);
        DgVec<R, 8> wk[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) wk[b] = dg_eight<R>(w[b], k + 8 * g, p.K);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double xi = dg_to_float(xk.e[i]);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) acc[b] = __builtin_amdgcn_mfma_f64_16x16x4f64(dg_to_float(wk[b].e[i]), xi, acc[b], 0, 0, 0);
        }
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) sums[wave][b][lane] = acc[b];
    __syncthreads();
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        if (b % WAVES != wave) continue;
        v4d s = sums[0][b][lane];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) s += sums[i][b][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t e = e0 + 16 * b + 4 * i + g;
            if (e < p.E && t0 + r < p.T) p.logits[(int64_t)(t0 + r) * p.E + e] = (float)s[i];
        }
    }
}

// ---- choices -------------------------------------------------------------------------------------------------------------
//
// A wavefront a token, HELD experts a lane.  A choice as a number of 64 bits that orders as it does: the largest is found half by half, by register moves, its expert by a ballot.

__device__ __forceinline__ uint32_t most_of_wave(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false));       // row_mirror
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));        // quad_perm 1, 0, 3, 2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));        // quad_perm 2, 3, 0, 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));       // row_half_mirror
    const auto near = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(near[0], near[1]);
    const auto far = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(far[0], far[1]);
}

// 0 for -infinity, which is not taken.  (Adding 0 makes one zero of the two.)
__device__ __forceinline__ uint64_t key_of(double choice)
{
    const uint64_t bits = (uint64_t)__double_as_longlong(choice + 0.0);
    return choice == -__builtin_inf() ? 0 : bits ^ ((uint64_t)((int64_t)bits >> 63) | 0x8000000000000000ull);
}

template <int HELD, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void route_choose_kernel(DgRoute p, int64_t first)
{
    const int lane = threadIdx.x & 63;
    const int64_t t = first + (int64_t)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (t >= p.T) return;
    const float *row = p.logits + t * p.E;
    const float none = -__builtin_inff();
    float logit[HELD];
    uint64_t key[HELD];
    bool whole = true;
#pragma unroll
    for (int i = 0; i < HELD; ++i) logit[i] = lane + 64 * i < p.E ? row[lane + 64 * i] : none;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const bool there = lane + 64 * i < p.E;
        double choice = logit[i];
        if (p.mode == DG_ROUTE_SIGMOID) choice = 1.0 / (1.0 + exp(-choice));
        if (p.bias && there) choice += (double)p.bias[lane + 64 * i];
        whole = whole && (!there || (choice == choice && logit[i] == logit[i]));
        key[i] = there ? key_of(choice) : 0;
    }
    int32_t *ids = p.ids + t * p.top;
    float *weights = p.weights + t * p.top;
    if (__ballot(!whole)) {
        if (lane < p.top) {
            ids[lane] = lane;
            weights[lane] = __builtin_nanf("");
        }
        return;
    }
    int32_t mine = -1;                          // lane j: choice j
    float its = none;
    for (int32_t j = 0; j < p.top; ++j) {
        uint64_t best = key[0];
#pragma unroll
        for (int i = 1; i < HELD; ++i) best = max(best, key[i]);
        const uint32_t high = most_of_wave((uint32_t)(best >> 32));
        const uint32_t low = most_of_wave((uint32_t)(best >> 32) == high ? (uint32_t)best : 0u);
        const uint64_t most = (uint64_t)high << 32 | low;
        if (most == 0) break;
        bool found = false;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const uint64_t which = __ballot(key[i] == most);
            if (!found && which) {                              // (uniform; the lowest expert of those with this choice)
                const int from = __builtin_ctzll(which);
                const float l = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(logit[i]), from));
                if (lane == j) {
                    mine = from + 64 * i;
                    its = l;
                }
                if (lane == from) key[i] = 0;
                found = true;
            }
        }
    }
    float w = 0.0f;
    if (p.mode == DG_ROUTE_SIGMOID) {
        if (mine >= 0) w = 1.0f / (1.0f + expf(-its));
        const float sum = dg_over_wave(w, DgAdd());
        w = sum > 0.0f ? w / sum : 0.0f;
    } else {
        float most = its, sum;
        if (p.mode == DG_ROUTE_SOFTMAX_ALL) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) most = fmaxf(most, logit[i]);
        }
        most = dg_over_wave(most, DgMax());
        if (mine >= 0) w = expf(its - most);
        sum = w;
        if (p.mode == DG_ROUTE_SOFTMAX_ALL) {
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < HELD; ++i) sum += logit[i] == none ? 0.0f : expf(logit[i] - most);
        }
        sum = dg_over_wave(sum, DgAdd());
        w = mine >= 0 ? w / sum : 0.0f;
    }
    if (lane < p.top) {
        ids[lane] = mine;
        weights[lane] = w * p.factor;
    }
}

template <int HELD>
void choose(const DgRoute &p, hipStream_t stream)
{
    dg_in_turns(p.T, 1 << 24, [&](int64_t t, int64_t count) {
        route_choose_kernel<HELD, 4><<<(uint32_t)((count + 3) / 4), 256, 0, stream>>>(p, t);
        return DG_OK;
    });
}

template <class X, class R>
void logits(const DgRoute &p, hipStream_t stream)
{
    dg_in_turns(p.T, 16 * 65535, [&](int64_t t, int64_t count) {
        DgRoute part = p;
        part.x = (const X *)p.x + t * p.stride_x;
        part.logits += t * p.E;
        part.T = (int32_t)count;
        route_logits_kernel<X, R, 8, 1><<<dim3((p.E + 15) / 16, (uint32_t)((count + 15) / 16)), 512, 0, stream>>>(part);
        return DG_OK;
    });
}

}   // namespace

dg_status dg_launch_route(const DgRoute &p, dg_dtype x_type, dg_dtype r_type, hipStream_t stream)
{
    dg_with_type(x_type, [&](auto t) {
        typedef decltype(t) X;
        if (r_type == DG_F32) logits<X, float>(p, stream);
        else logits<X, X>(p, stream);
        return 0;
    });
    if (p.E <= 64) choose<1>(p, stream);
    else if (p.E <= 128) choose<2>(p, stream);
    else if (p.E <= 256) choose<4>(p, stream);
    else if (p.E <= 512) choose<8>(p, stream);
    else choose<16>(p, stream);
    return dg_check_launch("dg_route_tokens");
}
