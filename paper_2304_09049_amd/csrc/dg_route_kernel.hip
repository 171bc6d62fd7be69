// A router: logits in binary64, each token's largest choices, their weights.
#include "dg_mx4.h"
#include "dg_route_rule.h"

namespace {

typedef double v4d __attribute__((ext_vector_type(4)));

constexpr int PARTS = DG_ROUTE_PARTS;

// ---- logits --------------------------------------------------------------------------------------------------------------
//
// Which experts a token goes to is decided by comparing sums that may lie as close as their rounding errors, and a choice that changes with the order of summation is
// another result, not one a little off.  In binary64 the products of 16- and 32-bit numbers are exact, and sums of thousands of them are good to 2^-50: rounded once to binary32
// they are the same whatever the order, but for sums within that of a border.
// v_mfma_f64_16x16x4f64: lane (r, g) holds number g of four of row r; sums 4 e + g (of 16 experts) of token r come out in a lane.  A lane loads eight neighbours, and number i of
// each lane's go into one instruction: any four positions may, as long as both operands take the same.

// Many tokens: 16 SIDE of them and 16 SIDE experts a workgroup, straight from memory, eight wavefronts sharing K, a step's loads under way while the one before is multiplied (2048 tokens
// of 4096 to 64 experts 34.7 -> 29.3 us with the choice).  With SIDE = 2 the matrix instruction bounds it, and what the address units take for loads of 16 rows (8192 tokens of 2048 to 128
// experts 78 us, 55 of the 70.8 TFLOP/s that a large binary64 matrix product reaches; with SIDE = 1 95); with SIDE = 1 and hundreds of tokens what a compute unit multiplies.  Tiles of 32 tokens and
// 128 experts staged in LDS took 75 us there, but 136 against 98 at 12000 tokens and up to four times as long where tokens are hundreds: few large tiles end in rounds that leave compute units without work.
template <class X, class R, int SIDE>
__global__ __launch_bounds__(512, 4) void route_many_kernel(DgRoute p)
{
    constexpr int WAVES = 8, COUNT = SIDE == 2 && sizeof(R) == 4 ? 4 : 8, EACH = 4 * COUNT;       // (a lane's neighbouring positions: with eight, two stages of binary32 rows do not fit into the registers)
    __shared__ v4d sums[WAVES][SIDE * SIDE][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t e0 = blockIdx.x * (16 * SIDE), t0 = blockIdx.y * (16 * SIDE);
    const int32_t share = (p.K + EACH * gridDim.z - 1) / (EACH * (int32_t)gridDim.z) * EACH, begin = blockIdx.z * share, end = min(p.K, begin + share);       // (whole steps, but for the last part's)
    const X *x[SIDE];
    const R *w[SIDE];
#pragma unroll
    for (int i = 0; i < SIDE; ++i) x[i] = (const X *)p.x + (int64_t)min(t0 + 16 * i + r, p.T - 1) * p.stride_x;
#pragma unroll
    for (int j = 0; j < SIDE; ++j) w[j] = (const R *)p.R + (int64_t)min(e0 + 16 * j + r, p.E - 1) * p.stride_r;
    v4d acc[SIDE * SIDE] = {};
    const auto load = [&](DgVec<X, COUNT> (&xk)[SIDE], DgVec<R, COUNT> (&wk)[SIDE], int32_t k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < SIDE; ++i) xk[i] = dg_load_vec<X, COUNT>(x[i] + k);
#pragma unroll
        for (int j = 0; j < SIDE; ++j) wk[j] = dg_load_vec<R, COUNT>(w[j] + k);
    };
    const auto add = [&](const DgVec<X, COUNT> (&xk)[SIDE], const DgVec<R, COUNT> (&wk)[SIDE]) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < COUNT; ++q) {
            double xq[SIDE], wq[SIDE];
#pragma unroll
            for (int i = 0; i < SIDE; ++i) xq[i] = dg_to_float(xk[i].e[q]);
#pragma unroll
            for (int j = 0; j < SIDE; ++j) wq[j] = dg_to_float(wk[j].e[q]);
#pragma unroll
            for (int i = 0; i < SIDE * SIDE; ++i) acc[i] = __builtin_amdgcn_mfma_f64_16x16x4f64(wq[i % SIDE], xq[i / SIDE], acc[i], 0, 0, 0);
        }
    };
    // (whole steps are loaded one ahead)
    constexpr int STEP = EACH * WAVES;
    DgVec<X, COUNT> xk[2][SIDE];
    DgVec<R, COUNT> wk[2][SIDE];
    int32_t k = begin + EACH * wave;
    if (k + EACH <= end) load(xk[0], wk[0], k + COUNT * g);
    while (k + EACH <= end) {
        if (k + STEP + EACH <= end) load(xk[1], wk[1], k + STEP + COUNT * g);
        __builtin_amdgcn_sched_barrier(0);
        add(xk[0], wk[0]);
        k += STEP;
        if (k + EACH > end) break;
        if (k + STEP + EACH <= end) load(xk[0], wk[0], k + STEP + COUNT * g);
        __builtin_amdgcn_sched_barrier(0);
        add(xk[1], wk[1]);
        k += STEP;
    }
    if (k < end) {                                                   // (one by one: unrolled it would take registers that the loop needs)
#pragma unroll 1
        for (int q = 0; q < COUNT; ++q) {
            const int32_t at = k + COUNT * g + q;
            double xq[SIDE], wq[SIDE];
#pragma unroll
            for (int i = 0; i < SIDE; ++i) xq[i] = at < end ? dg_to_float(x[i][at]) : 0.0f;
#pragma unroll
            for (int j = 0; j < SIDE; ++j) wq[j] = at < end ? dg_to_float(w[j][at]) : 0.0f;
#pragma unroll
            for (int i = 0; i < SIDE * SIDE; ++i) acc[i] = __builtin_amdgcn_mfma_f64_16x16x4f64(wq[i % SIDE], xq[i / SIDE], acc[i], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < SIDE * SIDE; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave >= SIDE * SIDE) return;
    v4d s = sums[0][wave][lane];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) s += sums[i][wave][lane];
    const int32_t t = t0 + 16 * (wave / SIDE) + r, e = e0 + 16 * (wave % SIDE) + g;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (e + 4 * i < p.E && t < p.T) {
            if (gridDim.z == 1) p.logits[(int64_t)t * p.E + e + 4 * i] = (float)s[i];
            else p.sums[((int64_t)blockIdx.z * p.T + t) * p.E + e + 4 * i] = s[i];
        }
}

// The sum over a wavefront's lanes, in each of them.
template <int CONTROL>
__device__ __forceinline__ double other_lane(double v)
{
    const uint64_t bits = (uint64_t)__double_as_longlong(v);
    const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CONTROL, 0xF, 0xF, false);
    const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), CONTROL, 0xF, 0xF, false);
    return __longlong_as_double((long long)((uint64_t)high << 32 | low));
}
__device__ __forceinline__ double sum_of_wave(double v)
{
    v += other_lane<0x140>(v);           // row_mirror
    v += other_lane<0xB1>(v);            // quad_perm 1, 0, 3, 2
    v += other_lane<0x4E>(v);            // quad_perm 2, 3, 0, 1
    v += other_lane<0x141>(v);           // row_half_mirror
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// Few tokens: a workgroup has an expert and TOKENS tokens, a lane eight neighbouring positions of 512 of a wavefront's.  One token of 4096 to 64 experts: 3.6 us, a launch and
// two waits.
template <class X, class R, int TOKENS>
__global__ __launch_bounds__(256) void route_few_kernel(DgRoute p)
{
    constexpr int WAVES = 4;
    __shared__ double sums[WAVES][TOKENS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t e = blockIdx.x, t0 = blockIdx.y * TOKENS;
    const R *w = (const R *)p.R + e * p.stride_r;
    const X *x[TOKENS];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) x[t] = (const X *)p.x + min(t0 + t, p.T - 1) * p.stride_x;
    double acc[TOKENS] = {};
    for (int64_t k = 8 * threadIdx.x; k < p.K; k += 512 * WAVES) {
        const DgVec<R, 8> wk = dg_eight<R>(w, (int32_t)k, p.K);
        DgVec<X, 8> xk[TOKENS];
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) xk[t] = dg_eight<X>(x[t], (int32_t)k, p.K);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double wi = dg_to_float(wk.e[i]);
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) acc[t] = __builtin_fma(wi, (double)dg_to_float(xk[t].e[i]), acc[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        const double s = sum_of_wave(acc[t]);
        if (lane == 0) sums[wave][t] = s;
    }
    __syncthreads();
    const int t = threadIdx.x;
    if (t < TOKENS && t0 + t < p.T) p.logits[(int64_t)(t0 + t) * p.E + e] = (float)(sums[0][t] + sums[1][t] + sums[2][t] + sums[3][t]);
}

// ---- choices -------------------------------------------------------------------------------------------------------------
//
// A wavefront a token, HELD experts a lane.  A choice as a number of 64 bits that orders as it does: the largest is found half by half, by register moves, its expert by a ballot.
// 8192 tokens to 8 of 128 9.6 us, vector instructions half of the cycles (exp in binary64 for the sigmoids, and some 40 a choice); one token 2.6.

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

template <int HELD, int WAVES, bool PARTED>
__global__ __launch_bounds__(64 * WAVES) void route_choose_kernel(DgRoute p, int64_t first)
{
    const int lane = threadIdx.x & 63;
    const int64_t t = first + (int64_t)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (t >= p.T) return;
    const float none = -__builtin_inff();
    float logit[HELD];
    uint64_t key[HELD];
    bool whole = true;
    if (PARTED) {
        double part[HELD][PARTS];
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int k = 0; k < PARTS; ++k) part[i][k] = lane + 64 * i < p.E ? p.sums[((int64_t)k * p.T + t) * p.E + lane + 64 * i] : 0.0;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            double sum = part[i][0];
#pragma unroll
            for (int k = 1; k < PARTS; ++k) sum += part[i][k];
            logit[i] = lane + 64 * i < p.E ? (float)sum : none;
        }
    } else {
        const float *row = p.logits + t * p.E;
#pragma unroll
        for (int i = 0; i < HELD; ++i) logit[i] = lane + 64 * i < p.E ? row[lane + 64 * i] : none;
    }
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
        if (__ballot(mine >= 0 && its < -80.0f)) {
            // (exp(88.8) is past binary32; below -87 a sigmoid has fewer bits)
            const double chance = mine >= 0 ? 1.0 / (1.0 + exp(-(double)its)) : 0.0, sum = sum_of_wave(chance);
            w = sum > 0.0 ? (float)(chance / sum) : 0.0f;
        } else {
            if (mine >= 0) w = 1.0f / (1.0f + expf(-its));
            const float sum = dg_over_wave(w, DgAdd());
            w = sum > 0.0f ? w / sum : 0.0f;
        }
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
void choose(const DgRoute &p, bool parted, hipStream_t stream)
{
    dg_in_turns(p.T, 1 << 24, [&](int64_t t, int64_t count) {
        const uint32_t grid = (uint32_t)((count + 3) / 4);
        if (parted) route_choose_kernel<HELD, 4, true><<<grid, 256, 0, stream>>>(p, t);
        else route_choose_kernel<HELD, 4, false><<<grid, 256, 0, stream>>>(p, t);
        return DG_OK;
    });
}

template <class X, class R>
bool logits(const DgRoute &p, hipStream_t stream)
{
    const int64_t units = dg_simd_count() / 4;
    const bool parted = dg_route_form(p.T, p.E, p.K, units) == DgRouteForm::Parts16;
    dg_in_turns(p.T, 16 * 65535, [&](int64_t t, int64_t count) {
        DgRoute part = p;
        part.x = (const X *)p.x + t * p.stride_x;
        if (!parted) part.logits += t * p.E;                        // (parts are of one turn)
        part.T = (int32_t)count;
        const dim3 tiles16((p.E + 15) / 16, (uint32_t)((count + 15) / 16), parted ? PARTS : 1);
        switch (dg_route_form(count, p.E, p.K, units)) {
        case DgRouteForm::One: route_few_kernel<X, R, 1><<<p.E, 256, 0, stream>>>(part); break;
        case DgRouteForm::Four: route_few_kernel<X, R, 4><<<dim3(p.E, (uint32_t)((count + 3) / 4)), 256, 0, stream>>>(part); break;
        case DgRouteForm::Tiles32: route_many_kernel<X, R, 2><<<dim3((p.E + 31) / 32, (uint32_t)((count + 31) / 32)), 512, 0, stream>>>(part); break;
        case DgRouteForm::Tiles16:
        case DgRouteForm::Parts16: route_many_kernel<X, R, 1><<<tiles16, 512, 0, stream>>>(part); break;
        }
        return DG_OK;
    });
    return parted;
}

}   // namespace

dg_status dg_launch_route(const DgRoute &p, dg_dtype x_type, dg_dtype r_type, hipStream_t stream)
{
    bool parted = false;
    dg_with_type(x_type, [&](auto t) {
        typedef decltype(t) X;
        parted = r_type == DG_F32 ? logits<X, float>(p, stream) : logits<X, X>(p, stream);
        return 0;
    });
    if (p.E <= 64) choose<1>(p, parted, stream);
    else if (p.E <= 128) choose<2>(p, parted, stream);
    else if (p.E <= 256) choose<4>(p, parted, stream);
    else if (p.E <= 512) choose<8>(p, parted, stream);
    else choose<16>(p, parted, stream);
    return dg_check_launch("dg_route_tokens");
}
