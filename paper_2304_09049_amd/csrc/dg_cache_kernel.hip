// The paged cache in 8 or 4 bits: new keys and values quantised as they are written, and read back.
#include "dg_decoder.h"

namespace {

struct WriteArgs {
    DgCache c;
    const void *k, *v;
    int64_t k_token, k_head, v_token, v_head;
    const int32_t *slots;
    int64_t T;
};

// Four consecutive tokens of a head make a group: a wavefront quantises it, 16 lanes a token (DIM / 16 channels each), for the keys and then for the values.
// Neighbouring lanes read neighbouring bytes.  A lane's keys are whole words of the cache.  A value's word in the cache is four tokens' bytes of one
// channel: where the group's slots are four in a row from a multiple of four, as a chunk of a prompt has them, the wavefront turns its 4 x DIM bytes over
// in LDS and stores words, side by side; a token by itself stores bytes.  (A lane a byte of two channels, one token a wavefront: 65536 tokens of 8 heads
// written and read back 596 us.)
// What a lane's PER channels of one token become: BYTES bytes, in 32-bit words, and the numbers.
template <class T, int BITS, int PER>
__device__ __forceinline__ void quantize_vector(const DgVec<T, PER> &x, uint32_t (&words)[(PER * BITS + 31) / 32], float &s, float &z)
{
    float lo = __builtin_inff(), hi = -__builtin_inff();
    bool finite = true;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float f = dg_to_float(x.e[i]);
        lo = fminf(lo, f);
        hi = fmaxf(hi, f);
        finite = finite && fabsf(f) < __builtin_inff();
    }
    // (an infinity where a value was none: a NaN compares false)
    lo = finite ? lo : -__builtin_inff();
#pragma unroll
    for (int i = 8; i; i >>= 1) {
        lo = fminf(lo, __shfl_xor(lo, i));
        hi = fmaxf(hi, __shfl_xor(hi, i));
    }
    const bool all = lo > -__builtin_inff();
    z = lo;
    if constexpr (BITS == 8) {
        s = all ? fmaxf(fabsf(lo), fabsf(hi)) / 127.0f : __builtin_nanf("");
        const DgDivisor by = dg_divisor(s);
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            int code[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) code[k] = dg_code8(dg_to_float(x.e[i + k]), by);
            words[i / 4] = (dg_bytes(code) & by.keep) ^ 0x80808080u;                 // (plus 128, byte by byte)
        }
    } else {
        s = all ? hi / 15.0f - lo / 15.0f : __builtin_nanf("");
        const DgDivisor by = dg_divisor(s);
        words[0] = 0;
        if constexpr (PER == 16) words[1] = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) words[i / 8] |= (uint32_t)(dg_code4(dg_to_float(x.e[i]), lo, by) & by.keep) << (4 * (i & 7));
    }
}

template <class T, int BITS, int DIM>
__global__ __launch_bounds__(256) void cache_write_kernel(WriteArgs a)
{
    constexpr int PER = DIM / 16, BYTES = PER * BITS / 8, WORDS = (BYTES + 3) / 4, STEP = DIM * BITS / 8;      // STEP: bytes of a token
    __shared__ __align__(16) uint8_t turned[4][4 * STEP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane & 15;
    const int64_t at = (int64_t)blockIdx.x * 4 + wave;
    if (at >= (a.T + 3) / 4 * a.c.heads) return;
    const int64_t group = at / a.c.heads, token = 4 * group + (lane >> 4);
    const int h = (int)(at % a.c.heads);
    const bool given = token < a.T;
    const int32_t slot = given ? a.slots[token] : -1;
    const bool there = slot >= 0 && slot < a.c.pages * a.c.page_size;
    const int64_t from = given ? token : a.T - 1;                                      // (a lane without a token reads the last one)
    const DgVec<T, PER> k = dg_load_vec<T, PER>((const T *)a.k + from * a.k_token + h * a.k_head + part * PER);
    const DgVec<T, PER> v = dg_load_vec<T, PER>((const T *)a.v + from * a.v_token + h * a.v_head + part * PER);
    const uint32_t place = there ? slot : 0, page = dg_fdiv(place, a.c.by_page), t = place - page * a.c.page_size;
    uint8_t *const block = a.c.base + page * a.c.page_bytes() + (int64_t)h * a.c.head;
    const int32_t first = __shfl(slot, 0);
    const bool whole = __all(there && slot == first + (lane >> 4)) && (first & 3) == 0;
    float *const numbers = (float *)(block + 2 * a.c.part) + t;
    uint32_t words[WORDS];
    float s, z;

    quantize_vector<T, BITS, PER>(k, words, s, z);
    if (there) {
        __builtin_memcpy(block + dg_key_byte<BITS>(t, part * PER, DIM), words, BYTES);
        if (part == 0) {
            numbers[0] = s;
            if (BITS == 4) numbers[2 * a.c.page_size] = z;
        }
    }
    quantize_vector<T, BITS, PER>(v, words, s, z);
    uint8_t *const values = block + a.c.part;
    if (there && part == 0) {
        numbers[a.c.page_size] = s;
        if (BITS == 4) numbers[3 * a.c.page_size] = z;
    }
    if (whole) {
        // token n's bytes in LDS, row n; word c of the cache: byte c of the four rows
        __builtin_memcpy(turned[wave] + (lane >> 4) * STEP + part * BYTES, words, BYTES);
        __builtin_amdgcn_wave_barrier();
        constexpr int MINE = STEP < 64 ? 1 : STEP / 64;                                // words a lane stores
        const int mine = min(lane, STEP / MINE - 1) * MINE;
        uint8_t row[4][MINE];
#pragma unroll
        for (int n = 0; n < 4; ++n) __builtin_memcpy(row[n], turned[wave] + n * STEP + mine, MINE);
        uint32_t out[MINE];
#pragma unroll
        for (int c = 0; c < MINE; ++c) out[c] = row[0][c] | row[1][c] << 8 | row[2][c] << 16 | (uint32_t)row[3][c] << 24;
        // (the first token's address: its lanes', the wavefront's first)
        const uint32_t first_t = __shfl(t, 0);
        if (STEP >= 64 || lane < STEP) __builtin_memcpy(values + (first_t >> 2) * (4 * STEP) + 4 * mine, out, 4 * MINE);
    } else if (there) {
#pragma unroll
        for (int i = 0; i < BYTES; ++i) values[(t >> 2) * (4 * STEP) + (part * BYTES + i) * 4 + (t & 3)] = (uint8_t)(words[i / 4] >> (8 * (i & 3)));
    }
}

struct ReadArgs {
    DgCache c;
    void *k, *v;
    const int32_t *slots;
    int64_t T;
};

// The same groups the other way round.
template <class T, int BITS, int DIM>
__global__ __launch_bounds__(256) void cache_read_kernel(ReadArgs a)
{
    constexpr int PER = DIM / 16, BYTES = PER * BITS / 8, WORDS = (BYTES + 3) / 4, STEP = DIM * BITS / 8;
    __shared__ __align__(16) uint8_t turned[4][4 * STEP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane & 15;
    const int64_t at = (int64_t)blockIdx.x * 4 + wave;
    if (at >= (a.T + 3) / 4 * a.c.heads) return;
    const int64_t group = at / a.c.heads, token = 4 * group + (lane >> 4);
    const int h = (int)(at % a.c.heads);
    const bool given = token < a.T;
    const int32_t slot = given ? a.slots[token] : -1;
    const bool there = slot >= 0 && slot < a.c.pages * a.c.page_size;
    const uint32_t place = there ? slot : 0, page = dg_fdiv(place, a.c.by_page), t = place - page * a.c.page_size;
    const uint8_t *const block = a.c.base + page * a.c.page_bytes() + (int64_t)h * a.c.head;
    const int32_t first = __shfl(slot, 0);
    const bool whole = __all(there && slot == first + (lane >> 4)) && (first & 3) == 0;
    const float *const numbers = (const float *)(block + 2 * a.c.part) + t;
    const auto put = [&](void *to, const uint32_t (&words)[WORDS], float s, float z) {
        DgVec<T, PER> x;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t code = words[i * BITS / 32] >> (i * BITS & 31) & (BITS == 8 ? 255 : 15);
            const float y = BITS == 8 ? (float)((int)code - 128) * s : (float)(int)code * s + z;
            x.e[i] = dg_from_float<T>(there ? y : 0.0f);
        }
        if (given) dg_store_vec<T, PER>((T *)to + (token * a.c.heads + h) * DIM + part * PER, x);
    };
    uint32_t words[WORDS] = {};
    if (a.k) {
        __builtin_memcpy(words, block + dg_key_byte<BITS>(t, part * PER, DIM), BYTES);
        put(a.k, words, numbers[0], BITS == 4 ? numbers[2 * a.c.page_size] : 0.0f);
    }
    if (!a.v) return;
    const uint8_t *const values = block + a.c.part;
    if (whole) {
        constexpr int MINE = STEP < 64 ? 1 : STEP / 64;
        const int mine = min(lane, STEP / MINE - 1) * MINE;
        uint32_t in[MINE];
        const uint32_t first_t = __shfl(t, 0);
        __builtin_memcpy(in, values + (first_t >> 2) * (4 * STEP) + 4 * mine, 4 * MINE);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            uint8_t row[MINE];
#pragma unroll
            for (int c = 0; c < MINE; ++c) row[c] = (uint8_t)(in[c] >> (8 * n));
            __builtin_memcpy(turned[wave] + n * STEP + mine, row, MINE);
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_memcpy(words, turned[wave] + (lane >> 4) * STEP + part * BYTES, BYTES);
    } else {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) words[i] = 0;
#pragma unroll
        for (int i = 0; i < BYTES; ++i) words[i / 4] |= (uint32_t)values[(t >> 2) * (4 * STEP) + (part * BYTES + i) * 4 + (t & 3)] << (8 * (i & 3));
    }
    put(a.v, words, numbers[a.c.page_size], BITS == 4 ? numbers[3 * a.c.page_size] : 0.0f);
}

// f(element type, bits, channels), the last two as constants
template <class F>
void with_form(const DgCache &c, dg_dtype type, F f)
{
    dg_with_type(type, [&](auto t) {
        auto by_dim = [&](auto bits) {
            switch (c.dim) {
            case 64: f(t, bits, std::integral_constant<int, 64>{}); break;
            case 128: f(t, bits, std::integral_constant<int, 128>{}); break;
            default: f(t, bits, std::integral_constant<int, 256>{}); break;
            }
        };
        if (c.bits == 8) by_dim(std::integral_constant<int, 8>{});
        else by_dim(std::integral_constant<int, 4>{});
        return 0;
    });
}

}   // namespace

dg_status dg_launch_cache_write(const DgCache &c, const void *k, const void *v, dg_dtype type, int64_t T, const int64_t strides[4],
                                const int32_t *slots, hipStream_t stream)
{
    const WriteArgs a = {c, k, v, strides[0], strides[1], strides[2], strides[3], slots, T};
    const uint32_t blocks = (uint32_t)(((T + 3) / 4 * c.heads + 3) / 4);
    with_form(c, type, [&](auto t, auto bits, auto dim) {
        cache_write_kernel<decltype(t), decltype(bits)::value, decltype(dim)::value><<<blocks, 256, 0, stream>>>(a);
    });
    return dg_check_launch("dg_cache_write");
}

dg_status dg_launch_cache_read(const DgCache &c, const int32_t *slots, int64_t T, void *k, void *v, dg_dtype type, hipStream_t stream)
{
    const ReadArgs a = {c, k, v, slots, T};
    const uint32_t blocks = (uint32_t)(((T + 3) / 4 * c.heads + 3) / 4);
    with_form(c, type, [&](auto t, auto bits, auto dim) {
        cache_read_kernel<decltype(t), decltype(bits)::value, decltype(dim)::value><<<blocks, 256, 0, stream>>>(a);
    });
    return dg_check_launch("dg_cache_read");
}
