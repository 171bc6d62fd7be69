// The paged cache in 8 or 4 bits: new keys and values quantised as they are written, and read back.
//
// 8 bits: s = max|x| / 127, code = rint(x / s), kept as code + 128; 4 bits: z = min, s = (max - min) / 15, code = rint((x - z) / s); rounded in binary32
// operation by operation (dg_decoder.h), so that a test can ask for the very bytes.  Bound by bytes where there are many tokens (65536 of 8 heads x 128 channels,
// 8 bits, written and read back: 177 us for 818 MB, 4.6 TB/s; 16384 of 8 heads x 256 channels 86 us, 4.7 TB/s, in 4 bits 84, 4.0; of 8 x 64 in 4 bits 31, 2.8),
// by two launches where there are few (32 tokens 7.4 us, 3.7 each).
#include "dg_decoder.h"

namespace {

struct WriteArgs {
    DgCache c;
    const void *k, *v;
    int64_t k_token, k_head, v_token, v_head;
    const int32_t *slots;
    int64_t T;
};

// A wavefront takes 64 / LANES consecutive tokens of a head, LANES lanes each: neighbouring lanes read neighbouring bytes.  A lane's keys are whole pieces
// of the cache, or halves.  A value's word in the cache is four tokens' bytes of one channel: where four tokens' slots follow one another from a
// multiple of four, the lanes of these four turn their 4 x DIM codes over by way of LDS and store words, side by side; other tokens store bytes.  So that a chunk
// of a prompt, which begins anywhere in a page, is mostly such fours, a wavefront leaves its last tokens to the next one if they share a word with that
// one's first (first_token).
// Eight lanes a token where there are many to write; sixteen, for wavefronts with less to do one after another, where there are few (`many`), and mostly to read.
template <int BITS, int DIM, int LANES>
struct Form {
    static constexpr int TOKENS = 64 / LANES, FOUR = 4 * LANES;          // lanes of four tokens
    static constexpr int PER = DIM / LANES;                              // channels of a lane
    static constexpr int STEP = DIM * BITS / 8;                          // bytes of a token
    static constexpr int BYTES = STEP / LANES, WORDS = (BYTES + 3) / 4;  // of a lane
    static constexpr int PIECE = (PER < 16 ? PER : 16) * BITS / 8;       // of a lane's keys that lie side by side
    static constexpr int MINE = STEP < FOUR ? 1 : STEP / FOUR;           // words of values that a lane stores, or reads, of four tokens
};

// A lane's channels of one token as codes, and the token's numbers.
template <class T, int BITS, int DIM, int LANES>
__device__ __forceinline__ void quantize_lane(const DgVec<T, DIM / LANES> &x, uint32_t (&words)[Form<BITS, DIM, LANES>::WORDS], float &s, float &z)
{
    constexpr int PER = DIM / LANES;
    float lo = __builtin_inff(), hi = BITS == 8 ? 0.0f : -__builtin_inff(), bad = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float f = dg_to_float(x.e[i]);
        if (BITS == 8) hi = fmaxf(hi, fabsf(f));
        else hi = fmaxf(hi, f), lo = fminf(lo, f);
        bad = __builtin_fmaf(f, 0.0f, bad);                   // (a NaN once there was an infinity or a NaN)
    }
    bad = bad == 0.0f ? 0.0f : 1.0f;
    hi = dg_over_lanes<LANES>(hi, DgMax());
    bad = dg_over_lanes<LANES>(bad, DgMax());
    if constexpr (BITS == 8) {
        s = bad == 0.0f ? hi / 127.0f : __builtin_nanf("");
        const DgDivisor by = dg_divisor(s);
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            int code[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) code[k] = dg_code8(dg_to_float(x.e[i + k]), by);
            words[i / 4] = (dg_bytes(code) & by.keep) ^ 0x80808080u;                 // (plus 128, byte by byte)
        }
        z = 0.0f;
    } else {
        lo = dg_over_lanes<LANES>(lo, DgMin());
        s = bad == 0.0f ? hi / 15.0f - lo / 15.0f : __builtin_nanf("");
        z = lo;
        const DgDivisor by = dg_divisor(s);
#pragma unroll
        for (int i = 0; i < PER; i += 8) {
            uint32_t w = 0;
#pragma unroll
            for (int k = 0; k < (PER < 8 ? PER : 8); ++k) w |= (uint32_t)dg_code4(dg_to_float(x.e[i + k]), lo, by) << (4 * k);
            words[i / 8] = w & by.keep;
        }
    }
}

// Four rows of MINE bytes <-> MINE words of one byte of each row.
template <int MINE>
__device__ __forceinline__ void turn(const uint32_t *in, uint32_t *out)
{
    if constexpr (MINE >= 4) {
#pragma unroll
        for (int k = 0; k < MINE / 4; ++k) {
            // (in: word k of rows 0 ... 3 at stride MINE / 4; out: four words)
            const uint32_t a = in[k], b = in[k + MINE / 4], c = in[k + 2 * (MINE / 4)], d = in[k + 3 * (MINE / 4)];
            const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
            const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
            out[4 * k] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
            out[4 * k + 1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
            out[4 * k + 2] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
            out[4 * k + 3] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
        }
    } else {
#pragma unroll
        for (int c = 0; c < MINE; ++c) {
            out[c] = 0;
#pragma unroll
            for (int n = 0; n < 4; ++n) out[c] |= (in[n] >> (8 * c) & 255u) << (8 * n);
        }
    }
}

// The first token of the wavefront whose tokens begin about token `base`: up to three before it, if these lie in one word of values with it.
__device__ __forceinline__ int64_t first_token(const int32_t *slots, int64_t T, int64_t base)
{
    const auto scalar = (const __attribute__((address_space(4))) int32_t *)slots;
    if (base >= T) return T;
    const int32_t slot = scalar[base], in_word = slot & 3;
    if (base < 3 || slot < 0) return base;
    const bool a = scalar[base - 1] == slot - 1, b = scalar[base - 2] == slot - 2, c = scalar[base - 3] == slot - 3;
    const bool together = in_word < 1 || (a && (in_word < 2 || (b && (in_word < 3 || c))));
    return together ? base - in_word : base;
}

// Where a lane's token lies, and whether it is one of four in a row of four.
struct Place {
    bool given, there, whole;
    uint32_t t, first_t;               // the token's, and the four's first one's, place in the page
    int64_t block;                     // the first byte of the page's head
};
template <int LANES>
__device__ __forceinline__ Place place_of(const DgCache &c, const int32_t *slots, int64_t token, int64_t end, int h, int lane)
{
    constexpr int FOUR = 4 * LANES;
    Place p;
    p.given = token < end;
    const int32_t slot = p.given ? slots[token] : -1;
    p.there = slot >= 0 && slot < c.pages * c.page_size;
    const uint32_t place = p.there ? slot : 0, page = dg_fdiv(place, c.by_page);
    p.t = place - page * c.page_size;
    p.block = page * c.page_bytes() + (int64_t)h * c.head;
    const int32_t first = FOUR == 64 || lane < 32 ? __builtin_amdgcn_readlane(slot, 0) : __builtin_amdgcn_readlane(slot, 32);
    const uint64_t in_row = __ballot(p.there && slot == first + (lane / LANES) % 4 && (first & 3) == 0);
    p.whole = FOUR == 64 ? in_row == ~0ull : (uint32_t)(lane < 32 ? in_row : in_row >> 32) == 0xFFFFFFFFu;
    p.first_t = p.t - (lane / LANES) % 4;
    return p;
}

template <class T, int BITS, int DIM, int LANES>
__global__ __launch_bounds__(256) void cache_write_kernel(WriteArgs a)
{
    typedef Form<BITS, DIM, LANES> F;
    __shared__ __align__(16) uint8_t turned[4][F::TOKENS * F::STEP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane % LANES, mine = lane % F::FOUR * F::MINE;
    const int64_t at = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + wave);
    if (at >= (a.T + F::TOKENS - 1) / F::TOKENS * a.c.heads) return;
    const int64_t base = at / a.c.heads * F::TOKENS, first = first_token(a.slots, a.T, base), end = first_token(a.slots, a.T, base + F::TOKENS);
    const int h = (int)(at % a.c.heads);
#pragma unroll 1
    for (int64_t token = first + lane / LANES; token - lane / LANES < end; token += F::TOKENS) {     // (once, but where a run of slots ends)
        const Place p = place_of<LANES>(a.c, a.slots, token, end, h, lane);
        const int64_t from = p.given ? token : end - 1;                                    // (a lane without a token reads the last one)
        const DgVec<T, F::PER> k = dg_load_vec<T, F::PER>((const T *)a.k + from * a.k_token + h * a.k_head + part * F::PER);
        const DgVec<T, F::PER> v = dg_load_vec<T, F::PER>((const T *)a.v + from * a.v_token + h * a.v_head + part * F::PER);
        uint8_t *const block = a.c.base + p.block;
        float *const numbers = (float *)(block + 2 * a.c.part) + p.t;
        uint32_t words[F::WORDS];
        float s, z;

        quantize_lane<T, BITS, DIM, LANES>(k, words, s, z);
        if (p.there) {
#pragma unroll
            for (int i = 0; i < F::BYTES / F::PIECE; ++i)
                __builtin_memcpy(block + dg_key_byte<BITS>(p.t, part * F::PER + 16 * i, DIM), (const uint8_t *)words + i * F::PIECE, F::PIECE);
            if (part == 0) {
                numbers[0] = s;
                if (BITS == 4) numbers[2 * a.c.page_size] = z;
            }
        }
        quantize_lane<T, BITS, DIM, LANES>(v, words, s, z);
        uint8_t *const values = block + a.c.part;
        if (p.there && part == 0) {
            numbers[a.c.page_size] = s;
            if (BITS == 4) numbers[3 * a.c.page_size] = z;
        }
        if (p.whole) {
            __builtin_memcpy(turned[wave] + (lane / LANES) * F::STEP + part * F::BYTES, words, F::BYTES);
            __builtin_amdgcn_wave_barrier();
            constexpr int ROW = (F::MINE + 3) / 4;                                         // words of a row
            uint32_t rows[4 * ROW] = {}, out[F::MINE];
            if (mine < F::STEP) {
#pragma unroll
                for (int n = 0; n < 4; ++n) __builtin_memcpy(rows + n * ROW, turned[wave] + (lane / F::FOUR * 4 + n) * F::STEP + mine, F::MINE);
                turn<F::MINE>(rows, out);
                __builtin_memcpy(values + (p.first_t >> 2) * (4 * F::STEP) + 4 * mine, out, 4 * F::MINE);
            }
        } else if (p.there) {
#pragma unroll
            for (int i = 0; i < F::BYTES; ++i) values[(p.t >> 2) * (4 * F::STEP) + (part * F::BYTES + i) * 4 + (p.t & 3)] = (uint8_t)(words[i / 4] >> (8 * (i & 3)));
        }
        __builtin_amdgcn_wave_barrier();
    }
}

struct ReadArgs {
    DgCache c;
    void *k, *v;
    const int32_t *slots;
    int64_t T;
};

// The same the other way round.
template <class T, int BITS, int DIM, int LANES>
__global__ __launch_bounds__(256) void cache_read_kernel(ReadArgs a)
{
    typedef Form<BITS, DIM, LANES> F;
    __shared__ __align__(16) uint8_t turned[4][F::TOKENS * F::STEP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane % LANES, mine = lane % F::FOUR * F::MINE;
    const int64_t at = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + wave);
    if (at >= (a.T + F::TOKENS - 1) / F::TOKENS * a.c.heads) return;
    const int64_t base = at / a.c.heads * F::TOKENS, first = first_token(a.slots, a.T, base), end = first_token(a.slots, a.T, base + F::TOKENS);
    const int h = (int)(at % a.c.heads);
#pragma unroll 1
    for (int64_t token = first + lane / LANES; token - lane / LANES < end; token += F::TOKENS) {
        const Place p = place_of<LANES>(a.c, a.slots, token, end, h, lane);
        const uint8_t *const block = a.c.base + p.block, *const values = block + a.c.part;
        const float *const numbers = (const float *)(block + 2 * a.c.part) + p.t;
        const auto put = [&](void *to, uint32_t (&words)[F::WORDS], float s, float z) {
            DgVec<T, F::PER> x;
            s = p.there ? s : 0.0f;
            z = p.there ? z : 0.0f;
#pragma unroll
            for (int i = 0; i < F::WORDS; ++i) words[i] = p.there ? words[i] : BITS == 8 ? 0x80808080u : 0u;
#pragma unroll
            for (int i = 0; i < F::PER; ++i) {
                const float code = (float)(words[i * BITS / 32] >> (i * BITS & 31) & (BITS == 8 ? 255u : 15u));
                x.e[i] = dg_from_float<T>(BITS == 8 ? (code - 128.0f) * s : code * s + z);
            }
            if (p.given) dg_store_vec<T, F::PER>((T *)to + (token * a.c.heads + h) * DIM + part * F::PER, x);
        };
        // everything is asked for before anything is waited for
        uint32_t keys[F::WORDS] = {}, words[F::WORDS] = {}, in[F::MINE] = {};
        float s[2] = {}, z[2] = {};
        if (a.k) {
#pragma unroll
            for (int i = 0; i < F::BYTES / F::PIECE; ++i)
                __builtin_memcpy((uint8_t *)keys + i * F::PIECE, block + dg_key_byte<BITS>(p.t, part * F::PER + 16 * i, DIM), F::PIECE);
            s[0] = numbers[0];
            if (BITS == 4) z[0] = numbers[2 * a.c.page_size];
        }
        if (a.v) {
            s[1] = numbers[a.c.page_size];
            if (BITS == 4) z[1] = numbers[3 * a.c.page_size];
            if (p.whole) {
                if (mine < F::STEP) __builtin_memcpy(in, values + (p.first_t >> 2) * (4 * F::STEP) + 4 * mine, 4 * F::MINE);
            } else {
#pragma unroll
                for (int i = 0; i < F::BYTES; ++i) words[i / 4] |= (uint32_t)values[(p.t >> 2) * (4 * F::STEP) + (part * F::BYTES + i) * 4 + (p.t & 3)] << (8 * (i & 3));
            }
        }
        if (a.k) put(a.k, keys, s[0], z[0]);
        if (!a.v) continue;
        if (p.whole) {
            constexpr int ROW = (F::MINE + 3) / 4;
            uint32_t rows[4 * ROW] = {};
            if constexpr (F::MINE >= 4) {
#pragma unroll
                for (int i = 0; i < F::MINE / 4; ++i) {
                    uint32_t four[4];
                    turn<4>(in + 4 * i, four);
#pragma unroll
                    for (int n = 0; n < 4; ++n) rows[n * ROW + i] = four[n];
                }
            } else {
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int c = 0; c < F::MINE; ++c) rows[n] |= (in[c] >> (8 * n) & 255u) << (8 * c);
            }
            if (mine < F::STEP)
#pragma unroll
                for (int n = 0; n < 4; ++n) __builtin_memcpy(turned[wave] + (lane / F::FOUR * 4 + n) * F::STEP + mine, rows + n * ROW, F::MINE);
            __builtin_amdgcn_wave_barrier();
            __builtin_memcpy(words, turned[wave] + (lane / LANES) * F::STEP + part * F::BYTES, F::BYTES);
        }
        put(a.v, words, s[1], z[1]);
        __builtin_amdgcn_wave_barrier();
    }
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

// Whether there are enough tokens to write for eight lanes each, which share a token's numbers among fewer (8 heads x 128 channels, 8 bits: 16384 tokens 21.4 us, by sixteen
// 25.1; 1024 3.85 either way; 256 3.6, by sixteen 3.2).
static bool many(int64_t T, int32_t heads) { return T * heads >= 8192; }

// Tokens a launch takes: whole eights, so that what a wavefront leaves to the next one stays with it, and at most 2^26 (token, head) rows, 16 threads each.
static int64_t tokens_a_launch(int32_t heads) { return std::max<int64_t>(((int64_t)1 << 26) / heads / 8 * 8, 8); }

dg_status dg_launch_cache_write(const DgCache &c, const void *k, const void *v, dg_dtype type, int64_t tokens, const int64_t strides[4],
                                const int32_t *slots, hipStream_t stream)
{
    const int64_t size = dg_type_size(type);
    dg_in_turns(tokens, tokens_a_launch(c.heads), [&](int64_t first, int64_t T) {
        const WriteArgs a = {c, (const uint8_t *)k + first * strides[0] * size, (const uint8_t *)v + first * strides[2] * size, strides[0], strides[1], strides[2], strides[3],
                             slots + first, T};
        with_form(c, type, [&](auto t, auto bits, auto dim) {
            constexpr int BITS = decltype(bits)::value, DIM = decltype(dim)::value;
            if (many(T, c.heads)) cache_write_kernel<decltype(t), BITS, DIM, 8><<<(uint32_t)(((T + 7) / 8 * c.heads + 3) / 4), 256, 0, stream>>>(a);
            else cache_write_kernel<decltype(t), BITS, DIM, 16><<<(uint32_t)(((T + 3) / 4 * c.heads + 3) / 4), 256, 0, stream>>>(a);
        });
        return DG_OK;
    });
    return dg_check_launch("dg_cache_write");
}

dg_status dg_launch_cache_read(const DgCache &c, const int32_t *slots, int64_t tokens, void *k, void *v, dg_dtype type, hipStream_t stream)
{
    const int64_t token = c.heads * c.dim * dg_type_size(type);
    dg_in_turns(tokens, tokens_a_launch(c.heads), [&](int64_t first, int64_t T) {
        const ReadArgs a = {c, k ? (uint8_t *)k + first * token : nullptr, v ? (uint8_t *)v + first * token : nullptr, slots + first, T};
        with_form(c, type, [&](auto t, auto bits, auto dim) {
            constexpr int BITS = decltype(bits)::value, DIM = decltype(dim)::value;
            // Sixteen lanes a token, which then store 16 bytes each side by side (16384 tokens x 8 heads x 128 channels, 8 bits 30 us, by eight 45; 4096 10.6,
            // 16.2); eight for many of 64 channels in 4 bits, where a lane of sixteen would have two bytes (16384 written and read 31.3 us, by sixteen 35.0).
            constexpr int LANES = BITS == 4 && DIM == 64 ? 8 : 16;
            if (many(T, c.heads)) cache_read_kernel<decltype(t), BITS, DIM, LANES><<<(uint32_t)(((T + 64 / LANES - 1) / (64 / LANES) * c.heads + 3) / 4), 256, 0, stream>>>(a);
            else cache_read_kernel<decltype(t), BITS, DIM, 16><<<(uint32_t)(((T + 3) / 4 * c.heads + 3) / 4), 256, 0, stream>>>(a);
        });
        return DG_OK;
    });
    return dg_check_launch("dg_cache_read");
}
