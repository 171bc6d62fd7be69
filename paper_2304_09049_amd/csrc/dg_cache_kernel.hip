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

// A wavefront per (token, head): lane l holds channels DIM / 64 * l ...
template <class T, int BITS, int DIM>
__global__ __launch_bounds__(256) void cache_write_kernel(WriteArgs a)
{
    constexpr int PER = DIM / 32;                                     // channels per lane (the upper 32 lanes take the values)
    const int lane = threadIdx.x & 63;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= a.T * a.c.heads) return;
    const int64_t token = at / a.c.heads;
    const int h = (int)(at % a.c.heads);
    const int32_t slot = a.slots[token];
    if (slot < 0 || slot >= (int64_t)a.c.pages * a.c.page_size) return;
    const uint32_t page = dg_fdiv((uint32_t)slot, a.c.by_page), t = (uint32_t)slot - page * a.c.page_size;
    uint8_t *block = a.c.base + page * a.c.page_bytes() + (int64_t)h * a.c.head;

    const bool values = lane >= 32;
    const int d = (lane & 31) * PER;
    const T *row = values ? (const T *)a.v + token * a.v_token + h * a.v_head : (const T *)a.k + token * a.k_token + h * a.k_head;
    const DgVec<T, PER> x = dg_load_vec<T, PER>(row + d);
    float lo = __builtin_inff(), hi = -__builtin_inff();
    bool finite = true;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float f = dg_to_float(x.e[i]);
        lo = fminf(lo, f);
        hi = fmaxf(hi, f);
        finite = finite && fabsf(f) < __builtin_inff();
    }
#pragma unroll
    for (int i = 16; i; i >>= 1) {
        lo = fminf(lo, __shfl_xor(lo, i));
        hi = fmaxf(hi, __shfl_xor(hi, i));
        finite = __shfl_xor((int)finite, i) && finite;
    }
    float *numbers = (float *)(block + 2 * a.c.part) + t;
    uint8_t *codes = block + (values ? a.c.part : 0);
    if constexpr (BITS == 8) {
        const float s = finite ? dg_scale8(fmaxf(fabsf(lo), fabsf(hi))) : __builtin_nanf("");
        const DgDivisor by = dg_divisor(s);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint8_t code = (uint8_t)((dg_code8(dg_to_float(x.e[i]), by) & by.keep) + 128);
            codes[values ? dg_value_byte<8>(t, d + i, DIM) : dg_key_byte<8>(t, d + i, DIM)] = code;
        }
        if ((lane & 31) == 0) numbers[values ? a.c.page_size : 0] = s;
    } else {
        const float s = finite ? hi / 15.0f - lo / 15.0f : __builtin_nanf("");
        const DgDivisor by = dg_divisor(s);
#pragma unroll
        for (int i = 0; i < PER; i += 2) {
            const int low = dg_code4(dg_to_float(x.e[i]), lo, by) & by.keep, high = dg_code4(dg_to_float(x.e[i + 1]), lo, by) & by.keep;
            codes[values ? dg_value_byte<4>(t, d + i, DIM) : dg_key_byte<4>(t, d + i, DIM)] = (uint8_t)(low | high << 4);
        }
        if ((lane & 31) == 0) {
            numbers[values ? a.c.page_size : 0] = s;
            numbers[(values ? 3 : 2) * a.c.page_size] = lo;
        }
    }
}

struct ReadArgs {
    DgCache c;
    void *k, *v;
    const int32_t *slots;
    int64_t T;
};

template <class T, int BITS, int DIM>
__global__ __launch_bounds__(256) void cache_read_kernel(ReadArgs a)
{
    constexpr int PER = DIM / 32;
    const int lane = threadIdx.x & 63;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= a.T * a.c.heads) return;
    const int h = (int)(at % a.c.heads);
    const bool values = lane >= 32;
    T *out = (T *)(values ? a.v : a.k);
    if (!out) return;
    const int d = (lane & 31) * PER;
    out += at * DIM + d;
    const int32_t slot = a.slots[at / a.c.heads];
    DgVec<T, PER> x = {};
    if (slot >= 0 && slot < (int64_t)a.c.pages * a.c.page_size) {
        const uint32_t page = dg_fdiv((uint32_t)slot, a.c.by_page), t = (uint32_t)slot - page * a.c.page_size;
        const uint8_t *block = a.c.base + page * a.c.page_bytes() + (int64_t)h * a.c.head;
        const uint8_t *codes = block + (values ? a.c.part : 0);
        const float *numbers = (const float *)(block + 2 * a.c.part) + t;
        const float s = numbers[values ? a.c.page_size : 0];
        if constexpr (BITS == 8) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int code = codes[values ? dg_value_byte<8>(t, d + i, DIM) : dg_key_byte<8>(t, d + i, DIM)];
                x.e[i] = dg_from_float<T>((float)(code - 128) * s);
            }
        } else {
            const float z = numbers[(values ? 3 : 2) * a.c.page_size];
#pragma unroll
            for (int i = 0; i < PER; i += 2) {
                const int two = codes[values ? dg_value_byte<4>(t, d + i, DIM) : dg_key_byte<4>(t, d + i, DIM)];
                x.e[i] = dg_from_float<T>((float)(two & 15) * s + z);
                x.e[i + 1] = dg_from_float<T>((float)(two >> 4) * s + z);
            }
        }
    }
    dg_store_vec<T, PER>(out, x);
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
    const uint32_t blocks = (uint32_t)((T * c.heads + 3) / 4);
    with_form(c, type, [&](auto t, auto bits, auto dim) {
        cache_write_kernel<decltype(t), decltype(bits)::value, decltype(dim)::value><<<blocks, 256, 0, stream>>>(a);
    });
    return dg_check_launch("dg_cache_write");
}

dg_status dg_launch_cache_read(const DgCache &c, const int32_t *slots, int64_t T, void *k, void *v, dg_dtype type, hipStream_t stream)
{
    const ReadArgs a = {c, k, v, slots, T};
    const uint32_t blocks = (uint32_t)((T * c.heads + 3) / 4);
    with_form(c, type, [&](auto t, auto bits, auto dim) {
        cache_read_kernel<decltype(t), decltype(bits)::value, decltype(dim)::value><<<blocks, 256, 0, stream>>>(a);
    });
    return dg_check_launch("dg_cache_read");
}
