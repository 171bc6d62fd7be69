// What the kernels that multiply microscaled 4-bit rows share: loads of such rows by way of LDS.
#pragma once

#include "dg_decoder.h"
#include "dg_lds_dma.h"

constexpr uint32_t DG_NOWHERE = 0xF0000000u;             // an offset that no buffer has: loads from there are zeros

// `have` rows from `first` on, of which `bytes` can be read.
__device__ __forceinline__ dg_v4i dg_rows_buffer(const uint8_t *rows, int64_t first, int64_t stride, int32_t have, int32_t bytes)
{
    return dg_buffer(rows + first * stride, (uint32_t)((have - 1) * (uint32_t)stride + bytes));
}

// 8 or 16 bytes to memory past the caches.
template <class T, int COUNT>
__device__ __forceinline__ void dg_store_past(T *to, const DgVec<T, COUNT> &v)
{
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(v) / 4)));
    typedef words anywhere __attribute__((aligned(2)));
    words w;
    __builtin_memcpy(&w, &v, sizeof(v));
    __builtin_nontemporal_store(w, (anywhere *)to);
}
// dg_load16_to_lds of what is not read again.
__device__ __forceinline__ void dg_load16_once_to_lds(const dg_v4i &buffer, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen nt lds" :: "v"(offset), "s"(buffer), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory", "m0");
}
