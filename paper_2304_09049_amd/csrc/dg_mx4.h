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
