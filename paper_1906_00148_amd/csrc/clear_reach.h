// What a token attends to of a row of a prefix's places and, behind them, its request's own (host and device).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace she { namespace clear {

// Lengths come from device memory and may be any numbers of 32 bits.  A place that they put further back than any table reaches is FAR, to which 1 can be added.
constexpr int FAR = 0x7FFFFFFE;
__host__ __device__ inline int as_place(int64_t at)
{
    return (int)(at < FAR ? at : FAR);
}

// The token has the place `place` (0 or more) of its request's own.  Of the prefix's places `own` have a column in its table and stand in the row, and
// `missing` that follow do not; they count for a window all the same.
__host__ __device__ inline int first_behind(int64_t place, uint32_t window, int own, int64_t missing)
{
    if (!window) return 0;
    const int64_t low = place - (int64_t)window + 1, before = low + own + missing;
    return as_place(low >= 0 ? low + own : before < own ? before < 0 ? 0 : before : own);
}
__host__ __device__ inline int last_behind(int64_t place, int own) { return as_place(place + own); }

}}  // namespace she::clear
