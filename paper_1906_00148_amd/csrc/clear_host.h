// What the host files of the clear calls share (she_clear.cpp has it): checks of the context, its counter and its scratch.
#pragma once
#include "clear_internal.h"
#include "she_ctx.h"

namespace she { namespace clear {

// so that no grid has more than 2^32 threads along one axis
constexpr uint64_t MOST_TOKENS = 1u << 24, MOST_SEGMENTS = 1u << 20, MOST_WIDTH = 1u << 24, MOST_PLACES = 1u << 26, MOST_GROUPS = 1u << 24;

int ready(she_ctx *c);                                  // the context's device is the current one, and its counter is there
int ensure_scratch(she_ctx *c, size_t bytes);
inline bool half_type(int32_t t) { return t == SHE_BF16 || t == SHE_F16; }
inline bool on16(const void *p) { return ((uintptr_t)p & 15) == 0; }

}}  // namespace she::clear
