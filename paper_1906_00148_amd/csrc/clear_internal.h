// Launchers of the clear side's kernels (she_clear.h) and what their host and device code share (internal).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/she_clear.h"

namespace she { namespace clear {

// Beside the count of bad ids the context keeps a unit of zeros, for kernels that bring tiles with holes.
constexpr uint32_t COUNTERS = 8, ZEROS_AT = 4;   // words of that memory, and where the unit starts
inline const void *zeros_of(const uint32_t *d_bad) { return d_bad + ZEROS_AT; }

inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// ---- queries and keys
struct QkShape {
    uint32_t lanes;          // lanes that hold a head, eight elements each: 8, 16, 32 or 64
    uint32_t heads;          // rows of a token: queries, keys and, with pages, values
    uint32_t steps;          // of 64 / lanes rows each, that a token's rows take
    uint32_t per_wave;       // steps that a wavefront does for one token
    uint32_t chunks;         // wavefronts' shares of a token
    uint32_t blocks;
    bool wide;               // every row starts on 16 bytes and has whole vectors
    bool aligned;            // and so do a lane's cosines and sines
};
QkShape qk_shape(const she_qk_rotate_args &a, uint32_t cus);
struct QkGradShape {
    uint32_t lanes;
    bool wide, aligned;
    QkShape q, k;            // their heads, steps, shares and workgroups
};
QkGradShape qk_grad_shape(const she_qk_rotate_grad_args &a, uint32_t cus);
size_t qk_grad_scratch(const QkGradShape &s, uint32_t head);
hipError_t launch_qk_rotate(const she_qk_rotate_args &a, const QkShape &s, uint32_t *d_bad, hipStream_t st);
hipError_t launch_qk_rotate_grad(const she_qk_rotate_grad_args &a, const QkGradShape &s, void *scratch, uint32_t *d_bad, hipStream_t st);

// ---- adapters
size_t adapters_scratch(const she_adapters_args &a);
size_t adapters_grad_scratch(const she_adapters_grad_args &a);
hipError_t launch_adapters(const she_adapters_args &a, void *scratch, uint32_t *d_bad, uint32_t cus, hipStream_t st);
hipError_t launch_adapters_grad(const she_adapters_grad_args &a, void *scratch, uint32_t *d_bad, uint32_t cus, hipStream_t st);

// ---- attention
// Rows of a workgroup of either kernel, places that k_attend_few looks up together at most, places of a step of k_attend_tile.
constexpr int FEW_ROWS = 16, TILE_ROWS = 128, MOST_CHUNK = 2048, STEP = 64;
struct AttendShape {
    bool few;                            // the kernel for few rows, and not that for many
    uint64_t slots;                      // tiles of rows, at most
    uint32_t chunk;                      // places of the cache that a workgroup walks
    uint32_t splits;                     // workgroups that share a tile's places, at most
};
AttendShape attend_shape(const she_attend_pages_args &a, uint32_t cus);
size_t attend_pieces(const she_attend_pages_args &a, const AttendShape &s);      // rows of pieces that wait to be joined
size_t attend_scratch(const she_attend_pages_args &a, const AttendShape &s);
hipError_t launch_attend_pages(const she_attend_pages_args &a, const AttendShape &s, void *scratch, uint32_t *d_bad, hipStream_t st);

}}  // namespace she::clear
