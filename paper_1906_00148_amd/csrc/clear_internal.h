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

// A call with shared prefixes: the walk over these, and the one over what the requests have behind them; or each request's over both.
struct SharedShape {
    bool whole;                          // `behind` is the walk over both
    bool two;                            // tiles of many rows take weights as two numbers of the type, as those of few rows always do
    AttendShape prefix, behind;          // either joined with the other, whatever its pieces
};
she_attend_pages_args shared_behind(const she_attend_shared_args &a);            // the walk over the requests' own places as a call
SharedShape shared_shape(const she_attend_shared_args &a, uint32_t cus);
size_t shared_pieces(const she_attend_shared_args &a, const SharedShape &s);     // rows of pieces that wait to be joined
size_t shared_scratch(const she_attend_shared_args &a, const SharedShape &s);
hipError_t launch_attend_shared(const she_attend_shared_args &a, const SharedShape &s, void *scratch, uint32_t *d_bad, hipStream_t st);

// ---- places of a step's new tokens
constexpr uint32_t PLAN_REQUESTS = 4096;             // requests that one workgroup scans at once
// Whether one workgroup does all of a call: its requests and tokens are few.
inline bool plan_few(const she_plan_pages_args &a) { return a.requests <= PLAN_REQUESTS && a.tokens <= 4096; }
size_t plan_scratch(const she_plan_pages_args &a);
hipError_t launch_plan_pages(const she_plan_pages_args &a, void *scratch, uint32_t *d_bad, hipStream_t st);

// ---- the next token
struct SampleShape {
    uint32_t parts, tiles;               // workgroups that share a row, none if one has all of it; tiles of logits of each, or of its wavefronts if `plain`
    bool plain;                          // no filters
    uint32_t rows;                       // of a set of launches
};
SampleShape sample_shape(const she_sample_args &a, uint32_t cus);
size_t sample_scratch(const she_sample_args &a, const SampleShape &s);
hipError_t launch_sample(const she_sample_args &a, const SampleShape &s, void *scratch, hipStream_t st);

}}  // namespace she::clear
