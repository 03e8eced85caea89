// The launchers of the clear side's kernels for a fake device: k_qk_rotate leaves three ids out, the others do nothing.
#pragma once
#include "clear_internal.h"

inline uint32_t *counter = nullptr;
namespace she { namespace clear {
QkShape qk_shape(const she_qk_rotate_args &, uint32_t) { return {}; }
QkGradShape qk_grad_shape(const she_qk_rotate_grad_args &, uint32_t) { return {}; }
size_t qk_grad_scratch(const QkGradShape &, uint32_t) { return 0; }
size_t adapters_scratch(const she_adapters_args &) { return 0; }
size_t adapters_grad_scratch(const she_adapters_grad_args &) { return 0; }
AttendShape attend_shape(const she_attend_pages_args &, uint32_t) { return {}; }
size_t attend_scratch(const she_attend_pages_args &, const AttendShape &) { return 0; }
hipError_t launch_qk_rotate(const she_qk_rotate_args &, const QkShape &, uint32_t *bad, hipStream_t) { counter = bad; *bad += 3; return hipSuccess; }
hipError_t launch_qk_rotate_grad(const she_qk_rotate_grad_args &, const QkGradShape &, void *, uint32_t *, hipStream_t) { return hipSuccess; }
hipError_t launch_adapters(const she_adapters_args &, void *, uint32_t *, uint32_t, hipStream_t) { return hipSuccess; }
hipError_t launch_adapters_grad(const she_adapters_grad_args &, void *, uint32_t *, uint32_t, hipStream_t) { return hipSuccess; }
hipError_t launch_attend_pages(const she_attend_pages_args &, const AttendShape &, void *, uint32_t *, hipStream_t) { return hipSuccess; }
}}
