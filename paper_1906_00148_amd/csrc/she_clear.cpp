// The clear side of split inference in the C ABI (declared in include/she_clear.h): checks of arguments, scratch, launches.
#include <algorithm>

#include "clear_host.h"

using namespace she;
using namespace she::clear;

namespace {

// Allocating would break a capture: the error says so before it does.
int may_allocate(she_ctx *c)
{
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    HIP_TRY(c, hipStreamIsCapturing(c->stream, &status));
    if (status == hipStreamCaptureStatusNone) return SHE_OK;
    return fail(c, SHE_ENOMEM, "this call needs more scratch than any before it: run it once before it is captured");
}

// Launches go to the current device, and the default stream is another one on each.
int on_device(she_ctx *c)
{
    int now = -1;
    HIP_TRY(c, hipGetDevice(&now));
    if (now == c->device) return SHE_OK;
    return fail(c, SHE_EINVAL, "the current device is " + std::to_string(now) + ", the context is on " + std::to_string(c->device));
}

}  // namespace

namespace she { namespace clear {

int ready(she_ctx *c)
{
    int code = on_device(c);
    if (code || c->clear.d_bad) return code;
    if ((code = may_allocate(c))) return code;
    HIP_TRY(c, hipMalloc((void **)&c->clear.d_bad, clear::COUNTERS * sizeof(uint32_t)));
    hipError_t rc = hipMemset(c->clear.d_bad, 0, clear::COUNTERS * sizeof(uint32_t));
    if (rc == hipSuccess) rc = hipStreamSynchronize(nullptr);
    if (rc != hipSuccess) {
        hipFree(c->clear.d_bad);
        c->clear.d_bad = nullptr;
    }
    HIP_TRY(c, rc);
    return SHE_OK;
}

int ensure_scratch(she_ctx *c, size_t bytes)
{
    if (bytes <= c->clear.bytes) return SHE_OK;
    int code = may_allocate(c);
    if (code) return code;
    c->clear.blocks.reserve(c->clear.blocks.size() + 1);
    bytes = std::max(bytes, 2 * c->clear.bytes);
    void *block = nullptr;
    HIP_TRY(c, hipMalloc(&block, bytes));
    c->clear.blocks.push_back(block);
    c->clear.bytes = bytes;
    return SHE_OK;
}

}}  // namespace she::clear

namespace {

// what both directions of the adapters have in common
template <class Args> int check_adapters(she_ctx *c, const Args &a, const char *name)
{
    const std::string at = std::string(name) + ": ";
    if (!half_type(a.type)) return fail(c, SHE_EINVAL, at + "type must be SHE_BF16 or SHE_F16");
    if (a.base_type != SHE_NO_BASE && a.base_type != a.type && a.base_type != SHE_F32 && a.base_type != SHE_I32)
        return fail(c, SHE_EINVAL, at + "base_type must be SHE_NO_BASE, the type, SHE_F32 or SHE_I32");
    if (!a.inputs || !a.outputs || !a.adapters || !a.rank) return fail(c, SHE_EINVAL, at + "a size is zero");
    if (a.rank > 512) return fail(c, SHE_ERANGE, at + "rank is at most 512");
    if (a.adapters > 65535) return fail(c, SHE_ERANGE, at + "at most 65535 adapters");
    if (a.tokens > MOST_TOKENS || a.segments > MOST_SEGMENTS || a.inputs > MOST_WIDTH || a.outputs > MOST_WIDTH)
        return fail(c, SHE_ERANGE, at + "tokens and widths are at most 2^24, segments 2^20");
    if (!a.down || !a.up || !a.scale || (a.segments && (!a.starts || !a.which)) || (a.tokens && !a.x) ||
        (a.tokens && a.base_type != SHE_NO_BASE && !a.base))
        return fail(c, SHE_EINVAL, at + "null argument");
    return SHE_OK;
}

int check_heads(she_ctx *c, const std::string &at, int32_t type, uint32_t tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t head,
                uint32_t rot, float eps)
{
    if (!half_type(type)) return fail(c, SHE_EINVAL, at + "type must be SHE_BF16 or SHE_F16");
    if (!q_heads || !kv_heads || !head) return fail(c, SHE_EINVAL, at + "a size is zero");
    if (head > 512 || q_heads > 65535 || kv_heads > 65535 || tokens > MOST_TOKENS)
        return fail(c, SHE_ERANGE, at + "head is at most 512, heads at most 65535, tokens at most 2^24");
    if (rot % 2 || rot > head) return fail(c, SHE_EINVAL, at + "rot must be even and at most head");
    if (!(eps >= 0)) return fail(c, SHE_EINVAL, at + "eps must not be negative");
    return SHE_OK;
}

}  // namespace

extern "C" {

int she_adapters(she_ctx *c, const she_adapters_args *args)
try {
    if (!c) return SHE_EINVAL;
    if (!args) return fail(c, SHE_EINVAL, "null argument");
    const she_adapters_args a = *args;
    int rc = check_adapters(c, a, "she_adapters");
    if (rc) return rc;
    if (!a.tokens || !a.segments) return SHE_OK;
    if (!a.out) return fail(c, SHE_EINVAL, "she_adapters: null argument");
    if ((rc = ready(c)) || (rc = ensure_scratch(c, clear::adapters_scratch(a)))) return rc;
    HIP_TRY(c, clear::launch_adapters(a, c->clear.scratch(), c->clear.d_bad, c->dk.cus, c->stream));
    return SHE_OK;
} SHE_NOTHROW(c)

int she_adapters_grad(she_ctx *c, const she_adapters_grad_args *args)
try {
    if (!c) return SHE_EINVAL;
    if (!args) return fail(c, SHE_EINVAL, "null argument");
    const she_adapters_grad_args a = *args;
    int rc = check_adapters(c, a, "she_adapters_grad");
    if (rc) return rc;
    if (a.base_type == SHE_I32) return fail(c, SHE_EINVAL, "she_adapters_grad: base_type must be SHE_NO_BASE, the type or SHE_F32");
    if (!a.ddown || !a.dup || (a.tokens && (!a.dy || !a.dx))) return fail(c, SHE_EINVAL, "she_adapters_grad: null argument");
    if ((rc = ready(c)) || (rc = ensure_scratch(c, clear::adapters_grad_scratch(a)))) return rc;
    HIP_TRY(c, clear::launch_adapters_grad(a, c->clear.scratch(), c->clear.d_bad, c->dk.cus, c->stream));
    return SHE_OK;
} SHE_NOTHROW(c)

int she_qk_rotate(she_ctx *c, const she_qk_rotate_args *args)
try {
    if (!c) return SHE_EINVAL;
    if (!args) return fail(c, SHE_EINVAL, "null argument");
    const she_qk_rotate_args a = *args;
    const std::string at = "she_qk_rotate: ";
    int rc = check_heads(c, at, a.type, a.tokens, a.q_heads, a.kv_heads, a.head, a.rot, a.eps);
    if (rc) return rc;
    if (!a.tokens) return SHE_OK;
    if (!a.q || !a.k || !a.q_out || !a.positions || (a.rot && a.places && (!a.cosines || !a.sines)) ||
        (a.k_pages ? !a.v || !a.v_pages || !a.slots : !a.k_out))
        return fail(c, SHE_EINVAL, at + "null argument");
    if (a.k_pages && !a.page_size) return fail(c, SHE_EINVAL, at + "a size is zero");
    if ((rc = ready(c))) return rc;
    HIP_TRY(c, clear::launch_qk_rotate(a, clear::qk_shape(a, c->dk.cus), c->clear.d_bad, c->stream));
    return SHE_OK;
} SHE_NOTHROW(c)

int she_qk_rotate_grad(she_ctx *c, const she_qk_rotate_grad_args *args)
try {
    if (!c) return SHE_EINVAL;
    if (!args) return fail(c, SHE_EINVAL, "null argument");
    const she_qk_rotate_grad_args a = *args;
    const std::string at = "she_qk_rotate_grad: ";
    int rc = check_heads(c, at, a.type, a.tokens, a.q_heads, a.kv_heads, a.head, a.rot, a.eps);
    if (rc) return rc;
    if (a.tokens && (!a.dq_out || !a.dk_out || !a.q || !a.k || !a.dq || !a.dk || !a.positions || (a.rot && a.places && (!a.cosines || !a.sines))))
        return fail(c, SHE_EINVAL, at + "null argument");
    if ((rc = ready(c))) return rc;
    const clear::QkGradShape s = clear::qk_grad_shape(a, c->dk.cus);
    if ((rc = ensure_scratch(c, clear::qk_grad_scratch(s, a.head)))) return rc;
    HIP_TRY(c, clear::launch_qk_rotate_grad(a, s, c->clear.scratch(), c->clear.d_bad, c->stream));
    return SHE_OK;
} SHE_NOTHROW(c)

int she_attend_pages(she_ctx *c, const she_attend_pages_args *args)
try {
    if (!c) return SHE_EINVAL;
    if (!args) return fail(c, SHE_EINVAL, "null argument");
    const she_attend_pages_args a = *args;
    const std::string at = "she_attend_pages: ";
    if (!half_type(a.type)) return fail(c, SHE_EINVAL, at + "type must be SHE_BF16 or SHE_F16");
    if (!a.q_heads || !a.kv_heads || !a.head || !a.page_size) return fail(c, SHE_EINVAL, at + "a size is zero");
    if (a.q_heads % a.kv_heads) return fail(c, SHE_EINVAL, at + "q_heads must be a multiple of kv_heads");
    if (a.head % 8 || a.head > 256) return fail(c, SHE_EINVAL, at + "head must be a multiple of 8, at most 256");
    if (a.q_heads > 65535 || a.tokens > MOST_TOKENS || a.requests > MOST_TOKENS || (uint64_t)a.table_width * a.page_size > MOST_PLACES ||
        (uint64_t)a.tokens * (a.q_heads / a.kv_heads) > 0x7FFFFFFF)
        return fail(c, SHE_ERANGE, at + "at most 2^24 tokens and requests, 65535 heads, 2^26 places of a request and 2^31 rows of a key head");
    if (!a.tokens || !a.requests) return SHE_OK;
    if (!a.q || !a.out || !a.starts || !a.lengths || (a.table_width && (!a.table || !a.k_pages || !a.v_pages)))
        return fail(c, SHE_EINVAL, at + "null argument");
    if (!on16(a.q) || !on16(a.k_pages) || !on16(a.v_pages) || !on16(a.out) ||
        (a.q_token | a.q_head | a.page_stride | a.slot_stride | a.page_head | a.out_token | a.out_head) % 8)
        return fail(c, SHE_EINVAL, at + "rows must start on 16 bytes");
    int rc = ready(c);
    if (rc) return rc;
    const clear::AttendShape s = clear::attend_shape(a, c->dk.cus);
    if ((s.few ? s.slots : s.slots * a.kv_heads) > MOST_GROUPS) return fail(c, SHE_ERANGE, at + "too many tokens and requests for one call");
    if ((rc = ensure_scratch(c, clear::attend_scratch(a, s)))) return rc;
    HIP_TRY(c, clear::launch_attend_pages(a, s, c->clear.scratch(), c->clear.d_bad, c->stream));
    return SHE_OK;
} SHE_NOTHROW(c)

int she_clear_bad_ids(she_ctx *c, uint64_t *count, int reset)
try {
    if (!c) return SHE_EINVAL;
    if (!count) return fail(c, SHE_EINVAL, "null argument");
    *count = 0;
    if (!c->clear.d_bad) return SHE_OK;
    if (int code = on_device(c)) return code;
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    HIP_TRY(c, hipStreamIsCapturing(c->stream, &status));
    if (status != hipStreamCaptureStatusNone) return fail(c, SHE_EINVAL, "she_clear_bad_ids: the stream is captured and cannot be waited for");
    uint32_t n = 0;
    HIP_TRY(c, hipStreamSynchronize(c->stream));
    HIP_TRY(c, hipMemcpy(&n, c->clear.d_bad, sizeof(n), hipMemcpyDeviceToHost));
    if (reset) {                         // on the stream whose next kernel counts, which need not wait for the default one
        HIP_TRY(c, hipMemsetAsync(c->clear.d_bad, 0, sizeof(n), c->stream));
        HIP_TRY(c, hipStreamSynchronize(c->stream));
    }
    *count = n;
    return SHE_OK;
} SHE_NOTHROW(c)

int she_clear_device(const she_ctx *c) { return c ? c->device : -1; }

}  // extern "C"
