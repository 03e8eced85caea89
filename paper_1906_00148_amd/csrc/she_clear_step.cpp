// What a step of generation needs around its block, in the C ABI (declared in include/she_clear.h): checks of arguments, scratch, launches.
#include "clear_host.h"

using namespace she;
using namespace she::clear;

extern "C" {

int she_plan_pages(she_ctx *c, const she_plan_pages_args *args)
try {
    if (!c) return SHE_EINVAL;
    if (!args) return fail(c, SHE_EINVAL, "null argument");
    const she_plan_pages_args a = *args;
    const std::string at = "she_plan_pages: ";
    if (!a.page_size) return fail(c, SHE_EINVAL, at + "a size is zero");
    if (a.requests > MOST_SEGMENTS || a.tokens > MOST_TOKENS || a.page_size > MOST_PLACES || a.pages > 0x7FFFFFFF || a.free_count > 0x7FFFFFFF ||
        (uint64_t)a.table_width * a.page_size > MOST_PLACES)
        return fail(c, SHE_ERANGE, at + "at most 2^20 requests, 2^24 tokens, 2^26 places of a request and 2^31 pages");
    if (!a.taken || !a.taken_out || !a.starts || (a.requests && (!a.cached || !a.news || !a.lengths)) || (a.tokens && (!a.positions || !a.slots)) ||
        (a.requests && a.table_width && !a.table) || (a.free_count && !a.free))
        return fail(c, SHE_EINVAL, at + "null argument");
    if (a.requests > 1 && (a.table_stride < 0 ? -(uint64_t)a.table_stride : (uint64_t)a.table_stride) < a.table_width)
        return fail(c, SHE_EINVAL, at + "rows of the table must not overlap");
    int rc;
    if ((rc = ready(c)) || (rc = ensure_scratch(c, plan_scratch(a)))) return rc;
    HIP_TRY(c, launch_plan_pages(a, c->clear.scratch(), c->clear.d_bad, c->stream));
    return SHE_OK;
} SHE_NOTHROW(c)

int she_attend_shared(she_ctx *c, const she_attend_shared_args *args)
try {
    if (!c) return SHE_EINVAL;
    if (!args) return fail(c, SHE_EINVAL, "null argument");
    const she_attend_shared_args a = *args;
    const std::string at = "she_attend_shared: ";
    if (!half_type(a.type)) return fail(c, SHE_EINVAL, at + "type must be SHE_BF16 or SHE_F16");
    if (!a.q_heads || !a.kv_heads || !a.head || !a.page_size) return fail(c, SHE_EINVAL, at + "a size is zero");
    if (a.q_heads % a.kv_heads) return fail(c, SHE_EINVAL, at + "q_heads must be a multiple of kv_heads");
    if (a.head % 8 || a.head > 256) return fail(c, SHE_EINVAL, at + "head must be a multiple of 8, at most 256");
    if (a.q_heads > 65535 || a.tokens > MOST_TOKENS || a.requests > MOST_TOKENS || a.prefixes > MOST_SEGMENTS ||
        (uint64_t)a.table_width * a.page_size > MOST_PLACES || (uint64_t)a.prefix_width * a.page_size > MOST_PLACES ||
        (uint64_t)a.tokens * (a.q_heads / a.kv_heads) > 0x7FFFFFFF)
        return fail(c, SHE_ERANGE, at + "at most 2^24 tokens and requests, 2^20 prefixes, 65535 heads, 2^26 places of a request or prefix and 2^31 rows of a key head");
    if (!a.tokens || !a.requests) return SHE_OK;
    if (!a.q || !a.out || !a.starts || !a.lengths || (a.table_width && !a.table) || (a.prefixes && (!a.prefix_requests || !a.prefix_lengths)) ||
        (a.prefixes && a.prefix_width && !a.prefix_table) || ((a.table_width || (a.prefixes && a.prefix_width)) && (!a.k_pages || !a.v_pages)))
        return fail(c, SHE_EINVAL, at + "null argument");
    if (!on16(a.q) || !on16(a.k_pages) || !on16(a.v_pages) || !on16(a.out) ||
        (a.q_token | a.q_head | a.page_stride | a.slot_stride | a.page_head | a.out_token | a.out_head) % 8)
        return fail(c, SHE_EINVAL, at + "rows must start on 16 bytes");
    int rc = ready(c);
    if (rc) return rc;
    const SharedShape s = shared_shape(a, c->dk.cus);
    if (s.prefix.slots * a.kv_heads * s.prefix.splits + s.behind.slots * a.kv_heads * s.behind.splits > MOST_GROUPS)
        return fail(c, SHE_ERANGE, at + "too many tokens and requests for one call");
    if ((rc = ensure_scratch(c, shared_scratch(a, s)))) return rc;
    HIP_TRY(c, launch_attend_shared(a, s, c->clear.scratch(), c->clear.d_bad, c->stream));
    return SHE_OK;
} SHE_NOTHROW(c)

int she_sample(she_ctx *c, const she_sample_args *args)
try {
    if (!c) return SHE_EINVAL;
    if (!args) return fail(c, SHE_EINVAL, "null argument");
    const she_sample_args a = *args;
    const std::string at = "she_sample: ";
    if (!half_type(a.type) && a.type != SHE_F32 && a.type != SHE_I32) return fail(c, SHE_EINVAL, at + "type must be SHE_BF16, SHE_F16, SHE_F32 or SHE_I32");
    if (!a.vocab) return fail(c, SHE_EINVAL, at + "a size is zero");
    if (a.vocab > 1u << 20 || a.rows > 1u << 20) return fail(c, SHE_ERANGE, at + "rows and vocab are at most 2^20");
    if (!a.rows) return SHE_OK;
    if (!a.logits || !a.uniform || !a.tokens) return fail(c, SHE_EINVAL, at + "null argument");
    if (a.step && a.type != SHE_I32) return fail(c, SHE_EINVAL, at + "step belongs to SHE_I32");
    const SampleShape s = sample_shape(a, c->dk.cus);
    int rc;
    if ((rc = ready(c)) || (rc = ensure_scratch(c, sample_scratch(a, s)))) return rc;
    HIP_TRY(c, launch_sample(a, s, c->clear.scratch(), c->stream));
    return SHE_OK;
} SHE_NOTHROW(c)

}  // extern "C"
