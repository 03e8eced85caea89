// Places in a paged cache for a step's new tokens.
//
// Two scans over the requests, of their new tokens and of the pages that these need, and then one look-up for each token: its request
// by a search among the starts, its page off the free list at the request's first entry plus the column's distance from the columns
// that the request has.  A new column's first place is always a new token's, so the token that has it writes the column.  Nothing here
// comes near a rate of the card's: 12 bytes a token, behind a chain of dependent latencies.  A step of up to 4096 requests and 4096 tokens takes
// 5 to 6 us in one launch; 2500 prompts of 250000 tokens 7.5 us for the requests and 6.6 for the tokens, at 0.5 TB/s.
#include "clear_device.h"
#include "clear_internal.h"

namespace she { namespace clear {
namespace {

constexpr int THREADS = 1024, EACH = PLAN_REQUESTS / THREADS;      // requests of a thread that a workgroup scans at once
constexpr uint64_t LAST = 0x7FFFFFFF;

// The sum of the workgroup's earlier threads' v; `total` gets that of all.  `sums` is free again after the next barrier.
__device__ inline uint64_t sum_before(uint64_t v, uint64_t *sums, uint64_t &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t run = v;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const uint64_t other = __shfl_up(run, m);
        if (lane >= m) run += other;
    }
    if (lane == 63) sums[wave] = run;
    __syncthreads();
    uint64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; w++) {
        const uint64_t s = sums[w];
        if (w < wave) before += s;
        total += s;
    }
    return before + run - v;
}

__device__ inline uint32_t columns(uint64_t places, const she_plan_pages_args &a)
{
    return min(((uint32_t)places + (a.page_size - 1)) / a.page_size, a.table_width);          // below 2^31 + 2^26
}

// What the tokens of a request need of it.
struct Request {
    uint32_t start, cached, first;       // its first token, its places so far, the entry of the list that its first new page is at
};

// The requests from r0 on, up to PLAN_REQUESTS of them: thread t has the EACH from r0 + EACH t on.  `tokens` and `pages` are those of the
// requests before, and afterwards of these too.
__device__ inline void scan_requests(const she_plan_pages_args &a, uint32_t r0, uint64_t &tokens, uint64_t &pages, uint64_t (*sums)[THREADS / 64], Request out[EACH], uint32_t length[EACH])
{
    uint32_t news[EACH];
    uint64_t mine = 0, all;
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const uint32_t r = r0 + threadIdx.x * EACH + e;
        out[e].cached = r < a.requests ? (uint32_t)max(a.cached[r], 0) : 0;
        news[e] = r < a.requests ? min((uint32_t)max(a.news[r], 0), a.tokens) : 0;
        mine += news[e];
    }
    uint64_t at = tokens + sum_before(mine, sums[0], all);
    tokens += all;
    mine = 0;
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        out[e].start = (uint32_t)min(at, (uint64_t)a.tokens);
        at += news[e];
        const uint32_t end = (uint32_t)min(at, (uint64_t)a.tokens);
        length[e] = (uint32_t)min((uint64_t)out[e].cached + (end - out[e].start), LAST);
        news[e] = columns(length[e], a) - columns(out[e].cached, a);
        mine += news[e];
    }
    at = pages + sum_before(mine, sums[1], all);
    pages += all;
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        out[e].first = (uint32_t)min(at, (uint64_t)a.free_count);
        at += news[e];
    }
}

// Token t, of request r; returns whether it has no place.
__device__ inline bool place_token(const she_plan_pages_args &a, uint32_t t, uint32_t r, const Request &q)
{
    const uint32_t place = q.cached + (t - q.start), column = place / a.page_size, in_page = place - column * a.page_size;
    int32_t page = -1;
    if (column < a.table_width) {
        int32_t *entry = a.table + r * a.table_stride + column;
        const uint32_t have = columns(q.cached, a);
        if (column < have) {
            page = *entry;
        } else {
            const uint32_t at = q.first + (column - have);
            if (at < a.free_count) page = a.free[at];
        }
        if (page < 0 || (uint32_t)page >= a.pages) page = -1;
        if (column >= have && in_page == 0) *entry = page;
    }
    const uint64_t before = a.before ? (uint64_t)max(a.before[r], 0) : 0;
    a.positions[t] = (int32_t)min(before + place, LAST);
    a.slots[t] = page < 0 ? -1 : (int64_t)page * a.page_size + in_page;
    return page < 0;
}
__device__ inline void no_token(const she_plan_pages_args &a, uint32_t t)
{
    a.positions[t] = 0;
    a.slots[t] = -1;
}
__device__ inline uint64_t taken_before(const she_plan_pages_args &a)
{
    return min((uint32_t)max(*a.taken, 0), a.free_count);
}

// A call of up to PLAN_REQUESTS requests and few tokens, by one workgroup.
__global__ __launch_bounds__(THREADS) void k_plan_few(she_plan_pages_args a, uint32_t *d_bad)
{
    __shared__ uint64_t sums[2][THREADS / 64];
    __shared__ uint32_t starts[PLAN_REQUESTS + 1], cached[PLAN_REQUESTS], first[PLAN_REQUESTS];
    uint64_t tokens = 0, pages = taken_before(a);
    Request q[EACH];
    uint32_t length[EACH];
    scan_requests(a, 0, tokens, pages, sums, q, length);           // everything has been read once it is through its barriers
    const uint32_t all = (uint32_t)min(tokens, (uint64_t)a.tokens);
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const uint32_t r = threadIdx.x * EACH + e;
        starts[r] = q[e].start;
        cached[r] = q[e].cached;
        first[r] = q[e].first;
        if (r < a.requests) {
            a.starts[r] = (int32_t)q[e].start;
            a.lengths[r] = (int32_t)length[e];
        }
    }
    if (threadIdx.x == 0) {
        starts[PLAN_REQUESTS] = all;
        a.starts[a.requests] = (int32_t)all;
        *a.taken_out = (int32_t)min(pages, (uint64_t)a.free_count);
    }
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < a.tokens; t += THREADS) {
        if (t >= all) {
            no_token(a, t);
            continue;
        }
        uint32_t low = 0, high = a.requests;                       // starts[low] <= t < starts[high]
        while (high - low > 1) {
            const uint32_t mid = (low + high) / 2;
            if (starts[mid] <= t) low = mid;
            else high = mid;
        }
        if (place_token(a, t, low, Request{starts[low], cached[low], first[low]})) count_bad(d_bad);
    }
}

// Larger calls: the requests first, by one workgroup, and then the tokens.
__global__ __launch_bounds__(THREADS) void k_plan_requests(she_plan_pages_args a, uint32_t *cached, uint32_t *first)
{
    __shared__ uint64_t sums[2][THREADS / 64];
    uint64_t tokens = 0, pages = taken_before(a);
    for (uint32_t r0 = 0; r0 < a.requests; r0 += PLAN_REQUESTS) {
        Request q[EACH];
        uint32_t length[EACH];
        scan_requests(a, r0, tokens, pages, sums, q, length);
#pragma unroll
        for (int e = 0; e < EACH; e++) {
            const uint32_t r = r0 + threadIdx.x * EACH + e;
            if (r >= a.requests) continue;
            a.starts[r] = (int32_t)q[e].start;
            a.lengths[r] = (int32_t)length[e];
            cached[r] = q[e].cached;
            first[r] = q[e].first;
        }
    }
    if (threadIdx.x) return;
    a.starts[a.requests] = (int32_t)min(tokens, (uint64_t)a.tokens);
    *a.taken_out = (int32_t)min(pages, (uint64_t)a.free_count);
}

__global__ __launch_bounds__(256) void k_plan_tokens(she_plan_pages_args a, const uint32_t *cached, const uint32_t *first, uint32_t *d_bad)
{
    const uint32_t t = blockIdx.x * 256 + threadIdx.x;
    const uint32_t *starts = reinterpret_cast<const uint32_t *>(a.starts), all = starts[a.requests];
    if (t >= a.tokens) return;
    if (t >= all) {
        no_token(a, t);
        return;
    }
    uint32_t low = 0, high = a.requests;
    while (high - low > 1) {
        const uint32_t mid = (low + high) / 2;
        if (starts[mid] <= t) low = mid;
        else high = mid;
    }
    if (place_token(a, t, low, Request{starts[low], cached[low], first[low]})) count_bad(d_bad);
}

}  // namespace

size_t plan_scratch(const she_plan_pages_args &a)
{
    return plan_few(a) ? 0 : 2 * sizeof(uint32_t) * (size_t)a.requests;
}

hipError_t launch_plan_pages(const she_plan_pages_args &a, void *scratch, uint32_t *d_bad, hipStream_t st)
{
    if (plan_few(a)) {
        k_plan_few<<<1, THREADS, 0, st>>>(a, d_bad);
        return hipGetLastError();
    }
    uint32_t *cached = static_cast<uint32_t *>(scratch), *first = cached + a.requests;
    k_plan_requests<<<1, THREADS, 0, st>>>(a, cached, first);
    const hipError_t rc = hipGetLastError();
    if (rc != hipSuccess || !a.tokens) return rc;
    k_plan_tokens<<<(a.tokens + 255) / 256, 256, 0, st>>>(a, cached, first, d_bad);
    return hipGetLastError();
}

}}  // namespace she::clear
