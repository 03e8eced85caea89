// The calls around a block (she_clear.h) on a fake device: what they refuse, what they launch, and their scratch.
#include <cstdint>

#include "clear_launchers.h"
#include "fake_device.h"

static int failures = 0, launches = 0;
#define CHECK(c, ...) do { if (!(c)) { failures++; std::printf(__VA_ARGS__); } } while (0)

static size_t wanted = 0;                                                    // scratch
static hipError_t launched() { launches++; return fake::step(); }
namespace she { namespace clear {
size_t plan_scratch(const she_plan_pages_args &) { return wanted; }
hipError_t launch_plan_pages(const she_plan_pages_args &, void *, uint32_t *, hipStream_t) { return launched(); }
SharedShape shared_shape(const she_attend_shared_args &a, uint32_t) { SharedShape s{}; s.prefix.slots = a.prefixes; s.behind.slots = a.requests; return s; }
size_t shared_scratch(const she_attend_shared_args &, const SharedShape &) { return wanted; }
hipError_t launch_attend_shared(const she_attend_shared_args &, const SharedShape &, void *, uint32_t *, hipStream_t) { return launched(); }
SampleShape sample_shape(const she_sample_args &, uint32_t) { return {}; }
size_t sample_scratch(const she_sample_args &, const SampleShape &) { return wanted; }
hipError_t launch_sample(const she_sample_args &, const SampleShape &, void *, hipStream_t) { return launched(); }
}}

static hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
extern "C" hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *status) { *status = capturing; return hipSuccess; }

static she_ctx *c;
template <class A> static void expect(int (*call)(she_ctx *, const A *), const A &good, int code, const char *what, void (*change)(A &))
{
    A a = good;
    change(a);
    launches = 0;
    const int rc = call(c, &a);
    CHECK(rc == code && launches == (code == SHE_OK) && (code == SHE_OK || *she_last_error(c)), "%s: returns %d, %d launches\n", what, rc, launches);
}
#define EXPECT(call, good, code, change) expect<decltype(good)>(call, good, code, #call ": " #change, [](decltype(good) &a) { change; })

int main()
{
    she_params P{};
    P.n = 4; P.N = 256; P.k = 1; P.bg_bit = 7; P.l = 3; P.ks_t = 1; P.ks_basebit = 1; P.lwe_std = 0; P.bk_std = 0;
    if (she_keygen(&P, 3, 4, &c)) { std::printf("keygen: %s\n", she_last_error(nullptr)); return 1; }
    alignas(16) static char mem[64];
    int32_t *ints = (int32_t *)mem;

    she_plan_pages_args p{};
    p.requests = 3; p.tokens = 7; p.pages = 9; p.page_size = 16; p.table_width = 4; p.free_count = 5; p.table_stride = 4;
    p.cached = p.news = p.before = p.free = p.taken = ints; p.table = p.starts = p.lengths = p.positions = p.taken_out = ints; p.slots = (int64_t *)mem;
    EXPECT(she_plan_pages, p, SHE_OK, (void)a);
    EXPECT(she_plan_pages, p, SHE_OK, a.before = nullptr);
    EXPECT(she_plan_pages, p, SHE_OK, a.free_count = 0; a.free = nullptr);
    EXPECT(she_plan_pages, p, SHE_OK, a.table_width = 0; a.table = nullptr);
    EXPECT(she_plan_pages, p, SHE_OK, a.tokens = 0; a.positions = nullptr; a.slots = nullptr);
    EXPECT(she_plan_pages, p, SHE_OK, a.requests = 0; a.cached = a.news = nullptr; a.lengths = a.table = nullptr);
    EXPECT(she_plan_pages, p, SHE_OK, a.pages = 0);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.page_size = 0);
    EXPECT(she_plan_pages, p, SHE_ERANGE, a.page_size = (1u << 26) + 1; a.table_width = 0);
    EXPECT(she_plan_pages, p, SHE_ERANGE, a.table_width = (1u << 22) + 1);
    EXPECT(she_plan_pages, p, SHE_ERANGE, a.requests = (1u << 20) + 1);
    EXPECT(she_plan_pages, p, SHE_ERANGE, a.tokens = (1u << 24) + 1);
    EXPECT(she_plan_pages, p, SHE_ERANGE, a.pages = 1u << 31);
    EXPECT(she_plan_pages, p, SHE_ERANGE, a.free_count = 1u << 31);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.cached = nullptr);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.news = nullptr);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.free = nullptr);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.taken = nullptr);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.taken_out = nullptr);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.table = nullptr);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.starts = nullptr);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.lengths = nullptr);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.positions = nullptr);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.slots = nullptr);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.table_stride = 3);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.table_stride = 0);
    EXPECT(she_plan_pages, p, SHE_EINVAL, a.table_stride = -3);
    EXPECT(she_plan_pages, p, SHE_OK, a.table_stride = -4);
    EXPECT(she_plan_pages, p, SHE_OK, a.table_stride = INT64_MIN);
    EXPECT(she_plan_pages, p, SHE_OK, a.table_stride = 0; a.requests = 1);
    EXPECT(she_plan_pages, p, SHE_OK, a.table_stride = 0; a.table_width = 0);
    CHECK(she_plan_pages(c, nullptr) == SHE_EINVAL && she_plan_pages(nullptr, &p) == SHE_EINVAL, "null struct or context\n");

    she_sample_args s{};
    s.type = SHE_F32; s.rows = 3; s.vocab = 100; s.logits = mem; s.row_stride = 100; s.uniform = (float *)mem; s.tokens = ints;
    EXPECT(she_sample, s, SHE_OK, (void)a);
    EXPECT(she_sample, s, SHE_OK, a.type = SHE_BF16);
    EXPECT(she_sample, s, SHE_OK, a.type = SHE_I32; a.step = a.uniform);
    EXPECT(she_sample, s, SHE_OK, a.vocab = 1u << 20);
    EXPECT(she_sample, s, SHE_OK, a.temperature = a.top_p = a.min_p = a.uniform; a.top_k = a.tokens; a.probs = (float *)a.tokens);
    EXPECT(she_sample, s, SHE_EINVAL, a.type = 4);
    EXPECT(she_sample, s, SHE_EINVAL, a.type = -1);
    EXPECT(she_sample, s, SHE_EINVAL, a.vocab = 0);
    EXPECT(she_sample, s, SHE_ERANGE, a.vocab = (1u << 20) + 1);
    EXPECT(she_sample, s, SHE_ERANGE, a.rows = (1u << 20) + 1);
    EXPECT(she_sample, s, SHE_EINVAL, a.step = a.uniform);
    EXPECT(she_sample, s, SHE_EINVAL, a.logits = nullptr);
    EXPECT(she_sample, s, SHE_EINVAL, a.uniform = nullptr);
    EXPECT(she_sample, s, SHE_EINVAL, a.tokens = nullptr);
    launches = 0;
    s.rows = 0;
    CHECK(she_sample(c, &s) == SHE_OK && !launches, "no rows\n");
    s.rows = 3;
    CHECK(she_sample(c, nullptr) == SHE_EINVAL && she_sample(nullptr, &s) == SHE_EINVAL, "null struct or context\n");

    she_attend_shared_args t{};
    t.type = SHE_F16; t.tokens = 2; t.requests = 1; t.q_heads = 4; t.kv_heads = 2; t.head = 64; t.page_size = 16; t.pages = 4; t.table_width = 3;
    t.prefixes = 1; t.prefix_width = 5; t.q = t.k_pages = t.v_pages = t.out = mem;
    t.table = t.starts = t.lengths = t.prefix_table = t.prefix_requests = t.prefix_lengths = ints;
    t.q_token = t.out_token = 256; t.q_head = t.out_head = t.page_head = 64; t.slot_stride = 128; t.page_stride = 2048;
    EXPECT(she_attend_shared, t, SHE_OK, (void)a);
    EXPECT(she_attend_shared, t, SHE_OK, a.table_width = 0; a.table = nullptr);
    EXPECT(she_attend_shared, t, SHE_OK, a.prefix_width = 0; a.prefix_table = nullptr);
    EXPECT(she_attend_shared, t, SHE_OK, a.prefixes = 0; a.prefix_table = a.prefix_requests = a.prefix_lengths = nullptr);
    EXPECT(she_attend_shared, t, SHE_OK, a.prefix_width = a.table_width = 0; a.prefix_table = a.table = nullptr; a.k_pages = a.v_pages = nullptr);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.type = SHE_F32);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.q_heads = 5);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.kv_heads = 0);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.head = 60);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.head = 264);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.page_size = 0);
    EXPECT(she_attend_shared, t, SHE_ERANGE, a.table_width = 1u << 23);
    EXPECT(she_attend_shared, t, SHE_ERANGE, a.prefix_width = 1u << 23);
    EXPECT(she_attend_shared, t, SHE_ERANGE, a.requests = (1u << 24) + 1);
    EXPECT(she_attend_shared, t, SHE_ERANGE, a.prefixes = (1u << 20) + 1);
    EXPECT(she_attend_shared, t, SHE_ERANGE, a.tokens = 1u << 24; a.q_heads = 1024);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.q = (char *)a.q + 8);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.page_head = 60);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.out_token = 252);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.lengths = nullptr);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.starts = nullptr);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.table = nullptr);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.prefix_table = nullptr);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.prefix_requests = nullptr);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.prefix_lengths = nullptr);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.v_pages = nullptr);
    EXPECT(she_attend_shared, t, SHE_EINVAL, a.out = nullptr);
    launches = 0;
    t.tokens = 0;
    CHECK(she_attend_shared(c, &t) == SHE_OK && !launches, "no tokens\n");
    t.tokens = 2;
    CHECK(she_attend_shared(c, nullptr) == SHE_EINVAL && she_attend_shared(nullptr, &t) == SHE_EINVAL, "null struct or context\n");

    // while the stream is captured, a call that would allocate is refused
    capturing = hipStreamCaptureStatusActive;
    wanted = 500;
    CHECK(she_plan_pages(c, &p) == SHE_ENOMEM && she_attend_shared(c, &t) == SHE_ENOMEM && she_sample(c, &s) == SHE_ENOMEM, "a capture with scratch to allocate\n");
    capturing = hipStreamCaptureStatusNone;
    CHECK(she_plan_pages(c, &p) == SHE_OK, "scratch\n");
    capturing = hipStreamCaptureStatusActive;
    CHECK(she_plan_pages(c, &p) == SHE_OK && she_attend_shared(c, &t) == SHE_OK && she_sample(c, &s) == SHE_OK, "a capture within the scratch\n");
    capturing = hipStreamCaptureStatusNone;
    she_free(c);
    CHECK(fake::held == 0, "%zu bytes are still held\n", fake::held);
    std::printf("failures %d\n", failures);
    return failures != 0;
}
