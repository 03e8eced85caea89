// The clear side's calls (she_clear.h) on a fake device: what they refuse, what they launch, and their scratch.
#include <cmath>
#include <cstdint>

#include "clear_internal.h"
#include "fake_device.h"

static int failures = 0, launches = 0;
#define CHECK(c, ...) do { if (!(c)) { failures++; std::printf(__VA_ARGS__); } } while (0)

static size_t wanted = 0;                                                    // scratch
static hipError_t launched() { launches++; return fake::step(); }
namespace she { namespace clear {
QkShape qk_shape(const she_qk_rotate_args &, uint32_t) { return {}; }
QkGradShape qk_grad_shape(const she_qk_rotate_grad_args &, uint32_t) { return {}; }
size_t qk_grad_scratch(const QkGradShape &, uint32_t) { return wanted; }
size_t adapters_scratch(const she_adapters_args &) { return wanted; }
size_t adapters_grad_scratch(const she_adapters_grad_args &) { return wanted; }
AttendShape attend_shape(const she_attend_pages_args &a, uint32_t) { AttendShape s{}; s.slots = a.requests; return s; }
size_t attend_scratch(const she_attend_pages_args &, const AttendShape &) { return wanted; }
hipError_t launch_qk_rotate(const she_qk_rotate_args &, const QkShape &, uint32_t *, hipStream_t) { return launched(); }
hipError_t launch_qk_rotate_grad(const she_qk_rotate_grad_args &, const QkGradShape &, void *, uint32_t *, hipStream_t) { return launched(); }
hipError_t launch_adapters(const she_adapters_args &, void *, uint32_t *, uint32_t, hipStream_t) { return launched(); }
hipError_t launch_adapters_grad(const she_adapters_grad_args &, void *, uint32_t *, uint32_t, hipStream_t) { return launched(); }
hipError_t launch_attend_pages(const she_attend_pages_args &, const AttendShape &, void *, uint32_t *, hipStream_t) { return launched(); }
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
    uint64_t count = 7;
    CHECK(she_clear_bad_ids(c, &count, 1) == SHE_OK && count == 0 && she_clear_bad_ids(c, nullptr, 0) == SHE_EINVAL, "bad ids before a call\n");
    CHECK(she_clear_bad_ids(nullptr, &count, 1) == SHE_EINVAL, "no context\n");

    she_adapters_args a{};
    a.type = SHE_BF16; a.base_type = SHE_F32; a.tokens = 3; a.inputs = a.outputs = 16; a.adapters = 2; a.rank = 4; a.segments = 1;
    a.x = a.down = a.up = a.base = a.out = mem; a.starts = a.which = (int32_t *)mem; a.scale = (float *)mem;
    EXPECT(she_adapters, a, SHE_OK, (void)a);
    EXPECT(she_adapters, a, SHE_OK, a.base_type = SHE_NO_BASE; a.base = nullptr);
    EXPECT(she_adapters, a, SHE_OK, a.base_type = SHE_I32);
    EXPECT(she_adapters, a, SHE_EINVAL, a.type = SHE_F32);
    EXPECT(she_adapters, a, SHE_EINVAL, a.base_type = SHE_F16);
    EXPECT(she_adapters, a, SHE_EINVAL, a.base_type = 9);
    EXPECT(she_adapters, a, SHE_EINVAL, a.inputs = 0);
    EXPECT(she_adapters, a, SHE_EINVAL, a.outputs = 0);
    EXPECT(she_adapters, a, SHE_EINVAL, a.adapters = 0);
    EXPECT(she_adapters, a, SHE_EINVAL, a.rank = 0);
    EXPECT(she_adapters, a, SHE_ERANGE, a.rank = 513);
    EXPECT(she_adapters, a, SHE_ERANGE, a.adapters = 65536);
    EXPECT(she_adapters, a, SHE_ERANGE, a.tokens = (1u << 24) + 1);
    EXPECT(she_adapters, a, SHE_ERANGE, a.segments = (1u << 20) + 1);
    EXPECT(she_adapters, a, SHE_ERANGE, a.outputs = 1u << 30);
    EXPECT(she_adapters, a, SHE_EINVAL, a.x = nullptr);
    EXPECT(she_adapters, a, SHE_EINVAL, a.down = nullptr);
    EXPECT(she_adapters, a, SHE_EINVAL, a.up = nullptr);
    EXPECT(she_adapters, a, SHE_EINVAL, a.starts = nullptr);
    EXPECT(she_adapters, a, SHE_EINVAL, a.which = nullptr);
    EXPECT(she_adapters, a, SHE_EINVAL, a.scale = nullptr);
    EXPECT(she_adapters, a, SHE_EINVAL, a.base = nullptr);
    EXPECT(she_adapters, a, SHE_EINVAL, a.out = nullptr);
    launches = 0;
    CHECK(she_adapters(c, nullptr) == SHE_EINVAL && she_adapters(nullptr, &a) == SHE_EINVAL, "null struct or context\n");
    a.tokens = 0; a.x = a.base = a.out = nullptr;
    CHECK(she_adapters(c, &a) == SHE_OK && !launches, "no tokens\n");

    she_adapters_grad_args g{};
    g.type = SHE_F16; g.base_type = SHE_F16; g.tokens = 3; g.inputs = g.outputs = 16; g.adapters = 2; g.rank = 4; g.segments = 1;
    g.dy = g.x = g.down = g.up = g.base = g.dx = g.ddown = g.dup = mem; g.starts = g.which = (int32_t *)mem; g.scale = (float *)mem;
    EXPECT(she_adapters_grad, g, SHE_OK, (void)a);
    EXPECT(she_adapters_grad, g, SHE_OK, a.tokens = a.segments = 0; a.starts = a.which = nullptr; a.dy = a.x = a.base = a.dx = nullptr);
    EXPECT(she_adapters_grad, g, SHE_EINVAL, a.base_type = SHE_I32);
    EXPECT(she_adapters_grad, g, SHE_EINVAL, a.dy = nullptr);
    EXPECT(she_adapters_grad, g, SHE_EINVAL, a.dx = nullptr);
    EXPECT(she_adapters_grad, g, SHE_EINVAL, a.ddown = nullptr);
    EXPECT(she_adapters_grad, g, SHE_EINVAL, a.dup = nullptr);
    EXPECT(she_adapters_grad, g, SHE_ERANGE, a.rank = 1000);

    she_qk_rotate_args q{};
    q.type = SHE_BF16; q.tokens = 2; q.q_heads = 4; q.kv_heads = 2; q.head = 64; q.rot = 32; q.places = 9; q.eps = 0;
    q.q = q.k = q.q_out = q.k_out = mem; q.cosines = q.sines = (float *)mem; q.positions = (int32_t *)mem;
    EXPECT(she_qk_rotate, q, SHE_OK, (void)a);
    EXPECT(she_qk_rotate, q, SHE_OK, a.rot = 0; a.cosines = a.sines = nullptr);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.type = SHE_I32);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.q_heads = 0);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.kv_heads = 0);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.rot = 31);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.rot = 66);
    EXPECT(she_qk_rotate, q, SHE_ERANGE, a.head = 520);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.eps = -1);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.eps = std::nanf(""));
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.q = nullptr);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.k_out = nullptr);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.positions = nullptr);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.sines = nullptr);
    q.k_out = nullptr; q.k_pages = q.v_pages = mem; q.v = mem; q.slots = (int64_t *)mem; q.pages = 2; q.page_size = 16;
    EXPECT(she_qk_rotate, q, SHE_OK, (void)a);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.v = nullptr);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.v_pages = nullptr);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.slots = nullptr);
    EXPECT(she_qk_rotate, q, SHE_EINVAL, a.page_size = 0);

    she_qk_rotate_grad_args d{};
    d.type = SHE_BF16; d.tokens = 2; d.q_heads = 4; d.kv_heads = 2; d.head = 64; d.rot = 32; d.places = 9;
    d.dq_out = d.dk_out = d.q = d.k = d.dq = d.dk = mem; d.cosines = d.sines = (float *)mem; d.positions = (int32_t *)mem;
    EXPECT(she_qk_rotate_grad, d, SHE_OK, (void)a);
    EXPECT(she_qk_rotate_grad, d, SHE_EINVAL, a.dk = nullptr);
    EXPECT(she_qk_rotate_grad, d, SHE_EINVAL, a.dq_out = nullptr);
    EXPECT(she_qk_rotate_grad, d, SHE_EINVAL, a.rot = 3);

    she_attend_pages_args t{};
    t.type = SHE_F16; t.tokens = 2; t.requests = 1; t.q_heads = 4; t.kv_heads = 2; t.head = 64; t.page_size = 16; t.pages = 4; t.table_width = 3;
    t.q = t.k_pages = t.v_pages = t.out = mem; t.table = t.starts = t.lengths = (int32_t *)mem;
    t.q_token = t.out_token = 256; t.q_head = t.out_head = t.page_head = 64; t.slot_stride = 128; t.page_stride = 2048;
    EXPECT(she_attend_pages, t, SHE_OK, (void)a);
    EXPECT(she_attend_pages, t, SHE_OK, a.table_width = 0; a.table = nullptr; a.k_pages = a.v_pages = nullptr);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.type = SHE_F32);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.q_heads = 5);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.kv_heads = 0);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.head = 60);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.head = 264);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.page_size = 0);
    EXPECT(she_attend_pages, t, SHE_ERANGE, a.table_width = 1u << 23);
    EXPECT(she_attend_pages, t, SHE_ERANGE, a.requests = (1u << 24) + 1);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.q = (char *)a.q + 8);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.page_head = 60);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.out_token = 252);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.lengths = nullptr);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.table = nullptr);
    EXPECT(she_attend_pages, t, SHE_EINVAL, a.out = nullptr);
    t.tokens = 0;
    launches = 0;
    CHECK(she_attend_pages(c, &t) == SHE_OK && !launches, "no tokens\n");
    t.tokens = 2;

    // while the stream is captured, a call that would allocate is refused
    capturing = hipStreamCaptureStatusActive;
    wanted = 500;
    CHECK(she_attend_pages(c, &t) == SHE_ENOMEM, "a capture with scratch to allocate\n");
    wanted = 0;
    CHECK(she_attend_pages(c, &t) == SHE_OK, "a capture without\n");
    capturing = hipStreamCaptureStatusNone;

    // scratch grows once, is used again, and a call that gets none says so and leaves nothing behind
    wanted = 1000;
    CHECK(she_attend_pages(c, &t) == SHE_OK, "scratch\n");
    const size_t held = fake::held;
    CHECK(she_attend_pages(c, &t) == SHE_OK && fake::held == held, "scratch is allocated again\n");
    capturing = hipStreamCaptureStatusActive;
    CHECK(she_attend_pages(c, &t) == SHE_OK && fake::held == held, "a capture within the scratch\n");
    capturing = hipStreamCaptureStatusNone;
    wanted = 5000;
    fake::limit = fake::held;
    CHECK(she_attend_pages(c, &t) == SHE_ENOMEM && hipGetLastError() == hipSuccess, "no memory\n");
    fake::limit = ~(size_t)0;
    bool freed = false;
    fake::on_free = [&](const char *, size_t) { freed = true; };
    CHECK(she_attend_pages(c, &t) == SHE_OK && fake::held > held && !freed, "memory again, or the old block is gone\n");
    fake::on_free = nullptr;
    she_free(c);
    CHECK(fake::held == 0, "%zu bytes are still held\n", fake::held);
    std::printf("failures %d\n", failures);
    return failures != 0;
}
