// The clear side's calls while another device than the context's is the current one (on a fake device).
#include <hip/hip_runtime.h>

#include <cstdint>

#define hipGetDevice plain_get_device
#include "fake_device.h"
#undef hipGetDevice
#include "clear_launchers.h"

static int failures = 0, current = 2;
#define CHECK(c, ...) do { if (!(c)) { failures++; std::printf(__VA_ARGS__); } } while (0)
extern "C" {
hipError_t hipGetDevice(int *d) { *d = current; return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *status) { *status = hipStreamCaptureStatusNone; return hipSuccess; }
}

int main()
{
    she_params P{};
    P.n = 4; P.N = 256; P.k = 1; P.bg_bit = 7; P.l = 3; P.ks_t = 1; P.ks_basebit = 1; P.lwe_std = 0; P.bk_std = 0;
    she_ctx *c = nullptr;
    if (she_keygen(&P, 3, 4, &c)) { std::printf("keygen: %s\n", she_last_error(nullptr)); return 1; }
    alignas(16) static char mem[64];
    she_adapters_args a{};
    a.type = SHE_BF16; a.base_type = SHE_NO_BASE; a.tokens = 3; a.inputs = a.outputs = 16; a.adapters = 2; a.rank = 4; a.segments = 1;
    a.x = a.down = a.up = a.out = mem; a.starts = a.which = (int32_t *)mem; a.scale = (float *)mem;
    she_adapters_grad_args g{};
    g.type = SHE_BF16; g.base_type = SHE_NO_BASE; g.tokens = 3; g.inputs = g.outputs = 16; g.adapters = 2; g.rank = 4; g.segments = 1;
    g.dy = g.x = g.down = g.up = g.dx = g.ddown = g.dup = mem; g.starts = g.which = (int32_t *)mem; g.scale = (float *)mem;
    she_qk_rotate_args q{};
    q.type = SHE_BF16; q.tokens = 2; q.q_heads = 4; q.kv_heads = 2; q.head = 64; q.rot = 32; q.places = 9;
    q.q = q.k = q.q_out = q.k_out = mem; q.cosines = q.sines = (float *)mem; q.positions = (int32_t *)mem;
    she_qk_rotate_grad_args d{};
    d.type = SHE_BF16; d.tokens = 2; d.q_heads = 4; d.kv_heads = 2; d.head = 64; d.rot = 32; d.places = 9;
    d.dq_out = d.dk_out = d.q = d.k = d.dq = d.dk = mem; d.cosines = d.sines = (float *)mem; d.positions = (int32_t *)mem;
    she_attend_pages_args t{};
    t.type = SHE_F16; t.tokens = 2; t.requests = 1; t.q_heads = 4; t.kv_heads = 2; t.head = 64; t.page_size = 16; t.pages = 4; t.table_width = 3;
    t.q = t.k_pages = t.v_pages = t.out = mem; t.table = t.starts = t.lengths = (int32_t *)mem;
    t.q_token = t.out_token = 256; t.q_head = t.out_head = t.page_head = 64; t.slot_stride = 128; t.page_stride = 2048;
    uint64_t n;
    CHECK(she_clear_device(c) == 2 && she_clear_device(nullptr) == -1, "the context's device\n");
    for (int before = 0; before < 2; before++) {              // a first call has its counter to allocate
        current = 0;
        const size_t held = fake::held;
        counter = nullptr;
        CHECK(she_adapters(c, &a) == SHE_EINVAL && she_adapters_grad(c, &g) == SHE_EINVAL && she_qk_rotate(c, &q) == SHE_EINVAL &&
              she_qk_rotate_grad(c, &d) == SHE_EINVAL && she_attend_pages(c, &t) == SHE_EINVAL, "another device is current\n");
        CHECK(!counter && fake::held == held && *she_last_error(c), "something is launched, allocated or not said\n");
        CHECK(!before || she_clear_bad_ids(c, &n, 1) == SHE_EINVAL, "the count on another device\n");
        current = 2;
        CHECK(she_adapters(c, &a) == SHE_OK && she_qk_rotate(c, &q) == SHE_OK && she_attend_pages(c, &t) == SHE_OK, "the context's own\n");
    }
    she_free(c);
    std::printf("failures %d\n", failures);
    return failures != 0;
}
