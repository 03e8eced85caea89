// she_clear_bad_ids on a fake device whose streams remember what has not been waited for.
#include <hip/hip_runtime.h>

#include <cstdint>

// the fake device's own versions, under other names
#define hipMemset plain_memset
#define hipMemsetAsync plain_memset_async
#define hipStreamSynchronize plain_stream_synchronize
#include "fake_device.h"
#undef hipMemset
#undef hipMemsetAsync
#undef hipStreamSynchronize
#include "clear_launchers.h"

static int failures = 0, waits = 0;
#define CHECK(c, ...) do { if (!(c)) { failures++; std::printf(__VA_ARGS__); } } while (0)
static std::map<hipStream_t, int> under_way;               // writes that a stream has been given and nobody has waited for
static hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;

extern "C" {
hipError_t hipMemset(void *d, int v, size_t n) { under_way[nullptr]++; return plain_memset(d, v, n); }
hipError_t hipMemsetAsync(void *d, int v, size_t n, hipStream_t s) { under_way[s]++; return plain_memset_async(d, v, n, s); }
hipError_t hipStreamSynchronize(hipStream_t s) { waits++; under_way.erase(s); return plain_stream_synchronize(s); }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *status) { *status = capturing; return hipSuccess; }
}

int main()
{
    she_params P{};
    P.n = 4; P.N = 256; P.k = 1; P.bg_bit = 7; P.l = 3; P.ks_t = 1; P.ks_basebit = 1; P.lwe_std = 0; P.bk_std = 0;
    she_ctx *c = nullptr;
    if (she_keygen(&P, 3, 4, &c)) { std::printf("keygen: %s\n", she_last_error(nullptr)); return 1; }
    int a_stream;
    CHECK(she_set_stream(c, &a_stream) == SHE_OK, "set_stream\n");
    alignas(16) static char mem[64];
    she_qk_rotate_args q{};
    q.type = SHE_BF16; q.tokens = 2; q.q_heads = 4; q.kv_heads = 2; q.head = 64; q.rot = 32; q.places = 9;
    q.q = q.k = q.q_out = q.k_out = mem; q.cosines = q.sines = (float *)mem; q.positions = (int32_t *)mem;
    CHECK(she_qk_rotate(c, &q) == SHE_OK && counter, "the call\n");
    under_way.clear();
    uint64_t n = 0;
    CHECK(she_clear_bad_ids(c, &n, 0) == SHE_OK && n == 3 && *counter == 3, "count %llu\n", (unsigned long long)n);
    CHECK(she_clear_bad_ids(c, &n, 1) == SHE_OK && n == 3 && *counter == 0, "count and reset\n");
    // the next call's kernel, on a stream that need not wait for any other, must not start before the counter is cleared
    CHECK(under_way.empty(), "the counter is cleared by work that is not waited for\n");
    // a captured stream cannot be waited for, and to try would end the capture
    CHECK(she_qk_rotate(c, &q) == SHE_OK, "the call again\n");
    capturing = hipStreamCaptureStatusActive;
    waits = 0;
    n = 9;
    CHECK(she_clear_bad_ids(c, &n, 1) == SHE_EINVAL && *she_last_error(c) && !waits && n == 0 && *counter == 3, "in a capture\n");
    capturing = hipStreamCaptureStatusNone;
    CHECK(she_clear_bad_ids(c, &n, 1) == SHE_OK && n == 3, "after it\n");
    she_free(c);
    std::printf("failures %d\n", failures);
    return failures != 0;
}
