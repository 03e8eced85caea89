// Norms of queries and keys for each head with the rotation of the position, forward (into a tensor or the pages of a cache) and
// backward.
//
// A head of D elements lies on `lanes` neighbouring lanes, eight elements each, so that a wavefront holds 64 / lanes heads and every
// access is 16 bytes a lane.  With r = 1/sqrt(mean x^2 + eps), u = x r and R the rotation,
//     y = R (w u)                      g = R^T dy,   dw = sum g u,   dx = r (w g - u mean(w g u))
// so one sum over a head's lanes serves the forward pass and two the backward.  The other member of a pair half the rotated part
// away comes from the wavefront's own row buffer in LDS; neighbours are in one lane.  A wavefront keeps a token's cosines and sines
// for all the heads that it does.  Bound by memory: every element is read and written once.
//
// Measured: 16383 tokens of 64 heads of 80 (f16, ten of sixteen lanes busy) 79 us, 4.3 TB/s of the 4.9 that a large copy reaches;
// backward, 8192 tokens of 40 heads of 128 (bf16) 63 us, 4.1 TB/s, and 4.6 us for the weights' sums.
#include <algorithm>
#include <type_traits>

#include "clear_device.h"
#include "clear_internal.h"

namespace she { namespace clear {
namespace {

constexpr int WAVES = 4;                       // wavefronts of a workgroup
constexpr uint32_t GRAD_RESIDENT = 4;           // of the backward kernel's workgroups on a compute unit
constexpr int BATCH = 4;                       // steps whose loads are requested before the first is used

// Sum over the LANES lanes of a head.
template <int LANES> __device__ inline float head_sum(float v)
{
#pragma unroll
    for (int m = 1; m < LANES; m *= 2) v += __shfl_xor(v, m);
    return v;
}

// A lane's eight cosines and signed sines; s[i] is taken with the other member of element i's pair.  Elements that do not turn
// keep 1 and 0.
struct Turn {
    float c[8], s[8];
};
__device__ inline Turn load_turn(const float *cosines, const float *sines, uint32_t rot, bool interleaved, bool aligned, uint32_t place, int d0, float sign)
{
    Turn t;
    const uint32_t half = rot / 2;
    const float *c = cosines + (size_t)place * half, *s = sines + (size_t)place * half;
    if (aligned) {                             // a lane's pairs are eight, or four, neighbours on 16 bytes
        const bool turns = (uint32_t)d0 < rot;
        const uint32_t pair = !turns ? 0 : interleaved ? d0 / 2 : (uint32_t)d0 < half ? d0 : d0 - half;
        f32x4 cv[2] = {f32x4{1, 1, 1, 1}, f32x4{1, 1, 1, 1}}, sv[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
        if (turns) {
            cv[0] = *reinterpret_cast<const f32x4 *>(c + pair);
            sv[0] = *reinterpret_cast<const f32x4 *>(s + pair);
            if (!interleaved) {
                cv[1] = *reinterpret_cast<const f32x4 *>(c + pair + 4);
                sv[1] = *reinterpret_cast<const f32x4 *>(s + pair + 4);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int k = interleaved ? i / 2 : i;
            const bool first = interleaved ? !(i & 1) : (uint32_t)d0 < half;
            t.c[i] = cv[k / 4][k % 4];
            t.s[i] = first ? -sign * sv[k / 4][k % 4] : sign * sv[k / 4][k % 4];
        }
        return t;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint32_t d = d0 + i;
        const bool turns = d < rot, first = interleaved ? !(d & 1) : d < half;
        const uint32_t pair = !turns ? 0 : interleaved ? d >> 1 : first ? d : d - half;
        t.c[i] = turns ? c[pair] : 1.0f;
        t.s[i] = turns ? (first ? -sign : sign) * s[pair] : 0.0f;
    }
    return t;
}

// The other members of a lane's eight pairs.  row: the head's elements in the wavefront's buffer.
template <bool INTERLEAVED> __device__ inline void partners(const float v[8], float *row, int d0, uint32_t rot, float out[8])
{
    if constexpr (INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < 8; i++) out[i] = v[i ^ 1];
    } else {
        wave_lds_fence();
        *reinterpret_cast<f32x4 *>(row + d0) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4 *>(row + d0 + 4) = f32x4{v[4], v[5], v[6], v[7]};
        wave_lds_fence();
        const uint32_t half = rot / 2;
        if (half % 8 == 0) {                   // a lane's eight lie on one side, and so do their partners
            const uint32_t from = (uint32_t)d0 < half ? d0 + half : (uint32_t)d0 < rot ? d0 - half : d0;
            const f32x4 a = *reinterpret_cast<const f32x4 *>(row + from), b = *reinterpret_cast<const f32x4 *>(row + from + 4);
#pragma unroll
            for (int i = 0; i < 4; i++) { out[i] = a[i]; out[i + 4] = b[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t d = d0 + i;
                out[i] = row[d < half ? d + half : d < rot ? d - half : d];
            }
        }
    }
}
__device__ inline void turn(const Turn &t, const float v[8], const float other[8], int d0, uint32_t rot, float out[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++) out[i] = (uint32_t)(d0 + i) < rot ? fmaf(v[i], t.c[i], other[i] * t.s[i]) : v[i];
}

template <class T, bool WIDE, bool INTERLEAVED, int LANES>
__global__ __launch_bounds__(64 * WAVES) void k_qk_rotate(she_qk_rotate_args a, uint32_t steps, uint32_t per_wave, uint32_t chunks, bool aligned,
                                                          uint32_t *d_bad)
{
    constexpr int ROWS = 64 / LANES;
    __shared__ float rows[WAVES][64 * 8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = lane % LANES, row = lane / LANES, d0 = 8 * c, D = (int)a.head;
    const uint64_t unit = (uint64_t)blockIdx.x * WAVES + wave;
    const uint32_t t = (uint32_t)(unit / chunks), chunk = (uint32_t)(unit % chunks);
    if (t >= a.tokens) return;
    const bool paged = a.k_pages != nullptr;
    const int32_t position = a.positions[t];
    const bool placed = position >= 0 && (uint32_t)position < a.places;
    int64_t slot = paged ? a.slots[t] : -1;
    const bool slot_bad = paged && slot != -1 && (slot < 0 || slot >= (int64_t)a.pages * a.page_size);
    if (slot_bad || !placed) slot = -1;
    if (lane == 0 && chunk == 0 && (slot_bad || !placed)) count_bad(d_bad);
    const uint32_t page = slot >= 0 ? (uint32_t)((uint64_t)slot / a.page_size) : 0;
    const int64_t at = slot >= 0 ? page * a.page_stride + (slot - (int64_t)page * a.page_size) * a.slot_stride : 0;
    const int here = D - d0 < 0 ? 0 : D - d0 > 8 ? 8 : D - d0;     // of the lane's eight elements

    const Turn tr = load_turn(a.cosines, a.sines, placed ? a.rot : 0, INTERLEAVED, aligned, placed ? (uint32_t)position : 0, d0, 1.0f);
    float wq[8], wk[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        wq[i] = a.wq ? (i < here ? a.wq[d0 + i] : 0.0f) : 1.0f;
        wk[i] = a.wk ? (i < here ? a.wk[d0 + i] : 0.0f) : 1.0f;
    }
    const uint32_t heads = a.q_heads + a.kv_heads * (paged ? 2 : 1);
    const uint32_t end = min((chunk + 1) * per_wave, steps);
    for (uint32_t step = chunk * per_wave; step < end; step += BATCH) {
        u32x4 raw[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; b++) {
            const uint32_t h = (step + b) * ROWS + row;
            if (step + b < end && h < heads) {
                const T *p = h < a.q_heads ? (const T *)a.q + (int64_t)t * a.q_token + (int64_t)h * a.q_head
                             : h < a.q_heads + a.kv_heads ? (const T *)a.k + (int64_t)t * a.k_token + (int64_t)(h - a.q_heads) * a.k_head
                                                          : (const T *)a.v + (int64_t)t * a.v_token + (int64_t)(h - a.q_heads - a.kv_heads) * a.v_head;
                raw[b] = load8<T, WIDE>(p + d0, here);
            } else raw[b] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int b = 0; b < BATCH; b++) {
            if (step + b >= end) break;
            const uint32_t h = (step + b) * ROWS + row;
            float x[8], other[8], y[8], sum = 0;
            unpack<T>(raw[b], x);
#pragma unroll
            for (int i = 0; i < 8; i++) sum = fmaf(x[i], x[i], sum);
            const float r = 1.0f / sqrtf(head_sum<LANES>(sum) / D + a.eps);
            const bool is_q = h < a.q_heads;
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] *= r * (is_q ? wq[i] : wk[i]);
            partners<INTERLEAVED>(x, rows[wave] + row * LANES * 8, d0, a.rot, other);
            turn(tr, x, other, d0, a.rot, y);
            if (h >= heads) continue;
            const u32x4 words = placed ? pack<T>(y) : u32x4{0, 0, 0, 0};
            if (is_q) {
                store8<T, WIDE>((T *)a.q_out + (int64_t)t * a.q_out_token + (int64_t)h * a.q_out_head + d0, words, here);
            } else if (!paged) {
                store8<T, WIDE>((T *)a.k_out + (int64_t)t * a.k_out_token + (int64_t)(h - a.q_heads) * a.k_out_head + d0, words, here);
            } else if (slot >= 0) {
                const bool key = h < a.q_heads + a.kv_heads;
                T *to = key ? (T *)a.k_pages + (int64_t)(h - a.q_heads) * a.page_head
                            : (T *)a.v_pages + (int64_t)(h - a.q_heads - a.kv_heads) * a.page_head;
                store8<T, WIDE>(to + at + d0, key ? words : raw[b], here);
            }
        }
    }
}

// What the backward pass does with the queries, or with the keys.
struct GradSide {
    const void *x, *dy;
    int64_t x_token, x_head, dy_token, dy_head, dx_token, dx_head;
    const float *w;
    void *dx;
    uint32_t heads, steps, per_wave, chunks;   // as in QkShape
};
struct GradTurn {
    const float *cosines, *sines;
    const int32_t *positions;
    uint32_t tokens, head, rot, places;
    float eps;
    bool aligned;
};

// The first q_blocks workgroups have the queries, the others the keys, so that a lane keeps one weight and its sums.  Wavefronts walk
// the shares of all tokens; partial [blocks][D].
template <class T, bool WIDE, bool INTERLEAVED, int LANES>
__global__ __launch_bounds__(64 * WAVES, GRAD_RESIDENT) void k_qk_rotate_grad(GradSide q, GradSide k, GradTurn a, uint32_t q_blocks, float *partial, uint32_t *d_bad)
{
    constexpr int ROWS = 64 / LANES, PAIR = 2;
    __shared__ float rows[WAVES][64 * 8];
    __shared__ float sums[WAVES][LANES * 8];
    const bool is_q = blockIdx.x < q_blocks;
    const GradSide &side = is_q ? q : k;
    const uint32_t block = is_q ? blockIdx.x : blockIdx.x - q_blocks, blocks = is_q ? q_blocks : gridDim.x - q_blocks;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = lane % LANES, row = lane / LANES, d0 = 8 * c, D = (int)a.head;
    const int here = D - d0 < 0 ? 0 : D - d0 > 8 ? 8 : D - d0;
    float w[8], dw[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        w[i] = side.w ? (i < here ? side.w[d0 + i] : 0.0f) : 1.0f;
        dw[i] = 0;
    }
    const uint64_t units = (uint64_t)a.tokens * side.chunks;
    for (uint64_t unit = (uint64_t)block * WAVES + wave; unit < units; unit += (uint64_t)blocks * WAVES) {
        const uint32_t t = (uint32_t)(unit / side.chunks), chunk = (uint32_t)(unit % side.chunks);
        const int32_t position = a.positions[t];
        const bool placed = position >= 0 && (uint32_t)position < a.places;
        if (lane == 0 && chunk == 0 && is_q && !placed) count_bad(d_bad);
        const Turn tr = load_turn(a.cosines, a.sines, placed ? a.rot : 0, INTERLEAVED, a.aligned, placed ? (uint32_t)position : 0, d0, -1.0f);
        const uint32_t end = min((chunk + 1) * side.per_wave, side.steps);
        for (uint32_t step = chunk * side.per_wave; step < end; step += PAIR) {
            u32x4 raw_x[PAIR], raw_y[PAIR];
#pragma unroll
            for (int b = 0; b < PAIR; b++) {
                const uint32_t h = (step + b) * ROWS + row;
                raw_x[b] = raw_y[b] = u32x4{0, 0, 0, 0};
                if (step + b >= end || h >= side.heads) continue;
                raw_x[b] = load8<T, WIDE>((const T *)side.x + t * side.x_token + h * side.x_head + d0, here);
                raw_y[b] = load8<T, WIDE>((const T *)side.dy + t * side.dy_token + h * side.dy_head + d0, here);
            }
#pragma unroll
            for (int b = 0; b < PAIR; b++) {
                if (step + b >= end) break;
                const uint32_t h = (step + b) * ROWS + row;
                float x[8], dy[8], other[8], g[8], sum = 0, dot = 0;
                unpack<T>(raw_x[b], x);
                unpack<T>(raw_y[b], dy);
#pragma unroll
                for (int i = 0; i < 8; i++) sum = fmaf(x[i], x[i], sum);
                const float r = 1.0f / sqrtf(head_sum<LANES>(sum) / D + a.eps);
                partners<INTERLEAVED>(dy, rows[wave] + row * LANES * 8, d0, a.rot, other);
                turn(tr, dy, other, d0, a.rot, g);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    x[i] *= r;
                    const float gu = placed && h < side.heads ? g[i] * x[i] : 0.0f;
                    dw[i] += gu;
                    g[i] *= w[i];
                    dot = fmaf(w[i], gu, dot);
                }
                dot = head_sum<LANES>(dot) / D;
                if (h >= side.heads) continue;
#pragma unroll
                for (int i = 0; i < 8; i++) g[i] = placed ? r * (g[i] - x[i] * dot) : 0.0f;
                store8<T, WIDE>((T *)side.dx + t * side.dx_token + h * side.dx_head + d0, pack<T>(g), here);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
#pragma unroll
        for (int m = LANES; m < 64; m *= 2) dw[i] += __shfl_xor(dw[i], m);
        if (row == 0) sums[wave][d0 + i] = dw[i];
    }
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += 64 * WAVES) {
        float v = 0;
        for (int k = 0; k < WAVES; k++) v += sums[k][d];
        partial[(size_t)blockIdx.x * D + d] = v;
    }
}

// dwq, dwk = sums of the workgroups' partial sums: SUM_COLS columns a workgroup, SUM_PARTS threads a column, whose loads are
// requested eight at a time.
constexpr int SUM_COLS = 8, SUM_PARTS = 128;
__global__ __launch_bounds__(SUM_COLS * SUM_PARTS) void k_qk_weight_sums(const float *partial, uint32_t q_blocks, uint32_t blocks, uint32_t D, float *dwq, float *dwk)
{
    __shared__ float sums[SUM_PARTS][SUM_COLS + 1];
    const uint32_t col = blockIdx.x * SUM_COLS + threadIdx.x % SUM_COLS, part = threadIdx.x / SUM_COLS;
    const uint32_t first = blockIdx.y ? q_blocks : 0, rows = blockIdx.y ? blocks : q_blocks;
    float v = 0;
    if (col < D)
        for (uint32_t r0 = first + part; r0 < rows; r0 += 8 * SUM_PARTS) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = r0 + i * SUM_PARTS < rows ? partial[(size_t)(r0 + i * SUM_PARTS) * D + col] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i++) v += x[i];
        }
    sums[part][threadIdx.x % SUM_COLS] = v;
    __syncthreads();
    if (part >= 8) return;                                        // eight threads a column, then one
    v = 0;
    for (int p = part; p < SUM_PARTS; p += 8) v += sums[p][threadIdx.x % SUM_COLS];
#pragma unroll
    for (int m = SUM_COLS; m < 64; m *= 2) v += __shfl_xor(v, m);
    float *to = blockIdx.y ? dwk : dwq;
    if (to && !part && col < D) to[col] = v;
}

bool on16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// whether a lane's cosines and sines are neighbours on 16 bytes
bool turn_aligned(const float *cosines, const float *sines, uint32_t rot, bool interleaved)
{
    return on16(cosines) && on16(sines) && rot % (interleaved ? 8 : 16) == 0;
}

uint32_t lanes_of(uint32_t head) { return head <= 64 ? 8 : head <= 128 ? 16 : head <= 256 ? 32 : 64; }

// A token's heads are shared out among wavefronts only as far as it takes to give every SIMD about eight of them.
void share_out(QkShape &s, uint32_t tokens, uint32_t cus)
{
    s.steps = (uint32_t)ceil_div(s.heads, 64 / s.lanes);
    const uint64_t wanted = 32ull * (cus ? cus : 1), all = (uint64_t)tokens * s.steps;
    s.per_wave = (uint32_t)std::min<uint64_t>(s.steps, std::max<uint64_t>(1, all / wanted));
    s.chunks = (uint32_t)ceil_div(s.steps, s.per_wave);
    s.blocks = (uint32_t)ceil_div((uint64_t)tokens * s.chunks, WAVES);
}

template <template <class, bool, bool, int> class Launch, class... A> hipError_t choose(int type, bool wide, bool interleaved, uint32_t lanes, A &&...args)
{
    auto lanes_next = [&](auto t, auto w, auto i) {
        using T = decltype(t);
        constexpr bool W = decltype(w)::value, I = decltype(i)::value;
        return lanes == 8 ? Launch<T, W, I, 8>::go(args...) : lanes == 16 ? Launch<T, W, I, 16>::go(args...)
             : lanes == 32 ? Launch<T, W, I, 32>::go(args...) : Launch<T, W, I, 64>::go(args...);
    };
    auto inter_next = [&](auto t, auto w) { return interleaved ? lanes_next(t, w, std::true_type{}) : lanes_next(t, w, std::false_type{}); };
    auto wide_next = [&](auto t) { return wide ? inter_next(t, std::true_type{}) : inter_next(t, std::false_type{}); };
    return type == SHE_BF16 ? wide_next((__bf16)0.0f) : wide_next((_Float16)0.0f);
}
template <class T, bool W, bool I, int L> struct Rotate {
    static hipError_t go(const she_qk_rotate_args &a, const QkShape &s, uint32_t *d_bad, hipStream_t st)
    {
        k_qk_rotate<T, W, I, L><<<s.blocks, 64 * WAVES, 0, st>>>(a, s.steps, s.per_wave, s.chunks, s.aligned, d_bad);
        return hipGetLastError();
    }
};
template <class T, bool W, bool I, int L> struct RotateGrad {
    static hipError_t go(const GradSide &q, const GradSide &k, const GradTurn &a, const QkGradShape &s, float *partial, uint32_t *d_bad, hipStream_t st)
    {
        k_qk_rotate_grad<T, W, I, L><<<s.q.blocks + s.k.blocks, 64 * WAVES, 0, st>>>(q, k, a, s.q.blocks, partial, d_bad);
        return hipGetLastError();
    }
};

}  // namespace

QkShape qk_shape(const she_qk_rotate_args &a, uint32_t cus)
{
    QkShape s{};
    const bool paged = a.k_pages != nullptr;
    s.lanes = lanes_of(a.head);
    s.heads = a.q_heads + a.kv_heads * (paged ? 2 : 1);
    int64_t strides = a.q_token | a.q_head | a.k_token | a.k_head | a.q_out_token | a.q_out_head | a.head;
    s.wide = on16(a.q) && on16(a.k) && on16(a.q_out);
    if (paged) {
        strides |= a.v_token | a.v_head | a.page_stride | a.slot_stride | a.page_head;
        s.wide = s.wide && on16(a.v) && on16(a.k_pages) && on16(a.v_pages);
    } else {
        strides |= a.k_out_token | a.k_out_head;
        s.wide = s.wide && on16(a.k_out);
    }
    s.wide = s.wide && strides % 8 == 0;
    s.aligned = turn_aligned(a.cosines, a.sines, a.rot, a.interleaved != 0);
    share_out(s, a.tokens, cus);
    return s;
}

QkGradShape qk_grad_shape(const she_qk_rotate_grad_args &a, uint32_t cus)
{
    QkGradShape s{};
    s.lanes = lanes_of(a.head);
    const int64_t strides = a.q_token | a.q_head | a.k_token | a.k_head | a.dq_out_token | a.dq_out_head | a.dk_out_token | a.dk_out_head |
                            a.dq_token | a.dq_head | a.dk_token | a.dk_head | a.head;
    s.wide = strides % 8 == 0 && on16(a.q) && on16(a.k) && on16(a.dq_out) && on16(a.dk_out) && on16(a.dq) && on16(a.dk);
    s.aligned = turn_aligned(a.cosines, a.sines, a.rot, a.interleaved != 0);
    // Each workgroup leaves a row of partial sums: no more than are resident together, the queries' and the keys' in proportion to
    // their heads, and all of a side with as many shares, so that they end together.
    const uint32_t resident = GRAD_RESIDENT * (cus ? cus : 1);
    const auto side = [&](QkShape &q, uint32_t heads) {
        q.lanes = s.lanes;
        q.heads = heads;
        share_out(q, a.tokens, cus);
        const uint32_t part = std::max(1u, (uint32_t)((uint64_t)resident * heads / (a.q_heads + a.kv_heads)));
        const uint32_t rounds = std::max(1u, (uint32_t)ceil_div(q.blocks, part));
        q.blocks = std::max(1u, (uint32_t)ceil_div(q.blocks, rounds));
    };
    side(s.q, a.q_heads);
    side(s.k, a.kv_heads);
    return s;
}

size_t qk_grad_scratch(const QkGradShape &s, uint32_t head) { return (size_t)(s.q.blocks + s.k.blocks) * head * sizeof(float); }

hipError_t launch_qk_rotate(const she_qk_rotate_args &a, const QkShape &s, uint32_t *d_bad, hipStream_t st)
{
    return choose<Rotate>(a.type, s.wide, a.interleaved != 0, s.lanes, a, s, d_bad, st);
}

hipError_t launch_qk_rotate_grad(const she_qk_rotate_grad_args &a, const QkGradShape &s, void *scratch, uint32_t *d_bad, hipStream_t st)
{
    float *partial = static_cast<float *>(scratch);
    const GradSide q{a.q, a.dq_out, a.q_token, a.q_head, a.dq_out_token, a.dq_out_head, a.dq_token, a.dq_head, a.wq, a.dq, s.q.heads, s.q.steps, s.q.per_wave, s.q.chunks};
    const GradSide k{a.k, a.dk_out, a.k_token, a.k_head, a.dk_out_token, a.dk_out_head, a.dk_token, a.dk_head, a.wk, a.dk, s.k.heads, s.k.steps, s.k.per_wave, s.k.chunks};
    const GradTurn t{a.cosines, a.sines, a.positions, a.tokens, a.head, a.rot, a.places, a.eps, s.aligned};
    hipError_t rc = choose<RotateGrad>(a.type, s.wide, a.interleaved != 0, s.lanes, q, k, t, s, partial, d_bad, st);
    if (rc != hipSuccess || (!a.dwq && !a.dwk)) return rc;
    k_qk_weight_sums<<<dim3((uint32_t)ceil_div(a.head, SUM_COLS), 2), SUM_COLS * SUM_PARTS, 0, st>>>(partial, s.q.blocks, s.q.blocks + s.k.blocks, a.head, a.dwq, a.dwk);
    return hipGetLastError();
}

}}  // namespace she::clear
