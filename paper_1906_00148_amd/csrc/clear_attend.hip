// Attention of each request's new tokens over its paged cache.
//
// The query heads that share a key head are packed with the tokens: the rows of a request at one key head are its new tokens times
// the `group` query heads, token by token, and a tile of rows reads the request's keys and values once for all of them.  Along the
// cache a tile's places are cut into pieces of `chunk`, each a workgroup of its own; where a tile has more than one, they leave
// (top, sum, weighted values) of every row behind and k_attend_join puts them together in order.
//
// Scores are taken transposed, S^T = K Q^T, so that the lanes' results are the operands of the second product O^T = V^T P^T as they
// lie: a lane's scores of one row become eight places of one column, if V's rows are taken in the same order.  The softmax is the
// running one: a top m and a sum l per row in 32 bits, weights exp2(s - m) with log2(e) in the scale.  The weights are rounded to the
// type for the second product (their sum is not): an error of the size of the result's own rounding.
//
// Masks: a place that no row of the tile attends to is not read at all.  A place that some rows attend to and others do not has weight
// 0 for the others, which a matrix instruction multiplies with the value all the same; so where values of such places are
// infinite or NaN, the step is done row by row with the hidden places' values taken out.
#include <algorithm>
#include <type_traits>

#include "clear_device.h"
#include "clear_internal.h"

namespace she { namespace clear {
namespace {

constexpr int FEW_ROWS = 16, FEW_WAVES = 4, MOST_CHUNK = 2048;
constexpr float LOG2E = 1.4426950408889634f;

struct Work {                            // of the pieces of a cut row, [tokens * q_heads][splits]
    float *o;                            // [..][head]
    float2 *ml;
    uint32_t chunk, splits;
};

// A tile of rows and the places that any of them attends to.
struct Span {
    int request;                         // -1: nothing here
    int row, rows;                       // first row in the request, rows of the tile
    int64_t token0;                      // the request's first token
    int first;                           // place of the request's first new token (negative: its length is short of them)
    int from, to;                        // places, `from` a multiple of 32; none if to <= from
    int parts;                           // pieces that they are cut into
};
template <int ROWS> __device__ inline Span span_of(const she_attend_pages_args &a, uint32_t group, const Piece &p, int row, uint32_t chunk)
{
    Span s{};
    s.request = p.segment;
    if (p.segment < 0) return s;
    const int all = (int)(p.last - p.first), news = all / (int)group;
    const int64_t room = (int64_t)a.table_width * a.page_size;
    const int length = max(a.lengths[p.segment], 0);
    s.row = row;
    s.rows = min(ROWS, all - row);
    s.token0 = p.first / group;
    s.first = length - news;
    const int p0 = s.first + row / (int)group, p1 = s.first + (row + s.rows - 1) / (int)group;
    const int64_t low = a.window ? (int64_t)p0 - (int64_t)a.window + 1 : 0;
    s.from = (int)max(low, (int64_t)0) & ~31;
    s.to = (int)min((int64_t)p1 + 1, room);
    s.parts = s.to > s.from ? (int)(((uint32_t)(s.to - s.from) + chunk - 1) / chunk) : 0;
    return s;
}

// Where the rows of the places [from, from + count) start, -1 for those that their page id keeps out; returns whether any is.
__device__ inline void look_up(const she_attend_pages_args &a, int request, int kv_head, int from, int count, int64_t *rows, int *any_bad, uint32_t *d_bad)
{
    for (int i = threadIdx.x; i < count; i += blockDim.x) {
        const uint32_t place = from + i, column = place / a.page_size, in_page = place - column * a.page_size;
        const int32_t page = a.table[request * a.table_stride + column];
        const bool good = page >= 0 && (uint32_t)page < a.pages;
        rows[i] = good ? page * a.page_stride + in_page * a.slot_stride + kv_head * a.page_head : -1;
        if (!good) {
            *any_bad = 1;
            if (in_page == 0 || i == 0) count_bad(d_bad);
        }
    }
}

template <class T> __device__ inline bool has_special(u32x4 v)
{
    constexpr uint32_t E = std::is_same<T, __bf16>::value ? 0x7F80u : 0x7C00u;
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; i++) any |= (v[i] & E) == E || (v[i] & E << 16) == E << 16;
    return any;
}

// Few rows: every wavefront walks places of its own, 32 a step, four steps of the workgroup side by side, straight from memory.  Lane
// l reads d = 32 s + 8 (l/16) .. of the key of place l%16 for the scores, and EL elements from EL (l%16) on of the values of the
// eight places that its scores belong to, whole rows over 16 lanes; the eight rows are transposed in registers.
template <class T, int DP>
__global__ __launch_bounds__(64 * FEW_WAVES, 2) void k_attend_few(she_attend_pages_args a, uint32_t group, Work w, uint32_t *d_bad)
{
    constexpr int EL = DP == 64 ? 4 : 8, NB = DP == 256 ? 2 : 1, KS = DP / 32;
    __shared__ int64_t rows[MOST_CHUNK];
    __shared__ float joined[FEW_WAVES][FEW_ROWS][DP];
    __shared__ float tops[FEW_WAVES][FEW_ROWS], sums[FEW_WAVES][FEW_ROWS];
    __shared__ int any_bad;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quarter = lane >> 4;
    const int kv_head = blockIdx.y, D = (int)a.head;
    const Piece piece = find_piece(a.starts, a.requests, a.tokens, group, FEW_ROWS, blockIdx.x);
    const Span sp = span_of<FEW_ROWS>(a, group, piece, piece.index * FEW_ROWS, w.chunk);
    if (sp.request < 0 || (int)blockIdx.z >= max(sp.parts, 1)) return;
    const int from = sp.from + (int)blockIdx.z * (int)w.chunk, count = sp.parts ? min((int)w.chunk, sp.to - from) : 0;
    if (tid == 0) any_bad = 0;
    __syncthreads();
    look_up(a, sp.request, kv_head, from, count, rows, &any_bad, d_bad);

    // this lane's row
    const int my_row = min(sp.row + col, sp.row + sp.rows - 1), my_token = my_row / (int)group, my_head = kv_head * (int)group + my_row % (int)group;
    const int high = sp.first + my_token, low = a.window ? (int)max((int64_t)high - (int64_t)a.window + 1, (int64_t)0) : 0;
    const int high_min = sp.first + sp.row / (int)group, low_max = a.window ? (int)max((int64_t)sp.first + (sp.row + sp.rows - 1) / (int)group - (int64_t)a.window + 1, (int64_t)0) : 0;
    x8<T> q[KS];
    {
        const T *p = (const T *)a.q + (sp.token0 + my_token) * a.q_token + my_head * a.q_head + quarter * 8;
#pragma unroll
        for (int s = 0; s < KS; s++) q[s] = as_x8<T>(load8<T, true>(p + s * 32, D - (s * 32 + quarter * 8)));
    }
    const float scale = a.scale * LOG2E;
    float m = -__builtin_inff(), l = 0;
    f32x4 acc[NB][EL];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < EL; e++) acc[b][e] = f32x4{0, 0, 0, 0};
    __syncthreads();
    const bool unsafe = any_bad != 0;

    for (int k0 = wave * 32; k0 < count; k0 += FEW_WAVES * 32) {
        u32x4 kraw[2][KS];
#pragma unroll
        for (int t = 0; t < 2; t++) {
            const int i = k0 + t * 16 + col;
            const int64_t row = i < count ? rows[i] : -1;
            const T *p = (const T *)a.k_pages + (row < 0 ? 0 : row) + quarter * 8;
#pragma unroll
            for (int s = 0; s < KS; s++) kraw[t][s] = load8<T, true>(p + s * 32, row < 0 ? 0 : D - (s * 32 + quarter * 8));
        }
        u32x4 vraw[NB][8];
        uint32_t there = 0;                                       // which of the lane's eight places exist
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const int i = k0 + (e < 4 ? 0 : 16) + quarter * 4 + (e & 3);
            const int64_t row = i < count ? rows[i] : -1;
            there |= row < 0 ? 0u : 1u << e;
#pragma unroll
            for (int b = 0; b < NB; b++) {
                const int d = b * 128 + col * EL;
                const T *p = (const T *)a.v_pages + (row < 0 ? 0 : row) + d;
                if constexpr (EL == 8) vraw[b][e] = load8<T, true>(p, row < 0 ? 0 : D - d);
                else {
                    const uint2 v = row >= 0 && d < D ? *reinterpret_cast<const uint2 *>(p) : uint2{0, 0};
                    vraw[b][e] = u32x4{v.x, v.y, 0, 0};
                }
            }
        }
        f32x4 st[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
            for (int s = 0; s < KS; s++) st[t] = mfma16(as_x8<T>(kraw[t][s]), q[s], st[t]);

        const bool masked = unsafe || k0 + 32 > count || from + k0 + 31 > high_min || from + k0 < low_max;
        float s[8], top = m;
        uint32_t hidden = 0;                                      // which of the lane's eight places its row does not attend to
#pragma unroll
        for (int e = 0; e < 8; e++) s[e] = st[e / 4][e % 4] * scale;
        if (masked) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const int place = from + k0 + (e < 4 ? 0 : 16) + quarter * 4 + (e & 3);
                if (!(there >> e & 1) || place > high || place < low) {
                    s[e] = -__builtin_inff();
                    hidden |= 1u << e;
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; e++) top = fmaxf(top, s[e]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float ref = top == -__builtin_inff() ? 0.0f : top, alpha = __builtin_amdgcn_exp2f(m - ref);
        m = top;
        x8<T> p;
        float sum = 0;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float v = __builtin_amdgcn_exp2f(s[e] - ref);
            sum += v;
            p[e] = (T)v;
        }
        l = fmaf(l, alpha, sum);
        if (__ballot(alpha != 1.0f)) {
#pragma unroll
            for (int b = 0; b < NB; b++)
#pragma unroll
                for (int e = 0; e < EL; e++)
#pragma unroll
                    for (int i = 0; i < 4; i++) acc[b][e][i] *= alpha;
        }
        bool special = false;
        if (masked) {
#pragma unroll
            for (int b = 0; b < NB; b++)
#pragma unroll
                for (int e = 0; e < 8; e++) special |= has_special<T>(vraw[b][e]);
        }
        if (!__ballot(special)) {
#pragma unroll
            for (int b = 0; b < NB; b++) {
                x8<T> v[EL];
                transpose8<T, EL>(vraw[b], v);
#pragma unroll
                for (int e = 0; e < EL; e++) acc[b][e] = mfma16(v[e], p, acc[b][e]);
            }
        } else {
            for (int c = 0; c < FEW_ROWS; c++) {
                // the places that row c does not attend to: a quarter's eight are known to the quarter's lane of column c
                const uint32_t out = __shfl(hidden, quarter * 16 + c);
#pragma unroll
                for (int b = 0; b < NB; b++) {
                    u32x4 kept[8];
#pragma unroll
                    for (int e = 0; e < 8; e++) kept[e] = out >> e & 1 ? u32x4{0, 0, 0, 0} : vraw[b][e];
                    x8<T> v[EL];
                    transpose8<T, EL>(kept, v);
#pragma unroll
                    for (int e = 0; e < EL; e++) {
                        const f32x4 o = mfma16(v[e], p, f32x4{0, 0, 0, 0});
#pragma unroll
                        for (int i = 0; i < 4; i++) acc[b][e][i] += col == c ? o[i] : 0.0f;
                    }
                }
            }
        }
    }

    // the wavefronts' results, and the piece's
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (quarter == 0) { tops[wave][col] = m; sums[wave][col] = l; }
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int e = 0; e < EL; e += 4)
                *reinterpret_cast<f32x4 *>(&joined[wave][col][b * 128 + (quarter * 4 + i) * EL + e]) =
                    f32x4{acc[b][e][i], acc[b][e + 1][i], acc[b][e + 2][i], acc[b][e + 3][i]};
    __syncthreads();
    constexpr int EACH = DP / 16;                                 // elements of a row that a thread joins
    const int r = tid / 16, d0 = tid % 16 * EACH;
    if (r >= sp.rows) return;
    float top = -__builtin_inff(), sum = 0, o[EACH];
#pragma unroll
    for (int k = 0; k < FEW_WAVES; k++) top = fmaxf(top, tops[k][r]);
#pragma unroll
    for (int i = 0; i < EACH; i++) o[i] = 0;
#pragma unroll
    for (int k = 0; k < FEW_WAVES; k++) {
        const float f = tops[k][r] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(tops[k][r] - top);
        sum = fmaf(sums[k][r], f, sum);
#pragma unroll
        for (int i = 0; i < EACH; i++) o[i] = fmaf(joined[k][r][d0 + i], f, o[i]);
    }
    const int row = sp.row + r;
    const int64_t token = sp.token0 + row / (int)group;
    const int head = kv_head * (int)group + row % (int)group;
    if (sp.parts <= 1) {
        const float inv = sum == 0 ? 0.0f : 1.0f / sum;
        T *to = (T *)a.out + token * a.out_token + head * a.out_head + d0;
#pragma unroll
        for (int i = 0; i < EACH; i++)
            if (d0 + i < D) to[i] = (T)(o[i] * inv);
    } else {
        const size_t at = (size_t)(token * a.q_heads + head) * w.splits + blockIdx.z;
        if (d0 == 0) w.ml[at] = float2{top, sum};
#pragma unroll
        for (int i = 0; i < EACH; i++)
            if (d0 + i < D) w.o[at * D + d0 + i] = o[i];
    }
}

// The rows that were cut: a wavefront a row.
template <class T>
__global__ __launch_bounds__(256) void k_attend_join(she_attend_pages_args a, uint32_t group, Work w)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = (int)a.head;
    const Piece piece = find_piece(a.starts, a.requests, a.tokens, group, FEW_ROWS, blockIdx.x);
    const Span sp = span_of<FEW_ROWS>(a, group, piece, piece.index * FEW_ROWS, w.chunk);
    if (sp.request < 0 || sp.parts <= 1) return;
    for (int r = wave; r < sp.rows; r += 4) {
        const int row = sp.row + r;
        const int64_t token = sp.token0 + row / (int)group;
        const int head = blockIdx.y * (int)group + row % (int)group;
        const size_t at = (size_t)(token * a.q_heads + head) * w.splits;
        float top = -__builtin_inff(), sum = 0;
        for (int k = 0; k < sp.parts; k++) top = fmaxf(top, w.ml[at + k].x);
        float o[4] = {0, 0, 0, 0};
        for (int k = 0; k < sp.parts; k++) {
            const float2 ml = w.ml[at + k];
            const float f = ml.x == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(ml.x - top);
            sum = fmaf(ml.y, f, sum);
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (lane + 64 * i < D) o[i] = fmaf(w.o[(at + k) * D + lane + 64 * i], f, o[i]);
        }
        const float inv = sum == 0 ? 0.0f : 1.0f / sum;
        T *to = (T *)a.out + token * a.out_token + head * a.out_head;
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (lane + 64 * i < D) to[lane + 64 * i] = (T)(o[i] * inv);
    }
}

template <class T> hipError_t attend(const she_attend_pages_args &a, const AttendShape &s, const Work &w, uint32_t *d_bad, hipStream_t st)
{
    const uint32_t group = a.q_heads / a.kv_heads;
    const dim3 grid((uint32_t)s.few_slots, a.kv_heads, s.splits);
    if (a.head <= 64) k_attend_few<T, 64><<<grid, 64 * FEW_WAVES, 0, st>>>(a, group, w, d_bad);
    else if (a.head <= 128) k_attend_few<T, 128><<<grid, 64 * FEW_WAVES, 0, st>>>(a, group, w, d_bad);
    else k_attend_few<T, 256><<<grid, 64 * FEW_WAVES, 0, st>>>(a, group, w, d_bad);
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess || s.splits <= 1) return rc;
    k_attend_join<T><<<dim3((uint32_t)s.few_slots, a.kv_heads), 256, 0, st>>>(a, group, w);
    return hipGetLastError();
}

}  // namespace

AttendShape attend_shape(const she_attend_pages_args &a, uint32_t cus)
{
    AttendShape s{};
    const uint64_t group = a.q_heads / a.kv_heads, longest = std::min<uint64_t>((uint64_t)a.table_width * a.page_size, 0x7FFFFFFF);
    s.few_slots = a.tokens * group / FEW_ROWS + a.requests;
    s.tile_slots = 0;
    // pieces short enough for eight workgroups per compute unit, long enough that joining them costs little
    const uint64_t places = s.few_slots * a.kv_heads * longest;
    s.chunk = (uint32_t)std::min<uint64_t>(MOST_CHUNK, std::max<uint64_t>(256, ceil_div(places / (8 * (cus ? cus : 1)), 128) * 128));
    // a span starts at a multiple of 32 below its first place
    s.splits = (uint32_t)std::max<uint64_t>(1, ceil_div(longest, s.chunk));
    return s;
}

size_t attend_scratch(const she_attend_pages_args &a, const AttendShape &s)
{
    return s.splits <= 1 ? 0 : (size_t)a.tokens * a.q_heads * s.splits * (a.head * sizeof(float) + sizeof(float2));
}

hipError_t launch_attend_pages(const she_attend_pages_args &a, const AttendShape &s, void *scratch, uint32_t *d_bad, hipStream_t st)
{
    const size_t rows = (size_t)a.tokens * a.q_heads * s.splits;
    const Work w{static_cast<float *>(scratch), reinterpret_cast<float2 *>(static_cast<float *>(scratch) + rows * a.head), s.chunk, s.splits};
    return a.type == SHE_BF16 ? attend<__bf16>(a, s, w, d_bad, st) : attend<_Float16>(a, s, w, d_bad, st);
}

}}  // namespace she::clear
