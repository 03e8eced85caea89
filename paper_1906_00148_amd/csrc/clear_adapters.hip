// Low-rank adapters of many requests beside a shared projection, forward and backward.
//
// All the products have one of three shapes, for a tile of 32 tokens of one segment and its adapter (rank r of tens, widths of
// thousands):
//     k_adapter_down   h[t][j] = scale sum_k w[j][k] x[t][k]      x . down^T, and dy . up^T backward
//     k_adapter_up     y[t][n] = base + sum_j h[t][j] w[j][n]     h . up, and g . down backward
//     k_adapter_outer  d[j][k] = sum_t h[t][j] x[t][k]            g^T x and h^T dy, over all of an adapter's tiles
// Both matrices are rank-major, so the first reads its operands of the matrix instructions as they lie, eight neighbours along k a
// lane.  The other two sum along the slow axis: a lane reads eight rows of eight neighbours and transposes that block in its
// registers, one byte permutation a word of two elements, which makes the operands of eight matrix instructions.
//
// h is held in 32 bits while it is summed and handed on as two numbers of the type, the rounded value and what the rounding left
// (17 bits of it in bf16, 22 in f16), each with a product of its own: as good as 32 bits beside results of 8 or 11.  In f16 a tile's h
// is scaled by a power of two first, so that the range of the type does not matter.
//
// Bound by memory: x, base and the adapters are read, and the result written, once; a tile's h is a few KB.
#include <algorithm>
#include <type_traits>

#include "clear_device.h"
#include "clear_internal.h"

namespace she { namespace clear {
namespace {

constexpr int TILE = 32;                 // tokens
constexpr int CHUNK = 64;                // ranks that a workgroup of k_adapter_down or k_adapter_outer does
constexpr int UP_WAVES = 4, SPAN = 128;  // wavefronts of k_adapter_up, outputs of one
constexpr int OUTER_WAVES = 8;

// The hidden values of all tiles.  rows: r rounded up to 16.
struct Hidden {
    uint16_t *by_token[2];               // [slots][TILE][rows], value and rest; null: not wanted
    uint16_t *by_rank[2];                // [slots][rows][TILE]
    float *unscale;                      // [slots][chunks]: f16, what a tile's values are to be multiplied by
};
struct Segments {
    const int32_t *starts, *which, *ranks;
    const float *scale;
    uint32_t tokens, segments, adapters, rank, rows, chunks;
    uint32_t share, most, places;        // backward: tiles of a workgroup, workgroups of an adapter at most, places for their sums
};
struct Matrix {                          // [adapters][rank][width]
    const void *p;
    int64_t adapter, row;
    uint32_t width;
};
struct Rows {                            // [tokens][width]
    const void *p;
    int64_t stride;
};

__device__ inline int adapter_of(const Segments &s, int segment, uint32_t *d_bad)
{
    const int32_t a = s.which[segment];
    if (a >= 0 && (uint32_t)a < s.adapters) return a;
    if (d_bad && a != -1) count_bad(d_bad);
    return -1;
}
__device__ inline uint32_t rank_of(const Segments &s, int a)
{
    if (!s.ranks) return s.rank;
    const int32_t r = s.ranks[a];
    return r < 0 ? 0 : min((uint32_t)r, s.rank);
}

// v as the type's nearest value and the rest.  An infinity has no rest.
template <class T> __device__ inline void split(float v, uint16_t &value, uint16_t &rest)
{
    const T a = (T)v;
    const float left = v - (float)a;
    value = __builtin_bit_cast(uint16_t, a);
    rest = __builtin_bit_cast(uint16_t, (T)(fabsf(left) < __builtin_inff() ? left : 0.0f));
}

struct Down {
    Rows x;
    Matrix w;
    Hidden h;
};

// One tile, up to CHUNK ranks (RT tiles of 16) of it: the wavefronts share the width out, 32 columns a step.
template <class T, bool WIDE, int RT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_adapter_down(Down job0, Down job1, Segments s, uint32_t *d_bad)
{
    __shared__ float part[WAVES][RT * 16][TILE];
    __shared__ float tops[WAVES];
    const Down &job = blockIdx.z ? job1 : job0;
    const uint32_t slot = blockIdx.x, r0 = blockIdx.y * CHUNK;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quarter = lane >> 4;
    const Piece piece = find_piece(s.starts, s.segments, s.tokens, 1, TILE, slot);
    if (piece.segment < 0) return;
    const int a = adapter_of(s, piece.segment, tid == 0 && blockIdx.y == 0 && blockIdx.z == 0 && piece.index == 0 ? d_bad : nullptr);
    if (a < 0) return;
    const uint32_t rank = rank_of(s, a), K = job.w.width;
    const int64_t t0 = piece.first + (int64_t)piece.index * TILE;
    const int live = (int)min((int64_t)TILE, piece.last - t0);

    const T *x[2], *w[RT];
    bool has_x[2], has_w[RT];
#pragma unroll
    for (int c = 0; c < 2; c++) {
        has_x[c] = c * 16 + col < live;
        x[c] = (const T *)job.x.p + (t0 + (has_x[c] ? c * 16 + col : 0)) * job.x.stride + quarter * 8;
    }
#pragma unroll
    for (int r = 0; r < RT; r++) {
        const uint32_t j = r0 + r * 16 + col;
        has_w[r] = j < rank;
        w[r] = (const T *)job.w.p + a * job.w.adapter + (has_w[r] ? j : 0) * job.w.row + quarter * 8;
    }
    f32x4 acc[RT][2];
#pragma unroll
    for (int r = 0; r < RT; r++) acc[r][0] = acc[r][1] = f32x4{0, 0, 0, 0};
    constexpr int AHEAD = !WIDE ? 1 : RT == 4 ? 2 : 4;     // steps whose loads are requested together
    for (uint32_t k0 = wave * 32; k0 < K; k0 += AHEAD * WAVES * 32) {
        x8<T> xv[AHEAD][2], wv[AHEAD][RT];
#pragma unroll
        for (int e = 0; e < AHEAD; e++) {
            const uint32_t k = k0 + e * WAVES * 32;
            const int count = (int)K - (int)(k + quarter * 8);
#pragma unroll
            for (int c = 0; c < 2; c++) xv[e][c] = as_x8<T>(load8<T, WIDE>(x[c] + k, has_x[c] ? min(count, 8) : 0));
#pragma unroll
            for (int r = 0; r < RT; r++) wv[e][r] = as_x8<T>(load8<T, WIDE>(w[r] + k, has_w[r] ? min(count, 8) : 0));
        }
#pragma unroll
        for (int e = 0; e < AHEAD; e++)
#pragma unroll
            for (int r = 0; r < RT; r++) {
                acc[r][0] = mfma16(wv[e][r], xv[e][0], acc[r][0]);
                if (live > 16) acc[r][1] = mfma16(wv[e][r], xv[e][1], acc[r][1]);
            }
    }
#pragma unroll
    for (int r = 0; r < RT; r++)
#pragma unroll
        for (int c = 0; c < 2; c++)
#pragma unroll
            for (int i = 0; i < 4; i++) part[wave][r * 16 + quarter * 4 + i][c * 16 + col] = acc[r][c][i];
    __syncthreads();

    constexpr int VALUES = RT * 16 * TILE, EACH = (VALUES + 64 * WAVES - 1) / (64 * WAVES);
    const float scale = s.scale[a];
    float v[EACH], top = 0;
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const int n = e * 64 * WAVES + tid;
        v[e] = 0;
        if (n >= VALUES) continue;
        const float *p = &part[0][0][0] + n;
#pragma unroll
        for (int k = 0; k < WAVES; k++) v[e] += p[k * VALUES];
        // what no token or rank stands behind is zero, not what an infinity makes of zeros
        v[e] = n % TILE < live && r0 + n / TILE < rank ? v[e] * scale : 0.0f;
        if (fabsf(v[e]) < __builtin_inff()) top = fmaxf(top, fabsf(v[e]));
    }
    float by = 1;
    if constexpr (std::is_same<T, _Float16>::value) {
#pragma unroll
        for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = 0;
#pragma unroll
        for (int k = 0; k < WAVES; k++) top = fmaxf(top, tops[k]);
        const int e = top > 0 ? min(max(ilogbf(top), -100), 120) : 0;          // the largest becomes 2^13 .. 2^14
        by = ldexpf(1.0f, 13 - e);
        if (tid == 0) job.h.unscale[(size_t)slot * s.chunks + blockIdx.y] = ldexpf(1.0f, e - 13);
    }
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const int n = e * 64 * WAVES + tid, j = r0 + n / TILE, t = n % TILE;
        if (n >= VALUES || (uint32_t)j >= s.rows) continue;
        uint16_t value, rest;
        split<T>(v[e] * by, value, rest);
        if (job.h.by_token[0]) {
            const size_t at = ((size_t)slot * TILE + t) * s.rows + j;
            job.h.by_token[0][at] = value;
            job.h.by_token[1][at] = rest;
        }
        if (job.h.by_rank[0]) {
            const size_t at = ((size_t)slot * s.rows + j) * TILE + t;
            job.h.by_rank[0][at] = value;
            job.h.by_rank[1][at] = rest;
        }
    }
}

struct Up {
    Matrix w;
    Hidden h;
    const void *base;
    int64_t base_stride;
    const float *step;
    int32_t base_type;
    void *out;
    int64_t out_stride;
};

// Eight elements of the base as numbers of 32 bits.
template <class T, bool WIDE> __device__ inline void load_base(const Up &u, int64_t t, uint32_t n, int count, float out[8])
{
    if (u.base_type == SHE_NO_BASE) {
#pragma unroll
        for (int i = 0; i < 8; i++) out[i] = 0;
    } else if (u.base_type == SHE_F32 || u.base_type == SHE_I32) {
        const uint32_t *p = (const uint32_t *)u.base + t * u.base_stride + n;
        u32x4 v[2] = {u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
        if constexpr (WIDE) {
            if (count > 0) { v[0] = *reinterpret_cast<const u32x4 *>(p); v[1] = *reinterpret_cast<const u32x4 *>(p + 4); }
        } else {
            for (int i = 0; i < 8; i++)
                if (i < count) v[i / 4][i % 4] = p[i];
        }
        const bool sums = u.base_type == SHE_I32;
#pragma unroll
        for (int i = 0; i < 8; i++)
            out[i] = !sums ? __uint_as_float(v[i / 4][i % 4])
                           : (float)(int32_t)v[i / 4][i % 4] * (u.step && i < count ? u.step[n + i] : 1.0f);
    } else {
        unpack<T>(load8<T, WIDE>((const T *)u.base + t * u.base_stride + n, count), out);
    }
}

// A wavefront: SPAN outputs of one tile.  Lane l reads the eight outputs of block (l%4)*4 + (l%16)/4, so that after the matrix
// instructions the four lanes that share a token hold four neighbouring blocks and write 64 bytes side by side.
// MANY: several chunks of ranks whose tiles' powers of two differ, summed apart.
template <class T, bool WIDE, bool MANY>
__global__ __launch_bounds__(64 * UP_WAVES) void k_adapter_up(Up u, Segments s)
{
    const uint32_t slot = blockIdx.x, N = u.w.width;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
    const uint32_t n_first = (blockIdx.y * UP_WAVES + wave) * SPAN;
    if (n_first >= N) return;
    const Piece piece = find_piece(s.starts, s.segments, s.tokens, 1, TILE, slot);
    if (piece.segment < 0) return;
    const int a = adapter_of(s, piece.segment, nullptr);
    const int64_t t0 = piece.first + (int64_t)piece.index * TILE;
    const int live = (int)min((int64_t)TILE, piece.last - t0);
    const uint32_t rank = a < 0 ? 0 : rank_of(s, a);
    const uint32_t n_lane = n_first + ((col & 3) * 4 + (col >> 2)) * 8;
    const int w_count = min(8, (int)N - (int)n_lane);

    constexpr bool SCALED = std::is_same<T, _Float16>::value;
    f32x4 total[MANY ? 8 : 1][2], acc[8][2];
#pragma unroll
    for (int m = 0; m < 8; m++) {
        acc[m][0] = acc[m][1] = f32x4{0, 0, 0, 0};
        if constexpr (MANY) total[m][0] = total[m][1] = f32x4{0, 0, 0, 0};
    }
    for (uint32_t r0 = 0; r0 < rank; r0 += CHUNK) {
        for (uint32_t j0 = r0; j0 < min(rank, r0 + CHUNK); j0 += 32) {
            const uint32_t j = j0 + quarter * 8;
            u32x4 raw[8];
#pragma unroll
            for (int i = 0; i < 8; i++)
                raw[i] = load8<T, WIDE>((const T *)u.w.p + (int64_t)a * u.w.adapter + (int64_t)min(j + i, rank - 1) * u.w.row + n_lane,
                                        j + i < rank ? w_count : 0);
            x8<T> h[2][2], cols[8];
#pragma unroll
            for (int c = 0; c < 2; c++)
#pragma unroll
                for (int p = 0; p < 2; p++)
                    h[c][p] = as_x8<T>(j < s.rows ? *reinterpret_cast<const u32x4 *>(u.h.by_token[p] + ((size_t)slot * TILE + c * 16 + col) * s.rows + j)
                                                  : u32x4{0, 0, 0, 0});
            transpose8<T, 8>(raw, cols);
#pragma unroll
            for (int m = 0; m < 8; m++)
#pragma unroll
                for (int c = 0; c < 2; c++) {
                    acc[m][c] = mfma16(cols[m], h[c][0], acc[m][c]);
                    acc[m][c] = mfma16(cols[m], h[c][1], acc[m][c]);
                }
        }
        if constexpr (SCALED) {
            const float unscale = u.h.unscale[(size_t)slot * s.chunks + r0 / CHUNK];
#pragma unroll
            for (int m = 0; m < 8; m++)
#pragma unroll
                for (int c = 0; c < 2; c++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        if constexpr (MANY) {
                            total[m][c][i] = fmaf(acc[m][c][i], unscale, total[m][c][i]);
                            acc[m][c][i] = 0;
                        } else acc[m][c][i] *= unscale;
                    }
        }
    }
#pragma unroll
    for (int c = 0; c < 2; c++) {
        if (c * 16 + col >= live) continue;
        const int64_t t = t0 + c * 16 + col;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t n = n_first + (i * 4 + quarter) * 8;
            const int count = min(8, (int)N - (int)n);
            if (count <= 0) continue;
            float v[8];
            load_base<T, WIDE>(u, t, n, count, v);
#pragma unroll
            for (int m = 0; m < 8; m++) v[m] += MANY ? total[MANY ? m : 0][c][i] : acc[m][c][i];
            store8<T, WIDE>((T *)u.out + t * u.out_stride + n, pack<T>(v), count);
        }
    }
}

// What an adapter's tiles are: `before` of adapters of lower numbers and `own` of its own.
struct Share {
    uint32_t before, own;
};
__device__ inline uint32_t tiles_of(const Segments &s, uint32_t segment)
{
    const int64_t n = bounded_start(s.starts, (int)segment + 1, s.tokens) - bounded_start(s.starts, (int)segment, s.tokens);
    return n > 0 ? (uint32_t)((n + TILE - 1) / TILE) : 0;
}
__device__ inline Share share_of(const Segments &s, int a)
{
    const uint32_t lane = threadIdx.x & 63;
    uint32_t before = 0, own = 0;
    for (uint32_t i = lane; i < s.segments; i += 64) {
        const int32_t w = s.which[i];
        if (w < 0 || w > a) continue;
        const uint32_t n = tiles_of(s, i);
        if (w == a) own += n; else before += n;
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) { before += __shfl_xor(before, m); own += __shfl_xor(own, m); }
    return Share{(uint32_t)__builtin_amdgcn_readfirstlane(before), (uint32_t)__builtin_amdgcn_readfirstlane(own)};
}

struct Outer {
    Rows x;
    uint32_t width;
    Hidden h;
    void *out;                           // [adapters][rank][width]
    float *partial;                      // [places][rank][width]
};

// One adapter, SPAN columns, up to CHUNK ranks, and `share` of its tiles: the wavefronts take every eighth and are summed in LDS.
// An adapter of more tiles has several such sums, in places of their own (as many before them as lower adapters can need), which
// k_adapter_sum adds in order.
template <class T, bool WIDE, int RT>
__global__ __launch_bounds__(64 * OUTER_WAVES) void k_adapter_outer(Outer job0, Outer job1, Segments s, uint32_t spans0)
{
    __shared__ float part[OUTER_WAVES][16][SPAN];
    const bool second = blockIdx.x >= spans0;
    const Outer &job = second ? job1 : job0;
    const uint32_t f_first = (blockIdx.x - (second ? spans0 : 0)) * SPAN;
    const int a = blockIdx.y;
    const uint32_t z = blockIdx.z / s.chunks, chunk = blockIdx.z % s.chunks, r0 = chunk * CHUNK;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quarter = lane >> 4;
    const Share mine = share_of(s, a);
    const uint32_t parts = min((mine.own + s.share - 1) / s.share, s.most);
    if (z >= max(parts, 1u)) return;

    const uint32_t f = f_first + col * 8;
    const int count = min(8, (int)job.width - (int)f);
    f32x4 acc[8][RT];
#pragma unroll
    for (int m = 0; m < 8; m++)
#pragma unroll
        for (int r = 0; r < RT; r++) acc[m][r] = f32x4{0, 0, 0, 0};

    uint32_t seen = 0;                   // of the adapter's tiles
    const uint32_t from = z * s.share, to = min(from + s.share, mine.own);
    for (uint32_t s0 = 0; s0 < s.segments && seen < to; s0 += 64) {
        uint64_t match = __ballot(s0 + lane < s.segments && s.which[min(s0 + lane, s.segments - 1)] == a);
        for (; match; match &= match - 1) {
            const uint32_t seg = s0 + __builtin_ctzll(match);
            const uint32_t n = tiles_of(s, seg);
            const int64_t first = bounded_start(s.starts, (int)seg, s.tokens), last = bounded_start(s.starts, (int)seg + 1, s.tokens);
            const uint32_t slot0 = (uint32_t)(first / TILE + seg);
            // tiles of this segment that are in [from, to) and this wavefront's
            uint32_t i = seen < from ? from - seen : 0;
            i += ((uint32_t)wave - (seen + i)) & (OUTER_WAVES - 1);
            for (; i < n && seen + i < to; i += OUTER_WAVES) {
                const int64_t t = first + (int64_t)i * TILE + quarter * 8;
                u32x4 raw[8];
#pragma unroll
                for (int k = 0; k < 8; k++)
                    raw[k] = load8<T, WIDE>((const T *)job.x.p + min(t + k, last - 1) * job.x.stride + f, t + k < last ? count : 0);
                x8<T> h[RT][2], cols[8];
                const size_t slot = slot0 + i;
#pragma unroll
                for (int r = 0; r < RT; r++)
#pragma unroll
                    for (int p = 0; p < 2; p++) {
                        const uint32_t j = r0 + r * 16 + col;
                        h[r][p] = as_x8<T>(j < s.rows ? *reinterpret_cast<const u32x4 *>(job.h.by_rank[p] + (slot * s.rows + j) * TILE + quarter * 8)
                                                      : u32x4{0, 0, 0, 0});
                    }
                transpose8<T, 8>(raw, cols);
                const float unscale = std::is_same<T, _Float16>::value ? job.h.unscale[slot * s.chunks + chunk] : 1.0f;
#pragma unroll
                for (int m = 0; m < 8; m++)
#pragma unroll
                    for (int r = 0; r < RT; r++) {
                        if constexpr (std::is_same<T, _Float16>::value) {
                            f32x4 v = mfma16(h[r][0], cols[m], f32x4{0, 0, 0, 0});
                            v = mfma16(h[r][1], cols[m], v);
#pragma unroll
                            for (int k = 0; k < 4; k++) acc[m][r][k] = fmaf(v[k], unscale, acc[m][r][k]);
                        } else {
                            acc[m][r] = mfma16(h[r][0], cols[m], acc[m][r]);
                            acc[m][r] = mfma16(h[r][1], cols[m], acc[m][r]);
                        }
                    }
            }
            seen += n;
        }
    }

    const size_t place = mine.before / s.share + a + z;
    if (parts > 1 && place >= s.places) return;        // only where starts is not ascending
    const uint32_t rank = rank_of(s, a);
#pragma unroll
    for (int r = 0; r < RT; r++) {
        if (r) __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int m = 0; m < 8; m += 4)
                *reinterpret_cast<f32x4 *>(&part[wave][quarter * 4 + i][col * 8 + m]) =
                    f32x4{acc[m][r][i], acc[m + 1][r][i], acc[m + 2][r][i], acc[m + 3][r][i]};
        __syncthreads();
        for (int n = tid; n < 16 * SPAN / 4; n += 64 * OUTER_WAVES) {
            const uint32_t j = r0 + r * 16 + n / (SPAN / 4), k = f_first + n % (SPAN / 4) * 4;
            if (j >= s.rank || k >= job.width) continue;
            f32x4 v{0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < OUTER_WAVES; w++) v += *reinterpret_cast<const f32x4 *>(&part[w][n / (SPAN / 4)][n % (SPAN / 4) * 4]);
            if (j >= rank) v = f32x4{0, 0, 0, 0};
            if (parts > 1) {
                float *p = job.partial + (place * s.rank + j) * job.width + k;
                for (int i = 0; i < 4; i++)
                    if (k + i < job.width) p[i] = v[i];
            } else {
                T *p = (T *)job.out + ((size_t)a * s.rank + j) * job.width + k;
                for (int i = 0; i < 4; i++)
                    if (k + i < job.width) p[i] = (T)v[i];
            }
        }
    }
}

template <class T> __global__ __launch_bounds__(256) void k_adapter_sum(Outer job0, Outer job1, Segments s)
{
    const Outer &job = blockIdx.z ? job1 : job0;
    const int a = blockIdx.y;
    const Share mine = share_of(s, a);
    const uint32_t parts = min((mine.own + s.share - 1) / s.share, s.most);
    if (parts <= 1 || mine.before / s.share + a + parts > s.places) return;
    const size_t each = (size_t)s.rank * job.width, first = (size_t)(mine.before / s.share + a) * each;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < each; i += (size_t)gridDim.x * 256) {
        float v = 0;
        for (uint32_t z = 0; z < parts; z++) v += job.partial[first + z * each + i];
        ((T *)job.out)[a * each + i] = (T)v;
    }
}

bool on16(const void *p) { return ((uintptr_t)p & 15) == 0; }

uint32_t slots_of(uint32_t tokens, uint32_t segments) { return tokens / TILE + segments; }

struct Room {                            // hands out the scratch, on 256-byte boundaries
    char *base;
    size_t used = 0;
    template <class U> U *take(size_t count)
    {
        U *p = base ? reinterpret_cast<U *>(base + used) : nullptr;
        used += (count * sizeof(U) + 255) & ~(size_t)255;
        return p;
    }
};
Hidden take_hidden(Room &room, uint32_t slots, uint32_t rows, uint32_t chunks, bool by_token, bool by_rank)
{
    Hidden h{};
    const size_t n = (size_t)slots * TILE * rows;
    for (int p = 0; p < 2; p++) {
        if (by_token) h.by_token[p] = room.take<uint16_t>(n);
        if (by_rank) h.by_rank[p] = room.take<uint16_t>(n);
    }
    h.unscale = room.take<float>((size_t)slots * chunks);
    return h;
}
// Backward, a workgroup sums four tiles a wavefront and more where an adapter would else be shared by more than 16.
template <class Args> Segments segments_of(const Args &a)
{
    Segments s{a.starts, a.which, a.ranks, a.scale, a.tokens, a.segments, a.adapters, a.rank};
    s.rows = (uint32_t)ceil_div(a.rank, 16) * 16;
    s.chunks = (uint32_t)ceil_div(a.rank, CHUNK);
    const uint32_t tiles = slots_of(a.tokens, a.segments);
    s.share = std::max<uint32_t>(4 * OUTER_WAVES, (uint32_t)ceil_div(tiles, 16));
    s.most = (uint32_t)std::max<uint64_t>(1, ceil_div(tiles, s.share));
    s.places = s.most > 1 ? tiles / s.share + a.adapters : 0;
    return s;
}

template <class T, bool WIDE> hipError_t down(const Down &d0, const Down &d1, int jobs, const Segments &s, uint32_t *d_bad, hipStream_t st)
{
    const dim3 grid(slots_of(s.tokens, s.segments), s.chunks, jobs);
    if (s.rank <= 16) k_adapter_down<T, WIDE, 1, 16><<<grid, 1024, 0, st>>>(d0, d1, s, d_bad);
    else if (s.rank <= 32) k_adapter_down<T, WIDE, 2, 16><<<grid, 1024, 0, st>>>(d0, d1, s, d_bad);
    else k_adapter_down<T, WIDE, 4, 8><<<grid, 512, 0, st>>>(d0, d1, s, d_bad);
    return hipGetLastError();
}
template <class T, bool WIDE> hipError_t up(const Up &u, const Segments &s, hipStream_t st)
{
    const dim3 grid(slots_of(s.tokens, s.segments), (uint32_t)ceil_div(u.w.width, SPAN * UP_WAVES));
    if (std::is_same<T, _Float16>::value && s.chunks > 1) k_adapter_up<T, WIDE, std::is_same<T, _Float16>::value><<<grid, 64 * UP_WAVES, 0, st>>>(u, s);
    else k_adapter_up<T, WIDE, false><<<grid, 64 * UP_WAVES, 0, st>>>(u, s);
    return hipGetLastError();
}
template <class T, bool WIDE> hipError_t outer(const Outer &o0, const Outer &o1, const Segments &s, hipStream_t st)
{
    const uint32_t spans0 = (uint32_t)ceil_div(o0.width, SPAN), spans1 = (uint32_t)ceil_div(o1.width, SPAN);
    const dim3 grid(spans0 + spans1, s.adapters, s.most * s.chunks);
    if (s.rank <= 16) k_adapter_outer<T, WIDE, 1><<<grid, 64 * OUTER_WAVES, 0, st>>>(o0, o1, s, spans0);
    else if (s.rank <= 32) k_adapter_outer<T, WIDE, 2><<<grid, 64 * OUTER_WAVES, 0, st>>>(o0, o1, s, spans0);
    else k_adapter_outer<T, WIDE, 4><<<grid, 64 * OUTER_WAVES, 0, st>>>(o0, o1, s, spans0);
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess || s.most <= 1) return rc;
    const size_t each = (size_t)s.rank * std::max(o0.width, o1.width);
    k_adapter_sum<T><<<dim3((uint32_t)std::min<uint64_t>(ceil_div(each, 1024), 1024), s.adapters, 2), 256, 0, st>>>(o0, o1, s);
    return hipGetLastError();
}

Hidden lay_out(Room &room, const she_adapters_args &a)
{
    const Segments s = segments_of(a);
    return take_hidden(room, slots_of(a.tokens, a.segments), s.rows, s.chunks, true, false);
}
struct GradRoom {
    Hidden h, g;
    float *ddown, *dup;
};
GradRoom lay_out(Room &room, const she_adapters_grad_args &a)
{
    const Segments s = segments_of(a);
    const uint32_t slots = slots_of(a.tokens, a.segments);
    GradRoom r;
    r.h = take_hidden(room, slots, s.rows, s.chunks, false, true);
    r.g = take_hidden(room, slots, s.rows, s.chunks, true, true);
    r.ddown = room.take<float>((size_t)s.places * a.rank * a.inputs);
    r.dup = room.take<float>((size_t)s.places * a.rank * a.outputs);
    return r;
}

template <class T> hipError_t forward(const she_adapters_args &a, void *scratch, uint32_t *d_bad, hipStream_t st)
{
    const Segments s = segments_of(a);
    Room room{static_cast<char *>(scratch)};
    const Hidden h = lay_out(room, a);
    const Down d{{a.x, a.x_stride}, {a.down, a.down_adapter, a.down_rank, a.inputs}, h};
    const Up u{{a.up, a.up_adapter, a.up_rank, a.outputs}, h, a.base, a.base_stride, a.step, a.base_type, a.out, a.out_stride};
    const bool wide_down = on16(a.x) && on16(a.down) && (a.x_stride | a.down_adapter | a.down_rank | a.inputs) % 8 == 0;
    const bool wide_up = on16(a.up) && on16(a.base) && on16(a.out) && (a.up_adapter | a.up_rank | a.base_stride | a.out_stride | a.outputs) % 8 == 0;
    hipError_t rc = hipSuccess;
    if (s.rank && s.adapters) rc = wide_down ? down<T, true>(d, d, 1, s, d_bad, st) : down<T, false>(d, d, 1, s, d_bad, st);
    if (rc == hipSuccess) rc = wide_up ? up<T, true>(u, s, st) : up<T, false>(u, s, st);
    return rc;
}

template <class T> hipError_t backward(const she_adapters_grad_args &a, void *scratch, uint32_t *d_bad, hipStream_t st)
{
    const Segments s = segments_of(a);
    Room room{static_cast<char *>(scratch)};
    const GradRoom r = lay_out(room, a);
    const Matrix w_down{a.down, a.down_adapter, a.down_rank, a.inputs}, w_up{a.up, a.up_adapter, a.up_rank, a.outputs};
    const Rows x{a.x, a.x_stride}, dy{a.dy, a.dy_stride};
    const bool wide_x = on16(a.x) && a.x_stride % 8 == 0, wide_dy = on16(a.dy) && a.dy_stride % 8 == 0;
    const bool wide_down = on16(a.down) && (a.down_adapter | a.down_rank | a.inputs) % 8 == 0;
    const bool wide_up = on16(a.up) && (a.up_adapter | a.up_rank | a.outputs) % 8 == 0;
    const bool wide = wide_x && wide_dy && wide_down && wide_up;
    const Down d0{x, w_down, r.h}, d1{dy, w_up, r.g};
    const Up u{w_down, r.g, a.base, a.base_stride, nullptr, a.base_type, a.dx, a.dx_stride};
    hipError_t rc = !slots_of(a.tokens, a.segments) ? hipSuccess
                  : wide ? down<T, true>(d0, d1, 2, s, d_bad, st) : down<T, false>(d0, d1, 2, s, d_bad, st);
    if (rc != hipSuccess) return rc;
    if (slots_of(a.tokens, a.segments))
        rc = wide_down && on16(a.base) && on16(a.dx) && (a.base_stride | a.dx_stride) % 8 == 0 ? up<T, true>(u, s, st) : up<T, false>(u, s, st);
    if (rc != hipSuccess) return rc;
    const Outer o0{x, a.inputs, r.g, a.ddown, r.ddown}, o1{dy, a.outputs, r.h, a.dup, r.dup};
    return wide_x && wide_dy && (a.inputs | a.outputs) % 8 == 0 ? outer<T, true>(o0, o1, s, st) : outer<T, false>(o0, o1, s, st);
}

}  // namespace

size_t adapters_scratch(const she_adapters_args &a)
{
    Room room{nullptr};
    lay_out(room, a);
    return room.used;
}
size_t adapters_grad_scratch(const she_adapters_grad_args &a)
{
    Room room{nullptr};
    lay_out(room, a);
    return room.used;
}
hipError_t launch_adapters(const she_adapters_args &a, void *scratch, uint32_t *d_bad, hipStream_t st)
{
    return a.type == SHE_BF16 ? forward<__bf16>(a, scratch, d_bad, st) : forward<_Float16>(a, scratch, d_bad, st);
}
hipError_t launch_adapters_grad(const she_adapters_grad_args &a, void *scratch, uint32_t *d_bad, hipStream_t st)
{
    return a.type == SHE_BF16 ? backward<__bf16>(a, scratch, d_bad, st) : backward<_Float16>(a, scratch, d_bad, st);
}

}}  // namespace she::clear
