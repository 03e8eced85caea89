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
// (17 bits of it in bf16, 22 in f16), each with a product of its own: as good as 32 bits beside results of 8 or 11.  In f16 h is
// scaled by a power of two first, one for each token (and 64 ranks) where tokens are the rows of the result, one for each rank (and the
// 32 tokens of a tile) where ranks are.  So a number of h that is more than 2^16 below the largest of its token, or of its rank in
// the tile, is held to 2^-38 of that largest one; no token's result depends on the tokens beside it.
//
// Bound by memory: x, base and the adapters are read, and the result written, once; a tile's h is a few KB.  Backward, x and dy are
// read twice, the second time from the memory-side cache if they fit it.
//
// Measured, on inputs that do not repeat: 4099 tokens of 4096 -> 6144, rank 64, f16 with sums as base: 23 us for h (136 workgroups, each
// with all of its adapter) and 45 for the result (157 MB).  Backward, 8192 tokens of 4096 -> 4096, rank 32, bf16: 34 us for both hidden
// values (134 MB), 21 for dx (67 MB written), 26 + 6 for the matrices' gradients.  96 requests of a token, rank 16, 4096 -> 4096: 13 us
// in one launch.
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

// The hidden values of all tiles, value and rest, in the order of the operands that they become, so that a wavefront reads 16 bytes
// a lane side by side.  rows: r rounded up to 16.  Null: not wanted.
struct Hidden {
    uint16_t *by_token[2];               // [slots][TILE / 16][rows / 8][16 tokens][8 ranks]
    uint16_t *by_rank[2];                // [slots][rows / 16][TILE / 8][16 ranks][8 tokens]
    float *token_by, *rank_by;           // f16, what they are to be multiplied by: [slots][chunks][TILE], [slots][rows]
};
__device__ inline size_t by_token_at(size_t slot, int t, int j, uint32_t rows)
{
    return slot * TILE * rows + ((t >> 4) * (rows / 8) + (j >> 3)) * 128 + (t & 15) * 8 + (j & 7);
}
__device__ inline size_t by_rank_at(size_t slot, int j, int t, uint32_t rows)
{
    return slot * TILE * rows + ((j >> 4) * (TILE / 8) + (t >> 3)) * 128 + (j & 15) * 8 + (t & 7);
}
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

template <class T> __device__ inline float whole(uint16_t value, uint16_t rest)
{
    return (float)__builtin_bit_cast(T, value) + (float)__builtin_bit_cast(T, rest);
}

struct Tile {                            // the tokens [first, first + live) of a segment whose adapter is `adapter` (-1: none)
    int adapter, live;
    int64_t first;
    uint32_t rank;
};
__device__ inline Tile tile_of(const Segments &s, const Piece &p, uint32_t *d_bad)
{
    Tile t;
    t.adapter = adapter_of(s, p.segment, d_bad);
    t.first = p.first + (int64_t)p.index * TILE;
    t.live = (int)min((int64_t)TILE, p.last - t.first);
    t.rank = t.adapter < 0 ? 0 : rank_of(s, t.adapter);
    return t;
}

// The power of two that brings `top` to f16's upper range, 2^13 .. 2^14, and its inverse; not beyond what brings 2^-100 there.
struct Power {
    float by, back;
};
__device__ inline Power power_for(float top)
{
    const uint32_t e = top > 0 ? max(__float_as_uint(top) >> 23, 27u) : 127u;        // biased: 2^(e - 127) <= top
    return Power{__uint_as_float((127 + 127 + 13 - e) << 23), __uint_as_float((e - 13) << 23)};
}

// One tile, up to CHUNK ranks (RT tiles of 16) of it from r0 on: the wavefronts share the width out and are
// summed in LDS.  keep(j, t, v, token, rank) gets every number, and in f16 its token's power of two and, with RANKS, its rank's.
template <class T, bool WIDE, int RT, int WAVES, bool RANKS, class Keep>
__device__ inline void hidden_values(const Rows &rows, const Matrix &matrix, const Segments &s, const Tile &tile, uint32_t r0, Keep keep)
{
    __shared__ float part[WAVES][RT * 16][TILE];
    __shared__ float tops[WAVES][TILE];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quarter = lane >> 4;
    const uint32_t K = matrix.width;
    const T *x[2], *w[RT];
    bool has_x[2], has_w[RT];
#pragma unroll
    for (int c = 0; c < 2; c++) {
        has_x[c] = c * 16 + operand_row() < tile.live;
        x[c] = (const T *)rows.p + (tile.first + (has_x[c] ? c * 16 + operand_row() : 0)) * rows.stride + operand_unit() * 8;
    }
#pragma unroll
    for (int r = 0; r < RT; r++) {
        const uint32_t j = r0 + r * 16 + operand_row();
        has_w[r] = j < tile.rank;
        w[r] = (const T *)matrix.p + tile.adapter * matrix.adapter + (has_w[r] ? j : 0) * matrix.row + operand_unit() * 8;
    }
    f32x4 acc[RT][2];
#pragma unroll
    for (int r = 0; r < RT; r++) acc[r][0] = acc[r][1] = f32x4{0, 0, 0, 0};
    constexpr int AHEAD = !WIDE ? 1 : RT == 4 ? 2 : 4;     // steps whose loads are requested together
    for (uint32_t k0 = wave * 32; k0 < K; k0 += AHEAD * WAVES * 32) {
        u32x4 xv[AHEAD][2], wv[AHEAD][RT];
#pragma unroll
        for (int e = 0; e < AHEAD; e++) {
            const uint32_t k = k0 + e * WAVES * 32;
            const int count = min(8, (int)K - (int)(k + operand_unit() * 8));
#pragma unroll
            for (int c = 0; c < 2; c++) xv[e][c] = load8<T, WIDE>(x[c] + k, has_x[c] ? count : 0);
#pragma unroll
            for (int r = 0; r < RT; r++) wv[e][r] = load8<T, WIDE>(w[r] + k, has_w[r] ? count : 0);
        }
#pragma unroll
        for (int e = 0; e < AHEAD; e++) {
            x8<T> xo[2];
#pragma unroll
            for (int c = 0; c < 2; c++) xo[c] = as_x8<T>(to_operand(xv[e][c]));
#pragma unroll
            for (int r = 0; r < RT; r++) {
                const x8<T> wo = as_x8<T>(to_operand(wv[e][r]));
                acc[r][0] = mfma16(wo, xo[0], acc[r][0]);
                if (tile.live > 16) acc[r][1] = mfma16(wo, xo[1], acc[r][1]);
            }
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
    const float scale = s.scale[tile.adapter];
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
        v[e] = n % TILE < tile.live && r0 + n / TILE < tile.rank ? v[e] * scale : 0.0f;
        if (fabsf(v[e]) < __builtin_inff()) top = fmaxf(top, fabsf(v[e]));
    }
    Power token{1, 1};
    if constexpr (std::is_same<T, _Float16>::value) {        // all of a thread's numbers are of token tid % TILE
        top = fmaxf(top, __shfl_xor(top, TILE));
        if (lane < TILE) tops[wave][lane] = top;
        __syncthreads();
        top = 0;
#pragma unroll
        for (int k = 0; k < WAVES; k++) top = fmaxf(top, tops[k][tid % TILE]);
        token = power_for(top);
    }
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const int n = e * 64 * WAVES + tid, j = r0 + n / TILE;
        Power rank{1, 1};
        if constexpr (RANKS && std::is_same<T, _Float16>::value) {
            float most = fabsf(v[e]) < __builtin_inff() ? fabsf(v[e]) : 0.0f;
#pragma unroll
            for (int m = 1; m < TILE; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
            rank = power_for(most);
        }
        if (n < VALUES && (uint32_t)j < s.rows) keep(j, n % TILE, v[e], token, rank);
    }
}

struct Down {
    Rows x;
    Matrix w;
    Hidden h;
};

// RANKS: by_rank is wanted of every job, and by_token of those that have room for it; else by_token alone.
template <class T, bool WIDE, int RT, int WAVES, bool RANKS>
__global__ __launch_bounds__(64 * WAVES) void k_adapter_down(Down job0, Down job1, Segments s, uint32_t *d_bad)
{
    const Down &job = blockIdx.z ? job1 : job0;
    const uint32_t slot = blockIdx.x, r0 = blockIdx.y * CHUNK;
    const Piece piece = find_piece(s.starts, s.segments, s.tokens, 1, TILE, slot);
    if (piece.segment < 0) return;
    const Tile tile = tile_of(s, piece, threadIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && piece.index == 0 ? d_bad : nullptr);
    if (tile.adapter < 0) return;
    hidden_values<T, WIDE, RT, WAVES, RANKS>(job.x, job.w, s, tile, r0, [&](int j, int t, float v, Power token, Power rank) {
        constexpr bool F16 = std::is_same<T, _Float16>::value;
        uint16_t value, rest;
        if (job.h.by_token[0]) {
            const size_t at = by_token_at(slot, t, j, s.rows);
            split<T>(v * token.by, value, rest);
            job.h.by_token[0][at] = value;
            job.h.by_token[1][at] = rest;
            if (F16 && j == (int)r0) job.h.token_by[((size_t)slot * s.chunks + blockIdx.y) * TILE + t] = token.back;
        }
        if constexpr (RANKS) {
            const size_t at = by_rank_at(slot, j, t, s.rows);
            split<T>(v * rank.by, value, rest);
            job.h.by_rank[0][at] = value;
            job.h.by_rank[1][at] = rest;
            if (F16 && t == 0) job.h.rank_by[(size_t)slot * s.rows + j] = rank.back;
        }
    });
}

// An infinity in an operand that h is multiplied with is to be multiplied with h as a whole: the products with value and rest may have
// opposite signs, or the rest may be 0, and their sum NaN.  So sums that are not finite are done again, one by one (write_one_by_one,
// sum_one).
template <int N> __device__ inline bool all_finite(const f32x4 (&acc)[N])
{
    float v = 0;
#pragma unroll
    for (int n = 0; n < N; n++)
#pragma unroll
        for (int i = 0; i < 4; i++) v = fmaf(acc[n][i], 0.0f, v);
    return v == 0;
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

// A wavefront's SPAN outputs from n_first on: lane l has four from n_first + 4 (l % 16) on and four from 64 later on, of the tokens
// 4 (l / 16) + i, i < 4, of sixteen, so that sixteen lanes read and write whole lines of a row, of 16-bit elements and of 32-bit ones.
__device__ inline uint32_t lane_output(uint32_t n_first) { return n_first + (threadIdx.x & 15) * 4; }
__device__ inline int lane_token(int i) { return (threadIdx.x >> 4 & 3) * 4 + i; }

// The operands of 32 ranks from j0 on: for each of the lane's eight outputs its numbers of ranks j0 + 8 (lane / 16) .. + 7.
template <class T, bool WIDE> __device__ inline void load_columns(const Matrix &w, int adapter, uint32_t rank, uint32_t j0, uint32_t n_first, x8<T> cols[8])
{
    const uint32_t j = j0 + (threadIdx.x >> 4 & 3) * 8, n = lane_output(n_first);
    const int count = (int)w.width - (int)n;
    u32x4 raw[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const bool there = j + i < rank;
        raw[i] = load_quads<T, WIDE>((const T *)w.p + (int64_t)adapter * w.adapter + (int64_t)(there ? j + i : 0) * w.row + n, there ? count : 0, there ? count - 64 : 0);
    }
    transpose8<T, 8>(raw, cols);
}

// Eight elements of the base: their words, and the numbers that these stand for.
struct BaseWords {
    u32x4 v[2];
};
template <class T, bool WIDE> __device__ inline BaseWords load_base(const Up &u, int64_t t, uint32_t n, int count)
{
    BaseWords b{{u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}}};
    if (u.base_type == SHE_F32 || u.base_type == SHE_I32) {
        const uint32_t *p = (const uint32_t *)u.base + t * u.base_stride + n;
        if constexpr (WIDE) {
            if (count > 0) b.v[0] = *reinterpret_cast<const u32x4 *>(p);
            if (count > 64) b.v[1] = *reinterpret_cast<const u32x4 *>(p + 64);
        } else if (count >= 68) {
            __builtin_memcpy(&b.v[0], p, 16);
            __builtin_memcpy(&b.v[1], p + 64, 16);
        } else {
            for (int i = 0; i < 8; i++)
                if (i / 4 * 64 + i % 4 < count) b.v[i / 4][i % 4] = p[i / 4 * 64 + i % 4];
        }
    } else if (u.base_type != SHE_NO_BASE) {
        b.v[0] = load_quads<T, WIDE>((const T *)u.base + t * u.base_stride + n, count, count - 64);
    }
    return b;
}
template <class T> __device__ inline void base_numbers(const Up &u, const BaseWords &b, const float step[8], float out[8])
{
    if (u.base_type == SHE_F32 || u.base_type == SHE_I32) {
        const bool sums = u.base_type == SHE_I32;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t w = b.v[i / 4][i % 4];
            out[i] = sums ? (float)(int32_t)w * step[i] : __uint_as_float(w);
        }
    } else {
        unpack<T>(b.v[0], out);                  // zeros without a base
    }
}

// Sixteen tokens from `first` on, `live` of them: their bases; and by(i) times acc[m][i] added to the lane's output m of its token i,
// and written.
template <class T, bool WIDE> __device__ inline void load_bases(const Up &u, int64_t first, int live, uint32_t n_first, BaseWords base[4])
{
    const uint32_t n = lane_output(n_first);
    const int count = (int)u.w.width - (int)n;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const bool there = lane_token(i) < live && count > 0;
        base[i] = load_base<T, WIDE>(u, first + (there ? lane_token(i) : 0), there ? n : 0, there ? count : 0);
    }
}
template <class T, bool WIDE, class By> __device__ inline void write_outputs(const Up &u, int64_t first, int live, uint32_t n_first, const BaseWords base[4], const f32x4 acc[8], By by)
{
    const uint32_t n = lane_output(n_first);
    const int count = (int)u.w.width - (int)n;
    if (count <= 0) return;
    float step[8];
#pragma unroll
    for (int m = 0; m < 8; m++) step[m] = u.step && m / 4 * 64 + m % 4 < count ? u.step[n + m / 4 * 64 + m % 4] : 1.0f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if (lane_token(i) >= live) break;
        float v[8];
        const float times = by(i);
        base_numbers<T>(u, base[i], step, v);
#pragma unroll
        for (int m = 0; m < 8; m++) v[m] = fmaf(acc[m][i], times, v[m]);
        store_quads<T, WIDE>((T *)u.out + (first + lane_token(i)) * u.out_stride + n, pack<T>(v), count, count - 64);
    }
}

// The same where sums are not finite: element by element, with hidden(t, j) for the hidden value of token t of the sixteen.
template <class T, class Value> __device__ inline void write_one_by_one(const Up &u, const Tile &tile, int64_t first, int live, uint32_t n_first, Value hidden)
{
#pragma unroll 1
    for (int e = 0; e < 32; e++) {
        const int t = lane_token(e & 3);
        const uint32_t n = lane_output(n_first) + e / 16 * 64 + e / 4 % 4;
        if (t >= live || n >= u.w.width) continue;
        const T *w = (const T *)u.w.p + (int64_t)tile.adapter * u.w.adapter + n;
        float sum = 0;
        for (uint32_t j = 0; j < tile.rank; j++) sum = fmaf(hidden(t, (int)j), (float)w[(int64_t)j * u.w.row], sum);
        const int64_t at = (first + t) * u.base_stride + n;
        const float base = u.base_type == SHE_NO_BASE ? 0.0f : u.base_type == SHE_F32 ? ((const float *)u.base)[at]
                           : u.base_type == SHE_I32   ? (float)((const int32_t *)u.base)[at] * (u.step ? u.step[n] : 1.0f) : (float)((const T *)u.base)[at];
        ((T *)u.out)[(first + t) * u.out_stride + n] = (T)(base + sum);
    }
}

// A wavefront: SPAN outputs of one tile, 32 ranks a step.  CHUNKS: several chunks of ranks whose powers of two (f16) differ, summed
// apart.
template <class T, bool WIDE, bool CHUNKS>
__global__ __launch_bounds__(64 * UP_WAVES, WIDE && !CHUNKS ? 3 : 1) void k_adapter_up(Up u, Segments s)
{
    const int wave = threadIdx.x >> 6, col = threadIdx.x & 15, quarter = threadIdx.x >> 4 & 3;
    const uint32_t slot = blockIdx.x, n_first = (blockIdx.y * UP_WAVES + wave) * SPAN;
    if (n_first >= u.w.width) return;
    const Piece piece = find_piece(s.starts, s.segments, s.tokens, 1, TILE, slot);
    if (piece.segment < 0) return;
    const Tile tile = tile_of(s, piece, nullptr);
    // what the sums of the lane's tokens are to be multiplied by
    const auto back_of = [&](int c, uint32_t chunk) {
        return *reinterpret_cast<const f32x4 *>(u.h.token_by + ((size_t)slot * s.chunks + chunk) * TILE + c * 16 + lane_token(0));
    };
    f32x4 acc[2][8], total[CHUNKS ? 2 : 1][8];
#pragma unroll
    for (int c = 0; c < 2; c++) {
#pragma unroll
        for (int m = 0; m < 8; m++) {
            acc[c][m] = f32x4{0, 0, 0, 0};
            if constexpr (CHUNKS) total[c][m] = acc[c][m];
        }
    }
    for (uint32_t j0 = 0; j0 < tile.rank; j0 += 32) {
        x8<T> cols[8], h[2][2];
        const uint32_t j = j0 + quarter * 8;
#pragma unroll
        for (int c = 0; c < 2; c++)
#pragma unroll
            for (int p = 0; p < 2; p++)
                h[c][p] = as_x8<T>(j < s.rows ? *reinterpret_cast<const u32x4 *>(u.h.by_token[p] + by_token_at(slot, c * 16 + col, j, s.rows))
                                              : u32x4{0, 0, 0, 0});
        load_columns<T, WIDE>(u.w, tile.adapter, tile.rank, j0, n_first, cols);
#pragma unroll
        for (int m = 0; m < 8; m++)
#pragma unroll
            for (int c = 0; c < 2; c++) {
                acc[c][m] = mfma16(h[c][0], cols[m], acc[c][m]);
                acc[c][m] = mfma16(h[c][1], cols[m], acc[c][m]);
            }
        if constexpr (CHUNKS) {
#pragma unroll
            for (int c = 0; c < 2; c++) {
                const f32x4 back = back_of(c, j0 / CHUNK);
#pragma unroll
                for (int m = 0; m < 8; m++) {
                    total[c][m] += acc[c][m] * back;
                    acc[c][m] = f32x4{0, 0, 0, 0};
                }
            }
        }
    }
    BaseWords base[2][4];
#pragma unroll
    for (int c = 0; c < 2; c++) load_bases<T, WIDE>(u, tile.first + c * 16, tile.live - c * 16, n_first, base[c]);
#pragma unroll
    for (int c = 0; c < 2; c++) {
        if (__ballot(!all_finite(CHUNKS ? total[CHUNKS ? c : 0] : acc[c]))) {
            write_one_by_one<T>(u, tile, tile.first + c * 16, tile.live - c * 16, n_first, [&](int t, int j) {
                const size_t at = by_token_at(slot, c * 16 + t, j, s.rows);
                const float by = std::is_same<T, _Float16>::value ? u.h.token_by[((size_t)slot * s.chunks + j / CHUNK) * TILE + c * 16 + t] : 1.0f;
                return whole<T>(u.h.by_token[0][at], u.h.by_token[1][at]) * by;
            });
            continue;
        }
        const f32x4 back = std::is_same<T, _Float16>::value && !CHUNKS && tile.rank ? back_of(c, 0) : f32x4{1, 1, 1, 1};
        write_outputs<T, WIDE>(u, tile.first + c * 16, tile.live - c * 16, n_first, base[c], CHUNKS ? total[CHUNKS ? c : 0] : acc[c], [&](int i) { return back[i]; });
    }
}

// Few tiles: a workgroup of sixteen wavefronts makes a tile's hidden values in LDS and takes SPAN outputs a wavefront of them, in one
// launch and without a word of scratch.  Tiles of more outputs than that have several workgroups, each with all of the values.
constexpr int STEP_WAVES = 16;
template <class T, bool WIDE, int RT>
__global__ __launch_bounds__(64 * STEP_WAVES) void k_adapter_step(Rows x, Matrix w_down, Up u, Segments s, uint32_t *d_bad)
{
    __shared__ __align__(16) uint16_t h[2][TILE][RT * 16];
    __shared__ __align__(16) float back[TILE];
    const int wave = threadIdx.x >> 6, col = threadIdx.x & 15, quarter = threadIdx.x >> 4 & 3;
    const Piece piece = find_piece(s.starts, s.segments, s.tokens, 1, TILE, blockIdx.x);
    if (piece.segment < 0) return;
    const Tile tile = tile_of(s, piece, threadIdx.x == 0 && blockIdx.y == 0 && piece.index == 0 ? d_bad : nullptr);
    const uint32_t n_first = (blockIdx.y * STEP_WAVES + wave) * SPAN;
    if (tile.adapter >= 0) {
        hidden_values<T, WIDE, RT, STEP_WAVES, false>(x, w_down, s, tile, 0, [&](int j, int t, float v, Power token, Power) {
            split<T>(v * token.by, h[0][t][j], h[1][t][j]);
            if (std::is_same<T, _Float16>::value && j == 0) back[t] = token.back;
        });
        __syncthreads();
    }
    if (n_first >= u.w.width) return;
    x8<T> cols[8];
    const bool some = tile.adapter >= 0 && tile.rank;
    if (some) load_columns<T, WIDE>(u.w, tile.adapter, tile.rank, 0, n_first, cols);
#pragma unroll 1
    for (int c = 0; c < 2 && c * 16 < tile.live; c++) {
        BaseWords base[4];
        load_bases<T, WIDE>(u, tile.first + c * 16, tile.live - c * 16, n_first, base);
        f32x4 acc[8];
#pragma unroll
        for (int m = 0; m < 8; m++) acc[m] = f32x4{0, 0, 0, 0};
        if (some) {
            x8<T> hv[2];
#pragma unroll
            for (int p = 0; p < 2; p++)
                hv[p] = as_x8<T>(quarter * 8 < RT * 16 ? *reinterpret_cast<const u32x4 *>(&h[p][c * 16 + col][quarter * 8]) : u32x4{0, 0, 0, 0});
#pragma unroll
            for (int m = 0; m < 8; m++) {
                acc[m] = mfma16(hv[0], cols[m], acc[m]);
                acc[m] = mfma16(hv[1], cols[m], acc[m]);
            }
        }
        if (__ballot(!all_finite(acc))) {
            write_one_by_one<T>(u, tile, tile.first + c * 16, tile.live - c * 16, n_first, [&](int t, int j) {
                return whole<T>(h[0][c * 16 + t][j], h[1][c * 16 + t][j]) * (std::is_same<T, _Float16>::value ? back[c * 16 + t] : 1.0f);
            });
            continue;
        }
        write_outputs<T, WIDE>(u, tile.first + c * 16, tile.live - c * 16, n_first, base, acc, [&](int i) {
            // read when it is needed: there is no register to keep it in
            return std::is_same<T, _Float16>::value && some ? *(volatile const float *)&back[c * 16 + lane_token(i)] : 1.0f;
        });
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

// Where the sums of an adapter that has several begin.  It has more than `share` tiles then, and ceil(own / share) sums are at most
// floor(2 own / share): no place is another adapter's, and 2 tiles / share places do for all of them, however many adapters there are.
__device__ inline uint32_t place_of(const Segments &s, const Share &mine) { return (uint32_t)(2ull * mine.before / s.share); }

struct Outer {
    Rows x;
    uint32_t width;
    Hidden h;
    void *out;                           // [adapters][rank][width]
    float *partial;                      // [places][rank][width]
};

// d[j][k] over the adapter's tiles [from, to), by one thread.
template <class T> __device__ float sum_one(const Outer &job, const Segments &s, int a, uint32_t from, uint32_t to, uint32_t j, uint32_t k)
{
    float sum = 0;
    uint32_t seen = 0;
    for (uint32_t seg = 0; seg < s.segments && seen < to; seg++) {
        if (s.which[seg] != a) continue;
        const int64_t first = bounded_start(s.starts, (int)seg, s.tokens), last = bounded_start(s.starts, (int)seg + 1, s.tokens);
        const uint32_t n = tiles_of(s, seg);
        for (uint32_t i = seen < from ? from - seen : 0; i < n && seen + i < to; i++) {
            const size_t slot = (size_t)(first / TILE + seg) + i;
            const float by = std::is_same<T, _Float16>::value ? job.h.rank_by[slot * s.rows + j] : 1.0f;
            const int64_t t0 = first + (int64_t)i * TILE;
            for (int t = 0; t < TILE && t0 + t < last; t++) {
                const size_t at = by_rank_at(slot, j, t, s.rows);
                sum = fmaf(whole<T>(job.h.by_rank[0][at], job.h.by_rank[1][at]) * by, (float)((const T *)job.x.p)[(t0 + t) * job.x.stride + k], sum);
            }
        }
        seen += n;
    }
    return sum;
}

// One adapter, SPAN columns, up to CHUNK ranks, and `share` of its tiles: the wavefronts take every eighth and are summed in LDS.
// An adapter of more tiles has several such sums, in places of their own, which k_adapter_sum adds in order.
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
                        h[r][p] = as_x8<T>(j < s.rows ? *reinterpret_cast<const u32x4 *>(job.h.by_rank[p] + by_rank_at(slot, j, quarter * 8, s.rows))
                                                      : u32x4{0, 0, 0, 0});
                    }
                transpose8<T, 8>(raw, cols);
                f32x4 back[RT];                           // of the lane's ranks in the results
                if constexpr (std::is_same<T, _Float16>::value) {
#pragma unroll
                    for (int r = 0; r < RT; r++) {
                        const uint32_t j = r0 + r * 16 + quarter * 4;
                        back[r] = j < s.rows ? *reinterpret_cast<const f32x4 *>(job.h.rank_by + slot * s.rows + j) : f32x4{0, 0, 0, 0};
                    }
                }
#pragma unroll
                for (int m = 0; m < 8; m++)
#pragma unroll
                    for (int r = 0; r < RT; r++) {
                        if constexpr (std::is_same<T, _Float16>::value) {
                            f32x4 v = mfma16(h[r][0], cols[m], f32x4{0, 0, 0, 0});
                            v = mfma16(h[r][1], cols[m], v);
#pragma unroll
                            for (int k = 0; k < 4; k++) acc[m][r][k] = fmaf(v[k], back[r][k], acc[m][r][k]);
                        } else {
                            acc[m][r] = mfma16(h[r][0], cols[m], acc[m][r]);
                            acc[m][r] = mfma16(h[r][1], cols[m], acc[m][r]);
                        }
                    }
            }
            seen += n;
        }
    }

    const size_t place = place_of(s, mine) + z;
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
            if (__builtin_expect(!all_finite<1>({v}), 0)) {
#pragma unroll 1
                for (uint32_t i = 0; i < 4 && k + i < job.width; i++) {
                    const float again = sum_one<T>(job, s, a, from, to, j, k + i);
                    for (uint32_t m = 0; m < 4; m++) v[m] = m == i ? again : v[m];
                }
            }
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
    if (parts <= 1 || place_of(s, mine) + parts > s.places) return;
    const size_t each = (size_t)s.rank * job.width, first = (size_t)place_of(s, mine) * each;
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
    if (by_token) h.token_by = room.take<float>((size_t)slots * chunks * TILE);
    if (by_rank) h.rank_by = room.take<float>((size_t)slots * rows);
    return h;
}
// Backward, a workgroup sums eight tiles a wavefront (four: 80 and not 74 us for 8192 tokens, on one input again and again), and more where an adapter
// would else be shared by more than 16.
template <class Args> Segments segments_of(const Args &a)
{
    Segments s{a.starts, a.which, a.ranks, a.scale, a.tokens, a.segments, a.adapters, a.rank};
    s.rows = (uint32_t)ceil_div(a.rank, 16) * 16;
    s.chunks = (uint32_t)ceil_div(a.rank, CHUNK);
    const uint32_t tiles = slots_of(a.tokens, a.segments);
    s.share = std::max<uint32_t>(8 * OUTER_WAVES, (uint32_t)ceil_div(tiles, 16));
    s.most = (uint32_t)std::max<uint64_t>(1, ceil_div(tiles, s.share));
    s.places = s.most > 1 ? 2 * tiles / s.share : 0;
    return s;
}

template <class T, bool WIDE, bool RANKS> hipError_t down(const Down &d0, const Down &d1, int jobs, const Segments &s, uint32_t *d_bad, hipStream_t st)
{
    const dim3 grid(slots_of(s.tokens, s.segments), s.chunks, jobs);
    if (s.rank <= 16) k_adapter_down<T, WIDE, 1, 16, RANKS><<<grid, 1024, 0, st>>>(d0, d1, s, d_bad);
    else if (s.rank <= 32) k_adapter_down<T, WIDE, 2, 16, RANKS><<<grid, 1024, 0, st>>>(d0, d1, s, d_bad);
    else k_adapter_down<T, WIDE, 4, 8, RANKS><<<grid, 512, 0, st>>>(d0, d1, s, d_bad);
    return hipGetLastError();
}
template <class T, bool WIDE> hipError_t up(const Up &u, const Segments &s, hipStream_t st)
{
    constexpr bool F16 = std::is_same<T, _Float16>::value;
    const dim3 grid(slots_of(s.tokens, s.segments), (uint32_t)ceil_div(u.w.width, SPAN * UP_WAVES));
    if (F16 && s.chunks > 1) k_adapter_up<T, WIDE, F16><<<grid, 64 * UP_WAVES, 0, st>>>(u, s);
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

template <class T> hipError_t forward(const she_adapters_args &a, void *scratch, uint32_t *d_bad, uint32_t cus, hipStream_t st)
{
    const Segments s = segments_of(a);
    Room room{static_cast<char *>(scratch)};
    const Hidden h = lay_out(room, a);
    const Down d{{a.x, a.x_stride}, {a.down, a.down_adapter, a.down_rank, a.inputs}, h};
    const Up u{{a.up, a.up_adapter, a.up_rank, a.outputs}, h, a.base, a.base_stride, a.step, a.base_type, a.out, a.out_stride};
    const bool wide_down = on16(a.x) && on16(a.down) && (a.x_stride | a.down_adapter | a.down_rank | a.inputs) % 8 == 0;
    const bool wide_up = on16(a.up) && on16(a.base) && on16(a.out) && (a.up_adapter | a.up_rank | a.base_stride | a.out_stride | a.outputs) % 8 == 0;
    const dim3 grid(slots_of(a.tokens, a.segments), (uint32_t)ceil_div(a.outputs, SPAN * STEP_WAVES));
    if (wide_down && wide_up && s.rank <= 32 && (uint64_t)grid.x * grid.y <= cus) {
        if (s.rank <= 16) k_adapter_step<T, true, 1><<<grid, 64 * STEP_WAVES, 0, st>>>(d.x, d.w, u, s, d_bad);
        else k_adapter_step<T, true, 2><<<grid, 64 * STEP_WAVES, 0, st>>>(d.x, d.w, u, s, d_bad);
        return hipGetLastError();
    }
    hipError_t rc = wide_down ? down<T, true, false>(d, d, 1, s, d_bad, st) : down<T, false, false>(d, d, 1, s, d_bad, st);
    if (rc == hipSuccess) rc = wide_up ? up<T, true>(u, s, st) : up<T, false>(u, s, st);
    return rc;
}

template <class T> hipError_t backward(const she_adapters_grad_args &a, void *scratch, uint32_t *d_bad, uint32_t cus, hipStream_t st)
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
                  : wide ? down<T, true, true>(d0, d1, 2, s, d_bad, st) : down<T, false, true>(d0, d1, 2, s, d_bad, st);
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
hipError_t launch_adapters(const she_adapters_args &a, void *scratch, uint32_t *d_bad, uint32_t cus, hipStream_t st)
{
    return a.type == SHE_BF16 ? forward<__bf16>(a, scratch, d_bad, cus, st) : forward<_Float16>(a, scratch, d_bad, cus, st);
}
hipError_t launch_adapters_grad(const she_adapters_grad_args &a, void *scratch, uint32_t *d_bad, uint32_t cus, hipStream_t st)
{
    return a.type == SHE_BF16 ? backward<__bf16>(a, scratch, d_bad, cus, st) : backward<_Float16>(a, scratch, d_bad, cus, st);
}

}}  // namespace she::clear
