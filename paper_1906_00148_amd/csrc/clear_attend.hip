// Attention of each request's new tokens over its paged cache.
//
// The query heads that share a key head are packed with the tokens: the rows of a request at one key head are its new tokens times
// the `group` query heads, token by token, and a tile of rows reads the request's keys and values once for all of them.  Along the
// cache a tile's places are cut into pieces of `chunk`, each a workgroup of its own; where a tile has more than one, they leave
// (top, sum, weighted values) of every row behind and k_attend_join puts them together in order.
//
// Scores are taken transposed, S^T = K Q^T, so that the lanes' results are the operands of the second product O^T = V^T P^T as they
// lie: a lane's scores of one row become eight places of one column, if V's rows are taken in the same order.  The softmax is the
// running one: a top m and a sum l per row in 32 bits, weights exp2(s - m) with log2(e) in the scale.  k_attend_few, which waits for
// memory, takes the second product with the weights as two numbers of the type, the rounded value and the rest, so that nothing but the
// result's own rounding shows.  k_attend_tile rounds the weights to the type (their sum is not): an error of the size of the result's
// own rounding, 0.0024 and not 0.0017 of a result in bf16; with two numbers 2048 tokens over 32768 places take 1434 us and not 1065.
// Behind shared prefixes tiles of many rows have one number or two by the requests' rows (beside shared_shape): 24 questions of up to 300 tokens behind
// 8192 places 500 us, 636 with two; 64 single tokens behind 32768 78, and 88 with two, which they have.
//
// Masks: a place that no row of the tile attends to is not read at all.  A place that some rows attend to and others do not has weight
// 0 for the others, which a matrix instruction multiplies with the value all the same.  So where some of such places' values are
// infinite or NaN, the tile's rows are done again, one by one and over the places that they attend to alone.
// So they are where a sum is NaN and its weights' sum is not: an infinite value that a row does attend to is NaN times a weight that the type rounds to
// 0, or in two products of different signs.
#include <algorithm>
#include <type_traits>

#include "clear_device.h"
#include "clear_internal.h"
#include "clear_reach.h"

namespace she { namespace clear {
namespace {

constexpr int FEW_WAVES = 4, TILE_WAVES = TILE_ROWS / 32;
constexpr float LOG2E = 1.4426950408889634f;

// What a kernel walks: a call's requests; or in a call with shared prefixes these, each as a request of all tokens that have it, or what
// the requests have behind them, or both as one, where sharing saves nothing: a request has many rows, or all places are few.
enum Walk { REQUESTS, PREFIXES, BEHIND, WHOLE };
// The first and the last of them write results, or pieces where a tile is cut; the others, which are joined, pieces only, all of them.
constexpr bool joined_with_another(Walk walk) { return walk == PREFIXES || walk == BEHIND; }
constexpr float NOTHING = -1;            // in place of a sum: a token that attends to nothing at all, prefix or not

// What is left behind of the pieces of cut rows: [rows of all requests][kv_heads][splits].
struct Pieces {
    float *o;                            // [..][head]
    float2 *ml;
    uint32_t splits;
    uint32_t first, most;                // of these, the ones of this walk
    uint32_t chunk;                      // places of a piece, unless a tile has more than `most` such pieces
};

// What a call with shared prefixes has beside the arguments of a walk: over prefixes these have prefixes for requests, otherwise the requests.
struct Owners {
    const int32_t *requests;             // [prefixes + 1]
    const int32_t *prefix_lengths;       // [prefixes]
    const int32_t *lengths;              // [count]
    const int32_t *prefix_table;
    int64_t prefix_stride;
    uint32_t count, prefixes, prefix_width;
};
__device__ inline int owner_start(const Owners &w, int g)
{
    return min(max(w.requests[g], 0), (int)w.count);
}
// The prefix of request r, or -1.
__device__ inline int prefix_of(const Owners &owners, int r)
{
    const int lane = threadIdx.x & 63;
    int found = 0;
    for (uint32_t g0 = 0; g0 < owners.prefixes; g0 += 64) {
        const bool before = g0 + lane < owners.prefixes && owner_start(owners, (int)g0 + lane) <= r;
        const int n = __popcll(__ballot(before));
        found += n;
        if (n < 64) break;
    }
    return __builtin_amdgcn_readfirstlane(found && r < owner_start(owners, found) ? found - 1 : -1);
}
// Of a prefix's places, those that its table has a column for.
__device__ inline int prefix_places(const she_attend_pages_args &a, int length, uint32_t width)
{
    return (int)min((int64_t)max(length, 0), (int64_t)width * a.page_size);
}

// A tile of rows and the places that any of them attends to.
struct Span {
    int request;                         // -1: nothing here
    int row, rows;                       // first row in the request, rows of the tile
    int64_t token0;                      // the request's first token
    int first;                           // place of the request's first new token (negative: its length is short of them)
    int low;                             // the first place that any row attends to
    int from, to;                        // places to walk, `from` down from `low` to a multiple of 32; none if to <= from
    int chunk, parts;                    // places of a piece, pieces that they are cut into
    int prefix, own;                     // WHOLE: the prefix (-1: none), and the first place behind it
    int64_t missing;                     // WHOLE, PREFIXES: places of the prefix that have no column
};
__device__ inline size_t pieces_at(const Pieces &p, uint32_t kv_heads, uint32_t group, const Span &s, int row, int kv_head)
{
    return ((size_t)(s.token0 * group + row) * kv_heads + kv_head) * p.splits;
}
template <Walk WALK> __device__ inline Piece tile_of(const she_attend_pages_args &a, const Owners &owners, uint32_t group, uint32_t tile, uint32_t slot)
{
    if constexpr (WALK == PREFIXES)
        return find_piece_by([&](int g) { return bounded_start(a.starts, owner_start(owners, g), a.tokens); }, a.requests, group, tile, slot);
    else
        return find_piece(a.starts, a.requests, a.tokens, group, tile, slot);
}
template <int ROWS, Walk WALK>
__device__ inline Span span_of(const she_attend_pages_args &a, const Owners &owners, uint32_t group, const Piece &p, int row, const Pieces &pieces)
{
    Span s{};
    s.request = p.segment;
    if (p.segment < 0) return s;
    const int all = (int)(p.last - p.first), news = all / (int)group;
    int64_t room = (int64_t)a.table_width * a.page_size;
    const int length = max(a.lengths[p.segment], 0);
    s.row = row;
    s.rows = min(ROWS, all - row);
    s.token0 = p.first / group;
    if constexpr (WALK == PREFIXES) {
        // cut alike for all of a prefix's tiles
        s.to = prefix_places(a, length, a.table_width);
        s.missing = length - s.to;
        s.first = s.to - 1;                                       // a token's window is looked up apart
        s.chunk = (int)max(pieces.chunk, (((uint32_t)s.to + pieces.most - 1) / pieces.most + 63) & ~63u);
        s.parts = s.to ? (s.to - 1) / s.chunk + 1 : 0;
        return s;
    }
    s.first = length - news;
    if constexpr (WALK == WHOLE) {
        s.prefix = prefix_of(owners, p.segment);
        if (s.prefix >= 0) {
            const int places = max(owners.prefix_lengths[s.prefix], 0);
            s.own = prefix_places(a, places, owners.prefix_width);
            s.missing = places - s.own;
        }
        room += s.own;
    }
    const int p0 = s.first + row / (int)group, p1 = s.first + (row + s.rows - 1) / (int)group;
    int64_t low = a.window ? (int64_t)p0 - (int64_t)a.window + 1 : 0, to = (int64_t)p1 + 1;
    if constexpr (WALK == WHOLE) {
        low = p1 < 0 ? 0 : first_behind(max(p0, 0), a.window, s.own, s.missing);
        to = p1 < 0 ? 0 : to + s.own;
    }
    s.low = (int)max(low, (int64_t)0);
    s.from = s.low & ~31;
    s.to = (int)min(to, room);
    const uint32_t places = s.to > s.from ? s.to - s.from : 0;
    uint32_t chunk = pieces.chunk;
    if (places > (uint64_t)pieces.most * chunk) chunk = ((places + pieces.most - 1) / pieces.most + 127) & ~127u;
    s.chunk = (int)chunk;
    s.parts = (int)((places + chunk - 1) / chunk);
    return s;
}

// Of a walk that is joined with another: the piece z of the tile's rows is none, and if `alone`, nor are those of a prefix.  Returns whether
// there is nothing more to do.
template <Walk WALK>
__device__ inline bool leave_none(const she_attend_pages_args &a, const Owners &owners, uint32_t group, const Pieces &pieces, const Span &s, int kv_head, int z)
{
    if (WALK == BEHIND && z == 0) {
        if (prefix_of(owners, s.request) < 0)
            for (uint32_t i = threadIdx.x; i < s.rows * pieces.first; i += blockDim.x)
                pieces.ml[pieces_at(pieces, a.kv_heads, group, s, s.row + (int)(i / pieces.first), kv_head) + i % pieces.first] = float2{-__builtin_inff(), 0};
        return false;
    }
    if (z < s.parts) return false;
    for (int i = threadIdx.x; i < s.rows; i += blockDim.x)
        pieces.ml[pieces_at(pieces, a.kv_heads, group, s, s.row + i, kv_head) + pieces.first + z] = float2{-__builtin_inff(), 0};
    return true;
}

// The places that a row of a tile attends to, from low to high.  In the walk over prefixes the request's own length says where its window
// reaches back to.  With a prefix before them, tokens without a place of their own attend to nothing.
struct Reach {
    int low, high;
};
template <Walk WALK> __device__ inline Reach reach_of(const she_attend_pages_args &a, const Owners &owners, uint32_t group, const Span &s, int row)
{
    Reach w{0, s.first};
    if constexpr (WALK == PREFIXES) {
        if (!a.window) return w;
        const int64_t token = s.token0 + row / (int)group;
        int r = owner_start(owners, s.request), end = owner_start(owners, s.request + 1);
        while (end - r > 1) {
            const int mid = (r + end) / 2;
            if (bounded_start(a.starts, mid, a.tokens) <= token) r = mid;
            else end = mid;
        }
        const int64_t place = (int64_t)max(owners.lengths[r], 0) - (bounded_start(a.starts, r + 1, a.tokens) - token);
        w.low = (int)min(max(s.to + s.missing + place - (int64_t)a.window + 1, (int64_t)0), (int64_t)s.to);
    } else {
        const int place = s.first + row / (int)group;
        if constexpr (WALK == WHOLE) {
            if (place < 0) return Reach{0, -1};
            return Reach{first_behind(place, a.window, s.own, s.missing), last_behind(place, s.own)};
        }
        w.high = place;
        if (a.window) w.low = (int)max((int64_t)place - (int64_t)a.window + 1, (int64_t)0);
    }
    return w;
}

// The page and slot of a place.  Whether page ids are in range is the caller's to see.
struct Slot {
    int32_t page;
    uint32_t in_page;
};
template <Walk WALK> __device__ inline Slot slot_of(const she_attend_pages_args &a, const Owners &owners, const Span &s, uint32_t place)
{
    const int32_t *row = a.table + s.request * a.table_stride;
    if constexpr (WALK == WHOLE) {
        if (place < (uint32_t)s.own) row = owners.prefix_table + s.prefix * owners.prefix_stride;
        else place -= s.own;
    }
    const uint32_t column = place / a.page_size;
    return Slot{row[column], place - column * a.page_size};
}

// Whether place `place`, whose page id is out of range and slot in_page, stands for that page in the count: its first place that is
// attended to here.  Pages that end before a window may be gone.
__device__ inline bool counts(const Span &s, int place, int in_page, bool first)
{
    return place >= s.low && (in_page == 0 || place == s.low || first);
}

// Where the rows of the places [from, from + count) start, -1 for those that their page id keeps out; *any_bad: some that is attended to.
template <Walk WALK>
__device__ inline void look_up(const she_attend_pages_args &a, const Owners &owners, const Span &s, int kv_head, int from, int count, int64_t *rows, int *any_bad, uint32_t *d_bad)
{
    for (int i = threadIdx.x; i < count; i += blockDim.x) {
        const Slot at = slot_of<WALK>(a, owners, s, from + i);
        const bool good = at.page >= 0 && (uint32_t)at.page < a.pages;
        rows[i] = good ? at.page * a.page_stride + at.in_page * a.slot_stride + kv_head * a.page_head : -1;
        if (!good && from + i >= s.low) {
            *any_bad = 1;
            if (counts(s, from + i, at.in_page, i == 0)) count_bad(d_bad);
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

// One row over those of the places [from, to) that it attends to, its piece `part`, by one wavefront: scores with a place a lane, sums with elements on
// the lanes.  Writes the row's result, or its piece's.
template <class T, Walk WALK>
__device__ void attend_row(const she_attend_pages_args &a, const Owners &owners, uint32_t group, const Pieces &pieces, bool cut, size_t part, const Span &sp, int kv_head, int row, Reach reach, int from, int to)
{
    const int lane = threadIdx.x & 63, D = (int)a.head;
    const int64_t token = sp.token0 + row / (int)group;
    const int head = kv_head * (int)group + row % (int)group;
    const T *q = (const T *)a.q + token * a.q_token + head * a.q_head;
    float top = -__builtin_inff(), sum = 0, o[4] = {0, 0, 0, 0};
    to = min(to, reach.high + 1);
    for (int first = max(from, reach.low); first < to; first += 64) {
        const int place = first + lane;
        const Slot its = place < to ? slot_of<WALK>(a, owners, sp, place) : Slot{-1, 0};
        const bool there = its.page >= 0 && (uint32_t)its.page < a.pages;
        const int64_t at = there ? its.page * a.page_stride + (int64_t)its.in_page * a.slot_stride + kv_head * a.page_head : 0;
        float s = 0;
        if (there)
            for (int d = 0; d < D; d += 8) {
                float x[8], y[8];
                unpack<T>(load8<T, true>(q + d, 8), x);
                unpack<T>(load8<T, true>((const T *)a.k_pages + at + d, 8), y);
                for (int i = 0; i < 8; i++) s = fmaf(x[i], y[i], s);
            }
        s = there ? s * a.scale * LOG2E : -__builtin_inff();
        float next = fmaxf(top, s);
        for (int m = 1; m < 64; m *= 2) next = fmaxf(next, __shfl_xor(next, m));
        const float ref = next == -__builtin_inff() ? 0.0f : next, alpha = __builtin_amdgcn_exp2f(top - ref), p = __builtin_amdgcn_exp2f(s - ref);
        top = next;
        sum *= alpha;
        for (int i = 0; i < 4; i++) o[i] *= alpha;
        for (uint64_t left = __ballot(there); left; left &= left - 1) {
            const int from_lane = __builtin_ctzll(left);
            const float weight = __shfl(p, from_lane);
            const T *v = (const T *)a.v_pages + __shfl(at, from_lane);
            sum += weight;
            for (int i = 0; i < 4; i++)
                if (lane + 64 * i < D) o[i] = fmaf(weight, (float)v[lane + 64 * i], o[i]);
        }
    }
    const float inv = cut ? 1.0f : sum == 0 ? 0.0f : 1.0f / sum;
    if (cut && lane == 0) pieces.ml[part] = float2{top, WALK == BEHIND && reach.high < 0 ? NOTHING : sum};
    for (int i = 0; i < 4; i++) {
        const int d = lane + 64 * i;
        if (d >= D) continue;
        if (cut) pieces.o[part * D + d] = o[i];
        else ((T *)a.out)[token * a.out_token + head * a.out_head + d] = (T)(o[i] * inv);
    }
}

// For small calls, where latencies add up: a token over 197 places (2 key heads of 64) 6.8 us, 16 tokens over 1000 (8 of 128) 21 us; but
// it reaches the memory's rate too: 64 tokens over 1 to 16384 places (2.1 GB) 425 us, 5.0 TB/s.
//
// Few rows: every wavefront walks places of its own, 32 a step, four steps of the workgroup side by side, straight from memory.  Lane
// l reads d = 32 s + 8 (l/16) .. of the key of place l%16 for the scores, and EL elements from EL (l%16) on of the values of the
// eight places that its scores belong to, whole rows over 16 lanes; the eight rows are transposed in registers.
template <int DP> struct FewShared {
    int64_t rows[MOST_CHUNK];
    float joined[FEW_WAVES][FEW_ROWS][DP];
    float tops[FEW_WAVES][FEW_ROWS], sums[FEW_WAVES][FEW_ROWS];
    int any_bad, any_special;
};
template <class T, int DP, Walk WALK>
__device__ __forceinline__ void attend_few(const she_attend_pages_args &a, uint32_t group, const Pieces &pieces, const Owners &owners, uint32_t *d_bad, FewShared<DP> &shared,
                                           uint32_t slot, int kv_head, int z)
{
    constexpr int EL = DP == 64 ? 4 : 8, NB = DP == 256 ? 2 : 1, KS = DP / 32;
    auto &rows = shared.rows;
    auto &joined = shared.joined;
    auto &tops = shared.tops, &sums = shared.sums;
    int &any_bad = shared.any_bad, &any_special = shared.any_special;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quarter = lane >> 4;
    const int D = (int)a.head;
    const Piece piece = tile_of<WALK>(a, owners, group, FEW_ROWS, slot);
    if (piece.segment < 0) return;
    Span sp = span_of<FEW_ROWS, WALK>(a, owners, group, piece, piece.index * FEW_ROWS, pieces);
    if constexpr (joined_with_another(WALK)) {
        if (leave_none<WALK>(a, owners, group, pieces, sp, kv_head, z)) return;
    } else {
        if (z >= max(sp.parts, 1)) return;
    }
    const bool cut = joined_with_another(WALK) || sp.parts > 1;
    const uint32_t part = pieces.first + z;
    int from = sp.from + z * sp.chunk, count = sp.parts ? min(sp.chunk, sp.to - from) : 0;

    // this lane's row
    const int my_row = min(sp.row + col, sp.row + sp.rows - 1), my_token = my_row / (int)group, my_head = kv_head * (int)group + my_row % (int)group;
    const Reach mine = reach_of<WALK>(a, owners, group, sp, my_row);
    const int high = mine.high, low = mine.low;
    int high_min = sp.first, low_max = 0;
    if constexpr (WALK == PREFIXES) {
        if (a.window) {                                           // requests in any order: the earliest and the latest place of the rows
            int low_min = low;
            low_max = low;
#pragma unroll
            for (int m = 1; m < 16; m *= 2) {
                low_min = min(low_min, __shfl_xor(low_min, m));
                low_max = max(low_max, __shfl_xor(low_max, m));
            }
            sp.low = low_min;
            const int end = from + count;
            from = max(from, low_min & ~31);
            count = max(end - from, 0);
        }
    } else if constexpr (WALK == WHOLE) {
        high_min = reach_of<WALK>(a, owners, group, sp, sp.row).high;
        low_max = reach_of<WALK>(a, owners, group, sp, sp.row + sp.rows - 1).low;
    } else {
        high_min = sp.first + sp.row / (int)group;
        low_max = a.window ? (int)max((int64_t)sp.first + (sp.row + sp.rows - 1) / (int)group - (int64_t)a.window + 1, (int64_t)0) : 0;
    }
    if (tid == 0) any_bad = any_special = 0;
    __syncthreads();
    look_up<WALK>(a, owners, sp, kv_head, from, min(count, MOST_CHUNK), rows, &any_bad, d_bad);
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
    bool unsafe = any_bad != 0;
    bool special = false;                                         // infinite or NaN values where not all rows attend

    for (int base = 0; base < count; base += FEW_WAVES * 32) {
        if (base && base % MOST_CHUNK == 0) {
            __syncthreads();                                      // the rows that were looked up before have been read
            look_up<WALK>(a, owners, sp, kv_head, from + base, min(count - base, MOST_CHUNK), rows, &any_bad, d_bad);
            __syncthreads();
            unsafe = any_bad != 0;
        }
        const int k0 = base + wave * 32, r0 = k0 % MOST_CHUNK - k0;
        if (k0 >= count) break;
        u32x4 kraw[2][KS];
#pragma unroll
        for (int t = 0; t < 2; t++) {
            const int i = k0 + t * 16 + col;
            const int64_t row = i < count ? rows[i + r0] : -1;
            const T *p = (const T *)a.k_pages + (row < 0 ? 0 : row) + quarter * 8;
#pragma unroll
            for (int s = 0; s < KS; s++) kraw[t][s] = load8<T, true>(p + s * 32, row < 0 ? 0 : D - (s * 32 + quarter * 8));
        }
        u32x4 vraw[NB][8];
        uint32_t there = 0;                                       // which of the lane's eight places exist
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const int i = k0 + (e < 4 ? 0 : 16) + quarter * 4 + (e & 3);
            const int64_t row = i < count ? rows[i + r0] : -1;
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
#pragma unroll
        for (int e = 0; e < 8; e++) s[e] = st[e / 4][e % 4] * scale;
        if (masked) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const int place = from + k0 + (e < 4 ? 0 : 16) + quarter * 4 + (e & 3);
                if (!(there >> e & 1) || place > high || place < low) s[e] = -__builtin_inff();
            }
        }
#pragma unroll
        for (int e = 0; e < 8; e++) top = fmaxf(top, s[e]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float ref = top == -__builtin_inff() ? 0.0f : top, alpha = __builtin_amdgcn_exp2f(m - ref);
        m = top;
        x8<T> p, rest;
        float sum = 0;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float v = __builtin_amdgcn_exp2f(s[e] - ref);
            sum += v;
            p[e] = (T)v;
            rest[e] = (T)(v - (float)p[e]);
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
        if (masked) {
#pragma unroll
            for (int b = 0; b < NB; b++)
#pragma unroll
                for (int e = 0; e < 8; e++) special |= has_special<T>(vraw[b][e]);
        }
#pragma unroll
        for (int b = 0; b < NB; b++) {
            x8<T> v[EL];
            transpose8<T, EL>(vraw[b], v);
#pragma unroll
            for (int e = 0; e < EL; e++) acc[b][e] = mfma16(v[e], p, mfma16(v[e], rest, acc[b][e]));
        }
    }
    // the wavefronts' results, and the piece's
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    f32x4 lost{0, 0, 0, 0};                                       // NaN where a sum is, or where infinities meet
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < EL; e++) lost += acc[b][e];
    const float lost_sum = lost[0] + lost[1] + lost[2] + lost[3];
    if (special || (lost_sum != lost_sum && l == l)) any_special = 1;
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
    if (any_special) {
        for (int r = wave; r < sp.rows; r += FEW_WAVES)
            attend_row<T, WALK>(a, owners, group, pieces, cut, pieces_at(pieces, a.kv_heads, group, sp, sp.row + r, kv_head) + part, sp, kv_head, sp.row + r,
                          Reach{__shfl(low, r), __shfl(high, r)}, from, from + count);
        return;
    }
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
    if (!cut) {
        const float inv = sum == 0 ? 0.0f : 1.0f / sum;
        T *to = (T *)a.out + token * a.out_token + head * a.out_head + d0;
#pragma unroll
        for (int i = 0; i < EACH; i++)
            if (d0 + i < D) to[i] = (T)(o[i] * inv);
    } else {
        const size_t at = pieces_at(pieces, a.kv_heads, group, sp, row, kv_head) + part;
        if (d0 == 0) pieces.ml[at] = float2{top, WALK == BEHIND && sp.first + row / (int)group < 0 ? NOTHING : sum};
#pragma unroll
        for (int i = 0; i < EACH; i++)
            if (d0 + i < D) pieces.o[at * D + d0 + i] = o[i];
    }
}
template <class T, int DP, Walk WALK>
__global__ __launch_bounds__(64 * FEW_WAVES, DP == 256 ? 1 : 2) void k_attend_few(she_attend_pages_args a, uint32_t group, Pieces pieces, Owners owners, uint32_t *d_bad)
{
    __shared__ FewShared<DP> shared;
    attend_few<T, DP, WALK>(a, group, pieces, owners, d_bad, shared, blockIdx.x, (int)blockIdx.y, (int)blockIdx.z);
}

// Bound by what a wavefront does one after the other: 2048 tokens over 32768 places (32 / 8 heads of 128, bf16) 1066 us, 1000 TFLOP/s
// where a product of 8192^3 reaches 1279 (946 on another card).  The matrix units are busy for 45 % of the cycles and the vector units for as many; taken
// out for a timing, the softmax was worth 11 %, the second product 23 % and the tiles' loads 17 %.  Tried and slower: the next
// step's scores beside a step's softmax (two forms), raised priority around the matrix instructions, pieces for more workgroups.
// 24 requests of up to 700 tokens, half of them single (16 heads of 64, f16, a window of 1024): 56 us, most of it in the same steps.
// Heads of 64, 96, 192 and 256 over those 32768 places: 737, 742, 551 and 713 TFLOP/s (192 is computed as 256, with one workgroup per
// compute unit).
// Eight wavefronts on 256 rows gain 3 % there and lose a third where a window makes the tiles' edges count.
//
// Many rows: a workgroup has TILE_ROWS of them, 32 a wavefront, and steps through the places STEP at a time with both tiles of the step
// in LDS, twice over, so that the next step's are on their way while this one's are used.  The matrix instructions are 32 x 32 x 16:
// lane l has row l%32 of the tile, and of every 32 places the scores of 8 (i/4) + 4 (l/32) + i%4.  The second product's operand is
// V transposed, which LDS reads hand over four places at a time.
//
// LDS: a place's row of DP elements, its 16-byte units exchanged by place so that neighbouring lanes, which read the same unit of
// neighbouring places (keys) or four places of one pair of units (values), reach all banks.
template <int DP> __device__ inline int key_unit(int place, int unit)
{
    return unit ^ (DP == 64 ? (place >> 1) & 7 : place & 15);
}
template <int DP> __device__ inline int value_unit(int place, int unit)
{
    return unit ^ (DP == 64 ? ((place >> 1) & 3) << 1 : (place & 7) << 1);
}

constexpr int TILE_BLOCK = 4 * STEP;                                                 // places that are looked up together
template <class T, int DP> struct alignas(16) TileShared {
    T even_keys[STEP * DP], even_values[STEP * DP], odd_keys[STEP * DP], odd_values[STEP * DP];
    int64_t rows[2][TILE_BLOCK];
    uint64_t missing[2][TILE_BLOCK / 64];                                            // places that their page id or the table's end keeps out
    int lows[TILE_WAVES];
};
// Its arrays one by one: what is on its way into one of them is not waited for where another is read.  TWO: weights are two numbers of the type.
template <class T, int DP, Walk WALK, bool TWO>
__device__ __forceinline__ void attend_tile(const she_attend_pages_args &a, uint32_t group, const Pieces &pieces, const Owners &owners, const void *zeros, uint32_t *d_bad,
                                            T *__restrict__ even_keys, T *__restrict__ even_values, T *__restrict__ odd_keys, T *__restrict__ odd_values,
                                            int64_t (*__restrict__ rows)[TILE_BLOCK], uint64_t (*__restrict__ missing)[TILE_BLOCK / 64], int *__restrict__ lows,
                                            uint32_t slot, int kv_head, int z)
{
    constexpr int UNITS = DP / 8, KS = DP / 16, DB = DP / 32, BLOCK = TILE_BLOCK;
    constexpr int EACH = STEP * UNITS / (64 * TILE_WAVES);                           // units of either tile that a thread brings
    constexpr float LEAD = std::is_same<T, __bf16>::value ? 8.0f : 0.0f;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;
    const int D = (int)a.head;
    const Piece piece = tile_of<WALK>(a, owners, group, TILE_ROWS, slot);
    if (piece.segment < 0) return;
    Span sp = span_of<TILE_ROWS, WALK>(a, owners, group, piece, piece.index * TILE_ROWS, pieces);
    if constexpr (joined_with_another(WALK)) {
        if (leave_none<WALK>(a, owners, group, pieces, sp, kv_head, z)) return;
    } else {
        if (z >= max(sp.parts, 1)) return;
    }
    const bool cut = joined_with_another(WALK) || sp.parts > 1;
    const uint32_t part = pieces.first + z;
    int from = sp.from + z * sp.chunk, count = sp.parts ? min(sp.chunk, sp.to - from) : 0;

    // this lane's row, and what the wavefront's rows attend to
    const int last_row = sp.row + sp.rows - 1, first_here = sp.row + wave * 32, last_here = min(first_here + 31, last_row);
    const int my_row = min(first_here + col, last_row), my_token = my_row / (int)group, my_head = kv_head * (int)group + my_row % (int)group;
    int high, low, high_min, high_max, low_min, low_max;
    if constexpr (WALK == WHOLE) {
        const Reach mine = reach_of<WALK>(a, owners, group, sp, my_row), least = reach_of<WALK>(a, owners, group, sp, min(first_here, last_row)),
                    most = reach_of<WALK>(a, owners, group, sp, last_here);
        high = mine.high, low = mine.low, high_min = least.high, high_max = most.high, low_min = least.low, low_max = most.low;
    } else if constexpr (WALK == PREFIXES) {
        const Reach mine = reach_of<WALK>(a, owners, group, sp, my_row);
        high = high_min = high_max = mine.high;
        low = low_min = low_max = mine.low;
        if (a.window) {                                           // requests in any order: the earliest and the latest place of the rows
#pragma unroll
            for (int m = 1; m < 32; m *= 2) {
                low_min = min(low_min, __shfl_xor(low_min, m));
                low_max = max(low_max, __shfl_xor(low_max, m));
            }
            if (lane == 0) lows[wave] = low_min;
            __syncthreads();
            for (int k = 0; k < TILE_WAVES; k++) sp.low = k ? min(sp.low, lows[k]) : lows[k];
            const int end = from + count;
            from = max(from, sp.low & ~31);
            count = max(end - from, 0);
        }
    } else {
        const int64_t reach = a.window ? (int64_t)a.window - 1 : (int64_t)1 << 40;
        high = sp.first + my_token, low = (int)max(high - reach, (int64_t)0);
        high_min = sp.first + min(first_here, last_row) / (int)group, high_max = sp.first + last_here / (int)group;
        low_min = (int)max(high_min - reach, (int64_t)0), low_max = (int)max(high_max - reach, (int64_t)0);
    }
    const int steps = (count + STEP - 1) / STEP;

    // the rows of a block of places: thread tid has place BLOCK * b + tid, a wavefront a step
    auto page_of = [&](int b) {
        const int i = b * BLOCK + tid;
        if (i >= count) return Slot{-1, 0};
        const Slot at = slot_of<WALK>(a, owners, sp, from + i);
        if (at.page >= 0 && (uint32_t)at.page < a.pages) return at;
        if (counts(sp, from + i, at.in_page, i == 0)) count_bad(d_bad);
        return Slot{-1, 0};
    };
    auto keep_rows = [&](int b, Slot at) {
        rows[b & 1][tid] = at.page < 0 ? -1 : at.page * a.page_stride + (int64_t)at.in_page * a.slot_stride + kv_head * a.page_head;
        const uint64_t out = __ballot(at.page < 0);                                     // from `count` on too: a row may reach beyond the table
        if (lane == 0) missing[b & 1][wave] = out;
    };
    // a step's tiles on their way into LDS: a wavefront's 64 units lie side by side there, so each lane picks the one that belongs in
    // its place; what is not there comes from a unit of zeros
    auto request = [&](int step, T *keys, T *values) {
        const int64_t *row = &rows[step / 4 & 1][step % 4 * STEP + tid / UNITS];
        constexpr int PLACES = 64 * TILE_WAVES / UNITS;
        const int unit = tid % UNITS;
        if (D == DP && (step + 1) * STEP <= count && !missing[step / 4 & 1][step % 4]) {
#pragma unroll
            for (int e = 0; e < EACH; e++) {
                const int place = tid / UNITS + e * PLACES;
                to_lds((const T *)a.k_pages + row[e * PLACES] + key_unit<DP>(place, unit) * 8, keys + (e * TILE_WAVES + wave) * 64 * 8);
                to_lds((const T *)a.v_pages + row[e * PLACES] + value_unit<DP>(place, unit) * 8, values + (e * TILE_WAVES + wave) * 64 * 8);
            }
        } else {
#pragma unroll
            for (int e = 0; e < EACH; e++) {
                const int place = tid / UNITS + e * PLACES, key = key_unit<DP>(place, unit) * 8, value = value_unit<DP>(place, unit) * 8;
                const bool there = row[e * PLACES] >= 0;
                to_lds(there && key < D ? (const T *)a.k_pages + row[e * PLACES] + key : (const T *)zeros, keys + (e * TILE_WAVES + wave) * 64 * 8);
                to_lds(there && value < D ? (const T *)a.v_pages + row[e * PLACES] + value : (const T *)zeros, values + (e * TILE_WAVES + wave) * 64 * 8);
            }
        }
    };

    x8<T> q[KS];
    {
        const T *p = (const T *)a.q + (sp.token0 + my_token) * a.q_token + my_head * a.q_head + half * 8;
#pragma unroll
        for (int s = 0; s < KS; s++) {
            u32x4 v = load8<T, true>(p + s * 16, D - (s * 16 + half * 8));
            if (a.scale < 0) v ^= 0x80008000u;                    // so that the largest score is the largest product
            q[s] = as_x8<T>(v);
        }
    }
    const float scale = fmaxf(fabsf(a.scale) * LOG2E, 1e-37f);    // not 0: hidden places are -inf before it
    float m = -__builtin_inff(), l = 0;
    f32x16 acc[DB];
#pragma unroll
    for (int b = 0; b < DB; b++) acc[b] = f32x16{};

    if (steps) {
        keep_rows(0, page_of(0));
        __syncthreads();
        request(0, even_keys, even_values);
    }
    // Bytes from a tile's start: of the key of place `col`, its unit `half`; and of the value of place half * 4 + (lane & 15) / 4, from
    // element (lane & 16) + (lane & 3) * 4 on.  Later units are exchanged alike, so that theirs follow by exclusive or, and the
    // same unit of 8, 16 or 32 places later follows by adding.
    const int key_at = col * DP * 2 + key_unit<DP>(col, half) * 16;
    const int value_place = half * 4 + (lane & 15) / 4, value_d = (lane & 16) + (lane & 3) * 4;
    const int value_at = value_place * DP * 2 + value_unit<DP>(value_place, value_d / 8) * 16 + value_d % 8 * 2;
    Slot page{-1, 0};
    // Infinite or NaN values where not all rows attend.  (A number, which has a vector register: as a mask in scalar ones it pushes others of these out, and
    // 24 requests of up to 700 tokens under a window take 54.8 us and not 53.8.)
    int special = 0;
    auto do_step = [&](int step, const T *key_tile, const T *value_tile, T *next_keys, T *next_values) {
        wait_for_lds_loads();
        __syncthreads();                                          // this step's tiles are there, the others are free
        if (step % 4 == 0) page = page_of(step / 4 + 1);
        if (step % 4 == 1) keep_rows(step / 4 + 1, page);
        if (step + 1 < steps) request(step + 1, next_keys, next_values);
        const char *keys = reinterpret_cast<const char *>(key_tile), *values = reinterpret_cast<const char *>(value_tile);
        const int p0 = from + step * STEP;
        const uint64_t gone = missing[step / 4 & 1][step % 4];
        if (first_here <= last_row && p0 <= high_max && p0 + STEP > low_min) {
            f32x16 s[2];
#pragma unroll
            for (int t = 0; t < 2; t++) {
                s[t] = f32x16{};
#pragma unroll
                for (int k = 0; k < KS; k++) s[t] = mfma32(*reinterpret_cast<const x8<T> *>(keys + t * 32 * DP * 2 + (key_at ^ k * 32)), q[k], s[t]);
            }
            const bool masked = gone || p0 + STEP - 1 > high_min || p0 < low_max || step * STEP + STEP > count;
            if (__builtin_expect(masked, 0)) {
                const int from_here = p0 + 4 * half, most = high - from_here, least = low - from_here;
                const uint64_t out = gone >> 4 * half;
#pragma unroll
                for (int t = 0; t < 2; t++)
#pragma unroll
                    for (int i = 0; i < 16; i++) {
                        const int n = t * 32 + 8 * (i / 4) + i % 4;
                        if (n > most || n < least || (out >> n & 1)) s[t][i] = -__builtin_inff();
                    }
                for (int i = lane; i < STEP * UNITS; i += 64) special |= has_special<T>(*reinterpret_cast<const u32x4 *>(values + i * 16));
            }
            float top = s[0][0];
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
                for (int i = 0; i < 16; i++) top = fmaxf(top, s[t][i]);
            top = other_half_max(top) * scale;
            // The reference need not be the top itself: it is raised where a top exceeds it by 8.  In bf16, whose largest numbers are
            // f32's, it is raised to 8 above the top, so that no weight is more than 1; f16's smallest weights need the room instead.
            if (__builtin_expect(__ballot(top > m + (8.0f - LEAD)) != 0, 0)) {
                const float to = top > m ? top + LEAD : m, ref = to == -__builtin_inff() ? 0.0f : to, alpha = __builtin_amdgcn_exp2f(m - ref);
                m = to;
                l *= alpha;
#pragma unroll
                for (int b = 0; b < DB; b++)
#pragma unroll
                    for (int i = 0; i < 16; i++) acc[b][i] *= alpha;
            }
            const float ref = m == -__builtin_inff() ? 0.0f : m;
            x8<T> p[4], rest[4];
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const float v = __builtin_amdgcn_exp2f(fmaf(s[t][i], scale, -ref));
                    l += v;
                    p[t * 2 + i / 8][i % 8] = (T)v;
                    if constexpr (TWO) rest[t * 2 + i / 8][i % 8] = (T)(v - (float)p[t * 2 + i / 8][i % 8]);
                }
            // V^T of the 32 elements from 32 b on and the sixteen places from 16 k on, in the scores' order
            auto columns = [&](int b, int k) {
                u32x4 v;
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const u32x2 c = lds_columns(values + (k * 16 + e * 8) * DP * 2 + (value_at ^ b * 64));
                    v[e * 2] = c[0];
                    v[e * 2 + 1] = c[1];
                }
                return v;
            };
#pragma unroll
            for (int k = 0; k < 4; k++)
#pragma unroll
                for (int b = 0; b < DB; b++) {
                    const x8<T> v = as_x8<T>(columns(b, k));
                    if constexpr (TWO) acc[b] = mfma32(v, rest[k], acc[b]);
                    acc[b] = mfma32(v, p[k], acc[b]);
                }
        }
    };
    for (int step = 0; step < steps; step += 2) {
        do_step(step, even_keys, even_values, odd_keys, odd_values);
        if (step + 1 < steps) do_step(step + 1, odd_keys, odd_values, even_keys, even_values);
    }

    l += __shfl_xor(l, 32);
    f32x4 lost{0, 0, 0, 0};                                       // NaN where a sum is, or where infinities meet
#pragma unroll
    for (int b = 0; b < DB; b++)
#pragma unroll
        for (int i = 0; i < 16; i++) lost[i % 4] += acc[b][i];
    const float lost_sum = lost[0] + lost[1] + lost[2] + lost[3];
    if (__ballot(special || (lost_sum != lost_sum && l == l))) {
        for (int row = first_here; row <= last_here; row++)
            attend_row<T, WALK>(a, owners, group, pieces, cut, pieces_at(pieces, a.kv_heads, group, sp, row, kv_head) + part, sp, kv_head, row,
                          Reach{__shfl(low, row - first_here), __shfl(high, row - first_here)}, from, from + count);
        return;
    }
    if (first_here + col > last_row) return;
    const int64_t token = sp.token0 + my_token;
    const size_t at = pieces_at(pieces, a.kv_heads, group, sp, my_row, kv_head) + part;
    const float inv = cut ? 1.0f : l == 0 ? 0.0f : 1.0f / l;
    if (cut && half == 0) pieces.ml[at] = float2{m, WALK == BEHIND && high < 0 ? NOTHING : l};
#pragma unroll
    for (int b = 0; b < DB; b++)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = b * 32 + 2 * i + 4 * half;
            if (d >= D) continue;
            if (cut) {
                *reinterpret_cast<f32x4 *>(pieces.o + at * D + d) = f32x4{acc[b][i], acc[b][i + 1], acc[b][i + 2], acc[b][i + 3]};
            } else {
                T *to = (T *)a.out + token * a.out_token + my_head * a.out_head + d;
                T v[4];
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] = (T)(acc[b][i + e] * inv);
                *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(v);
            }
        }
}
// A key head's tiles are one XCD's where there are eight of them: neighbouring workgroups have different heads.  Late tokens have
// most to attend to: they come first.
template <class T, int DP, Walk WALK, bool TWO>
__global__ __launch_bounds__(64 * TILE_WAVES, DP == 256 ? 1 : 2) void k_attend_tile(she_attend_pages_args a, uint32_t group, Pieces pieces, Owners owners, const void *zeros, uint32_t *d_bad)
{
    __shared__ alignas(16) T even_keys[STEP * DP], even_values[STEP * DP], odd_keys[STEP * DP], odd_values[STEP * DP];
    __shared__ int64_t rows[2][TILE_BLOCK];
    __shared__ uint64_t missing[2][TILE_BLOCK / 64];
    attend_tile<T, DP, WALK, TWO>(a, group, pieces, owners, zeros, d_bad, even_keys, even_values, odd_keys, odd_values, rows, missing, nullptr, gridDim.x / a.kv_heads - 1 - blockIdx.x / a.kv_heads, (int)(blockIdx.x % a.kv_heads), (int)blockIdx.z);
}

// Rows that were cut, `each` of a tile a workgroup.  Up to JOIN_AHEAD pieces are a wavefront's work, and a workgroup of the tile kernel's
// has sixteen rows then (with four, 99 and not 82 us for the whole call of 4063 tokens in two pieces at 16 heads of 64); more are
// shared out among all four wavefronts, a row after the other, four rows a workgroup or, of many pieces, one.  Pieces are requested
// JOIN_AHEAD at a time.  A token over 32768 places, 4 rows of 64 pieces at 8 key heads, takes 33 us so on one input again and again (38 on
// others in turn), 43 with four rows a workgroup and 78 with a row a wavefront.
constexpr int JOIN_AHEAD = 4;
template <class T>
__device__ inline void join_row(const she_attend_pages_args &a, const Pieces &w, size_t at, int parts, int from, int by, float &sum, float o[4])
{
    const int lane = threadIdx.x & 63, D = (int)a.head;
    float top = -__builtin_inff();
    for (int k = lane; k < parts; k += 64) top = fmaxf(top, w.ml[at + k].x);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    sum = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) o[i] = 0;
    for (int k0 = from; k0 < parts; k0 += by * JOIN_AHEAD) {
        float2 ml[JOIN_AHEAD];
        float v[JOIN_AHEAD][4];
#pragma unroll
        for (int e = 0; e < JOIN_AHEAD; e++) {
            const int k = k0 + by * e;
            ml[e] = k < parts ? w.ml[at + k] : float2{-__builtin_inff(), 0};
#pragma unroll
            for (int i = 0; i < 4; i++) v[e][i] = k < parts && lane + 64 * i < D ? w.o[(at + k) * D + lane + 64 * i] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < JOIN_AHEAD; e++) {
            const float f = ml[e].x == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(ml[e].x - top);
            sum = fmaf(ml[e].y, f, sum);
#pragma unroll
            for (int i = 0; i < 4; i++) o[i] = fmaf(v[e][i], f, o[i]);
        }
    }
}
template <class T, int ROWS, Walk WALK>
__global__ __launch_bounds__(256) void k_attend_join(she_attend_pages_args a, uint32_t group, Pieces pieces, Owners owners, int each)
{
    __shared__ float sums[4], joined[4][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = (int)a.head;
    const Piece piece = find_piece(a.starts, a.requests, a.tokens, group, ROWS, blockIdx.x);
    if (piece.segment < 0) return;
    const int64_t first = piece.first + (int64_t)piece.index * ROWS + blockIdx.z * each;
    if (first >= piece.last) return;
    const Span sp = span_of<ROWS, WALK>(a, owners, group, piece, piece.index * ROWS, pieces);
    const int parts = sp.parts, rows = (int)min((int64_t)each, piece.last - first);
    if (parts <= 1) return;
    for (int r = parts <= JOIN_AHEAD ? wave : 0; r < rows; r += parts <= JOIN_AHEAD ? 4 : 1) {
        const int64_t row = first + r, token = row / group;
        const int head = blockIdx.y * (int)group + (int)(row % group);
        const size_t at = pieces_at(pieces, a.kv_heads, group, sp, sp.row + (int)blockIdx.z * each + r, blockIdx.y);
        T *to = (T *)a.out + token * a.out_token + head * a.out_head;
        float sum, o[4];
        if (parts <= JOIN_AHEAD) {
            join_row<T>(a, pieces, at, parts, 0, 1, sum, o);
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (lane + 64 * i < D) to[lane + 64 * i] = (T)(o[i] * (sum == 0 ? 0.0f : 1.0f / sum));
            continue;
        }
        join_row<T>(a, pieces, at, parts, wave, 4, sum, o);
        if (r) __syncthreads();
        if (lane == 0) sums[wave] = sum;
#pragma unroll
        for (int i = 0; i < 4; i++) joined[wave][lane + 64 * i] = o[i];
        __syncthreads();
        const int d = threadIdx.x;
        sum = sums[0] + sums[1] + sums[2] + sums[3];
        if (d < D) to[d] = (T)((joined[0][d] + joined[1][d] + joined[2][d] + joined[3][d]) * (sum == 0 ? 0.0f : 1.0f / sum));
    }
}

// A call with shared prefixes, whose two walks are one launch: while the prefixes' workgroups, of many rows, wait for the matrix units, those
// of the requests' own places wait for memory (64 tokens behind 32768 places with up to 500 of their own, 32 / 8 heads of 128, bf16: 73 to 88 us,
// 67 to 76 with weights of one number and then 6 less without their own places; two launches 95 and not 87 for the whole call at that time).  Such a call
// is bound by what a wavefront does one after the other: with one number a step of 64 places takes 1.7 us where a compute unit has one tile's workgroup, and
// two have theirs in 2.0.  97 requests of up to 4 tokens behind five prefixes (16 heads of 64, f16) take 83 us, 3.3 TB/s.
template <class T, int DP, bool FEW> using SharedOf = typename std::conditional<FEW, FewShared<DP>, TileShared<T, DP>>::type;
template <class T, int DP, bool FEW, Walk WALK, bool TWO>
__device__ __forceinline__ void attend_block(const she_attend_pages_args &a, uint32_t group, const Pieces &pieces, const Owners &owners, const void *zeros, uint32_t *d_bad, char *shared,
                                             uint32_t slots, uint32_t block)
{
    const uint32_t i = block / a.kv_heads, kv_head = block - i * a.kv_heads, z = i / slots, slot = i - z * slots;
    auto &its = *reinterpret_cast<SharedOf<T, DP, FEW> *>(shared);
    if constexpr (FEW) attend_few<T, DP, WALK>(a, group, pieces, owners, d_bad, its, slot, (int)kv_head, (int)z);
    else
        attend_tile<T, DP, WALK, TWO>(a, group, pieces, owners, zeros, d_bad, its.even_keys, its.even_values, its.odd_keys, its.odd_values, its.rows, its.missing, its.lows, slot,
                                 (int)kv_head, (int)z);
}
template <class T, int DP, bool PREFIX_FEW, bool FEW, bool TWO>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void k_attend_shared(she_attend_pages_args a, uint32_t group, Pieces prefix, Pieces pieces, Owners owners, const void *zeros,
                                                                          uint32_t prefix_slots, uint32_t prefix_blocks, uint32_t slots, uint32_t *d_bad)
{
    __shared__ alignas(16) char shared[std::max(sizeof(SharedOf<T, DP, PREFIX_FEW>), sizeof(SharedOf<T, DP, FEW>))];
    if (blockIdx.x < prefix_blocks) {
        she_attend_pages_args p = a;
        p.requests = owners.prefixes;
        p.table = owners.prefix_table;
        p.table_stride = owners.prefix_stride;
        p.table_width = owners.prefix_width;
        p.lengths = owners.prefix_lengths;
        attend_block<T, DP, PREFIX_FEW, PREFIXES, TWO>(p, group, prefix, owners, zeros, d_bad, shared, prefix_slots, blockIdx.x);
    } else {
        attend_block<T, DP, FEW, BEHIND, TWO>(a, group, pieces, owners, zeros, d_bad, shared, slots, blockIdx.x - prefix_blocks);
    }
}

// Rows of such a call, in the order of the pieces: neighbours have different key heads, so that where there are eight a row's pieces come from
// the XCD that wrote them.  Bound by memory where rows are many: 115000 rows of 128 in two pieces 48 us, 118 MB; 2048 rows in 17 pieces
// 8.6 us.  D/4 lanes have a piece's elements, and 4 * `lanes` / D pieces are read side by side by as many threads as
// have the row: a workgroup for many pieces, a wavefront for few, which then needs no barrier.
template <class T, int ROW> __global__ __launch_bounds__(256) void k_shared_join(she_attend_pages_args a, uint32_t group, Pieces pieces)
{
    __shared__ f32x4 joined[256];
    const int tid = threadIdx.x % ROW, lane = threadIdx.x & 63, D = (int)a.head, lanes = D / 4, sets = ROW / lanes, set = tid / lanes, d = tid % lanes * 4, parts = (int)pieces.splits;
    f32x4 *mine = joined + (threadIdx.x - tid);
    const int64_t first = bounded_start(a.starts, 0, a.tokens), last = bounded_start(a.starts, (int)a.requests, a.tokens), rows = (int64_t)a.tokens * a.q_heads;
    for (int64_t row = (int64_t)blockIdx.x * (256 / ROW) + threadIdx.x / ROW; row < rows; row += (int64_t)gridDim.x * (256 / ROW)) {
        const int64_t token = row / a.q_heads;
        const int at_token = (int)(row - token * a.q_heads), kv_head = at_token % (int)a.kv_heads, head = kv_head * (int)group + at_token / (int)a.kv_heads;
        if (token < first || token >= last) continue;
        const float2 *ml = pieces.ml + (size_t)row * parts;
        float top = -__builtin_inff();
        for (int k = lane; k < parts; k += 64) top = fmaxf(top, ml[k].x);
#pragma unroll
        for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
        const auto factor = [&](float of) { return of == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(of - top); };
        float sum = 0;
        for (int k = lane; k < parts; k += 64) sum = fmaf(ml[k].y, factor(ml[k].x), sum);
#pragma unroll
        for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
        const bool none = ml[pieces.first].y == NOTHING;
        const float inv = sum == 0 ? 0.0f : 1.0f / sum;
        f32x4 o{0, 0, 0, 0};
        if (set < sets && !none) {
#pragma unroll 4
            for (int k = set; k < parts; k += sets) {
                const float f = factor(ml[k].x);
                const f32x4 v = f == 0 ? f32x4{0, 0, 0, 0} : *reinterpret_cast<const f32x4 *>(pieces.o + ((size_t)row * parts + k) * D + d);
#pragma unroll
                for (int i = 0; i < 4; i++) o[i] = fmaf(v[i], f, o[i]);
            }
        }
        mine[tid] = o;
        if constexpr (ROW == 64) wave_lds_fence();
        else __syncthreads();
        for (int e = tid; e < D; e += ROW) {
            float v = 0;
            for (int k = 0; k < sets; k++) v += mine[k * lanes + e / 4][e & 3];
            ((T *)a.out)[token * a.out_token + head * a.out_head + e] = none ? (T)0.0f : (T)(v * inv);
        }
        if constexpr (ROW == 64) wave_lds_fence();
        else __syncthreads();
    }
}

// By the padded size of a head.
template <class F> hipError_t by_head(uint32_t head, F launch)
{
    if (head <= 64) launch(std::integral_constant<int, 64>{});
    else if (head <= 128) launch(std::integral_constant<int, 128>{});
    else launch(std::integral_constant<int, 256>{});
    return hipGetLastError();
}

template <class T, Walk WALK, bool TWO>
hipError_t walk(const she_attend_pages_args &a, const AttendShape &s, const Pieces &pieces, const Owners &owners, uint32_t *d_bad, hipStream_t st)
{
    const uint32_t group = a.q_heads / a.kv_heads, slots = (uint32_t)s.slots;
    return by_head(a.head, [&](auto size) {
        constexpr int DP = decltype(size)::value;
        if (s.few) k_attend_few<T, DP, WALK><<<dim3(slots, a.kv_heads, s.splits), 64 * FEW_WAVES, 0, st>>>(a, group, pieces, owners, d_bad);
        else k_attend_tile<T, DP, WALK, TWO><<<dim3(slots * a.kv_heads, 1, s.splits), 64 * TILE_WAVES, 0, st>>>(a, group, pieces, owners, zeros_of(d_bad), d_bad);
    });
}

template <class T, Walk WALK, bool TWO = false> hipError_t attend(const she_attend_pages_args &a, const AttendShape &s, const Pieces &pieces, const Owners &owners, uint32_t *d_bad, hipStream_t st)
{
    const hipError_t rc = walk<T, WALK, TWO>(a, s, pieces, owners, d_bad, st);
    if (rc != hipSuccess || s.splits == 1) return rc;
    const uint32_t group = a.q_heads / a.kv_heads, slots = (uint32_t)s.slots;
    const int each = s.few && s.splits > 4 * JOIN_AHEAD ? 1 : s.few || s.splits > JOIN_AHEAD ? 4 : 16;
    if (s.few)
        k_attend_join<T, FEW_ROWS, WALK><<<dim3(slots, a.kv_heads, FEW_ROWS / each), 256, 0, st>>>(a, group, pieces, owners, each);
    else
        k_attend_join<T, TILE_ROWS, WALK><<<dim3(slots, a.kv_heads, TILE_ROWS / each), 256, 0, st>>>(a, group, pieces, owners, each);
    return hipGetLastError();
}

template <class T> hipError_t attend_shared(const she_attend_pages_args &a, const SharedShape &s, const Pieces &prefix, const Pieces &pieces, const Owners &owners, uint32_t *d_bad, hipStream_t st)
{
    const uint32_t group = a.q_heads / a.kv_heads, prefix_slots = (uint32_t)s.prefix.slots, prefix_blocks = prefix_slots * a.kv_heads * s.prefix.splits;
    const uint32_t slots = (uint32_t)s.behind.slots, blocks = prefix_blocks + slots * a.kv_heads * s.behind.splits;
    const hipError_t rc = by_head(a.head, [&](auto size) {
        constexpr int DP = decltype(size)::value;
        const auto launch = [&](auto kernel) { kernel<<<blocks, 256, 0, st>>>(a, group, prefix, pieces, owners, zeros_of(d_bad), prefix_slots, prefix_blocks, slots, d_bad); };
        if (s.prefix.few) launch(k_attend_shared<T, DP, true, true, false>);
        else if (s.behind.few) s.two ? launch(k_attend_shared<T, DP, false, true, true>) : launch(k_attend_shared<T, DP, false, true, false>);
        else s.two ? launch(k_attend_shared<T, DP, false, false, true>) : launch(k_attend_shared<T, DP, false, false, false>);
    });
    if (rc != hipSuccess) return rc;
    const uint64_t rows = (uint64_t)a.tokens * a.q_heads;
    if (pieces.splits <= 8) k_shared_join<T, 64><<<(uint32_t)std::min<uint64_t>(ceil_div(rows, 4), 1u << 20), 256, 0, st>>>(a, group, pieces);
    else k_shared_join<T, 256><<<(uint32_t)std::min<uint64_t>(rows, 1u << 20), 256, 0, st>>>(a, group, pieces);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_pages(const she_attend_pages_args &a, const AttendShape &s, void *scratch, uint32_t *d_bad, hipStream_t st)
{
    float *o = static_cast<float *>(scratch);
    const Pieces pieces{o, reinterpret_cast<float2 *>(o + attend_pieces(a, s) * a.head), s.splits, 0, s.splits, s.chunk};
    return a.type == SHE_BF16 ? attend<__bf16, REQUESTS>(a, s, pieces, Owners{}, d_bad, st) : attend<_Float16, REQUESTS>(a, s, pieces, Owners{}, d_bad, st);
}

hipError_t launch_attend_shared(const she_attend_shared_args &args, const SharedShape &s, void *scratch, uint32_t *d_bad, hipStream_t st)
{
    const she_attend_pages_args a = shared_behind(args);
    const Owners owners{args.prefix_requests, args.prefix_lengths, a.lengths, args.prefix_table, args.prefix_stride, a.requests, args.prefixes, args.prefix_width};
    float *o = static_cast<float *>(scratch);
    float2 *ml = reinterpret_cast<float2 *>(o + shared_pieces(args, s) * a.head);
    if (s.whole) {
        const Pieces pieces{o, ml, s.behind.splits, 0, s.behind.splits, s.behind.chunk};
        if (s.two) return a.type == SHE_BF16 ? attend<__bf16, WHOLE, true>(a, s.behind, pieces, owners, d_bad, st) : attend<_Float16, WHOLE, true>(a, s.behind, pieces, owners, d_bad, st);
        return a.type == SHE_BF16 ? attend<__bf16, WHOLE>(a, s.behind, pieces, owners, d_bad, st) : attend<_Float16, WHOLE>(a, s.behind, pieces, owners, d_bad, st);
    }
    const uint32_t splits = s.prefix.splits + s.behind.splits;
    const Pieces prefix{o, ml, splits, 0, s.prefix.splits, s.prefix.chunk}, pieces{o, ml, splits, s.prefix.splits, s.behind.splits, s.behind.chunk};
    return a.type == SHE_BF16 ? attend_shared<__bf16>(a, s, prefix, pieces, owners, d_bad, st) : attend_shared<_Float16>(a, s, prefix, pieces, owners, d_bad, st);
}

}}  // namespace she::clear
