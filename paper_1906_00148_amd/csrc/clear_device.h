// What the clear side's kernels share: element types, 16-byte accesses, matrix instructions, and the search of a tile's segment.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace she { namespace clear {

using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));

template <class T> struct Of;
template <> struct Of<__bf16> { using x8 = bf16x8; };
template <> struct Of<_Float16> { using x8 = f16x8; };
template <class T> using x8 = typename Of<T>::x8;

// C[16][16] += A[16][32] B[32][16].  Lane l holds A[l%16][8*(l/16) ..+7], B[8*(l/16) ..+7][l%16] and C[4*(l/16) + i][l%16].
__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
// C[32][32] += A[32][16] B[16][32].  Lane l holds A[l%32][8*(l/32) ..+7], B[8*(l/32) ..+7][l%32] and, for i < 16,
// C[8*(i/4) + 4*(l/32) + i%4][l%32].
__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

template <class T> __device__ inline x8<T> as_x8(u32x4 v) { return __builtin_bit_cast(x8<T>, v); }
template <class T> __device__ inline u32x4 as_words(x8<T> v) { return __builtin_bit_cast(u32x4, v); }

// Eight elements from p on, of which the first `count` exist; the others are zeros.  WIDE: count is 8 or at most 0, p on 16 bytes.
// Otherwise p is on its element's two bytes, where the device loads and stores as much at once, if with more requests for it.
template <class T, bool WIDE> __device__ inline u32x4 load8(const T *p, int count)
{
    if constexpr (WIDE) {
        return count > 0 ? *reinterpret_cast<const u32x4 *>(p) : u32x4{0, 0, 0, 0};
    } else {
        if (count >= 8) {
            u32x4 w;
            __builtin_memcpy(&w, p, 16);
            return w;
        }
        x8<T> v;
        for (int i = 0; i < 8; i++) v[i] = i < count ? p[i] : (T)0.0f;
        return as_words<T>(v);
    }
}
template <class T, bool WIDE> __device__ inline void store8(T *p, u32x4 words, int count)
{
    if constexpr (WIDE) {
        if (count > 0) *reinterpret_cast<u32x4 *>(p) = words;
    } else if (count >= 8) {
        __builtin_memcpy(p, &words, 16);
    } else {
        const x8<T> v = as_x8<T>(words);
        for (int i = 0; i < 8; i++)
            if (i < count) p[i] = v[i];
    }
}
// Four elements from p on and four from p + 64 on, of which the first `count` of the first and `more` of the others exist.  WIDE: all or
// none of either four, p on 8 bytes.
template <class T, bool WIDE> __device__ inline u32x4 load_quads(const T *p, int count, int more)
{
    if constexpr (WIDE) {
        const uint2 a = count > 0 ? *reinterpret_cast<const uint2 *>(p) : uint2{0, 0}, b = more > 0 ? *reinterpret_cast<const uint2 *>(p + 64) : uint2{0, 0};
        return u32x4{a.x, a.y, b.x, b.y};
    } else {
        if (count >= 4 && more >= 4) {
            uint2 a, b;
            __builtin_memcpy(&a, p, 8);
            __builtin_memcpy(&b, p + 64, 8);
            return u32x4{a.x, a.y, b.x, b.y};
        }
        x8<T> v;
        for (int i = 0; i < 4; i++) {
            v[i] = i < count ? p[i] : (T)0.0f;
            v[4 + i] = i < more ? p[64 + i] : (T)0.0f;
        }
        return as_words<T>(v);
    }
}
template <class T, bool WIDE> __device__ inline void store_quads(T *p, u32x4 words, int count, int more)
{
    if constexpr (WIDE) {
        if (count > 0) *reinterpret_cast<uint2 *>(p) = uint2{words[0], words[1]};
        if (more > 0) *reinterpret_cast<uint2 *>(p + 64) = uint2{words[2], words[3]};
    } else if (count >= 4 && more >= 4) {
        const uint2 a{words[0], words[1]}, b{words[2], words[3]};
        __builtin_memcpy(p, &a, 8);
        __builtin_memcpy(p + 64, &b, 8);
    } else {
        const x8<T> v = as_x8<T>(words);
        for (int i = 0; i < 4; i++) {
            if (i < count) p[i] = v[i];
            if (i < more) p[64 + i] = v[4 + i];
        }
    }
}
template <class T> __device__ inline void unpack(u32x4 words, float out[8])
{
    const x8<T> v = as_x8<T>(words);
#pragma unroll
    for (int i = 0; i < 8; i++) out[i] = (float)v[i];
}
template <class T> __device__ inline u32x4 pack(const float in[8])
{
    x8<T> v;
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (T)in[i];
    return as_words<T>(v);
}

// The operand of a matrix instruction of sixteen rows of 32 neighbours, loaded as memory has it: lane l the unit l % 4 of row l / 4, which
// keeps the requests of neighbouring lanes in one line.  Lane l gets unit l / 16 of row l % 16.  (Loaded the operand's way round, every
// lane's 16 bytes are a line of their own, and a compute unit takes in 16 bytes a cycle.)
__device__ inline int operand_row() { return threadIdx.x >> 2 & 15; }
__device__ inline int operand_unit() { return threadIdx.x & 3; }
__device__ inline u32x4 to_operand(u32x4 v)
{
    const int from = ((threadIdx.x & 15) * 4 + (threadIdx.x >> 4 & 3)) * 4;
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)v[i]);
    return v;
}

// Eight rows of COLS neighbours -> for each of these columns, its elements of the eight rows.
template <class T, int COLS> __device__ inline void transpose8(const u32x4 rows[8], x8<T> cols[COLS])
{
#pragma unroll
    for (int m = 0; m < COLS; m++) {
        u32x4 w;
#pragma unroll
        for (int p = 0; p < 4; p++)
            w[p] = __builtin_amdgcn_perm(rows[2 * p + 1][m / 2], rows[2 * p][m / 2], m & 1 ? 0x07060302u : 0x05040100u);
        cols[m] = as_x8<T>(w);
    }
}

// Of the 4 x 16 elements that sixteen neighbouring lanes point at, four neighbours each and four lanes a row, lane c gets column c.
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
using s16x4 = short __attribute__((ext_vector_type(4)));
__device__ inline u32x2 lds_columns(const void *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}

// A wavefront's 64 units of 16 bytes, each from its lane's address, to LDS from `to` on; they are there after wait_for_lds_loads.
__device__ inline void to_lds(const void *from, void *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}
__device__ inline void wait_for_lds_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }      // vmcnt(0)

// The larger of a lane's number and that of the lane 32 away.
__device__ inline float other_half_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// LDS that one wavefront alone uses: its operations run in order, and this keeps the compiler from moving them.
__device__ inline void wave_lds_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ inline void count_bad(uint32_t *d_bad) { atomicAdd(d_bad, 1u); }

// Ragged segments [starts[s], starts[s+1]) of `scale` rows a token are cut into tiles of `tile` rows without a list of them: segment
// s owns the slots from starts[s] * scale / tile + s on, at least as many as it has tiles, so that rows / tile + segments slots
// serve any lengths.  The wavefront looks 64 segments up at a time.  Whatever `starts` holds, the rows stay inside [0, rows).
struct Piece {
    int segment;             // -1: the slot has no rows
    int index;               // of the tile in its segment
    int64_t first, last;     // the segment's rows
};
__device__ inline int64_t bounded_start(const int32_t *starts, int s, uint32_t tokens)
{
    const int32_t v = starts[s];
    return v < 0 ? 0 : (uint32_t)v > tokens ? tokens : v;
}
// `start_of(s)`: where segment s starts, inside [0, tokens] whatever it is read from.
template <class F> __device__ inline Piece find_piece_by(F start_of, uint32_t segments, uint32_t scale, uint32_t tile, uint32_t slot)
{
    const int lane = threadIdx.x & 63;
    int found = 0;
    for (uint32_t s0 = 0; s0 < segments; s0 += 64) {
        const uint32_t s = s0 + lane;
        const bool before = s < segments && start_of((int)s) * scale / tile + s <= slot;
        const int n = __popcll(__ballot(before));
        found += n;
        if (n < 64) break;
    }
    Piece p{-1, 0, 0, 0};
    if (!found) return p;
    const int s = __builtin_amdgcn_readfirstlane(found - 1);
    const int64_t a = start_of(s), b = start_of(s + 1);
    const int64_t index = (int64_t)slot - (a * scale / tile + s);
    if (b > a && index >= 0 && index * tile < (b - a) * scale) {
        p.segment = s;
        p.index = __builtin_amdgcn_readfirstlane((int)index);
        p.first = a * scale;
        p.last = b * scale;
    }
    return p;
}
__device__ inline Piece find_piece(const int32_t *starts, uint32_t segments, uint32_t tokens, uint32_t scale, uint32_t tile, uint32_t slot)
{
    return find_piece_by([=](int s) { return bounded_start(starts, s, tokens); }, segments, scale, tile, slot);
}

}}  // namespace she::clear
