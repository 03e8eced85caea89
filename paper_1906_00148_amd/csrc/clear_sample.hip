// The next token of every row of logits.
//
// Weights are whole numbers: exp(x - max x) * 2^43, rounded, of at most 2^20 tokens, so that sums are exact in 64 bits and every order of
// adding gives the same.  One is computed in 64-bit floating point, since a draw next to a border shows an error of 32 bits: with
// y = (logit - max) log2(e) / T in units of 1/256, the nearest whole k and the rest r, it is 2^(k/256) from a table and a power of two,
// times 2^(r/256) by its series up to the fourth power (the fifth is below 2^-54).  What lies more than 44.5 octaves below the
// largest has no weight.
//
// The tokens that filters keep are the first of an order, larger logits first and of equals the lower index: all above a logit, and of
// those equal to it the ones up to an index.  The logit is found by histograms: over y in 32nds of an octave first, then over the
// bits of the bin's logits until a bin is one value.  top_k counts with ones, top_p with weights.
#include "clear_device.h"
#include "clear_internal.h"

namespace she { namespace clear {
namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64, TILE = 512, BINS = 2048;
constexpr int ONE_AT = 43;                                         // a weight of 1 is 2^43
constexpr uint64_t ONE = 1ull << ONE_AT;
constexpr double LOG2E = 1.4426950408889634074, DEAD = -256 * 44.5;

__device__ inline uint32_t key_of(float v)                         // ordered as the numbers are
{
    const uint32_t u = __float_as_uint(v);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ inline float number_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// Eight logits of a row from `at` on, -infinity beyond its end and for NaN, and no negative zero.
template <class T> struct Row {
    const T *p;
    const float *step;
    uint32_t vocab;
};
template <class T> __device__ inline void load_logits(const Row<T> &row, uint32_t at, float v[8])
{
    const int count = (int)min((int64_t)row.vocab - at, (int64_t)8);
    if constexpr (sizeof(T) == 2) {
        unpack<T>(load8<T, false>(row.p + at, count), v);
    } else {
        T raw[8];
        if (count >= 8) {
            __builtin_memcpy(raw, row.p + at, 32);
        } else {
            for (int i = 0; i < 8; i++) raw[i] = i < count ? row.p[at + i] : (T)0;
        }
        if constexpr (__is_same(T, float)) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = raw[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = (float)((double)raw[i] * (row.step && i < count ? (double)row.step[at + i] : 1.0));
        }
    }
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = i < count && v[i] == v[i] ? v[i] + 0.0f : -__builtin_inff();
}

// 2^(j/256), to which a whole exponent is added in place.
__device__ inline void make_table(double *table)
{
    for (int j = threadIdx.x; j < 256; j += blockDim.x) table[j] = exp2(j / 256.0);
}

// What the logits of a row weigh.
struct Weights {
    float top;                           // the largest logit
    double unit;                         // 256 log2(e) / T
    const double *table;

    // in units of 1/256 octave, from 0 down; DEAD where there is no weight
    __device__ double below(float v) const
    {
        const double s = v == top ? 0.0 : ((double)v - (double)top) * unit;
        return s >= DEAD ? s : DEAD;                               // NaN, of -infinity at T = infinity, has none either
    }
    __device__ static int nearest(double s) { return __double2loint(s + 6755399441055744.0); }
    __device__ uint64_t weight(double s) const
    {
        if (s <= DEAD) return 0;
        const double shifted = s + 6755399441055744.0;             // 1.5 * 2^52: the nearest whole number is in the low bits
        const int k = __double2loint(shifted);
        const double r = (s - (shifted - 6755399441055744.0)) * (0.69314718055994530942 / 256);
        const double f = fma(r * r, fma(r, fma(r, 1.0 / 24, 1.0 / 6), 0.5), r);      // 2^(r/256) - 1
        const double t = __longlong_as_double(__double_as_longlong(table[k & 255]) + ((int64_t)(k >> 8) << 52));
        // added to 2^9, whose last bit is 2^-43
        return (uint64_t)(__double_as_longlong(fma(t, f, t) + 512.0) - __double_as_longlong(512.0));
    }
};

__device__ inline uint64_t wave_sum(uint64_t v)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
    return v;
}

// f * all for f in [0, 1), rounded down or up and not by way of a shorter number: a border that falls on a token exactly stays there.
__device__ inline uint64_t share_of(uint64_t all, float f, bool up)
{
    const uint32_t bits = __float_as_uint(f), e = bits >> 23;
    const uint64_t m = e ? (bits & 0x7FFFFF) | 0x800000 : bits;    // f = m / 2^s, s >= 24
    const int s = e ? 150 - (int)e : 149;
    const uint64_t low = m * all, high = __umul64hi(m, all);
    uint64_t q, rest;
    if (s < 64) {
        q = high << (64 - s) | low >> s;
        rest = low << (64 - s);
    } else {
        q = s < 128 ? high >> (s - 64) : 0;
        rest = low | (s == 64 ? 0 : s < 128 ? high << (128 - s) : high);
    }
    return q + (up && rest);
}

// Of the workgroup's array of BINS numbers: the first bin with which their running sum reaches `target` (at least 1), and the sum of those
// before it.  -1: all of them do not reach it.
struct Crossing {
    int bin;
    uint64_t before;
};
__device__ inline Crossing find_crossing(const uint64_t *hist, uint64_t target, uint64_t *sums, Crossing *found)
{
    constexpr int EACH = BINS / THREADS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t mine[EACH], run = 0;
#pragma unroll
    for (int e = 0; e < EACH; e++) run += mine[e] = hist[threadIdx.x * EACH + e];
    const uint64_t own = run;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const uint64_t other = __shfl_up(run, m);
        if (lane >= m) run += other;
    }
    if (lane == 63) sums[wave] = run;
    if (threadIdx.x == 0) *found = Crossing{-1, 0};
    __syncthreads();
    uint64_t before = run - own;
    for (int w = 0; w < wave; w++) before += sums[w];
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        if (before < target && before + mine[e] >= target) *found = Crossing{(int)threadIdx.x * EACH + e, before};
        before += mine[e];
    }
    __syncthreads();
    const Crossing c = *found;
    __syncthreads();
    return c;
}

// The tokens that are kept: of the logits of `key` those up to index `last`, and all with larger keys.
struct Kept {
    uint32_t key, last;
    __device__ bool has(uint32_t k, uint32_t index) const { return k > key || (k == key && index <= last); }
};

struct Shared {
    uint64_t bins[BINS];                 // a histogram; sums or counts of tiles
    double table[256];
    uint64_t sums[WAVES];
    Crossing found;
    float tops[WAVES];
    uint32_t where[WAVES], answer;
};

template <class T, class F> __device__ inline void for_all(const Row<T> &row, F f)
{
    constexpr int AHEAD = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (uint32_t at = wave * TILE; at < row.vocab; at += WAVES * TILE * AHEAD) {
        float v[AHEAD][8];
#pragma unroll
        for (int k = 0; k < AHEAD; k++)
            if (at + k * WAVES * TILE < row.vocab) load_logits(row, at + k * WAVES * TILE + lane * 8, v[k]);
#pragma unroll
        for (int k = 0; k < AHEAD; k++)
            if (at + k * WAVES * TILE < row.vocab) f(at + k * WAVES * TILE + lane * 8, v[k]);
    }
}
__device__ inline void clear_bins(Shared &s)
{
    for (int i = threadIdx.x; i < BINS; i += THREADS) s.bins[i] = 0;
    __syncthreads();
}

// Of what `kept` has, the first of the order whose measure (ones or weights) together reaches `target`; `kept` itself if all does not.
template <bool COUNT, class T> __device__ inline Kept select(const Row<T> &row, const Weights &w, Kept kept, uint64_t target, Shared &s)
{
    const auto measure = [&](double y) { return COUNT ? 1 : w.weight(y); };
    clear_bins(s);
    for_all(row, [&](uint32_t at, const float v[8]) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const double y = w.below(v[i]);
            if (y > DEAD && kept.has(key_of(v[i]), at + i)) atomicAdd((unsigned long long *)&s.bins[-w.nearest(y) >> 3], (unsigned long long)measure(y));
        }
    });
    __syncthreads();
    Crossing c = find_crossing(s.bins, target, s.sums, &s.found);
    if (c.bin < 0) return kept;
    const int bin = c.bin;
    // Keys that surround the bin's, so wide that no rounding matters.  (Where unit is 0, all logits are in bin 0.)
    uint32_t high = key_of(w.top), low = high;
    if (w.top < __builtin_inff()) {
        low = key_of((float)((double)w.top - (8 * bin + 8) / w.unit));
        high = min(high, key_of((float)((double)w.top - (8 * bin - 1) / w.unit)));
    }
    target -= c.before;
    for (;;) {
        int shift = 0;
        while ((high - low) >> shift >= BINS) shift++;
        clear_bins(s);
        for_all(row, [&](uint32_t at, const float v[8]) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t key = key_of(v[i]);
                if (key < low || key > high || !kept.has(key, at + i)) continue;
                const double y = w.below(v[i]);
                if (y > DEAD && -w.nearest(y) >> 3 == bin) atomicAdd((unsigned long long *)&s.bins[(high - key) >> shift], (unsigned long long)measure(y));
            }
        });
        __syncthreads();
        c = find_crossing(s.bins, target, s.sums, &s.found);
        if (c.bin < 0) return kept;                                // not so: the bin reaches the target, and all of it is here
        target -= c.before;
        const uint32_t first = high - ((uint32_t)c.bin << shift);
        if (shift) {
            low = max(low, first - ((1u << shift) - 1));
            high = first;
            continue;
        }
        low = first;
        break;
    }
    // `low` is the last key that is kept; how many of the tokens that have it are
    const uint64_t each = measure(w.below(number_of(low))), all = s.bins[c.bin] / each, wanted = (target + each - 1) / each;
    __syncthreads();
    if (wanted >= all) return Kept{low, low == kept.key ? kept.last : ~0u};
    // the index of the last of them, by tile and then by place
    for_all(row, [&](uint32_t at, const float v[8]) {
        uint32_t here = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) here += key_of(v[i]) == low && kept.has(low, at + i);
        const uint64_t sum = wave_sum(here);
        if ((threadIdx.x & 63) == 0) s.bins[at / TILE] = sum;
    });
    for (int i = threadIdx.x + (row.vocab + TILE - 1) / TILE; i < BINS; i += THREADS) s.bins[i] = 0;
    __syncthreads();
    c = find_crossing(s.bins, wanted, s.sums, &s.found);
    if (threadIdx.x < 64) {
        float v[8];
        const uint32_t at = c.bin * TILE + threadIdx.x * 8;
        load_logits(row, at, v);
        uint32_t here = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) here += key_of(v[i]) == low && kept.has(low, at + i);
        uint32_t run = here;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const uint32_t other = __shfl_up(run, m);
            if ((int)threadIdx.x >= m) run += other;
        }
        uint32_t left = (uint32_t)(wanted - c.before), before = run - here;
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (key_of(v[i]) == low && kept.has(low, at + i) && ++before == left) s.answer = at + i;
    }
    __syncthreads();
    const uint32_t last = s.answer;
    __syncthreads();
    return Kept{low, last};
}

// One workgroup a row.
template <class T> __global__ __launch_bounds__(THREADS) void k_sample_rows(she_sample_args a)
{
    __shared__ Shared s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t r = blockIdx.x;
    const Row<T> row{(const T *)a.logits + r * a.row_stride, a.step, a.vocab};
    make_table(s.table);

    // the largest logit, and the first that is as large
    float top = -__builtin_inff();
    uint32_t where = 0;
    for_all(row, [&](uint32_t at, const float v[8]) {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (v[i] > top) {
                top = v[i];
                where = at + i;
            }
    });
    const auto join = [&](float other, uint32_t place) {
        if (other > top || (other == top && place < where)) {
            top = other;
            where = place;
        }
    };
#pragma unroll
    for (int m = 1; m < 64; m *= 2) join(__shfl_xor(top, m), __shfl_xor(where, m));
    if (lane == 0) {
        s.tops[wave] = top;
        s.where[wave] = where;
    }
    __syncthreads();
    for (int k = 0; k < WAVES; k++) join(s.tops[k], s.where[k]);
    const float temperature = a.temperature ? a.temperature[r] : 1.0f;
    const bool none = top == -__builtin_inff();
    if (none || !(temperature > 0)) {
        if (threadIdx.x == 0) {
            a.tokens[r] = none ? -1 : (int32_t)where;
            if (a.probs) a.probs[r] = none ? 0.0f : 1.0f;
        }
        return;
    }

    const Weights w{top, 256 * LOG2E / (double)temperature, s.table};
    Kept kept{0, ~0u};
    if (a.top_k && a.top_k[r] > 0 && (uint32_t)a.top_k[r] < a.vocab) kept = select<true>(row, w, kept, (uint64_t)a.top_k[r], s);
    const float top_p = a.top_p ? a.top_p[r] : 1.0f;
    const uint32_t tiles = (a.vocab + TILE - 1) / TILE;
    // the kept weights of every tile
    const auto sum_tiles = [&](uint64_t least) {
        for_all(row, [&](uint32_t at, const float v[8]) {
            uint64_t sum = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                if (!kept.has(key_of(v[i]), at + i)) continue;
                const uint64_t weight = w.weight(w.below(v[i]));
                if (weight >= least) sum += weight;
            }
            sum = wave_sum(sum);
            if (lane == 0) s.bins[at / TILE] = sum;
        });
        for (int i = threadIdx.x + tiles; i < BINS; i += THREADS) s.bins[i] = 0;
        __syncthreads();
        uint64_t all = 0;
        for (int i = lane; i < BINS; i += 64) all += s.bins[i];
        return wave_sum(all);
    };
    if (top_p < 1.0f) {
        const uint64_t all = sum_tiles(0);
        __syncthreads();
        kept = select<false>(row, w, kept, max(share_of(all, fmaxf(top_p, 0.0f), true), (uint64_t)1), s);
    }
    const float min_p = a.min_p ? a.min_p[r] : 0.0f;
    const uint64_t least = min_p > 0 ? (uint64_t)ceil((double)fminf(min_p, 1.0f) * (double)ONE) : 0, all = sum_tiles(least);
    const float u = a.uniform[r];
    const uint64_t drawn = share_of(all, u > 0 ? fminf(u, 1.0f - 0x1p-24f) : 0.0f, false);
    const Crossing c = find_crossing(s.bins, drawn + 1, s.sums, &s.found);
    if (threadIdx.x >= 64) return;
    float v[8];
    const uint32_t at = c.bin * TILE + lane * 8;
    load_logits(row, at, v);
    uint64_t weight[8], here = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        weight[i] = kept.has(key_of(v[i]), at + i) ? w.weight(w.below(v[i])) : 0;
        if (weight[i] < least) weight[i] = 0;
        here += weight[i];
    }
    uint64_t run = here;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const uint64_t other = __shfl_up(run, m);
        if (lane >= m) run += other;
    }
    run = run - here + c.before;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if (run <= drawn && run + weight[i] > drawn) {
            a.tokens[r] = (int32_t)(at + i);
            // the weight itself, since of a small one few bits are held
            if (a.probs) a.probs[r] = (float)(exp2(w.below(v[i]) / 256) * ((double)ONE / (double)all));
        }
        run += weight[i];
    }
}

}  // namespace

hipError_t launch_sample(const she_sample_args &a, uint32_t, hipStream_t st)
{
    switch (a.type) {
    case SHE_BF16: k_sample_rows<__bf16><<<a.rows, THREADS, 0, st>>>(a); break;
    case SHE_F16: k_sample_rows<_Float16><<<a.rows, THREADS, 0, st>>>(a); break;
    case SHE_F32: k_sample_rows<float><<<a.rows, THREADS, 0, st>>>(a); break;
    default: k_sample_rows<int32_t><<<a.rows, THREADS, 0, st>>>(a); break;
    }
    return hipGetLastError();
}

}}  // namespace she::clear
