// The next token of every row of logits.
//
// Weights are whole numbers: exp(x - max x) * 2^43, rounded, of at most 2^20 tokens, so that sums are exact in 64 bits and every order of
// adding gives the same.  One is computed in 64-bit floating point, since a draw next to a border shows an error of 32 bits: with
// y = (logit - max) log2(e) / T in units of 1/256, the nearest whole k and the rest r, it is 2^(k/256) from a table and a power of two,
// times 2^(r/256) by its series up to the fourth power (the fifth is below 2^-54).  What lies more than 44.5 octaves below the
// largest has no weight: it is taken as there, where the weight rounds to 0.
// Calls without filters on larger rows hold to this by tiles of 512 logits instead: weights are those against the tile's largest, and the running
// sums in a tile, scaled to the row's largest, are rounded to whole numbers (k_sample_tiles, k_sample_drawn).  Both roundings are of half a unit at
// most, for each token in the one and each tile in the other, and a border may fall as far from where the other forms have it.
//
// The tokens that filters keep are the first of an order, larger logits first and of equals the lower index: all above a logit, and of
// those equal to it the ones up to an index.  Which bin of 1/32 octave has that logit is seen from a histogram: of weights for top_p, which needs all
// of them anyway; for top_k of the largest of every eight neighbours, since k of these that reach a logit are k logits that do.  Where the tokens up to
// that bin are few, up to a thread of a workgroup each, they are picked out and sorted: by the order for the filters, by index for the draw.
// Where they are many, only the bin's own are sorted, and the weights of all others are summed up by tile in the same pass over the row.  A bin that
// is too full for that (equal or nearly equal logits) is divided by the bits of its logits until it is one value.
//
// Bound by latency where rows are few (one of 32001, bf16: 3.5, 5.0 and 10.5 us for the three launches), by memory and 64-bit arithmetic in turns where
// they are many: 256 rows of 131072 numbers of 32 bits take 25 us for the largest (5.4 TB/s), 24 for the weights, and 61 for the answers of rows
// with all kinds of filters; all three take 47 us with top_k = 50 for every row, 128 with top_p = 0.9 (19000 tokens kept), and the two without filters 47.
#include <algorithm>

#include "clear_device.h"
#include "clear_internal.h"

namespace she { namespace clear {
namespace {

constexpr int TILE = 512, BINS = 2048, THREADS = 1024, WAVES = THREADS / 64, PART_THREADS = 256;
constexpr int ONE_AT = 43;                                         // a weight of 1 is 2^43
constexpr uint64_t ONE = 1ull << ONE_AT;
constexpr double LOG2E = 1.4426950408889634074, LN2 = 0.69314718055994530942, DEAD = -256 * 44.5;

__device__ inline uint32_t key_of(float v)                         // ordered as the numbers are
{
    const uint32_t u = __float_as_uint(v + 0.0f);                  // no negative zero
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ inline float number_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

template <class T> struct Row {
    const T *p;
    const float *step;
    uint32_t vocab;
};
template <class T> __device__ inline Row<T> row_of(const she_sample_args &a, uint32_t r) { return Row<T>{(const T *)a.logits + r * a.row_stride, a.step, a.vocab}; }

// Eight logits of a row from `at` on, NaN beyond its end.
template <class T> __device__ __forceinline__ void load_logits(const Row<T> &row, uint32_t at, float v[8])
{
    const int64_t left = (int64_t)row.vocab - at;                  // any distance, also of a place that no row has
    const int count = left <= 0 ? 0 : left < 8 ? (int)left : 8;
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
            float step[8];
            if (row.step && count >= 8) {
                __builtin_memcpy(step, row.step + at, 32);
            } else {
                for (int i = 0; i < 8; i++) step[i] = row.step && i < count ? row.step[at + i] : 1.0f;
            }
            // one rounding: a sum need not be a number of 32 bits
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = (float)((double)raw[i] * (double)step[i]);
        }
    }
    if (count < 8) {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < count ? v[i] : __builtin_nanf("");
    }
}

// 2^(j/256), to which a whole exponent is added in place: the series of exp(j ln 2 / 256), which is worked out by the compiler, since exp2 takes
// as long as a few tiles (k_sample_tiles for 64 rows of 100000 13.6 us, 14.5 with it).
struct Powers {
    double of[256];
    constexpr Powers() : of()
    {
        for (int j = 0; j < 256; j++) {
            const long double x = j * 0.693147180559945309417232121458L / 256;
            long double sum = 1, term = 1;
            for (int n = 1; n < 24; n++) sum += term *= x / n;
            of[j] = (double)sum;
        }
    }
};
__device__ constexpr Powers POWERS{};
__device__ __forceinline__ void make_table(double *table)
{
    for (int j = threadIdx.x; j < 256; j += blockDim.x) table[j] = POWERS.of[j];
}

// What the logits of a row weigh.
struct Weights {
    float top;                           // the largest logit, 0 where that is infinite
    bool infinite;                       // it is: then those that are have 0 for a logit, and the others -infinity
    double unit;                         // 256 log2(e) / T, finite
    const double *table;

    __device__ __forceinline__ Weights(float largest, float temperature, const double *table)
        : top(largest + 0.0f), infinite(largest == __builtin_inff()), unit(fmin(256 * LOG2E / (double)temperature, 1e300)), table(table)
    {
        if (infinite) top = 0;
    }
    // logits as they are compared, which NaN is not
    __device__ __forceinline__ void plain(const float v[8], float l[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; i++) l[i] = v[i];
        if (infinite)
            for (int i = 0; i < 8; i++) l[i] = v[i] == __builtin_inff() ? 0.0f : -__builtin_inff();
    }
    // in units of 1/256 octave, from 0 down
    __device__ __forceinline__ double distance(float v) const
    {
        if (infinite) v = v == __builtin_inff() ? 0.0f : -__builtin_inff();
        return ((double)v - (double)top) * unit;
    }
    // down to DEAD, which is where NaN goes too
    __device__ __forceinline__ double below(float v) const { return fmax(distance(v), DEAD); }
    __device__ __forceinline__ double below_plain(float v) const { return fmax(((double)v - (double)top) * unit, DEAD); }
    __device__ __forceinline__ static int nearest(double s) { return __double2loint(s + 6755399441055744.0); }      // 1.5 * 2^52: the low bits have it
    __device__ __forceinline__ static int bin(double s) { return -nearest(s) >> 3; }
    // the weight, with the bits of 512.0 above it
    __device__ __forceinline__ uint64_t raw_weight(double s) const
    {
        constexpr double L = LN2 / 256;
        const double shifted = s + 6755399441055744.0;
        const int k = __double2loint(shifted);
        const double r = s - (shifted - 6755399441055744.0);
        const double f = r * fma(r, fma(r, fma(r, L * L * L * L / 24, L * L * L / 6), L * L / 2), L);       // 2^(r/256) - 1
        const double t = __longlong_as_double(__double_as_longlong(table[k & 255]) + ((int64_t)(k & ~255) << 44));
        return (uint64_t)__double_as_longlong(fma(t, f, t) + 512.0);                                       // whose last bit is 2^-43
    }
    __device__ __forceinline__ uint64_t weight(double s) const { return raw_weight(s) - (uint64_t)__double_as_longlong(512.0); }
};
constexpr uint64_t RAW = 0x4080000000000000ull;                    // the bits of 512.0
constexpr int DEAD_BIN = (int)(256 * 44.5) >> 3;

__device__ __forceinline__ uint64_t wave_sum(uint64_t v)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
    return v;
}

// f * all for f in [0, 1), rounded down or up and not by way of a shorter number: a border that falls on a token exactly stays there.
__device__ __forceinline__ uint64_t share_of(uint64_t all, float f, bool up)
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
__device__ __forceinline__ Crossing find_crossing(const uint64_t *hist, uint64_t target, uint64_t *sums, Crossing *found)
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

// The tokens that are kept: those above a logit, and of those that have it the ones up to index `last`.
struct Kept {
    float logit;
    uint32_t last;
    __device__ __forceinline__ bool has(float l, uint32_t index) const { return l > logit || (l == logit && index <= last); }
};
__device__ __forceinline__ Kept all_kept() { return Kept{-__builtin_inff(), ~0u}; }

struct Shared {
    uint64_t bins[BINS];                 // a histogram; sums or counts of tiles
    double table[256];
    uint64_t list[THREADS];              // tokens: the logit's key above the index turned round, so that larger ones come first
    uint64_t sums[WAVES], totals[WAVES];
    Crossing found;
    Kept cut;
    float tops[WAVES];
    uint32_t where[WAVES], answer, count, eights;
    uint32_t waiting[WAVES][TILE];       // logits that wait for their weight; places of eights
};
__device__ __forceinline__ uint64_t token_of(float l, uint32_t index) { return (uint64_t)key_of(l) << 32 | (uint32_t)~index; }
__device__ __forceinline__ float logit_of(uint64_t token) { return number_of((uint32_t)(token >> 32)); }

__device__ __host__ inline uint32_t eights_of(uint32_t vocab) { return (vocab + 7) / 8; }

// A row's logits eight by eight: f(index, logits, whether they are there) for whole wavefronts, a tile each.  Eights below `least` need not be there.
template <class T> struct FromMemory {
    Row<T> row;
    const float *eights;                 // the largest of each; may be null
    template <class F> __device__ __forceinline__ void all(float least, F f) const
    {
        // two at a time: while they are used the next two are on their way, and whether those after them have to be there
        constexpr int AHEAD = 2;
        const uint32_t lane = threadIdx.x & 63, end = eights_of(row.vocab);
        struct Two {
            float largest[AHEAD], v[AHEAD][8];
            bool there[AHEAD];
        } a, b;
        const auto ask = [&](Two &t, uint32_t e0) {
#pragma unroll
            for (int k = 0; k < AHEAD; k++) t.largest[k] = eights && e0 + k * THREADS < end ? eights[e0 + k * THREADS] : __builtin_inff();
        };
        const auto fetch = [&](Two &t, uint32_t e0) {
#pragma unroll
            for (int k = 0; k < AHEAD; k++) {
                t.there[k] = e0 + k * THREADS < end && t.largest[k] >= least;
                if (t.there[k]) load_logits(row, (e0 + k * THREADS) * 8, t.v[k]);
            }
        };
        const auto use = [&](const Two &t, uint32_t e0) {
#pragma unroll
            for (int k = 0; k < AHEAD; k++)
                if (e0 + k * THREADS - lane < end) f((e0 + k * THREADS) * 8, t.v[k], t.there[k]);
        };
        constexpr uint32_t BY = AHEAD * THREADS;
        ask(a, threadIdx.x);
        ask(b, threadIdx.x + BY);
        fetch(a, threadIdx.x);
#pragma unroll 1
        for (uint32_t e0 = threadIdx.x; e0 - lane < end; e0 += 2 * BY) {
            fetch(b, e0 + BY);
            ask(a, e0 + 2 * BY);
            use(a, e0);
            fetch(a, e0 + 2 * BY);
            ask(b, e0 + 3 * BY);
            use(b, e0 + BY);
        }
    }
};
template <class T> struct Held {         // by the workgroup, eight a thread
    Row<T> row;
    float v[8];
    template <class F> __device__ __forceinline__ void all(float, F f) const
    {
        if ((threadIdx.x & ~63u) * 8 < row.vocab) f(threadIdx.x * 8, v, true);
    }
};
__device__ __forceinline__ void clear_bins(Shared &s)
{
    for (int i = threadIdx.x; i < BINS; i += THREADS) s.bins[i] = 0;
    __syncthreads();
}

// The running sum of v over the workgroup's threads; `all` gets the last.
__device__ __forceinline__ uint64_t running_sum(uint64_t v, uint64_t &all, Shared &s)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const uint64_t other = __shfl_up(v, m);
        if (lane >= m) v += other;
    }
    if (lane == 63) s.totals[wave] = v;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int k = 0; k < WAVES; k++) {
        if (k == wave) v += all;
        all += s.totals[k];
    }
    __syncthreads();
    return v;
}
__device__ __forceinline__ uint64_t block_sum(uint64_t v, Shared &s)
{
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) s.totals[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int k = 0; k < WAVES; k++) v += s.totals[k];
    __syncthreads();
    return v;
}

// The numbers of the threads, the largest first, where those from `count` on have 0: a bitonic sort.
__device__ __forceinline__ uint64_t sorted(uint64_t v, uint32_t count, Shared &s)
{
    const uint32_t i = threadIdx.x;
#pragma unroll 1
    for (uint32_t k = 2; k < 2 * count; k *= 2)
#pragma unroll 1
        for (uint32_t d = k / 2; d; d /= 2) {
            uint64_t other;
            if (d >= 64) {
                __syncthreads();
                s.list[i] = v;
                __syncthreads();
                other = s.list[i ^ d];
            } else {
                other = __shfl_xor(v, (int)d);
            }
            if ((((i & d) == 0) == ((i & k) == 0)) != (v > other)) v = other;
        }
    return v;
}

// A logit that is no larger than any of y or more, in units of 1/256 octave; one that is no smaller than any of a bin.
__device__ __forceinline__ float least_at(const Weights &w, double y) { return (float)((double)w.top + (y - 1) / w.unit); }
__device__ __forceinline__ float most_at(const Weights &w, int bin) { return bin ? (float)((double)w.top - (8 * bin - 1) / w.unit) : __builtin_inff(); }

// Of what `kept` has, the tokens of a bin, if they are no more than threads, in no order.  Returns how many there are.
template <class S> __device__ __forceinline__ uint32_t pick_out(const S &row, const Weights &w, Kept kept, int bin, Shared &s)
{
    __syncthreads();
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
    const float least = least_at(w, -8 * bin - 8), most = most_at(w, bin);
    row.all(least, [&](uint32_t at, const float v[8], bool there) {
        if (!there || s.count > THREADS) return;
        float l[8];
        w.plain(v, l);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (!(l[i] >= least) || l[i] > most) continue;
            const double y = w.below_plain(l[i]);
            if (!(y > DEAD) || w.bin(y) != bin || !kept.has(l[i], at + i)) continue;
            const uint32_t n = atomicAdd(&s.count, 1u);
            if (n < THREADS) s.list[n] = token_of(l[i], at + i);
        }
    });
    __syncthreads();
    return s.count;
}

// Of what `kept` has, the first of the order whose measure (ones or weights) together reaches `target`; `kept` itself if all does not.
// No token of a bin behind `bound` is among them.
template <bool COUNT, class S> __device__ __forceinline__ Kept select(const S &source, const Weights &w, Kept kept, uint64_t target, int bound, Shared &s)
{
    const auto &row = source.row;
    const auto measure = [&](double y) { return COUNT ? 1 : w.weight(y); };
    const float least = fmaxf(kept.logit, least_at(w, -8 * bound - 8));
    clear_bins(s);
    source.all(least, [&](uint32_t at, const float v[8], bool there) {
        if (!there) return;
        float l[8];
        w.plain(v, l);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (!(l[i] >= least) || !kept.has(l[i], at + i)) continue;
            const double y = w.below_plain(l[i]);
            if (y > DEAD) atomicAdd((unsigned long long *)&s.bins[w.bin(y)], (unsigned long long)measure(y));
        }
    });
    __syncthreads();
    Crossing c = find_crossing(s.bins, target, s.sums, &s.found);
    if (c.bin < 0) return kept;
    const int bin = c.bin;
    target -= c.before;
    const uint32_t count = pick_out(source, w, kept, bin, s);
    if (count <= THREADS) {
        const uint64_t token = sorted(threadIdx.x < count ? s.list[threadIdx.x] : 0, count, s), mine = threadIdx.x < count ? measure(w.below_plain(logit_of(token))) : 0;
        uint64_t all;
        const uint64_t run = running_sum(mine, all, s);
        if (run >= target && run - mine < target) s.cut = Kept{logit_of(token), ~(uint32_t)token};
        __syncthreads();
        return s.cut;
    }
    // Keys that surround the bin's, so wide that no rounding matters.  (Where unit is 0, all logits are in bin 0.)
    uint32_t low = key_of((float)((double)w.top - (8 * bin + 8) / w.unit)), high = min(key_of(w.top), key_of((float)((double)w.top - (8 * bin - 1) / w.unit)));
    for (;;) {
        int shift = 0;
        while ((high - low) >> shift >= BINS) shift++;
        clear_bins(s);
        source.all(number_of(low), [&](uint32_t at, const float v[8], bool there) {
            if (!there) return;
            float l[8];
            w.plain(v, l);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t key = key_of(l[i]);
                if (key < low || key > high || !kept.has(l[i], at + i)) continue;
                const double y = w.below_plain(l[i]);
                if (y > DEAD && w.bin(y) == bin) atomicAdd((unsigned long long *)&s.bins[(high - key) >> shift], (unsigned long long)measure(y));
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
    // `border` is the last logit that is kept; how many of the tokens that have it are
    const float border = number_of(low);
    const uint64_t each = measure(w.below_plain(border)), all = s.bins[c.bin] / each, wanted = (target + each - 1) / each;
    __syncthreads();
    if (wanted >= all) return Kept{border, border == kept.logit ? kept.last : ~0u};
    // the index of the last of them, by tile and then by place
    source.all(border, [&](uint32_t at, const float v[8], bool there) {
        float l[8];
        w.plain(v, l);
        uint32_t here = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) here += there && l[i] == border && kept.has(border, at + i);
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
        w.plain(v, v);
        uint32_t here = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) here += v[i] == border && kept.has(border, at + i);
        uint32_t run = here;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const uint32_t other = __shfl_up(run, m);
            if ((int)threadIdx.x >= m) run += other;
        }
        uint32_t left = (uint32_t)(wanted - c.before), before = run - here;
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (v[i] == border && kept.has(border, at + i) && ++before == left) s.answer = at + i;
    }
    __syncthreads();
    const uint32_t last = s.answer;
    __syncthreads();
    return Kept{border, last};
}

struct Settings {
    float temperature, top_p, uniform;
    uint32_t top_k;                      // vocab: all
    uint64_t least;                      // the weight that min_p asks for
    float share;                         // of the largest: min_p, 0 to 1
    __device__ __forceinline__ Settings(const she_sample_args &a, uint32_t r) : temperature(a.temperature ? a.temperature[r] : 1.0f), top_p(a.top_p ? a.top_p[r] : 1.0f), uniform(a.uniform[r])
    {
        const int32_t k = a.top_k ? a.top_k[r] : 0;
        top_k = k > 0 && (uint32_t)k < a.vocab ? (uint32_t)k : a.vocab;
        const float m = a.min_p ? a.min_p[r] : 0.0f;
        share = m > 0 ? fminf(m, 1.0f) : 0.0f;
        least = (uint64_t)ceil((double)share * (double)ONE);
        uniform = uniform > 0 ? fminf(uniform, 1.0f - 0x1p-24f) : 0.0f;
    }
    __device__ __forceinline__ float least_logit(const Weights &w) const { return share > 0 ? least_at(w, 256 * log2((double)share)) : -__builtin_inff(); }
    __device__ __forceinline__ uint64_t head(uint64_t all) const { return max(share_of(all, fmaxf(top_p, 0.0f), true), (uint64_t)1); }    // of a whole weight, for top_p below 1
};

__device__ inline void answer(const she_sample_args &a, uint32_t r, int32_t token, float prob)
{
    a.tokens[r] = token;
    if (a.probs) a.probs[r] = prob;
}
// The weight itself, since of a small one few bits are held.
__device__ __forceinline__ float prob_of(double y, uint64_t all) { return (float)(exp2(y / 256) * ((double)ONE / (double)all)); }

// The draw from sums of the kept weights of every tile, in s.bins.
template <class T> __device__ __forceinline__ void draw_by_tiles(const she_sample_args &a, uint32_t r, const Row<T> &row, const Weights &w, const Settings &set, const Kept &kept, Shared &s)
{
    const int lane = threadIdx.x & 63;
    uint64_t all = 0;
    for (int i = lane; i < BINS; i += 64) all += s.bins[i];
    all = wave_sum(all);
    const uint64_t drawn = share_of(all, set.uniform, false);
    const Crossing c = find_crossing(s.bins, drawn + 1, s.sums, &s.found);
    if (threadIdx.x >= 64) return;
    float v[8];
    const uint32_t at = c.bin * TILE + lane * 8;
    load_logits(row, at, v);
    w.plain(v, v);
    uint64_t weight[8], here = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        weight[i] = kept.has(v[i], at + i) ? w.weight(w.below_plain(v[i])) : 0;
        if (weight[i] < set.least) weight[i] = 0;
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
        if (run <= drawn && run + weight[i] > drawn) answer(a, r, (int32_t)(at + i), prob_of(w.below_plain(v[i]), all));
        run += weight[i];
    }
}

// The weights of a tile's logits, of which a wavefront's lanes hold eight each, `which` a bit for each that counts.  Few do mostly, and a weight is
// many instructions: they are moved together first.
__device__ __forceinline__ uint64_t tile_sum(const Weights &w, const float l[8], uint32_t which, uint64_t least, Shared &s)
{
    const uint32_t lane = threadIdx.x & 63;
    float *waiting = reinterpret_cast<float *>(s.waiting[threadIdx.x >> 6]);
    uint32_t count = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint64_t those = __ballot(which >> i & 1);
        if (which >> i & 1) waiting[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(those >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)those, 0))] = l[i];
        count += __popcll(those);
    }
    wave_lds_fence();
    uint64_t sum = 0;
#pragma unroll 2
    for (uint32_t i = lane; i < count; i += 64) {
        const uint64_t weight = w.weight(w.below_plain(waiting[i]));
        if (weight >= least) sum += weight;
    }
    wave_lds_fence();
    return count ? wave_sum(sum) : 0;
}

// The weights that are kept of every tile.
template <class S> __device__ __forceinline__ void sum_tiles(const S &source, const Weights &w, const Kept &kept, const Settings &set, bool filtered, Shared &s)
{
    const uint64_t least = filtered ? set.least : 0;
    const float floor = fmaxf(kept.logit, filtered ? set.least_logit(w) : -__builtin_inff());
    __syncthreads();
    source.all(floor, [&](uint32_t at, const float v[8], bool there) {
        float l[8];
        w.plain(v, l);
        uint32_t which = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) which |= (there && l[i] >= floor && kept.has(l[i], at + i)) << i;
        const uint64_t sum = tile_sum(w, l, which, least, s);
        if ((threadIdx.x & 63) == 0) s.bins[at / TILE] = sum;
    });
    for (int i = threadIdx.x + (source.row.vocab + TILE - 1) / TILE; i < BINS; i += THREADS) s.bins[i] = 0;
    __syncthreads();
}

// Both for top_p alone, in one pass: with the histogram of all weights in s.bins, the bin that has the border is picked out and the weights above it
// are summed up.  Returns whether the bin has no more tokens than there are threads; if it has, s.bins is not as it was.
template <class S> __device__ __forceinline__ bool head_sums(const S &source, const Weights &w, const Settings &set, uint64_t target, Kept &kept, Shared &s)
{
    const Crossing c = find_crossing(s.bins, target, s.sums, &s.found);
    const int bin = c.bin;                                         // there is one: the target is at most all of it
    target -= c.before;
    if (threadIdx.x == 0) {
        s.count = 0;
        s.cut = all_kept();                                        // where min_p leaves none of the bin, or none behind the border
    }
    clear_bins(s);
    // logits below `least` are behind the bin, and those above `most` before it
    const float least = least_at(w, -8 * bin - 8), most = most_at(w, bin), floor = set.least_logit(w);
    source.all(fmaxf(least, floor), [&](uint32_t at, const float v[8], bool there) {
        float l[8];
        w.plain(v, l);
        uint32_t which = 0, close = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            which |= (there && l[i] > most) << i;
            close |= (there && l[i] >= least && !(l[i] > most)) << i;
        }
        for (; close; close &= close - 1) {
            const int at_i = __builtin_ctz(close);
            float its = l[0];
#pragma unroll
            for (int i = 1; i < 8; i++) its = at_i == i ? l[i] : its;
            const double y = w.below_plain(its);
            if (!(y > DEAD) || w.bin(y) > bin) continue;
            if (w.bin(y) < bin) {
                which |= 1u << at_i;
                continue;
            }
            const uint32_t n = atomicAdd(&s.count, 1u);
            if (n < THREADS) s.list[n] = token_of(its, at + at_i);
        }
        const uint64_t sum = tile_sum(w, l, which, set.least, s);
        if ((threadIdx.x & 63) == 0) s.bins[at / TILE] = sum;
    });
    __syncthreads();
    const uint32_t count = s.count;
    if (count > THREADS) return false;
    const uint64_t token = sorted(threadIdx.x < count ? s.list[threadIdx.x] : 0, count, s), mine = threadIdx.x < count ? w.weight(w.below_plain(logit_of(token))) : 0;
    uint64_t all;
    const uint64_t before = running_sum(mine, all, s) - mine;
    const uint32_t index = ~(uint32_t)token;
    if (threadIdx.x < count && before < target) {
        if (mine >= set.least) atomicAdd((unsigned long long *)&s.bins[index / TILE], (unsigned long long)mine);
        if (before + mine >= target) s.cut = Kept{logit_of(token), index};
    }
    __syncthreads();
    kept = s.cut;
    return true;
}

// A row of any kind by passes over all of it.  `known`: s.bins has the histogram of all weights, there is no top_k, and `target` is top_p of
// them.  `bound`: as in select, of the first filter.
template <class T, class S> __device__ __forceinline__ void pass_by_pass(const she_sample_args &a, uint32_t r, const S &source, const Weights &w, const Settings &set, bool known, uint64_t target, int bound, Shared &s)
{
    Kept kept = all_kept();
    if (set.top_k < a.vocab) kept = select<true>(source, w, kept, set.top_k, bound, s);
    if (known) {
        if (head_sums(source, w, set, target, kept, s)) {
            draw_by_tiles(a, r, source.row, w, set, kept, s);
            return;
        }
        kept = select<false>(source, w, kept, target, bound, s);
    } else if (set.top_p < 1.0f) {
        sum_tiles(source, w, kept, set, false, s);
        uint64_t all = 0;
        for (int i = threadIdx.x; i < BINS; i += THREADS) all += s.bins[i];
        all = block_sum(all, s);
        kept = select<false>(source, w, kept, set.head(all), DEAD_BIN, s);
    }
    sum_tiles(source, w, kept, set, true, s);
    draw_by_tiles(a, r, source.row, w, set, kept, s);
}

// The draw from `count` tokens in s.list; `whole`: the row's weight, which top_p is of where there is no top_k.
__device__ __forceinline__ void draw_by_list(const she_sample_args &a, uint32_t r, const Weights &w, const Settings &set, uint64_t whole, uint32_t count, Shared &s)
{
    const uint32_t i = threadIdx.x;
    const auto weight_of = [&](float logit) { return w.weight(w.below_plain(logit)); };
    const uint64_t token = sorted(i < count ? s.list[i] : 0, count, s);
    bool kept = i < count && i < set.top_k;
    uint64_t weight = kept ? weight_of(logit_of(token)) : 0, all;
    if (set.top_p < 1.0f) {
        const uint64_t before = running_sum(weight, all, s) - weight;
        kept &= before < set.head(set.top_k < a.vocab ? all : whole);
    }
    // the first threads have what is kept: now by its index, the lowest first
    const uint32_t left = (uint32_t)__syncthreads_count(kept);
    const uint64_t turned = sorted(kept && weight >= set.least ? token << 32 | token >> 32 : 0, left, s);
    const float logit = number_of((uint32_t)turned);
    weight = turned ? weight_of(logit) : 0;
    const uint64_t run = running_sum(weight, all, s), drawn = share_of(all, set.uniform, false);
    if (run > drawn && run - weight <= drawn) answer(a, r, (int32_t)~(uint32_t)(turned >> 32), prob_of(w.below_plain(logit), all));
}

// Rows of few logits, which a workgroup holds.
template <class T> __global__ __launch_bounds__(THREADS) void k_sample_rows(she_sample_args a)
{
    __shared__ Shared s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t r = blockIdx.x;
    const Settings set(a, r);                                      // which the answer may overwrite: barriers follow
    Held<T> source{row_of<T>(a, r)};
    load_logits(source.row, threadIdx.x * 8, source.v);
    make_table(s.table);

    // the largest logit, and the first that is as large
    float top = -__builtin_inff();
    uint32_t where = 0;
    source.all(-__builtin_inff(), [&](uint32_t at, const float v[8], bool there) {
        if (!there) return;
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
    const bool none = top == -__builtin_inff();
    if (none || !(set.temperature > 0)) {
        if (threadIdx.x == 0) answer(a, r, none ? -1 : (int32_t)where, none ? 0.0f : 1.0f);
        return;
    }
    const Weights w(top, set.temperature, s.table);
    if (a.vocab <= THREADS && (set.top_k < a.vocab || set.top_p < 1.0f)) {
        // all of them are few (148 rows of 214 with all filters 24.9 us by passes, 18.1 so)
        float l[8];
        w.plain(source.v, l);
        uint64_t sum = 0;
        for (int i = 0; i < 8; i++) {
            const uint32_t at = threadIdx.x * 8 + i;
            if (at >= a.vocab) break;
            s.list[at] = l[i] > -__builtin_inff() ? token_of(l[i], at) : 0;
            sum += w.weight(w.below_plain(l[i]));
        }
        sum = block_sum(sum, s);
        draw_by_list(a, r, w, set, sum, a.vocab, s);
        return;
    }
    pass_by_pass<T>(a, r, source, w, set, false, 0, DEAD_BIN, s);
}

// Larger rows, in three launches.  First a row's parts have the largest logit of every eight neighbours, and their own.
struct Parts {
    float2 *tops;                        // [rows][parts]: the largest logit of each part, and the first eight neighbours that have it
    float *eights;                       // [rows][ceil(vocab / 8)]; null where no filter asks for them
    uint64_t *bins;                      // [rows][BINS]: the histogram of weights for top_p, or the weights of tiles without a filter
    uint32_t parts, tiles;               // tiles of a part, a multiple of PART_THREADS * 8 / TILE
};

template <class T> __global__ __launch_bounds__(PART_THREADS) void k_sample_largest(she_sample_args a, Parts w)
{
    constexpr int AHEAD = 4;
    __shared__ float tops[PART_THREADS / 64];
    __shared__ uint32_t wheres[PART_THREADS / 64];
    const uint32_t r = blockIdx.x / w.parts, part = blockIdx.x - r * w.parts;         // one axis: another one ends at 65535
    const Row<T> row = row_of<T>(a, r);
    for (uint32_t i = part * PART_THREADS + threadIdx.x; i < BINS; i += w.parts * PART_THREADS) w.bins[(size_t)r * BINS + i] = 0;
    const uint32_t first = part * w.tiles * (TILE / 8), last = min(first + w.tiles * (TILE / 8), eights_of(a.vocab));
    float top = -__builtin_inff();
    uint32_t where = first;
    for (uint32_t e0 = first + threadIdx.x; e0 < last; e0 += PART_THREADS * AHEAD) {
        float v[AHEAD][8];
#pragma unroll
        for (int k = 0; k < AHEAD; k++)
            if (e0 + k * PART_THREADS < last) load_logits(row, (e0 + k * PART_THREADS) * 8, v[k]);
#pragma unroll
        for (int k = 0; k < AHEAD; k++) {
            const uint32_t e = e0 + k * PART_THREADS;
            if (e >= last) break;
            float m = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 8; i++) m = fmaxf(m, v[k][i]);
            if (w.eights) w.eights[(size_t)r * eights_of(a.vocab) + e] = m;
            if (m > top) {
                top = m;
                where = e;
            }
        }
    }
    const auto join = [&](float other, uint32_t place) {
        if (other > top || (other == top && place < where)) {
            top = other;
            where = place;
        }
    };
#pragma unroll
    for (int m = 1; m < 64; m *= 2) join(__shfl_xor(top, m), __shfl_xor(where, m));
    if ((threadIdx.x & 63) == 0) {
        tops[threadIdx.x >> 6] = top;
        wheres[threadIdx.x >> 6] = where;
    }
    __syncthreads();
    if (threadIdx.x) return;
    for (int k = 1; k < PART_THREADS / 64; k++) join(tops[k], wheres[k]);
    w.tops[(size_t)r * w.parts + part] = float2{top, __uint_as_float(where)};
}
// The largest logit of a row, and the first eight neighbours that have it.  Every wavefront has both.
__device__ __forceinline__ void largest_of(const Parts &w, uint32_t r, float &top, uint32_t &where)
{
    const uint32_t lane = threadIdx.x & 63;
    const float2 mine = w.tops[(size_t)r * w.parts + min(lane, w.parts - 1)];
    top = mine.x;
    where = __float_as_uint(mine.y);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const float other = __shfl_xor(top, m);
        const uint32_t place = __shfl_xor(where, m);
        if (other > top || (other == top && place < where)) {
            top = other;
            where = place;
        }
    }
}

// Then the weights of rows without top_k: a histogram for top_p, or their sums over tiles.
template <class T> __global__ __launch_bounds__(PART_THREADS) void k_sample_weights(she_sample_args a, Parts w)
{
    constexpr int AHEAD = 2;
    __shared__ double table[256];
    __shared__ uint64_t bins[DEAD_BIN + 1];
    const uint32_t r = blockIdx.x / w.parts, part = blockIdx.x - r * w.parts;
    const Settings set(a, r);
    float top;
    uint32_t where;
    largest_of(w, r, top, where);
    if (top == -__builtin_inff() || !(set.temperature > 0) || set.top_k < a.vocab) return;
    const Row<T> row = row_of<T>(a, r);
    const Weights weights(top, set.temperature, table);
    make_table(table);
    const bool by_bin = set.top_p < 1.0f;
    if (by_bin)
        for (int i = threadIdx.x; i <= DEAD_BIN; i += PART_THREADS) bins[i] = 0;
    __syncthreads();
    const uint32_t first = part * w.tiles * (TILE / 8), last = min(first + w.tiles * (TILE / 8), eights_of(a.vocab));
    const uint64_t least = set.least + RAW;
    // whole wavefronts stay together: a tile is one's 64 times eight
    for (uint32_t e0 = first + threadIdx.x; e0 - (threadIdx.x & 63) < last; e0 += PART_THREADS * AHEAD) {
        float v[AHEAD][8];
#pragma unroll
        for (int k = 0; k < AHEAD; k++) load_logits(row, (e0 + k * PART_THREADS) * 8, v[k]);
#pragma unroll
        for (int k = 0; k < AHEAD; k++) {
            const uint32_t e = e0 + k * PART_THREADS;
            if (e - (threadIdx.x & 63) >= last) break;
            if (by_bin) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const double y = weights.below(v[k][i]);
                    if (y > DEAD) atomicAdd((unsigned long long *)&bins[weights.bin(y)], (unsigned long long)weights.weight(y));
                }
            } else {
                uint64_t sum = 0;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const uint64_t raw = weights.raw_weight(weights.below(v[k][i]));
                    sum += raw >= least ? raw - RAW : 0;
                }
                sum = wave_sum(sum);
                if ((threadIdx.x & 63) == 0) w.bins[(size_t)r * BINS + e / (TILE / 8)] = sum;
            }
        }
    }
    if (!by_bin) return;
    __syncthreads();
    for (int i = threadIdx.x; i <= DEAD_BIN; i += PART_THREADS)
        if (bins[i]) atomicAdd((unsigned long long *)&w.bins[(size_t)r * BINS + i], (unsigned long long)bins[i]);
}

// The tokens of the bins up to `last`, if they are no more than threads, in no order: first the eights that have any, then these.  Returns how many there
// are, or more than threads.
template <class T> __device__ __forceinline__ uint32_t pick_few(const FromMemory<T> &source, const Weights &w, int last, Shared &s)
{
    constexpr int AHEAD = 16;
    const uint32_t end = eights_of(source.row.vocab);
    uint32_t *places = s.waiting[0];
    __syncthreads();
    if (threadIdx.x == 0) s.count = s.eights = 0;
    __syncthreads();
    const float least = least_at(w, -8 * last - 8);
#pragma unroll 1
    for (uint32_t e0 = threadIdx.x; e0 < end; e0 += THREADS * AHEAD) {
        float m[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; k++) m[k] = e0 + k * THREADS < end ? source.eights[e0 + k * THREADS] : -__builtin_inff();
#pragma unroll
        for (int k = 0; k < AHEAD; k++) {
            if (!(m[k] >= least) || m[k] == -__builtin_inff()) continue;
            const uint32_t n = atomicAdd(&s.eights, 1u);
            if (n < THREADS) places[n] = (e0 + k * THREADS) * 8;
        }
    }
    __syncthreads();
    const uint32_t eights = s.eights;
    if (threadIdx.x < min(eights, (uint32_t)THREADS)) {
        float v[8];
        const uint32_t at = places[threadIdx.x];
        load_logits(source.row, at, v);
        w.plain(v, v);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const double y = w.below_plain(v[i]);
            if (!(y > DEAD) || w.bin(y) > last) continue;
            const uint32_t n = atomicAdd(&s.count, 1u);
            if (n < THREADS) s.list[n] = token_of(v[i], at + i);
        }
    }
    __syncthreads();
    // the eights that are left out, if any, may have no token: rounding is on the safe side there
    return eights <= THREADS ? s.count : THREADS + 1;
}

// And the rows' answers.
template <class T> __global__ __launch_bounds__(THREADS) void k_sample_answers(she_sample_args a, Parts parts)
{
    __shared__ Shared s;
    const uint32_t r = blockIdx.x;
    const Row<T> row = row_of<T>(a, r);
    const Settings set(a, r);
    float top;
    uint32_t where;
    largest_of(parts, r, top, where);
    const bool none = top == -__builtin_inff();
    if (none || !(set.temperature > 0)) {
        __syncthreads();                                           // all have read the settings, which the answer may overwrite
        if (threadIdx.x >= 64) return;
        float v[8];
        load_logits(row, where * 8, v);
        if (threadIdx.x) return;
        int i = 0;
        while (i < 7 && v[i] != top) i++;
        answer(a, r, none ? -1 : (int32_t)(where * 8 + i), none ? 0.0f : 1.0f);
        return;
    }
    make_table(s.table);
    const Weights w(top, set.temperature, s.table);
    const FromMemory<T> source{row, parts.eights + (size_t)r * eights_of(a.vocab)};
    const bool counted = set.top_k < a.vocab, headed = set.top_p < 1.0f;
    uint64_t all = 0;
    if (counted) {
        // the k-th of the eights' largest is no larger than the k-th logit
        clear_bins(s);
        constexpr int AHEAD = 8;
        const uint32_t end = eights_of(a.vocab);
#pragma unroll 1
        for (uint32_t e0 = threadIdx.x; e0 < end; e0 += THREADS * AHEAD) {
            float m[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; k++) m[k] = e0 + k * THREADS < end ? source.eights[e0 + k * THREADS] : -__builtin_inff();
#pragma unroll
            for (int k = 0; k < AHEAD; k++) {
                const double y = w.below(m[k]);
                if (y > DEAD) atomicAdd((unsigned long long *)&s.bins[w.bin(y)], 1ull);
            }
        }
        __syncthreads();
    } else {
        for (int i = threadIdx.x; i < BINS; i += THREADS) all += s.bins[i] = parts.bins[(size_t)r * BINS + i];
        all = block_sum(all, s);
        if (!headed) {
            draw_by_tiles(a, r, row, w, set, all_kept(), s);
            return;
        }
    }
    const uint64_t target = counted ? set.top_k : set.head(all);
    const Crossing c = find_crossing(s.bins, target, s.sums, &s.found);
    const int bound = c.bin < 0 ? DEAD_BIN : c.bin;
    uint32_t count = 0;
    if (!counted) {
        // at least as many tokens as their weight is of the largest that their bin has room for
        float many = 0;
        for (int b = threadIdx.x; b <= bound; b += THREADS) many += (float)s.bins[b] * (0.98f / (float)ONE) * __builtin_amdgcn_exp2f(b / 32.0f);
        count = (uint32_t)block_sum((uint64_t)fminf(many, 2 * THREADS), s);
    }
    if (count <= THREADS) count = pick_few(source, w, bound, s);
    if (count <= THREADS) draw_by_list(a, r, w, set, all, count, s);
    else pass_by_pass<T>(a, r, source, w, set, !counted, target, bound, s);
}

// Larger rows of calls without filters, in two launches.  A wavefront has a tile of 512 logits, whose weights and sum are those against the tile's
// own largest logit; what a tile counts in its row is its sum times 2^(how far its largest is below the row's), rounded.
struct Tiles {
    uint64_t *sums;                      // [rows][count]
    float *tops;                         // [rows][count]
    uint32_t count, each;                // tiles of a row, tiles of a wavefront
};
template <class T> __global__ __launch_bounds__(PART_THREADS) void k_sample_tiles(she_sample_args a, Tiles w)
{
    constexpr int AHEAD = 2;
    __shared__ double table[256];
    const uint32_t parts = (w.count + w.each * (PART_THREADS / 64) - 1) / (w.each * (PART_THREADS / 64)), lane = threadIdx.x & 63;
    const uint32_t r = blockIdx.x / parts, part = blockIdx.x - r * parts, first = (part * (PART_THREADS / 64) + (threadIdx.x >> 6)) * w.each, last = min(first + w.each, w.count);
    const Row<T> row = row_of<T>(a, r);
    const float temperature = a.temperature ? a.temperature[r] : 1.0f;
    float v[AHEAD][8];
#pragma unroll
    for (int k = 0; k < AHEAD; k++) load_logits(row, (first + k) * TILE + lane * 8, v[k]);
    make_table(table);
    __syncthreads();
    for (uint32_t t0 = first; t0 < last; t0 += AHEAD) {
#pragma unroll
        for (int k = 0; k < AHEAD; k++) {
            if (t0 + k >= last) break;
            float top = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 8; i++) top = fmaxf(top, v[k][i]);
#pragma unroll
            for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
            uint64_t sum = 0;
            if (temperature > 0 && top > -__builtin_inff()) {
                const Weights weights(top, temperature, table);
#pragma unroll
                for (int i = 0; i < 8; i++) sum += weights.raw_weight(weights.below(v[k][i])) - RAW;
                sum = wave_sum(sum);
            }
            load_logits(row, (t0 + k + AHEAD < last ? t0 + k + AHEAD : w.count) * TILE + lane * 8, v[k]);
            if (lane == 0) {
                w.sums[(size_t)r * w.count + t0 + k] = sum;
                w.tops[(size_t)r * w.count + t0 + k] = top;
            }
        }
    }
}
// A wavefront a row, which needs no barriers.  (Both launches with a workgroup of sixteen for each row, and so, in us on the device: 2000 rows of 20000
// 99 and 58, one of 32001 12.5 and 9.3, 64 of 100000 21.7 and 21.5; two of 1000000, whose 1954 tiles are much for one, 14.9 and 23.5.)
template <class T> __global__ __launch_bounds__(64) void k_sample_drawn(she_sample_args a, Tiles w)
{
    __shared__ double table[256];
    __shared__ uint64_t in_row[BINS];                              // what the tiles count
    const uint32_t r = blockIdx.x, lane = threadIdx.x;
    const Settings set(a, r);
    const uint64_t *sums = w.sums + (size_t)r * w.count;
    const float *tops = w.tops + (size_t)r * w.count;
    make_table(table);
    float top = -__builtin_inff();
    uint32_t where = 0;
#pragma unroll 4
    for (uint32_t t = lane; t < w.count; t += 64) {
        const float its = tops[t];
        where = its > top ? t : where;
        top = fmaxf(top, its);
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const float other = __shfl_xor(top, m);
        const uint32_t place = __shfl_xor(where, m);
        if (other > top || (other == top && place < where)) {
            top = other;
            where = place;
        }
    }
    __syncthreads();
    const Row<T> row = row_of<T>(a, r);
    const bool none = top == -__builtin_inff();
    if (none || !(set.temperature > 0)) {
        float v[8];
        load_logits(row, where * TILE + lane * 8, v);
        uint32_t here = 8;
#pragma unroll
        for (int i = 7; i >= 0; i--) here = v[i] == top ? i : here;
        const uint64_t those = __ballot(here < 8);
        if (none ? lane == 0 : (int)lane == __builtin_ctzll(those)) answer(a, r, none ? -1 : (int32_t)(where * TILE + lane * 8 + here), none ? 0.0f : 1.0f);
        return;
    }
    const Weights weights(top, set.temperature, table);
    // whole numbers below 2^53 times a factor, which every running sum is rounded with alike.  A tile whose largest has no weight counts nothing, however
    // many logits it has that are equal to that.
    const auto factor = [&](float its) {
        const double y = weights.below(its);
        return y > DEAD ? exp2(y / 256) : 0.0;
    };
    const auto counted = [](uint64_t sum, double f) { return (uint64_t)((double)sum * f + 0.5); };
    uint64_t all = 0;
#pragma unroll 4
    for (uint32_t t = lane; t < w.count; t += 64) {
        const uint64_t sum = sums[t];
        const double f = factor(tops[t]);
        all += in_row[t] = counted(sum, f);
    }
    all = wave_sum(all);
    const uint64_t drawn = share_of(all, set.uniform, false);
    // the tile that it falls into, and what is before that
    Crossing c{0, 0};
    for (uint32_t t0 = 0; t0 < w.count; t0 += 64) {
        const uint64_t mine = t0 + lane < w.count ? in_row[t0 + lane] : 0;
        uint64_t run = mine;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const uint64_t other = __shfl_up(run, m);
            if ((int)lane >= m) run += other;
        }
        const uint64_t those = __ballot(c.before + run > drawn);
        if (those) {
            const int it = __builtin_ctzll(those);
            c.bin = (int)t0 + it;
            c.before += __shfl(run - mine, it);
            break;
        }
        c.before += __shfl(run, 63);
    }
    float v[8];
    const uint32_t at = c.bin * TILE + lane * 8;
    load_logits(row, at, v);
    const float its = tops[c.bin];
    const Weights mine(its, set.temperature, table);
    const double f = factor(its);
    uint64_t weight[8], run = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) run += weight[i] = mine.weight(mine.below(v[i]));
    const uint64_t own = run;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const uint64_t other = __shfl_up(run, m);
        if ((int)lane >= m) run += other;
    }
    run -= own;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint64_t before = c.before + counted(run, f);
        run += weight[i];
        // a tile that begins above DEAD has tokens beyond it
        if (before <= drawn && c.before + counted(run, f) > drawn) answer(a, r, (int32_t)(at + i), prob_of(weights.distance(v[i]), all));
    }
}

template <class T> hipError_t sample_rows(const she_sample_args &a, const SampleShape &s, void *scratch, hipStream_t st)
{
    if (!s.parts) {
        k_sample_rows<T><<<a.rows, THREADS, 0, st>>>(a);
        return hipGetLastError();
    }
    if (s.plain) {
        Tiles w{};
        w.count = (uint32_t)ceil_div(a.vocab, TILE);
        w.each = s.tiles;
        w.sums = static_cast<uint64_t *>(scratch);
        w.tops = reinterpret_cast<float *>(w.sums + (size_t)a.rows * w.count);
        k_sample_tiles<T><<<a.rows * s.parts, PART_THREADS, 0, st>>>(a, w);
        const hipError_t rc = hipGetLastError();
        if (rc != hipSuccess) return rc;
        k_sample_drawn<T><<<a.rows, 64, 0, st>>>(a, w);
        return hipGetLastError();
    }
    Parts w{};
    w.bins = static_cast<uint64_t *>(scratch);
    w.tops = reinterpret_cast<float2 *>(w.bins + (size_t)a.rows * BINS);
    w.eights = a.top_k || a.top_p ? reinterpret_cast<float *>(w.tops + (size_t)a.rows * s.parts) : nullptr;
    w.parts = s.parts;
    w.tiles = s.tiles;
    k_sample_largest<T><<<a.rows * s.parts, PART_THREADS, 0, st>>>(a, w);
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess) return rc;
    k_sample_weights<T><<<a.rows * s.parts, PART_THREADS, 0, st>>>(a, w);
    if ((rc = hipGetLastError()) != hipSuccess) return rc;
    k_sample_answers<T><<<a.rows, THREADS, 0, st>>>(a, w);
    return hipGetLastError();
}

template <class T> hipError_t sample(const she_sample_args &a, const SampleShape &s, void *scratch, hipStream_t st)
{
    for (uint32_t r = 0; r < a.rows; r += s.rows) {
        she_sample_args b = a;
        b.rows = std::min(s.rows, a.rows - r);
        b.logits = (const T *)a.logits + r * a.row_stride;
        b.uniform += r;
        b.tokens += r;
        if (a.temperature) b.temperature += r;
        if (a.top_k) b.top_k += r;
        if (a.top_p) b.top_p += r;
        if (a.min_p) b.min_p += r;
        if (a.probs) b.probs += r;
        const hipError_t rc = sample_rows<T>(b, s, scratch, st);
        if (rc != hipSuccess) return rc;
    }
    return hipSuccess;
}

}  // namespace

SampleShape sample_shape(const she_sample_args &a, uint32_t cus)
{
    SampleShape s{};
    s.rows = a.rows;
    if (a.vocab <= 8 * THREADS) return s;
    s.plain = !a.top_k && !a.top_p && !a.min_p;
    s.rows = std::min({a.rows, (1u << 28) / a.vocab, s.plain ? a.rows : 8192u});       // what rows with filters leave behind takes up to 270 MB
    if (s.plain) {
        // a tile a wavefront, or more of them where there are many
        const uint64_t tiles = ceil_div(a.vocab, TILE), steps = ceil_div(tiles, PART_THREADS / 64), parts = std::max<uint64_t>(1, std::min<uint64_t>(steps, ceil_div(16 * cus, s.rows)));
        s.tiles = (uint32_t)ceil_div(steps, parts);
        s.parts = (uint32_t)ceil_div(tiles, s.tiles * (PART_THREADS / 64));
        return s;
    }
    constexpr uint32_t STEP = PART_THREADS * 8;                    // logits that a workgroup of a part has at once
    const uint64_t steps = ceil_div(a.vocab, STEP), parts = std::max<uint64_t>(1, std::min<uint64_t>({16, steps, ceil_div(8 * cus, s.rows)}));
    s.tiles = (uint32_t)(ceil_div(steps, parts) * (STEP / TILE));
    s.parts = (uint32_t)ceil_div(a.vocab, (uint64_t)s.tiles * TILE);
    return s;
}

size_t sample_scratch(const she_sample_args &a, const SampleShape &s)
{
    if (!s.parts) return 0;
    if (s.plain) return (size_t)s.rows * ceil_div(a.vocab, TILE) * (sizeof(uint64_t) + sizeof(float));
    return (size_t)s.rows * (BINS * sizeof(uint64_t) + s.parts * sizeof(float2) + (a.top_k || a.top_p ? eights_of(a.vocab) * sizeof(float) : 0));
}

hipError_t launch_sample(const she_sample_args &a, const SampleShape &s, void *scratch, hipStream_t st)
{
    switch (a.type) {
    case SHE_BF16: return sample<__bf16>(a, s, scratch, st);
    case SHE_F16: return sample<_Float16>(a, s, scratch, st);
    case SHE_F32: return sample<float>(a, s, scratch, st);
    default: return sample<int32_t>(a, s, scratch, st);
    }
}

}}  // namespace she::clear
