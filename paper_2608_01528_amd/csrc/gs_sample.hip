// An entry drawn from a row of scores: temperature, top-k, top-p, min-p, and a
// given random number.
//
// Scores are ranked exactly, by an order-preserving integer key.  Weights are
// formed in fp64 and held as whole multiples, at least one, of 2^-shift of the
// largest one, so their sums are integer sums: the same in any order, whatever
// the split of a row over threads, and atomic sums are as good as ordered ones.
// Up to LONG_ROW entries the shift goes by the row's length: a sum is off by less
// than M 2^-shift <= 2^-26 of the largest weight.  For longer rows that grows as
// M^2 (a tail of no weight would come to a quarter of the largest entry at 2^30),
// and the shift is taken from the row's total, which two more launches find: a
// sum is off by less than M 2^-60 of the total (8 rows of 262145: 42 us, 30 with
// the shift by length; with top_p 313 and 295).
//
// What is kept is a run of the entries in rank order (falling scores, equal
// ones by index), thinned by min_p from its end: top_k and top_p each end it
// after some entry.  No row is sorted.  Forms by the size of a row:
//   a thread a row      up to 32 entries: every pair compared
//   a wave a row        up to 2048 entries, in registers: the end of the run is
//                       found by halving the range of keys
//   a work-group a row  up to 8189 entries, in registers: a histogram of the
//                       scores below the largest finds the bin the run ends in
//   work-groups a row   more entries: the same over chunks of 8192, in five
//                       launches (largest scores, histogram, where the run ends,
//                       entries in question, ranking and draw; the two for the
//                       total after the first).  A launch
//                       boundary hands a row's data on faster than fences and
//                       counters did, which write caches back from every
//                       work-group: 200 rows of 128001 took 402 and 511 us in
//                       the launches that had them, 97 and 128 without
//   the same, few kept  where top_k keeps up to half as many entries as the row
//                       has parts of 256: a second launch reads the parts whose
//                       largest scores reach k parts' ones, and draws.  Where
//                       each row has a top_k of its own the other launches
//                       follow for the rest, from 256 parts on (131072 entries,
//                       one row, top_k 50: 24 us for all rows alike, 31 for each
//                       its own, 38 without; 32000: 24, 33 and 37, but 70 with a
//                       row among them that keeps more, 44 without)
//
// Few rows are bound by the launches and the latency within them (4 us a
// launch that does nothing), many by the fp64 work of the weights: some 40
// instructions an entry, 25.6 million of which take 30 us of 53 in the histogram
// launch for 200 rows of 128001; the scores alone would be read in 11.
#include <algorithm>

#include "gs_internal.h"

namespace gs {
namespace {

typedef float f4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));

// Key of a score: larger scores have larger keys, equal scores (the two zeros
// among them) equal keys; 0 for entries that cannot be drawn (-inf, NaN).
__device__ __forceinline__ uint32_t key_of(float x) {
    if (!(x > -INFINITY)) return 0;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t LOWEST = 0x00800000u;     // key of the lowest finite score
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// 2^(i / 64), i = 0..63, in LDS: the table that weights are formed from.
constexpr int TABLE = 64;
__device__ __forceinline__ void fill_table(double *table, int t) {
    if (t < TABLE) table[t] = exp2((double)t / TABLE);
}

// Weight of an entry, exp((x - max) / temperature) = 2^(y / 64): the whole part
// of y from the table and the exponent, the rest, |f| <= 1/2, by its series up
// to f^4 (the next term is below 4e-14 of the weight).  Whole parts and
// multiples are taken by adding a power of two whose last place is the unit
// (no conversions between fp64 and integers).
// LONG: rows of more than LONG_ROW entries.
template <bool LONG> struct WeighOf {
    double m, c;                // largest score; 64 log2(e) / temperature
    int shift;                  // a mass of 2^shift (at most 2^51; LONG: 2^61) is the largest weight
    const double *table;
    // an infinite largest score leaves weight to its equals alone
    __device__ __forceinline__ WeighOf(uint32_t top, double c64, int s, const double *t)
        : m(fmin((double)value_of(top), 1e300)), c(c64), shift(s), table(t) {}
    __device__ __forceinline__ double scaled(uint32_t key) const { return fmin(((double)value_of(key) - m) * c, 0.); }
    __device__ __forceinline__ double part(double y, int &n) const {     // 2^(y / 64) = part 2^n
        const double z = y + 6755399441055744.;                         // 1.5 2^52
        const int whole = (int)(uint32_t)__double_as_longlong(z);
        const double f = y - (z - 6755399441055744.);
        constexpr double L = 0.693147180559945309417 / TABLE;
        n = whole >> 6;
        return fma(fma(fma(fma(f, L * L * L * L / 24, L * L * L / 6), f, L * L / 2), f, L), f, 1.) * table[whole & (TABLE - 1)];
    }
    __device__ __forceinline__ double weight(uint32_t key) const {
        int n;
        const double w = part(fmax(scaled(key), -1100. * TABLE), n);
        return ldexp(w, n);
    }
    // The weight in whole multiples of 2^-shift, at least one (zero only below
    // the smallest fp64 number); weights below 2^-70 all round to that one.
    __device__ __forceinline__ uint64_t mass(uint32_t key) const {
        const double y = scaled(key);
        int n;
        const double w = part(fmax(y, -70. * TABLE), n);
        const double v = __longlong_as_double(__double_as_longlong(w) + (int64_t)(n + shift) * (1ll << 52));
        const uint64_t r = LONG ? (uint64_t)(v + 0.5)
                                : (uint64_t)__double_as_longlong(v + 4503599627370496.) & 0xfffffffffffffull;   // 2^52
        return r ? r : (y > -1074. * TABLE ? 1 : 0);
    }
};
typedef WeighOf<false> Weigh;
constexpr int64_t LONG_ROW = (int64_t)1 << 18;

// A row's parameters, brought into range.
struct Row {
    int64_t k;                  // entries kept by rank, M: all
    double p;                   // share of the weight kept, >= 1: all
    double least;               // smallest weight kept
    double c;                   // 64 log2(e) / temperature
    float temp;
    __device__ __forceinline__ Row(const SampleArgs &a, int64_t b) {
        temp = a.temperature ? a.temperature[b] : a.temperature_all;
        k = a.top_k ? a.top_k[b] : a.top_k_all;
        const float tp = a.top_p ? a.top_p[b] : a.top_p_all, mp = a.min_p ? a.min_p[b] : a.min_p_all;
        if (k <= 0 || k > a.M) k = a.M;
        if (!(temp > 0.f)) {
            k = 1;
            temp = 1.f;
        }
        p = tp < 1.f ? (tp > 0.f ? (double)tp : 0.) : 1.;
        least = mp > 0.f ? fmin(1., (double)mp) : 0.;
        c = fmax(TABLE * 1.4426950408889634074 / (double)temp, 1e-290);     // (infinite temperature: all weights 1)
    }
    __device__ __forceinline__ bool keeps_all(int64_t M) const { return k >= M && p >= 1.; }
    __device__ __forceinline__ bool takes_first() const { return k == 1; }
};

// The sum that the drawn entry's has to exceed.
__device__ __forceinline__ double goal_of(float u, uint64_t total) {
    return u > 0.f ? (u < 1.f ? (double)u * (double)total : (double)total) : 0.;
}

__device__ __forceinline__ void put(const SampleArgs &a, int64_t b, int64_t j, uint64_t w, uint64_t total, int64_t kept) {
    a.idx[b] = (int32_t)j;
    if (a.prob) a.prob[b] = total ? (float)((double)w / (double)total) : 0.f;
    if (a.kept) a.kept[b] = (int32_t)kept;
}

template <typename T> struct Quad;
template <> struct Quad<float> {
    typedef f4v Raw;
    static __device__ __forceinline__ f4v scores(Raw r) { return r; }
};
template <> struct Quad<bf16_t> {
    typedef u2v Raw;
    static __device__ __forceinline__ f4v scores(Raw r) {
        return f4v{__uint_as_float(r[0] << 16), __uint_as_float(r[0] & 0xffff0000u), __uint_as_float(r[1] << 16),
                   __uint_as_float(r[1] & 0xffff0000u)};
    }
};

// Entries are dealt out by places: place 0 is the last one at or before a row's
// start that lies on a boundary of four entries, so that quads of places load
// as one piece whatever the row's alignment; index = place - skew.
template <typename T> __device__ __forceinline__ int skew_of(const T *row) {
    return (int)(reinterpret_cast<uintptr_t>(row) / sizeof(T) & 3);
}
// Keys of the four entries from index j on (0 outside the row).  The load and
// what is made of it are apart, so that a thread asks for several pieces before
// it waits for the first.
template <typename T> struct Piece {
    typename Quad<T>::Raw raw;
    bool whole;
    __device__ __forceinline__ void ask(const T *row, int32_t j, uint32_t M) {
        whole = (uint32_t)j < M && (uint32_t)(j + 3) < M;
        raw = {};
        if (whole) raw = *reinterpret_cast<const typename Quad<T>::Raw *>(row + j);
    }
    __device__ __forceinline__ void keys(uint32_t *key, const T *row, int32_t j, uint32_t M) const {
        const f4v x = Quad<T>::scores(raw);
#pragma unroll
        for (int c = 0; c < 4; ++c) key[c] = key_of(x[c]);
        if (whole) return;
#pragma unroll
        for (int c = 0; c < 4; ++c) key[c] = (uint32_t)(j + c) < M ? key_of(ld_f32<T>(row, j + c)) : 0;
    }
};

// ---------------------------------------------------------------- in a wave

// Sums and maxima over a wave by moves between lanes within the vector unit:
// within rows of 16 lanes by 1, 2, 4, 8, then from the rows before.  Lanes
// without a source contribute 0.
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS> __device__ __forceinline__ uint64_t moved(uint64_t v) {
    return (uint64_t)moved<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | moved<CTRL, ROWS>((uint32_t)v);
}
template <typename V, typename F> __device__ __forceinline__ V wave_scan(V v, F f) {
    v = f(v, moved<0x111, 0xf>(v));
    v = f(v, moved<0x112, 0xf>(v));
    v = f(v, moved<0x114, 0xf>(v));
    v = f(v, moved<0x118, 0xf>(v));
    v = f(v, moved<0x142, 0xa>(v));     // lane 15 of the row before, into rows 1 and 3
    return f(v, moved<0x143, 0xc>(v));  // lane 31, into rows 2 and 3
}
__device__ __forceinline__ uint64_t plus(uint64_t a, uint64_t b) { return a + b; }
// sum over this and the lanes before it
__device__ __forceinline__ uint64_t wave_upto(uint64_t v) { return wave_scan(v, plus); }
__device__ __forceinline__ uint64_t read_lane64(uint64_t v, int i) {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, i), hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), i);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t v) { return read_lane64(wave_upto(v), 63); }
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    return __builtin_amdgcn_readlane(wave_scan(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; }), 63);
}
// Hand-over through LDS between the lanes of one wave.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ int below(uint64_t ballot, int l) { return __popcll(ballot & (((uint64_t)1 << l) - 1)); }

// The smallest key in [lo, hi] with `has`, which holds for hi and, with a key,
// for all larger ones: 64 candidates a step.
template <typename F> __device__ __forceinline__ uint32_t least_key(uint32_t lo, uint32_t hi, int l, F has) {
    while (lo < hi) {
        const uint32_t step = (hi - lo + 63) / 64;
        const uint64_t at = (uint64_t)lo + (uint64_t)l * step;
        const uint64_t on = __ballot(at >= hi || has((uint32_t)at));
        const int first = on ? __ffsll((unsigned long long)on) - 1 : 64;    // (64 steps reach hi)
        const uint64_t next = (uint64_t)lo + (uint64_t)first * step;
        if (first) lo = lo + (uint32_t)((first - 1) * (uint64_t)step) + 1;
        else return lo;
        hi = next < hi ? (uint32_t)next : hi;
    }
    return hi;
}

// Draws from the n <= 64 E entries of a list in index order, E l + e in lane l
// (all others of the row rank behind them and are not kept).  top_k and top_p
// end the run of kept entries after the first `ties`, by index, of those equal
// to `cut`, found by halving the range of keys.
template <int E>
__device__ __forceinline__ void draw_lanes(const SampleArgs &a, int64_t b, const Row &r, const Weigh &wt, uint32_t top,
                                           const uint32_t (&key)[E], const int32_t (&j)[E], int n, uint32_t *lds, int l) {
    auto count_from = [&](uint32_t c) {
        int m = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) m += __popcll(__ballot(key[e] >= c));
        return m;
    };
    uint64_t mass[E];
#pragma unroll
    for (int e = 0; e < E; ++e) mass[e] = key[e] ? wt.mass(key[e]) : 0;
    uint32_t cut = 1;
    int ties = n;
    if (n > r.k) {
        uint32_t lo = 1, hi = top;
        int m = n;
        while (lo < hi && m != (int)r.k) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            const int x = count_from(mid);
            if (x >= (int)r.k) lo = mid, m = x;
            else hi = mid - 1;
        }
        cut = lo;
        if (m > r.k) ties = (int)r.k - (cut == top ? 0 : count_from(cut + 1));
    }
    bool keep[E];
    auto cut_ties = [&](uint32_t c, int most) {     // keep[] without the ties past `most`
        int at = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) at += below(__ballot(keep[e] && key[e] == c), l);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (keep[e] && key[e] == c) keep[e] = at++ < most;
    };
#pragma unroll
    for (int e = 0; e < E; ++e) keep[e] = key[e] >= cut;
    if (ties < n) cut_ties(cut, ties);
    if (r.p < 1.) {
        uint64_t sum = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) sum += keep[e] ? mass[e] : 0;
        const double goal = r.p * (double)wave_sum(sum);
        // the smallest key over which less than the goal lies: its entries, or some of them, end the run
        uint32_t lo = cut, hi = top;
        uint64_t above = 0;                         // mass over hi
        int in = 0, over = 0;                       // entries of [lo, hi], and over hi
#pragma unroll
        for (int e = 0; e < E; ++e) in += __popcll(__ballot(keep[e]));
        // (m, x: mass and number of the entries from mid on)
        auto halved = [&](uint32_t mid, uint64_t m, int x) {
            if (x > 0 && (double)m >= goal) {
                lo = mid;
                in = x - over;
            } else {
                hi = mid - 1;
                above = m;
                in -= x - over;
                over = x;
            }
        };
        while (lo < hi && in > (E > 2 ? 64 : 1)) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            uint64_t m = 0;
            int x = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool on = keep[e] && key[e] >= mid;
                m += on ? mass[e] : 0;
                x += __popcll(__ballot(on));
            }
            halved(mid, wave_sum(m), x);
        }
        if (E > 2 && lo < hi && in > 1) {
            // the entries still in question, one a lane
            int at = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) at += below(__ballot(keep[e] && key[e] >= lo && key[e] <= hi), l);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (keep[e] && key[e] >= lo && key[e] <= hi) lds[at++] = key[e];
            wave_sync();
            const uint32_t k = l < in ? lds[l] : 0;
            wave_sync();
            const uint64_t one = k ? wt.mass(k) : 0, before = above;
            const int ahead = over;
            while (lo < hi && in > 1) {
                const uint32_t mid = lo + (hi - lo) / 2 + 1;
                const bool on = k >= mid;
                halved(mid, before + wave_sum(on ? one : 0), ahead + __popcll(__ballot(on)));
            }
        }
        // [lo, hi] holds entries of one key at most: it is theirs
        uint32_t found = 0;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (keep[e] && key[e] >= lo && key[e] <= hi) found = key[e];
        found = wave_max(found);
        if (!found) found = lo;
        const uint64_t one = wt.mass(found);
        // as many of them as reach the goal, one at least
        double need = one ? ceil((goal - (double)above) / (double)one) : 1.;
        need = need < 1. ? 1. : need;
#pragma unroll
        for (int e = 0; e < E; ++e) keep[e] = keep[e] && key[e] >= found;
        if (need < (double)n) cut_ties(found, (int)need);
    }
    const uint32_t floor = r.least > 0. ? least_key(LOWEST, top, l, [&](uint32_t k) { return wt.weight(k) >= r.least; }) : 1;
    int kept = 0;
    uint64_t mine = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        keep[e] = keep[e] && key[e] >= floor;
        if (!keep[e]) mass[e] = 0;
        kept += __popcll(__ballot(keep[e]));
        mine += mass[e];
    }
    const uint64_t upto = wave_upto(mine), total = read_lane64(upto, 63);
    const double goal = goal_of(a.u[b], total);
    const uint64_t has = __ballot(mine != 0), past = __ballot(mine != 0 && (double)upto > goal);
    const int at = past ? __ffsll((unsigned long long)past) - 1 : 63 - __clzll(has);
    if (l != at) return;
    uint64_t sum = upto - mine, hw = 0;
    int hit = -1;
    bool done = false;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (!done && mass[e]) {
            sum += mass[e];
            hit = j[e], hw = mass[e];
            done = (double)sum > goal;
        }
    put(a, b, hit, hw, total, kept);
}

// A wave a row of up to 64 E places (E a multiple of 4, or 1).  The entries are
// loaded in pieces of four a lane and handed over to lie E side by side in a
// lane, so that lanes are in index order; what top_k leaves, if it fits, moves
// on to lists of one or two entries a lane.
template <typename T, int E>
__global__ void __launch_bounds__(256, 4) sample_wave_kernel(SampleArgs a) {
    constexpr int V = E < 4 ? 1 : 4, Q = E / V, STEP = E + 1;       // (an odd step: 64 lanes on different banks)
    __shared__ double table[TABLE];
    __shared__ uint32_t rows[4][E == 1 ? 1 : 64 * STEP];
    const int t = threadIdx.x, l = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6);
    fill_table(table, t);
    __syncthreads();
    const int64_t b = a.row0 + (int64_t)blockIdx.x * 4 + wv;
    if (b >= a.row1) return;
    uint32_t *const lds = rows[wv];
    const T *const row = static_cast<const T *>(a.S) + b * a.lds;
    const int skew = E == 1 ? 0 : skew_of(row);
    uint32_t key[E], top = 0;
    Piece<T> piece[V == 4 ? Q : 1];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int32_t j = (64 * q + l) * V - skew;
        if constexpr (V == 1) key[q] = (uint32_t)j < (uint32_t)a.M ? key_of(ld_f32<T>(row, j)) : 0;
        else piece[q].ask(row, j, (uint32_t)a.M);
    }
    if constexpr (V == 4) {
#pragma unroll
        for (int q = 0; q < Q; ++q) piece[q].keys(key + V * q, row, (64 * q + l) * V - skew, (uint32_t)a.M);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) top = max(top, key[e]);
    top = wave_max(top);
    if (!top) {
        if (l == 0) put(a, b, -1, 0, 0, 0);
        return;
    }
    if constexpr (E > 1) {
        // place p = E x + y of lane x lies at STEP x + y
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int c = 0; c < V; ++c) {
                const int p = (64 * q + l) * V + c;
                lds[p / E * STEP + p % E] = key[V * q + c];
            }
        wave_sync();
#pragma unroll
        for (int e = 0; e < E; ++e) key[e] = lds[STEP * l + e];
        wave_sync();
    }
    const Row r(a, b);
    const Weigh wt(top, r.c, a.shift, table);
    if constexpr (E > 2) {
        // top_k's halving on whole rows, from the 64th largest or lower on: the least of the lanes' largest
        uint32_t best = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) best = max(best, key[e]);
        auto count_from = [&](uint32_t c) {
            int m = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) m += __popcll(__ballot(key[e] >= c));
            return m;
        };
        uint32_t lo = 1, hi = top;
        int n = count_from(1);
        if (n > r.k) {
            if (r.k <= 64) {
                lo = max(1u, ~wave_max(~best));
                n = count_from(lo);
            }
            while (r.k <= 128 && lo < hi && n > 128) {
                const uint32_t mid = lo + (hi - lo) / 2 + 1;
                const int m = count_from(mid);
                if (m >= (int)r.k) lo = mid, n = m;
                else hi = mid - 1;
            }
        }
        if (n <= 128) {
            // entries from lo on, in index order: 16 bits of place are enough
            int at = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) at += below(__ballot(key[e] >= lo), l);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (key[e] >= lo) {
                    lds[at] = key[e];
                    lds[128 + at++] = E * l + e - skew;
                }
            wave_sync();
            if (n <= 64) {
                const uint32_t k[1] = {l < n ? lds[l] : 0};
                const int32_t j[1] = {l < n ? (int32_t)lds[128 + l] : 0};
                draw_lanes<1>(a, b, r, wt, top, k, j, n, lds, l);
            } else {
                uint32_t k[2];
                int32_t j[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const bool in = 2 * l + e < n;
                    k[e] = in ? lds[2 * l + e] : 0;
                    j[e] = in ? (int32_t)lds[128 + 2 * l + e] : 0;
                }
                draw_lanes<2>(a, b, r, wt, top, k, j, n, lds, l);
            }
            return;
        }
    }
    int32_t j[E];
#pragma unroll
    for (int e = 0; e < E; ++e) j[e] = E * l + e - skew;
    int n = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) n += __popcll(__ballot(key[e] != 0));
    draw_lanes<E>(a, b, r, wt, top, key, j, n, lds, l);
}

// ------------------------------------------------------------- a thread a row

// Up to P entries of a row in a thread's registers: 64 rows a wave where a wave
// a row would leave most lanes idle.
template <typename T, int P>
__global__ void __launch_bounds__(64) sample_thread_kernel(SampleArgs a) {
    __shared__ double table[TABLE];
    __shared__ uint64_t sorted[P][64];
    fill_table(table, threadIdx.x);
    __syncthreads();
    const int64_t b = a.row0 + (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (b >= a.row1) return;
    const T *const row = static_cast<const T *>(a.S) + b * a.lds;
    const int M = (int)a.M;
    uint32_t key[P], top = 0;
#pragma unroll
    for (int j = 0; j < P; ++j) {
        key[j] = j < M ? key_of(ld_f32<T>(row, j)) : 0;
        top = max(top, key[j]);
    }
    if (!top) {
        put(a, b, -1, 0, 0, 0);
        return;
    }
    const Row r(a, b);
    const Weigh wt(top, r.c, a.shift, table);
    uint64_t mass[P];
    uint32_t light = 0;                     // entries below min_p, told by their exponents
    // (a weight within 2^-54 of 1 is 1: 64 log2(e) 2^-54 below the exponent 0)
    const double limit = r.least > 0. ? log2(r.least) * TABLE - 5.2e-15 : -INFINITY;
#pragma unroll
    for (int j = 0; j < P; ++j) {
        mass[j] = key[j] ? wt.mass(key[j]) : 0;
        if (key[j] && wt.scaled(key[j]) < limit) light |= 1u << j;
    }
    uint32_t keep = ~0u;
    if (r.k < M || r.p < 1.) {
        // ranks by comparing every pair once; entries that cannot be drawn come last
        int rank[P];
#pragma unroll
        for (int j = 0; j < P; ++j) rank[j] = P - 1 - j;
#pragma unroll
        for (int j = 1; j < P; ++j)
#pragma unroll
            for (int i = 0; i < j; ++i) {
                const bool c = key[i] >= key[j];
                rank[j] += c;
                rank[i] -= c;
            }
        // masses in rank order, a column of LDS a thread
#pragma unroll
        for (int j = 0; j < P; ++j) sorted[rank[j]][threadIdx.x] = mass[j];
        const int most = r.k < P ? (int)r.k : P;
        int end = most;
        if (r.p < 1.) {
            uint64_t all = 0, m = 0;
#pragma unroll
            for (int i = 0; i < P; ++i)
                if (i < most) all += sorted[i][threadIdx.x];
            const double goal = r.p * (double)all;
            end = 1;
#pragma unroll
            for (int i = 0; i < P - 1; ++i) {
                m += sorted[i][threadIdx.x];
                if (i + 1 < most && (double)m < goal) end = i + 2;
            }
        }
        keep = 0;
#pragma unroll
        for (int j = 0; j < P; ++j)
            if (key[j] && rank[j] < end) keep |= 1u << j;
    } else {
#pragma unroll
        for (int j = 0; j < P; ++j)
            if (!key[j]) keep &= ~(1u << j);
        if (P < 32) keep &= (1u << (P & 31)) - 1;
    }
    keep &= ~light;
    uint64_t total = 0;
#pragma unroll
    for (int j = 0; j < P; ++j)
        if ((keep >> j) & 1) total += mass[j];
    const double goal = goal_of(a.u[b], total);
    uint64_t sum = 0, hw = 0;
    int hit = -1;
    bool past = false;
#pragma unroll
    for (int j = 0; j < P; ++j) {
        if (!((keep >> j) & 1) || !mass[j] || past) continue;
        sum += mass[j];
        hit = j, hw = mass[j];
        past = (double)sum > goal;
    }
    put(a, b, hit, hw, total, __popc(keep));
}

// --------------------------------------------------------- work-groups a row

// What the threads hold, 32 places each, is a chunk: PARTS parts of 256 places
// (four a lane of one wave), in index order.  PARTS_HERE: parts of a row whose
// masses fit a work-group's LDS.
constexpr int NT = 256, Q = 8, PARTS = NT / 64 * Q, CHUNK = 256 * PARTS, BINS = 2048, CAP = 1024, PARTS_HERE = 1024;
constexpr uint32_t LAST = 0x7fffffff;       // an index behind every entry

struct Block {
    uint64_t tmp[NT / 64];
    __device__ __forceinline__ uint64_t all() const {
        uint64_t v = 0;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) v += tmp[i];
        return v;
    }
    __device__ __forceinline__ uint64_t sum(uint64_t v) {
        v = wave_sum(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
        __syncthreads();
        return all();
    }
    __device__ __forceinline__ uint32_t most(uint32_t v) {
        v = wave_max(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
        __syncthreads();
        uint64_t m = tmp[0];
#pragma unroll
        for (int i = 1; i < NT / 64; ++i) m = max(m, tmp[i]);
        return (uint32_t)m;
    }
    // sum over the threads before this one; *sum_all: over all of them
    __device__ __forceinline__ uint64_t before(uint64_t v, uint64_t *sum_all) {
        const int w = threadIdx.x >> 6;
        const uint64_t x = wave_upto(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 63) tmp[w] = x;
        __syncthreads();
        uint64_t base = 0;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i)
            if (i < w) base += tmp[i];
        *sum_all = all();
        return base + x - v;
    }
};

// Bins of the scores below the largest: a rank-preserving map, so that a run of
// the first entries is some whole bins and a part of the next.  The bins cover
// the row's range, or the 32 temperatures below the largest score (weights
// above e^-32) if that is less, down to the smallest key that min_p keeps; the
// last one takes the rest.  (Where a run ends among entries that min_p takes
// away is of no account; only with both top_k and top_p is the one's end there
// needed for the other's.)
struct Binning {
    uint32_t floor;
    float m, scale;
    __device__ __forceinline__ Binning(uint32_t top, uint32_t low, const Row &r, int64_t M, uint32_t least)
        : floor(r.k < M && r.p < 1. ? 0 : least), m(value_of(top)) {
        const float range = fminf(m - value_of(max(low, floor)), 32.f * r.temp);
        scale = (float)BINS / range;
    }
    __device__ __forceinline__ int bin(uint32_t key) const {
        if (key < floor) return BINS - 1;
        const float x = value_of(key);
        if (x == m) return 0;
        const float at = (m - x) * scale;
        return at < (float)(BINS - 2) ? (int)at : BINS - 2;     // (NaN and infinities: the last but one)
    }
};

// Where the run of kept entries ends, as far as the histogram tells.  Keys from
// `sure` on are kept; those of [p_lo, p_hi] (the bins top_p may end in) and of
// [k_lo, k_hi] (the bin top_k ends in) have to be ranked.  An empty range asks
// for nothing.
struct Plan {
    uint32_t sure, p_lo, p_hi, k_lo, k_hi;
    uint32_t listed;            // entries to rank
    uint64_t mass_p, mass_k, all;       // mass over p_hi, over k_hi, of all entries
    uint64_t count_k;                   // entries over k_hi
    __device__ __forceinline__ bool in_p(uint32_t x) const { return x >= p_lo && x <= p_hi; }
    __device__ __forceinline__ bool in_k(uint32_t x) const { return x >= k_lo && x <= k_hi; }
    __device__ __forceinline__ bool asks(uint32_t x) const { return in_p(x) || in_k(x); }
};

// The end of the run: entries over `key`, and those equal to it up to index j.
struct End {
    uint32_t key, j;
    __device__ __forceinline__ bool has(uint32_t x, uint32_t i) const { return x > key || (x == key && x && i <= j); }
};
constexpr End NO_END = {1, LAST};

// Bin i lies in slot(i): a thread reads eight bins in a row, and 64 threads then
// read 64 slots in a row.
struct Hist {
    uint32_t count[BINS];
    uint64_t mass[BINS];
};
__device__ __forceinline__ int slot(int i) { return (i & 7) * (BINS / 8) + (i >> 3); }
static_assert(BINS == 8 * NT, "eight bins a thread");

// Workspace of a row that several work-groups share; chunks x ChunkSpace follow.
struct RowSpace {
    Hist hist;
    Plan plan;
    uint32_t listed, floor;     // entries listed; the smallest key that min_p keeps
    uint32_t top, low;          // the largest key and (long rows) the smallest
    uint64_t total;             // long rows: the sum of all masses at the shift that goes by the length
    uint32_t done, pad;         // drawn from already
    uint64_t list[CAP];
};
struct ChunkSpace {
    uint64_t mass[PARTS];       // of the entries that are surely kept, by parts
    uint32_t most[PARTS];       // each part's largest key
    uint32_t count, top, low, pad;
};

// Shared memory of a work-group.
struct Shared {
    Block block;
    double table[TABLE];
    alignas(16) Hist hist;
    uint64_t list[CAP];
    Plan plan;
    End end;
    uint32_t n, bins[4];
    uint64_t base, wave[2][NT / 64];
    uint64_t mass[PARTS_HERE];  // masses of a row's parts
};

template <typename T> struct Chunk {
    uint32_t key[Q][4];
    int32_t j0;                 // index of the first place
    __device__ __forceinline__ uint32_t at(int q, int c) const { return (uint32_t)(j0 + (int)(NT * q + threadIdx.x) * 4 + c); }
    __device__ __forceinline__ void load(const SampleArgs &a, int64_t b, int chunk) {
        const T *const row = static_cast<const T *>(a.S) + b * a.lds;
        j0 = (int32_t)((uint32_t)chunk * CHUNK - (uint32_t)skew_of(row));
        Piece<T> piece[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) piece[q].ask(row, (int32_t)at(q, 0), (uint32_t)a.M);
#pragma unroll
        for (int q = 0; q < Q; ++q) piece[q].keys(key[q], row, (int32_t)at(q, 0), (uint32_t)a.M);
    }
    template <typename F> __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (key[q][c]) f(key[q][c], q, c);
    }
    // the same without the parts whose largest key is below `from`
    __device__ __forceinline__ void load_from(const SampleArgs &a, int64_t b, int chunk, const ChunkSpace &cs, uint32_t from) {
        uint32_t largest[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) largest[q] = cs.most[q * (NT / 64) + (threadIdx.x >> 6)];
        load_from(a, b, chunk, largest, from);
    }
    __device__ __forceinline__ void load_from(const SampleArgs &a, int64_t b, int chunk, const uint32_t (&largest)[Q], uint32_t from) {
        const T *const row = static_cast<const T *>(a.S) + b * a.lds;
        j0 = (int32_t)((uint32_t)chunk * CHUNK - (uint32_t)skew_of(row));
        Piece<T> piece[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q)
            if (largest[q] >= from) piece[q].ask(row, (int32_t)at(q, 0), (uint32_t)a.M);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
#pragma unroll
            for (int c = 0; c < 4; ++c) key[q][c] = 0;
            if (largest[q] >= from) piece[q].keys(key[q], row, (int32_t)at(q, 0), (uint32_t)a.M);
        }
    }
    // largest key, and the complement of the smallest, of this thread's entries
    __device__ __forceinline__ void range(uint32_t &top, uint32_t &low) const {
        top = 0, low = 0;
        each([&](uint32_t x, int, int) { top = max(top, x), low = max(low, ~x); });
    }
};

__device__ __forceinline__ void clear(Hist &h) {
    for (int i = threadIdx.x; i < BINS; i += NT) h.count[i] = 0, h.mass[i] = 0;
}

// Lists the entries that the plan asks for, CAP of them at most, in any order.
template <typename T>
__device__ __forceinline__ void list_asked(const Chunk<T> &ch, const Plan &p, uint32_t *count, uint64_t *list) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        bool ask[4], any = false;
#pragma unroll
        for (int c = 0; c < 4; ++c) any |= ask[c] = p.asks(ch.key[q][c]);       // (no range has key 0)
        if (!any) continue;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (!ask[c]) continue;
            const uint32_t at = atomicAdd(count, 1u);
            if (at < CAP) list[at] = (uint64_t)ch.key[q][c] << 32 | ch.at(q, c);
        }
    }
}

// The smallest key that min_p keeps.
template <typename W> __device__ __forceinline__ uint32_t floor_of(const Row &r, const W &wt, uint32_t top) {
    if (!(r.least > 0.)) return 1;
    return least_key(LOWEST, top, threadIdx.x & 63, [&](uint32_t k) { return wt.weight(k) >= r.least; });
}

// Reads the plan off the histogram (which holds counts where top_k asks, masses
// where top_p does).
__device__ __forceinline__ void make_plan(Shared &sh, const Row &r, const Binning &bins, uint32_t top, uint32_t floor) {
    constexpr int PER = BINS / NT;
    const int t = threadIdx.x, w = t >> 6, l = t & 63, i0 = t * PER;
    Hist &h = sh.hist;
    uint64_t n = 0, m = 0, all_n, all_m;
    for (int i = i0; i < i0 + PER; ++i) n += h.count[slot(i)], m += h.mass[slot(i)];
    const uint64_t n0 = sh.block.before(n, &all_n), m0 = sh.block.before(m, &all_m);
    // bins 0: top_k's; 1, 2: the first and last that top_p may end in; BINS: none
    if (t < 4) sh.bins[t] = BINS;
    if (t == 0) sh.plan = Plan{1, 1, 0, 1, 0, 0, 0, 0, all_m, 0};
    __syncthreads();
    const bool by_k = (uint64_t)r.k < all_n, by_p = r.p < 1.;
    if (by_k) {
        uint64_t c = n0, x = m0;
        for (int i = i0; i < i0 + PER; ++i) {
            if (c < (uint64_t)r.k && c + h.count[slot(i)] >= (uint64_t)r.k) {
                sh.bins[0] = i;
                sh.plan.count_k = c;
                sh.plan.mass_k = x;
            }
            c += h.count[slot(i)], x += h.mass[slot(i)];
        }
    }
    __syncthreads();
    if (by_p) {
        // top_k leaves between mass_k and mass_k + the mass of its bin
        const double least = r.p * (double)(by_k ? sh.plan.mass_k : all_m);
        const double most = r.p * (double)(by_k ? sh.plan.mass_k + h.mass[slot(sh.bins[0])] : all_m);
        uint64_t x = m0;
        for (int i = i0; i < i0 + PER; ++i) {
            const uint64_t y = x + h.mass[slot(i)];
            if (y > x) {        // the first bin whose sum reaches (the largest score's, if that is no more than 0)
                if ((x == 0 || (double)x < least) && (double)y >= least) {
                    sh.bins[1] = i;
                    sh.plan.mass_p = x;
                }
                if ((x == 0 || (double)x < most) && (double)y >= most) sh.bins[2] = i;
            }
            x = y;
        }
    }
    __syncthreads();
    // the keys at the bins' edges, one a wave: the smallest key of a bin or of a smaller one
    const int k = (int)sh.bins[0], p1 = (int)sh.bins[1], p2 = (int)sh.bins[2];
    const int edge = w == 0 ? k : (w == 1 ? k - 1 : (w == 2 ? p2 : p1 - 1));
    const bool ask = w < 2 ? k < BINS : p1 < BINS;
    uint32_t key = 0;
    if (ask) key = edge < 0 ? top + 1 : least_key(LOWEST, top, l, [&](uint32_t x) { return bins.bin(x) <= edge; });
    if (l == 0 && ask) {
        if (w == 0) sh.plan.k_lo = key;
        if (w == 1) sh.plan.k_hi = key - 1;
        if (w == 2) sh.plan.p_lo = key;
        if (w == 3) sh.plan.p_hi = key - 1;
    }
    uint64_t listed = 0;
    if (by_k) {
        for (int i = i0; i < i0 + PER; ++i)
            if (i == k || (i >= p1 && i <= p2)) listed += h.count[slot(i)];
    }
    listed = sh.block.sum(listed);
    if (t == 0) {
        Plan &p = sh.plan;
        p.sure = p1 < BINS ? p.p_hi + 1 : (k < BINS ? p.k_hi + 1 : 1);
        p.listed = (uint32_t)(listed < CAP + 1 ? listed : CAP + 1);     // (without top_k: counted as they are listed)
        if (floor > p.p_hi && floor > p.k_hi) {       // min_p takes away all that is in question
            p.p_lo = p.k_lo = 1, p.p_hi = p.k_hi = 0;
            p.listed = 0;
        }
    }
    __syncthreads();
}

// Entries of a work-group, CAP / NT a thread in any order, key 0 for none.
struct Listed {
    static constexpr int PER = CAP / NT;
    uint32_t key[PER], j[PER];
    uint64_t mass[PER];
    uint32_t places;            // indices lie below this
    int turn = 0;               // (two sets of partial sums: one barrier a sum)
    // sums over the entries that `on` takes, of 1 or of their masses
    template <typename F> __device__ __forceinline__ uint64_t sum(Shared &sh, bool by_mass, F on) {
        uint64_t v = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (key[i] && on(i)) v += by_mass ? mass[i] : 1;
        v = wave_sum(v);
        uint64_t *const to = sh.wave[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) to[threadIdx.x >> 6] = v;
        __syncthreads();
        uint64_t all = 0;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) all += to[i];
        return all;
    }
    // The end of the run of entries in rank order that has n of them (by_mass:
    // that reaches the mass n), among the keys of [lo, most] and with the sum
    // `above` before them.  The run is known to end there.
    __device__ __forceinline__ End run(Shared &sh, uint32_t lo, uint32_t most, bool by_mass, double n, uint64_t above) {
        uint32_t hi = most;
        uint64_t over = above;          // the sum over hi
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            const uint64_t x = above + sum(sh, by_mass, [&](int i) { return key[i] >= mid && key[i] <= most; });
            if (!by_mass && (double)x == n) return End{mid, LAST};
            if (x > above && (double)x >= n) lo = mid;
            else hi = mid - 1, over = x;
        }
        // ends among the entries equal to lo: after as many of them as are needed
        const uint64_t same = sum(sh, false, [&](int i) { return key[i] == lo; });
        uint64_t one = 0;
        if (by_mass) {
            const uint64_t all = sum(sh, true, [&](int i) { return key[i] == lo; });
            one = same ? all / same : 0;
        }
        double need = by_mass ? (one ? ceil((n - (double)over) / (double)one) : 1.) : n - (double)over;
        if (need < 1.) need = 1.;
        if (need >= (double)same) return End{lo, LAST};
        uint32_t a = 0, b = places - 1;     // the smallest index with `need` of them up to it
        while (a < b) {
            const uint32_t mid = a + (b - a) / 2;
            if ((double)sum(sh, false, [&](int i) { return key[i] == lo && j[i] <= mid; }) >= need) b = mid;
            else a = mid + 1;
        }
        return End{lo, a};
    }
};

// The same for up to 64 entries, by every wave for itself: an entry a lane,
// compared with all of them.
template <typename W> __device__ __forceinline__ End end_of_short_list(const Shared &sh, const Row &r, const W &wt, int n) {
    const Plan &p = sh.plan;
    const int l = threadIdx.x & 63;
    const uint64_t v = l < n ? sh.list[l] : 0;
    const uint32_t key = (uint32_t)(v >> 32), j = (uint32_t)v;
    const bool in_k = key && p.in_k(key), in_p = key && p.in_p(key);
    const uint64_t mass = key && r.p < 1. ? wt.mass(key) : 0, mass_p = in_p ? mass : 0;
    const uint64_t ks = __ballot(in_k);
    uint64_t before_p = 0;
    int rank = 0, rank_k = 0;
    for (int i = 0; i < n; ++i) {
        const uint32_t k = __builtin_amdgcn_readlane(key, i), ji = __builtin_amdgcn_readlane(j, i);
        const uint64_t m = read_lane64(mass_p, i);
        const bool first = k > key || (k == key && ji < j);
        rank += first;
        rank_k += first && ((ks >> i) & 1);
        before_p += first ? m : 0;
    }
    bool keep = key && (!in_k || (uint64_t)rank_k + p.count_k < (uint64_t)r.k);
    if (r.p < 1.) {
        const uint64_t all = p.k_lo <= p.k_hi ? p.mass_k + wave_sum(keep && in_k ? mass : 0) : p.all;
        const uint64_t before = p.mass_p + before_p;
        keep = keep && in_p && (before == 0 || (double)before < r.p * (double)all);
    }
    // the last one kept (one is: the run ends among these)
    const uint32_t last = wave_max(keep ? rank + 1 : 0);
    const int at = __ffsll((unsigned long long)__ballot(keep && rank + 1 == (int)last)) - 1;
    return End{(uint32_t)__builtin_amdgcn_readlane(key, at < 0 ? 0 : at), (uint32_t)__builtin_amdgcn_readlane(j, at < 0 ? 0 : at)};
}

typedef uint64_t u8v __attribute__((ext_vector_type(2)));

// The same for up to 256 entries, one a thread, in the place of the histogram.
// (More are searched by halving the range of keys, a sum over the work-group a
// step: some 10 us, where 256 comparisons take 3.)
template <typename W> __device__ __forceinline__ End end_of_ranked_list(Shared &sh, const Row &r, const W &wt, int n) {
    const Plan &p = sh.plan;
    const int t = threadIdx.x;
    const uint64_t v = t < n ? sh.list[t] : 0, mine = v ^ 0xffffffffu;      // in rank order: larger keys, then smaller indices
    const uint32_t key = (uint32_t)(v >> 32);
    const bool in_k = key && p.in_k(key), in_p = key && p.in_p(key);
    const uint64_t mass = key && r.p < 1. ? wt.mass(key) : 0;
    // order and mass side by side; nothing behind the last entry
    u8v *const pairs = reinterpret_cast<u8v *>(sh.hist.mass);
    pairs[t] = t < n ? u8v{mine, in_p ? mass : 0} : u8v{0, 0};
    __syncthreads();
    const uint64_t k_lo = (uint64_t)p.k_lo << 32, k_hi = (uint64_t)p.k_hi << 32 | LAST | 0x80000000u;
    uint64_t before_p = 0;
    int rank = 0, rank_k = 0;
#pragma unroll 8
    for (int i = 0; i < (n + 7) / 8 * 8; ++i) {
        const u8v o = pairs[i];
        const bool first = o[0] > mine;
        rank += first;
        rank_k += first && o[0] >= k_lo && o[0] <= k_hi;
        before_p += first ? o[1] : 0;
    }
    bool keep = key && (!in_k || (uint64_t)rank_k + p.count_k < (uint64_t)r.k);
    if (r.p < 1.) {
        const uint64_t kept = sh.block.sum(keep && in_k ? mass : 0);
        const uint64_t all = p.k_lo <= p.k_hi ? p.mass_k + kept : p.all;
        const uint64_t before = p.mass_p + before_p;
        keep = keep && in_p && (before == 0 || (double)before < r.p * (double)all);
    }
    // the last one kept (one is: the run ends among these)
    const uint32_t last = sh.block.most(keep ? rank + 1 : 0);
    if (keep && rank + 1 == (int)last) sh.end = End{key, (uint32_t)v};
    __syncthreads();
    return sh.end;
}

// The end of the run from the listed entries (n <= CAP, in sh.list as key and
// index): top_k's, then top_p's within it.
template <typename W>
__device__ __forceinline__ End end_of_list(Shared &sh, const Row &r, const W &wt, int n, uint32_t places) {
    if (n <= 64) return end_of_short_list(sh, r, wt, n);
    if (n <= NT) return end_of_ranked_list(sh, r, wt, n);
    const Plan p = sh.plan;
    Listed e;
    e.places = places;
#pragma unroll
    for (int i = 0; i < Listed::PER; ++i) {
        const int x = i * NT + threadIdx.x;
        const uint64_t v = x < n ? sh.list[x] : 0;
        e.key[i] = (uint32_t)(v >> 32);
        e.j[i] = (uint32_t)v;
        e.mass[i] = e.key[i] && r.p < 1. ? wt.mass(e.key[i]) : 0;
    }
    End end = NO_END;
    uint64_t all = p.all;
    if (p.k_lo <= p.k_hi) {
        end = e.run(sh, p.k_lo, p.k_hi, false, (double)r.k, p.count_k);
        all = p.mass_k + e.sum(sh, true, [&](int i) { return p.in_k(e.key[i]) && end.has(e.key[i], e.j[i]); });
    }
    if (r.p < 1.) {
        // entries that top_k leaves out weigh nothing
#pragma unroll
        for (int i = 0; i < Listed::PER; ++i)
            if (!p.in_p(e.key[i]) || !end.has(e.key[i], e.j[i])) e.key[i] = 0;
        const uint32_t lo = p.k_lo <= p.k_hi && end.key > p.p_lo ? end.key : p.p_lo;
        const End ends = e.run(sh, lo, p.p_hi, true, r.p * (double)all, p.mass_p);
        if (ends.key > end.key || (ends.key == end.key && ends.j < end.j)) end = ends;
    }
    return end;
}

// The end of the run for rows whose bins hold too many entries: the range of
// keys in question is divided by 2048 until it is one key, by whole passes over
// the row, or over the parts of it that reach `least`, the entries below which
// are known to lie behind the end (cs: the row's chunks, null if it is one).
template <typename T, typename W>
__device__ __forceinline__ End end_by_passes(Shared &sh, const SampleArgs &a, int64_t b, const Row &r, const W &wt,
                                              uint32_t top, const ChunkSpace *cs, uint32_t least) {
    const int t = threadIdx.x;
    auto load = [&](Chunk<T> &ch, int c, uint32_t from) {
        if (cs) ch.load_from(a, b, c, cs[c], from);
        else ch.load(a, b, c);
    };
    auto pass = [&](auto f) {
        Chunk<T> ch;
#pragma unroll 1
        for (int c = 0; c < a.chunks; ++c) {
            load(ch, c, least);
            ch.each([&](uint32_t x, int, int) { f(x); });
        }
    };
    // the largest key from which on at least `goal` (entries, or mass) lies, not
    // below `from`; *above: what lies over it
    auto find = [&](uint32_t from, double goal, bool by_mass, uint64_t *above) {
        uint32_t lo = from, hi = top;
        *above = 0;
        while (lo < hi) {
            const uint64_t step = ((uint64_t)hi - lo + BINS) / BINS;
            clear(sh.hist);
            __syncthreads();
            pass([&](uint32_t x) {
                if (x >= lo && x <= hi)
                    atomicAdd((unsigned long long *)&sh.hist.mass[slot((int)((hi - x) / step))], by_mass ? (unsigned long long)wt.mass(x) : 1ull);
            });
            __syncthreads();
            // the bin in which the sum comes to the goal; the last one if it does not
            const int end = (int)((hi - lo) / step);
            auto there = [&](uint64_t m) { return m && (double)m >= goal; };
            uint64_t m = 0, all;
            for (int i = 8 * t; i < 8 * t + 8; ++i) m += sh.hist.mass[slot(i)];
            m = *above + sh.block.before(m, &all);
            for (int i = 8 * t; i < 8 * t + 8; ++i) {
                const uint64_t next = m + sh.hist.mass[slot(i)];
                if (!there(m) && (there(next) || (i == end && !there(*above + all)))) sh.n = i, sh.base = m;
                m = next;
            }
            __syncthreads();
            const uint32_t i = sh.n;
            *above = sh.base;
            const uint64_t down = (uint64_t)(i + 1) * step - 1;
            const uint32_t low = (uint64_t)hi - lo < down ? lo : (uint32_t)(hi - down);
            hi -= (uint32_t)(i * step);
            lo = low;
            __syncthreads();
        }
        return lo;
    };
    auto count_mass = [&](uint32_t from, uint64_t *m) {         // entries and mass of keys >= from
        uint64_t n = 0, w = 0;
        pass([&](uint32_t x) {
            if (x >= from) ++n, w += wt.mass(x);
        });
        *m = sh.block.sum(w);
        return sh.block.sum(n);
    };
    uint64_t all_mass, above = 0;
    uint32_t cut = 1;
    uint64_t ties = (uint64_t)a.M;
    if (count_mass(1, &all_mass) > (uint64_t)r.k) {
        cut = find(1, (double)r.k, false, &above);
        ties = (uint64_t)r.k - above;
        uint64_t m = 0;
        if (cut < top) count_mass(cut + 1, &m);
        all_mass = m + ties * wt.mass(cut);
    }
    if (r.p < 1.) {
        const double goal = r.p * (double)all_mass;
        const uint32_t at = find(cut, goal, true, &above);
        if (at > cut) cut = at, ties = (uint64_t)a.M;
        const uint64_t one = cut > 1 ? wt.mass(cut) : 0;
        double n = one ? ceil((goal - (double)above) / (double)one) : 1.;
        if (n < 1.) n = 1.;
        if (n < (double)ties) ties = (uint64_t)n;
    }
    // index of the last tie kept: the chunk that has it, then the place in it
    if (t == 0) sh.end = End{cut, LAST};
    uint64_t seen = 0;
    Chunk<T> ch;
#pragma unroll 1
    for (int c = 0; c < a.chunks && ties < (uint64_t)a.M; ++c) {
        load(ch, c, cut);
        uint64_t here = 0;
        ch.each([&](uint32_t x, int, int) { here += x == cut; });
        here = sh.block.sum(here);
        seen += here;
        if (seen < ties) continue;
        seen -= here;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            uint64_t mine = 0, all;
#pragma unroll
            for (int e = 0; e < 4; ++e) mine += ch.key[q][e] == cut;
            uint64_t at = seen + sh.block.before(mine, &all);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (ch.key[q][e] == cut && ++at == ties) sh.end.j = ch.at(q, e);
            seen += all;
        }
        break;
    }
    __syncthreads();
    return sh.end;
}

// Masses, by parts, and number of the entries of a chunk that `has` keeps.
// MOST of them: masses are formed for all, without branches, several side by
// side; otherwise for those kept, where a wave has any (the nucleus of 200 rows
// of 128001: 39 us for their list launch, 54 with all masses).
template <bool MOST, typename T, typename W, typename F>
__device__ __forceinline__ uint64_t chunk_parts(Block &block, const Chunk<T> &ch, const W &wt, F has, uint64_t *mass) {
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    uint64_t n = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        uint64_t m = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t x = ch.key[q][c];
            const bool on = x && has(x, ch.at(q, c));
            if constexpr (MOST) {
                const uint64_t one = wt.mass(x);
                m += on ? one : 0;
                n += on;
            } else if (on) {
                m += wt.mass(x);
                ++n;
            }
        }
        if (MOST || __ballot(m != 0)) m = wave_sum(m);
        if (l == 0) mass[q * (NT / 64) + w] = m;
    }
    return block.sum(n);
}

// Draws from a row of whose `parts` parts `mass_of` tells the masses.
template <typename T, typename W, typename F>
__device__ __forceinline__ void draw_parts(Shared &sh, const SampleArgs &a, int64_t b, const W &wt, End end,
                                           uint32_t floor, uint64_t kept, int parts, F mass_of) {
    const int t = threadIdx.x, l = t & 63;
    const float u = a.u[b];
    uint64_t total = 0;
    for (int i = t; i < parts; i += NT) total += mass_of(i);
    total = sh.block.sum(total);
    const double goal = goal_of(u, total);
    // the part in which the sum passes the goal, in index order: the last one
    // with a mass before which it has not (that is also right where it never does)
    if (t == 0) sh.n = 0;
    __syncthreads();
    uint64_t run = 0;
    for (int i0 = 0; i0 < parts; i0 += NT) {
        const int i = i0 + t;
        const uint64_t m = i < parts ? mass_of(i) : 0;
        uint64_t all;
        const uint64_t before = run + sh.block.before(m, &all);
        if (m && !((double)before > goal)) atomicMax(&sh.n, (uint32_t)i + 1);
        run += all;
    }
    __syncthreads();
    const int at = (int)sh.n - 1;
    // what lies before it, again in a fixed order
    uint64_t base = 0;
    for (int i = t; i < at; i += NT) base += mass_of(i);
    base = sh.block.sum(base);
    if (t >= 64) return;
    const T *const row = static_cast<const T *>(a.S) + b * a.lds;
    const int32_t j = (int32_t)((uint32_t)at * 256 + 4 * l - (uint32_t)skew_of(row));
    uint32_t key[4];
    uint64_t mass[4], mine = 0;
    Piece<T> piece;
    piece.ask(row, j, (uint32_t)a.M);
    piece.keys(key, row, j, (uint32_t)a.M);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const bool on = key[c] && key[c] >= floor && end.has(key[c], (uint32_t)(j + c));
        mass[c] = on ? wt.mass(key[c]) : 0;
        mine += mass[c];
    }
    const uint64_t upto = wave_upto(mine);
    const uint64_t has = __ballot(mine != 0), past = __ballot(mine != 0 && (double)(base + upto) > goal);
    const int lane = past ? __ffsll((unsigned long long)past) - 1 : 63 - __clzll(has);
    if (l != lane) return;
    uint64_t s = base + upto - mine, hw = 0;
    int32_t hit = -1;
    bool done = false;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        if (done || !mass[c]) continue;
        s += mass[c];
        hit = j + c, hw = mass[c];
        done = (double)s > goal;
    }
    put(a, b, hit, hw, total, kept);
}

// The first of the largest entries, which temperature 0 and top_k 1 take.
template <typename T>
__device__ __forceinline__ void draw_first(Shared &sh, const SampleArgs &a, int64_t b, const Chunk<T> &ch, uint32_t top) {
    uint32_t mine = 0;          // complement of the index: the largest is the first
    ch.each([&](uint32_t x, int q, int c) {
        if (x == top) mine = max(mine, ~ch.at(q, c));
    });
    mine = sh.block.most(mine);
    if (threadIdx.x == 0) put(a, b, (int32_t)~mine, 1, 1, 1);
}

template <typename T, typename W>
__device__ __forceinline__ void count_bins(Hist &h, const Chunk<T> &ch, const Row &r, const W &wt, const Binning &bins,
                                           bool by_k) {
    const bool by_p = r.p < 1.;
    uint32_t rest_n = 0;        // of the last bin, which many entries may share
    uint64_t rest = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        uint64_t mass[4];
        int at[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            at[c] = bins.bin(ch.key[q][c]);
            mass[c] = by_p ? wt.mass(ch.key[q][c]) : 0;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (!ch.key[q][c]) continue;
            if (at[c] == BINS - 1) {
                ++rest_n, rest += mass[c];
                continue;
            }
            if (by_k) atomicAdd(&h.count[slot(at[c])], 1u);
            if (by_p) atomicAdd((unsigned long long *)&h.mass[slot(at[c])], (unsigned long long)mass[c]);
        }
    }
    rest_n = (uint32_t)wave_sum(rest_n);
    rest = wave_sum(rest);
    if ((threadIdx.x & 63) == 0 && rest_n) {
        if (by_k) atomicAdd(&h.count[slot(BINS - 1)], rest_n);
        if (by_p) atomicAdd((unsigned long long *)&h.mass[slot(BINS - 1)], (unsigned long long)rest);
    }
}

// A work-group a row, up to a chunk of places.
template <typename T>
__global__ void __launch_bounds__(NT, 3) sample_group_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x;
    const int64_t b = a.row0 + blockIdx.x;
    fill_table(sh.table, t);
    clear(sh.hist);
    Chunk<T> ch;
    ch.load(a, b, 0);
    uint32_t top, low;
    ch.range(top, low);
    top = sh.block.most(top);
    low = ~sh.block.most(low);
    if (!top) {
        if (t == 0) put(a, b, -1, 0, 0, 0);
        return;
    }
    const Row r(a, b);
    if (r.takes_first()) {
        draw_first(sh, a, b, ch, top);
        return;
    }
    const Weigh wt(top, r.c, a.shift, sh.table);
    const uint32_t floor = floor_of(r, wt, top);
    End end = NO_END;
    if (!r.keeps_all(a.M)) {
        const Binning bins(top, low, r, a.M, floor);
        count_bins(sh.hist, ch, r, wt, bins, r.k < a.M);
        if (t == 0) sh.n = 0;
        __syncthreads();
        make_plan(sh, r, bins, top, floor);
        const Plan p = sh.plan;
        uint32_t listed = p.listed;
        if (listed <= CAP) {
            list_asked(ch, p, &sh.n, sh.list);
            __syncthreads();
            listed = sh.n;
            __syncthreads();
        }
        if (listed > CAP) end = end_by_passes<T>(sh, a, b, r, wt, top, nullptr, 1);
        else if (listed) end = end_of_list(sh, r, wt, (int)listed, (uint32_t)a.M);
    }
    const uint64_t kept =
        chunk_parts<true>(sh.block, ch, wt, [&](uint32_t x, uint32_t j) { return x >= floor && end.has(x, j); }, sh.mass);
    draw_parts<T>(sh, a, b, wt, end, floor, kept, PARTS, [&](int i) { return sh.mass[i]; });
}

__device__ __forceinline__ RowSpace *row_space(const SampleArgs &a, int64_t slot) {
    return reinterpret_cast<RowSpace *>(static_cast<char *>(a.ws) + slot * a.row_bytes);
}
__device__ __forceinline__ ChunkSpace *chunk_space(RowSpace *rs) { return reinterpret_cast<ChunkSpace *>(rs + 1); }

// Launch 1: each chunk's largest and smallest score; the row's space cleared.
template <typename T>
__global__ void __launch_bounds__(NT) sample_top_kernel(SampleArgs a) {
    __shared__ Block block;
    const int t = threadIdx.x, chunk = blockIdx.x % a.chunks;
    const int64_t slot = blockIdx.x / a.chunks, b = a.row0 + slot;
    RowSpace *const rs = row_space(a, slot);
    for (int i = chunk * NT + t; i < BINS; i += a.chunks * NT) rs->hist.count[i] = 0, rs->hist.mass[i] = 0;
    if (chunk == 0 && t == 0) rs->listed = 0, rs->done = 0, rs->total = 0;
    Chunk<T> ch;
    ch.load(a, b, chunk);
    ChunkSpace &cs = chunk_space(rs)[chunk];
    uint32_t top, low;
    ch.range(top, low);
#pragma unroll
    for (int q = 0; q < Q && a.most; ++q) {
        uint32_t x = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) x = max(x, ch.key[q][c]);
        x = wave_max(x);
        if ((t & 63) == 0) cs.most[q * (NT / 64) + (t >> 6)] = x;
    }
    top = block.most(top);
    low = ~block.most(low);
    if (t == 0) cs.top = top, cs.low = low;
}

// The row's largest and smallest key from the chunks' ones.
__device__ __forceinline__ void row_range(Block &block, const SampleArgs &a, const ChunkSpace *cs, uint32_t &top, uint32_t &low) {
    top = 0;
    low = 0;
    for (int i = threadIdx.x; i < a.chunks; i += NT) top = max(top, cs[i].top), low = max(low, ~cs[i].low);
    top = block.most(top);
    low = ~block.most(low);
}

// Long rows, after launch 1: their range, a work-group a row (that every chunk of
// the launches that follow reads the ranges of all of them costs more than the
// row's scores from some 2^26 entries on) ...
__global__ void __launch_bounds__(NT) sample_range_kernel(SampleArgs a) {
    __shared__ Block block;
    RowSpace *const rs = row_space(a, blockIdx.x);
    uint32_t top, low;
    row_range(block, a, chunk_space(rs), top, low);
    if (threadIdx.x == 0) rs->top = top, rs->low = low;
}
// ... and their total, at the shift that goes by the length.
template <typename T>
__global__ void __launch_bounds__(NT) sample_total_kernel(SampleArgs a) {
    __shared__ Block block;
    __shared__ double table[TABLE];
    const int t = threadIdx.x, chunk = blockIdx.x % a.chunks;
    const int64_t slot = blockIdx.x / a.chunks, b = a.row0 + slot;
    const Row r(a, b);
    if (r.takes_first()) return;
    RowSpace *const rs = row_space(a, slot);
    const uint32_t top = rs->top;
    if (!top) return;
    Chunk<T> ch;
    ch.load(a, b, chunk);
    fill_table(table, t);
    __syncthreads();
    const Weigh wt(top, r.c, a.shift, table);
    uint64_t m = 0;
    ch.each([&](uint32_t x, int, int) { m += wt.mass(x); });
    m = block.sum(m);
    if (t == 0) atomicAdd((unsigned long long *)&rs->total, (unsigned long long)m);
}
// With total < 2^e at the shift s a row's weight is below 3/2 2^(e - s) of its
// largest one (no mass is less than 2/3 of its weight), so that its masses at the
// shift s + 62 - e sum up to less than 3/2 2^62 + M; and as rounding up to one adds
// at most M 2^-s <= 1, that is to say the largest weight at most, to the total, a
// unit of that shift is below 2^-60 of the row's weight.
template <bool LONG> __device__ __forceinline__ int shift_of(const SampleArgs &a, const RowSpace *rs) {
    return LONG ? a.shift + __clzll((long long)rs->total) - 2 : a.shift;
}

// Rows of which top_k keeps a few, a work-group a row: a key that the largest
// ones of k parts reach has k entries from it on, so that only parts that reach
// it can hold kept entries, and few others do.  Those entries are listed, ranked
// and drawn from at once.  A row with more than CAP of them (few parts that hold
// all that counts, or many equal scores) is left to the other launches, or, ONLY
// where there are none, ranked by passes over it.
template <typename T, bool ONLY>
__global__ void __launch_bounds__(NT) sample_pick_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x, l = t & 63;
    const int64_t slot = blockIdx.x, b = a.row0 + slot;
    const Row r(a, b);
    const int parts = a.chunks * PARTS;
    if (!ONLY && (r.takes_first() || r.k > parts / 2)) return;
    RowSpace *const rs = row_space(a, slot);
    const ChunkSpace *const cs = chunk_space(rs);
    constexpr int PER = PARTS_HERE / NT;
    uint32_t *const ids = sh.hist.count;
    uint32_t most[PER], top = 0;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const int i = NT * x + t;
        most[x] = i < parts ? cs[i / PARTS].most[i % PARTS] : 0;
        top = max(top, most[x]);
    }
    fill_table(sh.table, t);
    if (t == 0) sh.bins[0] = sh.bins[1] = 0;
    top = sh.block.most(top);
    if (!top) {
        if (ONLY && t == 0) put(a, b, -1, 0, 0, 0);
        return;
    }
    // a key that k parts reach, within 2^-16 of the largest such (1 if there are
    // fewer parts with entries): by halving
    uint32_t from = 1;
    for (uint32_t hi = top, step = 0; step < 16 && from < hi; ++step) {
        const uint32_t mid = hi - (hi - from) / 2;
        uint32_t n = 0;
#pragma unroll
        for (int x = 0; x < PER; ++x) n += __popcll(__ballot(most[x] >= mid));
        uint64_t *const to = sh.wave[step & 1];
        if (l == 0) to[t >> 6] = n;
        __syncthreads();
        uint64_t all = 0;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) all += to[i];
        if (all >= (uint64_t)r.k) from = mid;
        else hi = mid - 1;
    }
#pragma unroll
    for (int x = 0; x < PER; ++x)
        if (most[x] >= from) ids[atomicAdd(&sh.bins[0], 1u)] = NT * x + t;
    __syncthreads();
    const int listed_parts = (int)sh.bins[0];
    const T *const row = static_cast<const T *>(a.S) + b * a.lds;
    const int skew = skew_of(row);
    constexpr int U = 8;
    for (int i0 = t >> 6; i0 < listed_parts; i0 += U * (NT / 64)) {
        Piece<T> piece[U];
        int32_t j[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {       // (behind the last: the last once more, not used)
            j[u] = (int32_t)(ids[min(i0 + u * (NT / 64), listed_parts - 1)] * 256 + 4 * l) - skew;
            piece[u].ask(row, j[u], (uint32_t)a.M);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * (NT / 64) >= listed_parts) continue;
            uint32_t key[4];
            piece[u].keys(key, row, j[u], (uint32_t)a.M);
            uint64_t on[4];
            uint32_t n = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) on[c] = __ballot(key[c] >= from), n += __popcll(on[c]);
            uint32_t at = l == 0 ? atomicAdd(&sh.bins[1], n) : 0;
            at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t to = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(on[c] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)on[c], 0));
                if (key[c] >= from && to < CAP) sh.list[to] = (uint64_t)key[c] << 32 | (uint32_t)(j[u] + c);
                at += __popcll(on[c]);
            }
        }
    }
    __syncthreads();
    const int n = (int)sh.bins[1];
    if (n > CAP && !ONLY) return;
    const Weigh wt(top, r.c, a.shift, sh.table);
    const uint32_t floor = max(floor_of(r, wt, top), from);
    if (n > CAP) {
        const End end = end_by_passes<T>(sh, a, b, r, wt, top, cs, from);
        uint64_t kept = 0;
        Chunk<T> ch;
#pragma unroll 1
        for (int i = 0; i < a.chunks; ++i) {
            ch.load_from(a, b, i, cs[i], floor);
            kept += chunk_parts<false>(sh.block, ch, wt, [&](uint32_t x, uint32_t j) { return x >= floor && end.has(x, j); },
                                       sh.mass + i * PARTS);
        }
        draw_parts<T>(sh, a, b, wt, end, floor, kept, parts, [&](int i) { return sh.mass[i]; });
        return;
    }
    const bool by_k = n > (int)r.k;
    uint64_t all = 0;
    if (!by_k && r.p < 1.) {
        for (int i = t; i < n; i += NT) all += wt.mass((uint32_t)(sh.list[i] >> 32));
        all = sh.block.sum(all);
    }
    // everything listed is in question
    if (t == 0) sh.plan = Plan{top + 1, from, top, by_k ? from : 1, by_k ? top : 0, (uint32_t)n, 0, 0, all, 0};
    for (int i = t; i < parts; i += NT) sh.mass[i] = 0;
    __syncthreads();
    End end = NO_END;
    if (by_k || r.p < 1.) end = end_of_list(sh, r, wt, n, (uint32_t)a.M);
    uint64_t kept = 0;
    for (int i = t; i < n; i += NT) {
        const uint32_t x = (uint32_t)(sh.list[i] >> 32), at = (uint32_t)sh.list[i];
        if (x < floor || !end.has(x, at)) continue;
        ++kept;
        atomicAdd((unsigned long long *)&sh.mass[(at + skew) / 256], (unsigned long long)wt.mass(x));
    }
    if (!ONLY && t == 0) rs->done = 1;
    kept = sh.block.sum(kept);
    draw_parts<T>(sh, a, b, wt, end, floor, kept, parts, [&](int i) { return sh.mass[i]; });
}

// Launch 2: the histogram of the row; for rows without top_k and top_p the
// chunk's mass.
template <typename T, bool LONG>
__global__ void __launch_bounds__(NT) sample_bins_kernel(SampleArgs a) {
    __shared__ Block block;
    __shared__ double table[TABLE];
    __shared__ Hist hist;
    const int t = threadIdx.x, chunk = blockIdx.x % a.chunks;
    const int64_t slot = blockIdx.x / a.chunks, b = a.row0 + slot;
    const Row r(a, b);
    if (r.takes_first()) return;
    RowSpace *const rs = row_space(a, slot);
    if (a.picked && rs->done) return;
    ChunkSpace *const cs = chunk_space(rs);
    Chunk<T> ch;
    ch.load(a, b, chunk);
    fill_table(table, t);
    clear(hist);
    uint32_t top, low;
    if constexpr (LONG) {
        top = rs->top, low = rs->low;
        __syncthreads();
    } else {
        row_range(block, a, cs, top, low);
    }
    if (!top) return;
    const WeighOf<LONG> wt(top, r.c, shift_of<LONG>(a, rs), table);
    const uint32_t floor = floor_of(r, wt, top);
    if (r.keeps_all(a.M)) {
        const uint64_t n = chunk_parts<true>(block, ch, wt, [&](uint32_t x, uint32_t) { return x >= floor; }, cs[chunk].mass);
        if (t == 0) cs[chunk].count = (uint32_t)n;
        return;
    }
    const bool by_k = r.k < a.M;
    count_bins(hist, ch, r, wt, Binning(top, low, r, a.M, floor), by_k);
    __syncthreads();
    for (int i = t; i < BINS; i += NT) {
        if (by_k && hist.count[i]) atomicAdd(&rs->hist.count[i], hist.count[i]);
        if (hist.mass[i]) atomicAdd((unsigned long long *)&rs->hist.mass[i], (unsigned long long)hist.mass[i]);
    }
}

// Launch 3, a work-group a row: the plan.
__global__ void __launch_bounds__(NT) sample_plan_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x;
    const int64_t slot = blockIdx.x, b = a.row0 + slot;
    const Row r(a, b);
    if (r.takes_first() || r.keeps_all(a.M)) return;
    RowSpace *const rs = row_space(a, slot);
    if (a.picked && rs->done) return;
    for (int i = t; i < BINS; i += NT) sh.hist.count[i] = rs->hist.count[i], sh.hist.mass[i] = rs->hist.mass[i];
    fill_table(sh.table, t);
    uint32_t top, low;
    row_range(sh.block, a, chunk_space(rs), top, low);
    if (!top) {
        if (t == 0) rs->top = 0;
        return;
    }
    const uint32_t floor = floor_of(r, Weigh(top, r.c, a.shift, sh.table), top);
    make_plan(sh, r, Binning(top, low, r, a.M, floor), top, floor);
    if (t == 0) rs->plan = sh.plan, rs->floor = floor, rs->top = top;
}

// Launch 4: the entries in question listed, the mass of those before them
// summed.
template <typename T, bool LONG>
__global__ void __launch_bounds__(NT) sample_list_kernel(SampleArgs a) {
    __shared__ Block block;
    __shared__ double table[TABLE];
    const int t = threadIdx.x, chunk = blockIdx.x % a.chunks;
    const int64_t slot = blockIdx.x / a.chunks, b = a.row0 + slot;
    const Row r(a, b);
    if (r.takes_first() || r.keeps_all(a.M)) return;
    RowSpace *const rs = row_space(a, slot);
    if (a.picked && rs->done) return;
    ChunkSpace &cs = chunk_space(rs)[chunk];
    // asked for at once
    uint32_t largest[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) largest[q] = cs.most[q * (NT / 64) + (t >> 6)];
    const uint32_t top = rs->top, floor = rs->floor;
    const Plan p = rs->plan;
    if (!top || p.listed > CAP) return;
    const uint32_t from = max(p.sure, floor);
    uint32_t least = from;
    if (p.p_lo <= p.p_hi) least = min(least, p.p_lo);
    if (p.k_lo <= p.k_hi) least = min(least, p.k_lo);
    Chunk<T> ch;
    ch.load_from(a, b, chunk, largest, least);
    fill_table(table, t);
    __syncthreads();
    const WeighOf<LONG> wt(top, r.c, shift_of<LONG>(a, rs), table);
    list_asked(ch, p, &rs->listed, rs->list);
    const uint64_t n = chunk_parts<false>(block, ch, wt, [&](uint32_t x, uint32_t) { return x >= from; }, cs.mass);
    if (t == 0) cs.count = (uint32_t)n;
}

// Launch 5, a work-group a row: the listed entries ranked, and the draw.
template <typename T, bool LONG>
__global__ void __launch_bounds__(NT) sample_draw_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x;
    const int64_t slot = blockIdx.x, b = a.row0 + slot;
    RowSpace *const rs = row_space(a, slot);
    if (a.picked && rs->done) return;
    ChunkSpace *const cs = chunk_space(rs);
    // asked for at once, whether the row needs it or not
    const Row r(a, b);
    const uint32_t planned = rs->plan.listed, sure = rs->plan.sure, in_question = rs->listed, least = rs->floor;
    const uint64_t entry = rs->list[t];
    const int parts = a.chunks * PARTS;
    const bool here = parts <= PARTS_HERE;
    if (here)
        for (int i = t; i < parts; i += NT) sh.mass[i] = cs[i / PARTS].mass[i % PARTS];
    fill_table(sh.table, t);
    uint32_t top, low;
    row_range(sh.block, a, cs, top, low);
    if (!top) {
        if (t == 0) put(a, b, -1, 0, 0, 0);
        return;
    }
    if (r.takes_first()) {
        uint32_t first = 0;     // complement of the first chunk that has it
        for (int i = t; i < a.chunks; i += NT)
            if (cs[i].top == top) first = max(first, ~(uint32_t)i);
        Chunk<T> ch;
        ch.load(a, b, (int)~sh.block.most(first));
        draw_first(sh, a, b, ch, top);
        return;
    }
    const WeighOf<LONG> wt(top, r.c, shift_of<LONG>(a, rs), sh.table);
    End end = NO_END;
    uint32_t floor;
    bool again = false;
    uint64_t more = 0;
    if (r.keeps_all(a.M)) {
        floor = floor_of(r, wt, top);
    } else {
        if (t == 0) sh.plan = rs->plan;
        const uint32_t listed = planned > CAP ? planned : in_question;
        floor = least;
        if (listed > CAP) {
            end = end_by_passes<T>(sh, a, b, r, wt, top, cs, 1);
            again = true;
        } else if (listed) {
            sh.list[t] = entry;
            for (int i = NT + t; i < (int)listed; i += NT) sh.list[i] = rs->list[i];
            __syncthreads();
            end = end_of_list(sh, r, wt, (int)listed, (uint32_t)a.M);
            again = !here;
            if (here) {
                // their masses to their parts' (exact sums: the order is of no account)
                const int skew = skew_of(static_cast<const T *>(a.S) + b * a.lds);
                for (int i = t; i < (int)listed; i += NT) {
                    const uint32_t x = (uint32_t)(sh.list[i] >> 32), j = (uint32_t)sh.list[i];
                    if (x >= sure || x < floor || !end.has(x, j)) continue;
                    ++more;
                    atomicAdd((unsigned long long *)&sh.mass[(j + skew) / 256], (unsigned long long)wt.mass(x));
                }
            }
        }
    }
    if (again) {
        // the whole row once more, now that the end of the run is known
        Chunk<T> ch;
        for (int i = 0; i < a.chunks; ++i) {
            ch.load_from(a, b, i, cs[i], floor);
            const uint64_t n = chunk_parts<false>(sh.block, ch, wt, [&](uint32_t x, uint32_t j) { return x >= floor && end.has(x, j); },
                                           here ? sh.mass + i * PARTS : cs[i].mass);
            if (t == 0) cs[i].count = (uint32_t)n;
        }
    }
    __syncthreads();
    for (int i = t; i < a.chunks; i += NT) more += cs[i].count;
    const uint64_t kept = sh.block.sum(more);
    if (here) draw_parts<T>(sh, a, b, wt, end, floor, kept, parts, [&](int i) { return sh.mass[i]; });
    else draw_parts<T>(sh, a, b, wt, end, floor, kept, parts, [&](int i) { return cs[i / PARTS].mass[i % PARTS]; });
}

// Rows a launch: the space of rows that several work-groups share is reused, and
// the threads of a launch are counted in 32 bits.
constexpr int64_t SHARED_ROWS = 2048, ROWS = (int64_t)1 << 22;

size_t row_bytes(int64_t chunks) { return sizeof(RowSpace) + (size_t)chunks * sizeof(ChunkSpace); }
int64_t chunks_of(int64_t M) { return (M + 3 + CHUNK - 1) / CHUNK; }     // (a row's places: its entries and up to 3 before)
int64_t shared_rows(int64_t M) { return std::min(SHARED_ROWS, ROWS / chunks_of(M)); }

template <typename T, int E> void launch_wave(const SampleArgs &a, int64_t rows, hipStream_t s) {
    sample_wave_kernel<T, E><<<dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s>>>(a);
}
template <typename T, int P> void launch_thread(const SampleArgs &a, int64_t rows, hipStream_t s) {
    sample_thread_kernel<T, P><<<dim3((unsigned)((rows + 63) / 64)), dim3(64), 0, s>>>(a);
}

// A thread a row or a wave a row, up to 32 entries (top_k 5 and top_p, fp32, in
// us, thread and wave):
//   5 entries   512 rows 5.6, 7.2;   65536 rows 7.8, 72
//   12 entries  2048 rows 8.9, 8.1;  4096 rows 8.9, 9.9;    65536 rows 9.5, 66
//   22 entries  8192 rows 13.4, 11.7;  16384 rows 13.5, 18.8;  65536 rows 14.3, 59
//   32 entries  8192 rows 18.3, 11.7;  16384 rows 18.5, 18.9;  65536 rows 21.6, 59
bool thread_a_row(int64_t M, int64_t B) { return M <= 8 || (M <= 32 && B >= (M <= 16 ? 4096 : (M <= 24 ? 12288 : 16384))); }

// Launches 2 to 5 (3 and 4 have nothing to do if `all` rows have no run to end).
template <typename T, bool LONG> void launch_shared(const SampleArgs &a, dim3 grid, dim3 one, bool all, hipStream_t s) {
    sample_bins_kernel<T, LONG><<<grid, dim3(NT), 0, s>>>(a);
    if (!all) {
        sample_plan_kernel<<<one, dim3(NT), 0, s>>>(a);
        sample_list_kernel<T, LONG><<<grid, dim3(NT), 0, s>>>(a);
    }
    sample_draw_kernel<T, LONG><<<one, dim3(NT), 0, s>>>(a);
}

// Rows row0 .. row1 - 1.  A wave a row while its lanes hold the row (2045
// entries, top_k 50 and top_p, one row: 12 us, a work-group 24; 2000 rows: 17,
// 83), a work-group while it does (8000 entries, one row: 26 us, shared by
// work-groups 39; 2000 rows: 93, 147).
template <typename T> void launch_rows(SampleArgs a, hipStream_t s) {
    const int64_t rows = a.row1 - a.row0, places = a.vec ? a.M : a.M + 3;
    if (thread_a_row(a.M, a.B)) {
        if (a.M <= 8) return launch_thread<T, 8>(a, rows, s);
        if (a.M <= 16) return launch_thread<T, 16>(a, rows, s);
        return a.M <= 24 ? launch_thread<T, 24>(a, rows, s) : launch_thread<T, 32>(a, rows, s);
    }
    if (a.M <= 64) return launch_wave<T, 1>(a, rows, s);
    if (places <= 256) return launch_wave<T, 4>(a, rows, s);
    if (places <= 512) return launch_wave<T, 8>(a, rows, s);
    if (places <= 1024) return launch_wave<T, 16>(a, rows, s);
    if (places <= 2048) return launch_wave<T, 32>(a, rows, s);
    if (a.M + 3 <= CHUNK) {
        sample_group_kernel<T><<<dim3((unsigned)rows), dim3(NT), 0, s>>>(a);
        return;
    }
    // no row with a run to end
    const bool all = !a.top_k && !a.top_p && (a.top_k_all <= 1 || a.top_k_all >= a.M) && !(a.top_p_all < 1.f);
    const dim3 grid((unsigned)(rows * a.chunks)), one((unsigned)rows);
    // one top_k for all rows, and a small one (temperature 0: one entry), in rows
    // whose parts' sums fit: see the head for both sides' times
    const int parts = a.chunks * PARTS;
    const bool fits = parts <= PARTS_HERE, first = !a.temperature && !(a.temperature_all > 0.f);
    const bool few = fits && (first || (!a.top_k && a.top_k_all >= 1 && a.top_k_all <= parts / 2));
    a.most = few || !all;
    sample_top_kernel<T><<<grid, dim3(NT), 0, s>>>(a);
    if (few) {
        sample_pick_kernel<T, true><<<one, dim3(NT), 0, s>>>(a);
        return;
    }
    a.picked = fits && a.top_k && parts >= 256;
    if (a.picked) sample_pick_kernel<T, false><<<one, dim3(NT), 0, s>>>(a);
    if (a.M > LONG_ROW) {
        sample_range_kernel<<<one, dim3(NT), 0, s>>>(a);
        sample_total_kernel<T><<<grid, dim3(NT), 0, s>>>(a);
        launch_shared<T, true>(a, grid, one, all, s);
    } else {
        launch_shared<T, false>(a, grid, one, all, s);
    }
}

template <typename T> hipError_t launch_typed(SampleArgs a, void *ws, hipStream_t s) {
    const bool shared = a.M + 3 > CHUNK;
    a.chunks = (int)chunks_of(a.M);
    a.row_bytes = row_bytes(a.chunks);
    a.ws = ws;
    const int64_t most = shared ? shared_rows(a.M) : ROWS;
    for (a.row0 = 0; a.row0 < a.B; a.row0 = a.row1) {
        a.row1 = a.row0 + most < a.B ? a.row0 + most : a.B;
        launch_rows<T>(a, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t sample_workspace(int64_t B, int64_t M) {
    if (M + 3 <= CHUNK) return 0;
    return (size_t)std::min(B, shared_rows(M)) * row_bytes(chunks_of(M));
}

hipError_t launch_sample(gs_dtype st, SampleArgs a, void *ws, hipStream_t s) {
    int bits = 0;
    while (((int64_t)1 << bits) < a.M) ++bits;
    a.shift = 62 - bits < 51 ? 62 - bits : 51;
    return st == GS_F32 ? launch_typed<float>(a, ws, s) : launch_typed<bf16_t>(a, ws, s);
}

}  // namespace gs
