// An entry drawn from a row of scores: temperature, top-k, top-p, min-p, and a
// given random number.
//
// Everything that decides is exact or in 64 bits.  Scores are ranked by an
// order-preserving integer key; weights are formed in fp64 and held as whole
// multiples of 2^-shift of the largest one, so their sums are integer sums: the
// same in any order, whatever the split of a row over threads, and atomic sums
// are as good as ordered ones.
//
// What is kept is a run of the entries in rank order (falling scores, equal
// ones by index), thinned by min_p from its end: top_k and top_p each end it
// after some entry.  No row is sorted.  Forms by the size of a row:
//   a thread a row      up to 32 entries, many rows: every pair compared
//   a wave a row        up to 2048 entries, in registers: the end of the run is
//                       found by halving the range of keys until at most 64
//                       entries are in question, and these are ranked
//   a work-group a row  up to 8192 entries, in registers: a histogram of the
//                       scores below the largest finds the bin the run ends in
//   work-groups a row   more entries: the same over chunks of 8192, in four
//                       launches (largest score, histogram, entries of the bin,
//                       ranking and draw): a launch boundary hands a row's data
//                       on faster than fences and counters did, which write the
//                       caches back from every work-group (402 and 511 us for
//                       the two launches they were in, against TIMES)
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
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// 2^(i / 64), i = 0..63, in LDS: the table that weights are formed from.
constexpr int TABLE = 64;
__device__ __forceinline__ void fill_table(double *table, int t) {
    if (t < TABLE) table[t] = exp2((double)t / TABLE);
}

// Weight of an entry, exp((x - max) / temperature): 2^y with y in 64ths taken
// from the table and the rest, |t| <= ln 2 / 128, by its series up to t^4 (the
// next term is below 4e-14 of the weight).
struct Weigh {
    double m, c;                // largest score; log2(e) / temperature
    int shift;                  // a mass of 2^shift is the largest weight
    const double *table;
    __device__ __forceinline__ double weight(uint32_t key) const {
        const double x = value_of(key);
        if (x == m) return 1.;
        const double y = fmax((x - m) * c, -1100.);     // (2^-1100 is zero)
        const double n = rint(y * TABLE);
        const double t = fma(n, -1. / TABLE, y) * 0.693147180559945309417;
        const int i = (int)n;
        const double s = fma(fma(fma(fma(t, 1. / 24, 1. / 6), t, 0.5), t, 1.), t, 1.);
        return ldexp(s * table[i & (TABLE - 1)], i >> 6);
    }
    __device__ __forceinline__ uint64_t mass_of(double w) const {
        return w > 0. ? (uint64_t)fmax(1., rint(ldexp(w, shift))) : 0;
    }
    __device__ __forceinline__ uint64_t mass(uint32_t key) const { return key ? mass_of(weight(key)) : 0; }
};

// A row's parameters, brought into range.
struct Row {
    int64_t k;                  // entries kept by rank, M: all
    double p;                   // share of the weight kept, >= 1: all
    double least;               // smallest weight kept
    double c;                   // log2(e) / temperature
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
        c = 1.4426950408889634074 / (double)temp;
    }
    __device__ __forceinline__ bool keeps_all(int64_t M) const { return k >= M && p >= 1.; }
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
template <> struct Quad<float> { static __device__ __forceinline__ f4v load(const float *p) { return *reinterpret_cast<const f4v *>(p); } };
template <> struct Quad<bf16_t> {
    static __device__ __forceinline__ f4v load(const bf16_t *p) {
        const u2v r = *reinterpret_cast<const u2v *>(p);
        return f4v{__uint_as_float(r[0] << 16), __uint_as_float(r[0] & 0xffff0000u), __uint_as_float(r[1] << 16),
                   __uint_as_float(r[1] & 0xffff0000u)};
    }
};

// Keys of V consecutive entries from j on (0 past the row's end).
template <typename T, int V>
__device__ __forceinline__ void load_keys(uint32_t *key, const T *row, int64_t j, int64_t M, bool vec) {
    if (V == 4 && vec && j + 4 <= M) {
        const f4v x = Quad<T>::load(row + j);
#pragma unroll
        for (int c = 0; c < V; ++c) key[c] = key_of(x[c]);
    } else {
#pragma unroll
        for (int c = 0; c < V; ++c) key[c] = j + c < M ? key_of(ld_f32<T>(row, j + c)) : 0;
    }
}

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

// Lists of up to 64 E entries in index order: lane l holds entries E l + e.
// Entries in rank order before each of this lane's: their number and mass.
template <int E>
__device__ __forceinline__ void rank_lanes(const uint32_t (&key)[E], const uint64_t (&mass)[E], int n, int l, int (&rank)[E],
                                           uint64_t (&before)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) rank[e] = 0, before[e] = 0;
    for (int i = 0; i < n; i += E) {
#pragma unroll
        for (int f = 0; f < E; ++f) {
            const uint32_t k = __builtin_amdgcn_readlane(key[f], i / E);
            const uint64_t m = read_lane64(mass[f], i / E);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (k > key[e] || (k == key[e] && i + f < E * l + e)) {
                    ++rank[e];
                    before[e] += m;
                }
        }
    }
}

// Draws from the n entries of a list (all others of the row rank behind them
// and are not kept).
template <int E>
__device__ __forceinline__ void draw_lanes(const SampleArgs &a, int64_t b, const Row &r, const Weigh &wt,
                                           const uint32_t (&key)[E], const int32_t (&j)[E], int n, int l) {
    double w[E];
    uint64_t mass[E];
    bool keep[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        w[e] = key[e] ? wt.weight(key[e]) : 0.;
        mass[e] = wt.mass_of(w[e]);
        keep[e] = key[e] != 0;
    }
    if (r.k < n || r.p < 1.) {
        int rank[E];
        uint64_t before[E], sum = 0;
        rank_lanes<E>(key, mass, n, l, rank, before);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            keep[e] = keep[e] && rank[e] < r.k;
            if (keep[e]) sum += mass[e];
        }
        if (r.p < 1.) {
            const double goal = r.p * (double)wave_sum(sum);
#pragma unroll
            for (int e = 0; e < E; ++e) keep[e] = keep[e] && (rank[e] == 0 || (double)before[e] < goal);
        }
    }
    int kept = 0;
    uint64_t mine = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        keep[e] = keep[e] && w[e] >= r.least;
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

// A wave a row.  Lane l holds the entries 64 V q + V l + c, q < Q, c < V.
template <typename T, int V, int Q>
__global__ void __launch_bounds__(256) sample_wave_kernel(SampleArgs a) {
    __shared__ double table[TABLE];
    __shared__ uint2 list_of[4][128];
    const int t = threadIdx.x, l = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6);
    fill_table(table, t);
    __syncthreads();
    const int64_t b = (int64_t)blockIdx.x * 4 + wv;
    if (b >= a.B) return;
    uint2 *const list = list_of[wv];
    const int64_t M = a.M;
    const T *const row = static_cast<const T *>(a.S) + b * a.lds;
    uint32_t key[Q][V];
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        load_keys<T, V>(key[q], row, (64 * q + l) * V, M, a.vec);
#pragma unroll
        for (int c = 0; c < V; ++c) top = max(top, key[q][c]);
    }
    top = wave_max(top);
    if (!top) {
        if (l == 0) put(a, b, -1, 0, 0, 0);
        return;
    }
    const Row r(a, b);
    const Weigh wt{(double)value_of(top), r.c, a.shift, table};
    if constexpr (V == 1 && Q == 1) {
        const int32_t j[1] = {l};
        draw_lanes<1>(a, b, r, wt, key[0], j, (int)M, l);
        return;
    }
    auto count_from = [&](uint32_t c0) {
        int n = 0;
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int c = 0; c < V; ++c) n += __popcll(__ballot(key[q][c] >= c0));
        return n;
    };
    // entries of [lo, hi] into the list, in index order; at most 128 of them
    auto gather = [&](uint32_t lo, uint32_t hi) {
        int n = 0;
        wave_sync();
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            int at = n;
#pragma unroll
            for (int c = 0; c < V; ++c) {
                const uint64_t on = __ballot(key[q][c] >= lo && key[q][c] <= hi);
                at += below(on, l);
                n += __popcll(on);
            }
#pragma unroll
            for (int c = 0; c < V; ++c)
                if (key[q][c] >= lo && key[q][c] <= hi) list[at++] = make_uint2(key[q][c], (64 * q + l) * V + c);
        }
        wave_sync();
        return n;
    };

    // top_k: the largest cut with at least k entries from it on (cut is a key
    // that entries have, or all the entries above cut - 1 are exactly k)
    uint32_t cut = 1;
    int n = count_from(1);
    if (n > r.k) {
        uint32_t lo = 1, hi = top;
        while (lo < hi && n != (int)r.k) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            const int m = count_from(mid);
            if (m >= (int)r.k) lo = mid, n = m;
            else hi = mid - 1;
        }
        cut = lo;
    }
    if (n <= 64) {
        gather(cut, top);
        const uint2 e = l < n ? list[l] : make_uint2(0, 0);
        const uint32_t k[1] = {e.x};
        const int32_t j[1] = {(int32_t)e.y};
        draw_lanes<1>(a, b, r, wt, k, j, n, l);
        return;
    }
    if (n <= 128) {
        gather(cut, top);
        uint32_t k[2];
        int32_t j[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint2 x = 2 * l + e < n ? list[2 * l + e] : make_uint2(0, 0);
            k[e] = x.x, j[e] = (int32_t)x.y;
        }
        draw_lanes<2>(a, b, r, wt, k, j, n, l);
        return;
    }
    // more than 128 entries: of those equal to cut the first `ties` by index
    int ties = n;
    uint64_t mass[Q][V];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int c = 0; c < V; ++c) {
            const double w = key[q][c] >= cut && key[q][c] ? wt.weight(key[q][c]) : 0.;
            mass[q][c] = wt.mass_of(w);
        }
    if (n > r.k) ties = (int)r.k - (cut == top ? 0 : count_from(cut + 1));
    if (r.p < 1.) {
        uint64_t all = 0;
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int c = 0; c < V; ++c)
                if (key[q][c] > cut) all += mass[q][c];
        const uint64_t one = wt.mass(cut), above_cut = wave_sum(all);
        const int equal = n - (cut == top ? 0 : count_from(cut + 1));
        if (ties > equal) ties = equal;     // (a cut of 1 that no entry has)
        const double goal = r.p * (double)(above_cut + (uint64_t)ties * one);
        // the run ends among the keys of [lo, hi]; `above`: the mass over hi
        uint32_t lo = cut, hi = top;
        uint64_t above = 0;
        int over = 0;                       // entries over hi
        int in = n;                         // entries of [lo, hi]
        while (lo < hi && in > 24) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            uint64_t s = 0;
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int c = 0; c < V; ++c)
                    if (key[q][c] >= mid) s += mass[q][c];
            s = wave_sum(s);
            const int m = count_from(mid);
            if ((double)s >= goal && m > 0) {
                lo = mid;
                in = m - over;
            } else {
                hi = mid - 1;
                above = s;
                in -= m - over;
                over = m;
            }
        }
        if (lo > cut) {
            cut = lo;
            ties = n;
        }
        if (in <= 64) {
            gather(lo, hi);
            const uint2 e = l < in ? list[l] : make_uint2(0, 0);
            int rank[1];
            uint64_t before[1];
            const uint32_t k[1] = {e.x};
            const uint64_t m[1] = {wt.mass(e.x)};
            rank_lanes<1>(k, m, in, l, rank, before);
            bool keep = e.x != 0 && ((rank[0] == 0 && over == 0) || (double)(above + before[0]) < goal);
            if (e.x == cut) {               // top_k's ties
                const uint64_t same = __ballot(keep && e.x == cut);
                keep = keep && below(same, l) < ties;
            }
            // the last one kept ends the run; if none is, all of it is over hi
            const uint64_t kb = __ballot(keep);
            if (!kb) {
                cut = hi == top ? top : hi + 1;
                ties = n;
            } else {
                cut = ~wave_max(keep ? ~e.x : 0);
                ties = __popcll(__ballot(keep && e.x == cut));
            }
        } else {                            // equal entries alone
            const uint64_t w1 = wt.mass(lo);
            double need = w1 ? ceil((goal - (double)above) / (double)w1) : 1.;
            if (over == 0 && need < 1.) need = 1.;
            if (need < 0.) need = 0.;
            if (need < (double)ties) ties = (int)need;
            cut = lo;
        }
    }
    // min_p: the smallest key that weighs enough (weights do not fall as keys rise)
    uint32_t floor = 1;
    if (r.least > 0.) {
        uint32_t light = 0;
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int c = 0; c < V; ++c)
                if (key[q][c] >= cut && key[q][c] > light && wt.weight(key[q][c]) < r.least) light = key[q][c];
        floor = wave_max(light) + 1;
    }
    // the kept entries, block by block of 64 V: masses, and where the sum passes
    uint64_t part[Q];
    int kept = 0, seen = 0;
    auto each = [&](int q, int &tie, auto use) {
        int at = tie;
#pragma unroll
        for (int c = 0; c < V; ++c) {
            const uint64_t on = __ballot(key[q][c] == cut);
            at += below(on, l);
            tie += __popcll(on);
        }
#pragma unroll
        for (int c = 0; c < V; ++c) {
            const uint32_t x = key[q][c];
            if (!x || x < cut) continue;
            if (x == cut && at++ >= ties) continue;
            if (x >= floor) use(c, mass[q][c]);
        }
    };
    uint64_t total = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        uint64_t s = 0;
        each(q, seen, [&](int, uint64_t w) { s += w, ++kept; });
        part[q] = wave_sum(s);
        total += part[q];
    }
    kept = (int)wave_sum(kept);
    const double goal = goal_of(a.u[b], total);
    uint64_t base = 0;
    seen = 0;
    bool done = false;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const bool last = base + part[q] == total && part[q];
        if (!done && part[q] && ((double)(base + part[q]) > goal || last)) {
            done = true;
            int tie = seen;
            uint64_t mine = 0;
            each(q, tie, [&](int, uint64_t w) { mine += w; });
            const uint64_t upto = wave_upto(mine);
            const uint64_t has = __ballot(mine != 0), past = __ballot(mine != 0 && (double)(base + upto) > goal);
            const int at = past ? __ffsll((unsigned long long)past) - 1 : 63 - __clzll(has);
            uint64_t sum = base + upto - mine, hw = 0;
            int hit = -1, end = -1;
            uint64_t ew = 0;
            tie = seen;
            each(q, tie, [&](int c, uint64_t w) {
                if (!w) return;
                sum += w;
                end = c, ew = w;
                if (hit < 0 && (double)sum > goal) hit = c, hw = w;
            });
            if (hit < 0) hit = end, hw = ew;
            if (l == at) put(a, b, (64 * q + l) * V + hit, hw, total, kept);
        }
        base += part[q];
#pragma unroll
        for (int c = 0; c < V; ++c) seen += __popcll(__ballot(key[q][c] == cut));
    }
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
    const int64_t b = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (b >= a.B) return;
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
    const Weigh wt{(double)value_of(top), r.c, a.shift, table};
    uint64_t mass[P];
    uint32_t light = 0;                     // entries below min_p
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const double w = key[j] ? wt.weight(key[j]) : 0.;
        mass[j] = wt.mass_of(w);
        if (w < r.least) light |= 1u << j;
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

// ---------------------------------------------------- work-groups of 256 a row

constexpr int NT = 256, Q = 8, CHUNK = NT * 4 * Q, BINS = 2048, CAP = 1024, MORE = 256;

struct Block {
    uint64_t tmp[NT / 64];
    __device__ __forceinline__ uint64_t sum(uint64_t v) {
        v = wave_sum(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
        __syncthreads();
        return tmp[0] + tmp[1] + tmp[2] + tmp[3];
    }
    __device__ __forceinline__ uint32_t most(uint32_t v) {
        v = wave_max(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
        __syncthreads();
        return (uint32_t)max(max(tmp[0], tmp[1]), max(tmp[2], tmp[3]));
    }
    // sum over the threads before this one; *all: over all of them
    __device__ __forceinline__ uint64_t before(uint64_t v, uint64_t *all) {
        const int w = threadIdx.x >> 6;
        const uint64_t x = wave_upto(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 63) tmp[w] = x;
        __syncthreads();
        uint64_t base = 0;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i)
            if (i < w) base += tmp[i];
        *all = tmp[0] + tmp[1] + tmp[2] + tmp[3];
        return base + x - v;
    }
};

// Bins of the scores below the largest: a rank-preserving map, so that a run of
// the first entries is some whole bins and a part of the next.  The bins cover
// the row's range, or the 32 temperatures below the largest score (weights
// above e^-32) if that is less; the last one takes the rest.
struct Binning {
    float m, scale;
    __device__ __forceinline__ Binning(float top, float low, float temp) : m(top) {
        const float range = fminf(top - low, 32.f * temp);
        scale = (float)BINS / range;
    }
    __device__ __forceinline__ int bin(uint32_t key) const {
        const float x = value_of(key);
        if (x == m) return 0;
        const float at = (m - x) * scale;
        return at < (float)(BINS - 1) ? (int)at : BINS - 1;     // (NaN and infinities: the last)
    }
};

// Where the run of kept entries ends, as far as the histogram tells: bins below
// `sure` are kept; the entries of the bins lo..hi (top_p), and of bin bk
// (top_k), have to be ranked.
struct Plan {
    int lo, hi, bk;             // bk = BINS: top_k keeps all; lo..hi empty: top_p does
    uint64_t mass_lo, mass_k, all;      // mass below bin lo / below bk; mass of all entries
    uint32_t count_lo, count_k;         // entries below bin lo / below bk
    uint32_t listed;            // entries to rank
    __device__ __forceinline__ int sure() const { return lo <= hi ? lo : bk; }
    __device__ __forceinline__ bool asks(int bin) const { return (bin >= lo && bin <= hi) || bin == bk; }
};

// The end of the run: entries over `key`, and those equal to it up to index j.
struct End {
    uint32_t key, j;
    __device__ __forceinline__ bool has(uint32_t x, uint32_t i) const { return x > key || (x == key && x && i <= j); }
};

struct Hist {
    uint32_t count[BINS];
    uint64_t mass[BINS];
};

// Workspace of a row that several work-groups share.
struct RowSpace {
    Hist hist;
    uint32_t listed, pad;
    uint64_t list[CAP];
    // then chunks x { mass u64, count u32, top u32, low u32, pad u32 }
};
struct ChunkSpace {
    uint64_t mass;
    uint32_t count, top, low, pad;
};

// Shared memory of a work-group.
struct Shared {
    Block block;
    double table[TABLE];
    Hist hist;
    uint64_t list[CAP];
    Plan plan;
    End end;
    uint32_t n, flag;
    uint64_t found, total, base;
    uint64_t part[NT / 64][Q];
    uint64_t more[MORE];        // masses of listed entries by chunk
};

template <typename T> struct Chunk {
    uint32_t key[Q][4];
    uint32_t j0;
    __device__ __forceinline__ uint32_t at(int q, int c) const { return j0 + (NT * q + threadIdx.x) * 4 + c; }
    __device__ __forceinline__ void load(const SampleArgs &a, int64_t b, int chunk) {
        j0 = (uint32_t)chunk * CHUNK;
        const T *const row = static_cast<const T *>(a.S) + b * a.lds;
#pragma unroll
        for (int q = 0; q < Q; ++q) load_keys<T, 4>(key[q], row, at(q, 0), a.M, a.vec);
    }
    template <typename F> __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (key[q][c]) f(key[q][c], q, c);
    }
};

__device__ __forceinline__ void clear(Hist &h) {
    for (int i = threadIdx.x; i < BINS; i += NT) h.count[i] = 0, h.mass[i] = 0;
}

// Reads the plan off the histogram (masses are there if top_p or min_p asks).
__device__ __forceinline__ void make_plan(Shared &sh, const Row &r, int64_t M) {
    constexpr int PER = BINS / NT;
    const int t = threadIdx.x, i0 = t * PER;
    Hist &h = sh.hist;
    uint64_t n = 0, w = 0, all_n, all_w;
    for (int i = i0; i < i0 + PER; ++i) n += h.count[i], w += h.mass[i];
    const uint64_t n0 = sh.block.before(n, &all_n), w0 = sh.block.before(w, &all_w);
    if (t == 0) {
        sh.plan = Plan{1, 0, BINS, 0, 0, all_w, 0, 0, 0};
    }
    __syncthreads();
    const bool by_k = (uint64_t)r.k < all_n, by_p = r.p < 1.;
    if (by_k) {
        uint64_t c = n0, m = w0;
        for (int i = i0; i < i0 + PER; ++i) {
            if (c < (uint64_t)r.k && c + h.count[i] >= (uint64_t)r.k) {
                sh.plan.bk = i;
                sh.plan.count_k = (uint32_t)c;
                sh.plan.mass_k = m;
            }
            c += h.count[i], m += h.mass[i];
        }
    }
    __syncthreads();
    if (by_p) {
        // top_k leaves between mass_k and mass_k + the mass of bin bk
        const double least = r.p * (double)(by_k ? sh.plan.mass_k : all_w);
        const double most = r.p * (double)(by_k ? sh.plan.mass_k + h.mass[sh.plan.bk] : all_w);
        uint64_t c = n0, m = w0;
        for (int i = i0; i < i0 + PER; ++i) {
            const uint64_t m1 = m + h.mass[i];
            if (h.count[i]) {
                // the first bin whose sum reaches: (an empty row has been dealt with)
                const bool start = c == 0;
                if ((start || (double)m < least) && (double)m1 >= least) {
                    sh.plan.lo = i;
                    sh.plan.count_lo = (uint32_t)c;
                    sh.plan.mass_lo = m;
                }
                if ((start || (double)m < most) && (double)m1 >= most) sh.plan.hi = i;
            }
            c += h.count[i], m = m1;
        }
    }
    __syncthreads();
    uint64_t ask = 0;
    for (int i = i0; i < i0 + PER; ++i)
        if (sh.plan.asks(i)) ask += h.count[i];
    ask = sh.block.sum(ask);
    if (t == 0) sh.plan.listed = (uint32_t)ask;
    __syncthreads();
}

// Ranks the listed entries (at most CAP, in sh.list as ~key, index) and finds
// the end of the run.
__device__ __forceinline__ void rank_list(Shared &sh, const Row &r, const Weigh &wt, const Binning &bins, int n) {
    const int t = threadIdx.x;
    int size = 64;
    while (size < n) size *= 2;
    for (int i = n + t; i < size; i += NT) sh.list[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int d = k / 2; d; d /= 2) {
            for (int i = t; i < size / 2; i += NT) {
                const int x = (i / d) * 2 * d + i % d, y = x + d;
                const uint64_t u = sh.list[x], v = sh.list[y];
                if ((u > v) == ((x & k) == 0)) sh.list[x] = v, sh.list[y] = u;
            }
            __syncthreads();
        }
    constexpr int PER = CAP / NT;
    const Plan &p = sh.plan;
    uint32_t key[PER];
    uint64_t mass[PER], of_k = 0, of_p = 0, all;
    int bin[PER], first_k = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int x = t * PER + i;
        key[i] = x < n ? ~(uint32_t)(sh.list[x] >> 32) : 0;
        bin[i] = key[i] ? bins.bin(key[i]) : -1;
        mass[i] = wt.mass(key[i]);
        if (key[i] && bin[i] >= p.lo && bin[i] <= p.hi) of_p += mass[i];
        if (key[i] && bin[i] < p.bk) ++first_k;
    }
    // listed entries below bin bk come first
    const int start_k = (int)sh.block.sum(first_k);
    uint32_t keep = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int x = t * PER + i;
        if (!key[i]) continue;
        if (bin[i] < p.bk || (uint64_t)(x - start_k) + p.count_k < (uint64_t)r.k) {
            keep |= 1u << i;
            if (bin[i] == p.bk) of_k += mass[i];
        }
    }
    if (r.p < 1.) {
        of_k = sh.block.sum(of_k);
        const double goal = r.p * (double)(p.bk < BINS ? p.mass_k + of_k : p.all);
        uint64_t m = p.mass_lo + sh.block.before(of_p, &all);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (!key[i]) continue;
            const bool in = bin[i] >= p.lo && bin[i] <= p.hi;
            const bool first = t == 0 && i == 0 && p.count_lo == 0;
            if (!in || !(first || (double)m < goal)) keep &= ~(1u << i);
            if (in) m += mass[i];
        }
    }
    // the last one kept (its rank + 1; none: everything below bin `sure`)
    uint32_t last = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if ((keep >> i) & 1) last = t * PER + i + 1;
    last = sh.block.most(last);
    if (t == 0) {
        if (last) {
            sh.end.key = ~(uint32_t)(sh.list[last - 1] >> 32);
            sh.end.j = (uint32_t)sh.list[last - 1];
        }
        sh.n = last;
    }
    __syncthreads();
}

// The end of the run for rows whose bins hold too many entries: the range of
// keys in question is divided by 2048 until it is one key, by whole passes over
// the row.
template <typename T>
__device__ __forceinline__ void end_by_passes(Shared &sh, const SampleArgs &a, int64_t b, const Row &r, const Weigh &wt,
                                              uint32_t top) {
    const int t = threadIdx.x;
    const T *const row = static_cast<const T *>(a.S) + b * a.lds;
    auto pass = [&](auto f) {
        for (int64_t j = t; j < a.M; j += NT) {
            const uint32_t x = key_of(ld_f32<T>(row, j));
            if (x) f(x, j);
        }
    };
    // the largest key from which on at least `goal` (entries, or mass) lies, not
    // below `floor`; *above: what lies over it
    auto find = [&](uint32_t floor, double goal, bool by_mass, uint64_t *above) {
        uint32_t lo = floor, hi = top;
        *above = 0;
        while (lo < hi) {
            const uint64_t step = ((uint64_t)hi - lo + BINS) / BINS;
            clear(sh.hist);
            __syncthreads();
            pass([&](uint32_t x, int64_t) {
                if (x >= lo && x <= hi)
                    atomicAdd((unsigned long long *)&sh.hist.mass[(hi - x) / step], by_mass ? (unsigned long long)wt.mass(x) : 1ull);
            });
            __syncthreads();
            if (t == 0) {
                uint64_t m = *above;
                int i = 0;
                const int last = (int)((hi - lo) / step);
                while (i < last && !((double)(m + sh.hist.mass[i]) >= goal && m + sh.hist.mass[i])) m += sh.hist.mass[i++];
                sh.n = i;
                sh.base = m;
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
        pass([&](uint32_t x, int64_t) {
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
        const uint64_t one = wt.mass(cut);
        double n = one ? ceil((goal - (double)above) / (double)one) : 1.;
        if (n < 1.) n = 1.;
        if (n < (double)ties) ties = (uint64_t)n;
    }
    // index of the last tie kept
    uint64_t seen = 0;
    if (t == 0) sh.end = End{cut, 0xffffffffu};
    __syncthreads();
    if (ties < (uint64_t)a.M) {
        for (int64_t j0 = 0; j0 < a.M && seen < ties; j0 += NT) {
            const int64_t j = j0 + t;
            const bool is = j < a.M && key_of(ld_f32<T>(row, j)) == cut;
            uint64_t all;
            const uint64_t before = seen + sh.block.before(is, &all);
            if (is && before + 1 == ties) sh.end.j = (uint32_t)j;
            seen += all;
        }
    }
    __syncthreads();
}

// Mass and number of a chunk's kept entries.
template <typename T, typename F>
__device__ __forceinline__ void chunk_sums(Shared &sh, const Chunk<T> &ch, const Row &r, const Weigh &wt, F has,
                                           uint64_t *mass, uint64_t *count) {
    uint64_t m = 0, n = 0;
    ch.each([&](uint32_t x, int q, int c) {
        if (!has(x, ch.at(q, c))) return;
        const double w = wt.weight(x);
        if (w >= r.least) m += wt.mass_of(w), ++n;
    });
    *mass = sh.block.sum(m);
    *count = sh.block.sum(n);
}

// Draws from a chunk: `base` is the mass of the chunks before it, and the sum
// passes the goal in it (or it is the last with a mass).
template <typename T>
__device__ __forceinline__ void draw_chunk(Shared &sh, const SampleArgs &a, int64_t b, const Chunk<T> &ch, const Row &r,
                                           const Weigh &wt, End end, uint64_t base, uint64_t total, uint64_t kept,
                                           double goal) {
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    auto mass_at = [&](int q, int c) -> uint64_t {
        const uint32_t x = ch.key[q][c];
        if (!x || !end.has(x, ch.at(q, c))) return 0;
        const double v = wt.weight(x);
        return v >= r.least ? wt.mass_of(v) : 0;
    };
    uint64_t mine[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        mine[q] = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) mine[q] += mass_at(q, c);
        const uint64_t s = wave_sum(mine[q]);
        if (l == 0) sh.part[w][q] = s;
    }
    if (t == 0) sh.found = ~0ull, sh.base = 0;
    __syncthreads();
    // the wave and block of 256 entries in which the sum passes, in index order
    uint64_t run = base;
    int at_q = -1, at_w = -1, end_q = -1, end_w = -1;
    uint64_t at_base = 0, end_base = 0;
    for (int q = 0; q < Q; ++q)
        for (int v = 0; v < NT / 64; ++v) {
            const uint64_t s = sh.part[v][q];
            if (!s) continue;
            end_q = q, end_w = v, end_base = run;
            if (at_q < 0 && (double)(run + s) > goal) at_q = q, at_w = v, at_base = run;
            run += s;
        }
    if (at_q < 0) at_q = end_q, at_w = end_w, at_base = end_base;
    if (w != at_w) return;
    uint64_t sum = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q)
        if (q == at_q) sum = mine[q];
    const uint64_t upto = wave_upto(sum);
    const uint64_t has = __ballot(sum != 0), past = __ballot(sum != 0 && (double)(at_base + upto) > goal);
    const int lane = past ? __ffsll((unsigned long long)past) - 1 : 63 - __clzll(has);
    if (l != lane) return;
    uint64_t s = at_base + upto - sum, hw = 0;
    int64_t hit = -1;
#pragma unroll
    for (int q = 0; q < Q; ++q)
        if (q == at_q) {
            bool done = false;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint64_t m = mass_at(q, c);
                if (done || !m) continue;
                s += m;
                hit = ch.at(q, c), hw = m;
                done = (double)s > goal;
            }
        }
    put(a, b, hit, hw, total, kept);
}

template <typename T>
__device__ __forceinline__ void count_bins(Shared &sh, const Chunk<T> &ch, const Row &r, const Weigh &wt, const Binning &bins) {
    const bool by_p = r.p < 1.;
    ch.each([&](uint32_t x, int, int) {
        const int i = bins.bin(x);
        atomicAdd(&sh.hist.count[i], 1u);
        if (by_p) atomicAdd((unsigned long long *)&sh.hist.mass[i], (unsigned long long)wt.mass(x));
    });
}

// A work-group a row, up to CHUNK entries.
template <typename T>
__global__ void __launch_bounds__(NT) sample_group_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x;
    const int64_t b = blockIdx.x;
    fill_table(sh.table, t);
    clear(sh.hist);
    Chunk<T> ch;
    ch.load(a, b, 0);
    uint32_t top = 0, low = 0;
    ch.each([&](uint32_t x, int, int) { top = max(top, x), low = max(low, ~x); });
    top = sh.block.most(top);
    low = ~sh.block.most(low);
    if (!top) {
        if (t == 0) put(a, b, -1, 0, 0, 0);
        return;
    }
    const Row r(a, b);
    const Weigh wt{(double)value_of(top), r.c, a.shift, sh.table};
    End end{1, 0xffffffffu};
    if (r.k < a.M || r.p < 1.) {
        const Binning bins(value_of(top), value_of(low), r.temp);
        count_bins(sh, ch, r, wt, bins);
        __syncthreads();
        make_plan(sh, r, a.M);
        const Plan p = sh.plan;
        if (p.listed > CAP) {
            end_by_passes<T>(sh, a, b, r, wt, top);
            end = sh.end;
        } else if (p.lo <= p.hi || p.bk < BINS) {
            if (t == 0) sh.n = 0;
            __syncthreads();
            ch.each([&](uint32_t x, int q, int c) {
                if (p.asks(bins.bin(x))) sh.list[atomicAdd(&sh.n, 1u)] = (uint64_t)~x << 32 | ch.at(q, c);
            });
            __syncthreads();
            rank_list(sh, r, wt, bins, (int)p.listed);
            end = sh.end;
            if (!sh.n) end = End{0xffffffffu, 0};       // (not reached: the run ends in a listed bin)
        }
    }
    uint64_t total, kept;
    chunk_sums(sh, ch, r, wt, [&](uint32_t x, uint32_t j) { return end.has(x, j); }, &total, &kept);
    draw_chunk(sh, a, b, ch, r, wt, end, 0, total, kept, goal_of(a.u[b], total));
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
    if (chunk == 0 && t == 0) rs->listed = 0;
    Chunk<T> ch;
    ch.load(a, b, chunk);
    uint32_t top = 0, low = 0;
    ch.each([&](uint32_t x, int, int) { top = max(top, x), low = max(low, ~x); });
    top = block.most(top);
    low = ~block.most(low);
    if (t == 0) chunk_space(rs)[chunk].top = top, chunk_space(rs)[chunk].low = low;
}

// The row's largest and smallest key from the chunks' ones.
__device__ __forceinline__ void row_range(Shared &sh, const SampleArgs &a, const ChunkSpace *cs, uint32_t &top, uint32_t &low) {
    top = 0;
    low = 0;
    for (int i = threadIdx.x; i < a.chunks; i += NT) top = max(top, cs[i].top), low = max(low, ~cs[i].low);
    top = sh.block.most(top);
    low = ~sh.block.most(low);
}

// Draws once the end of the run is known: every chunk's mass is in cs, but for
// the masses `more` of listed entries.
template <typename T>
__device__ __forceinline__ void draw_row(Shared &sh, const SampleArgs &a, int64_t b, const ChunkSpace *cs, const Row &r,
                                         const Weigh &wt, End end, uint64_t more_count) {
    const int t = threadIdx.x;
    auto mass_of = [&](int i) { return i < a.chunks ? cs[i].mass + (i < MORE ? sh.more[i] : 0) : 0; };
    uint64_t n = 0, m = 0;
    for (int i = t; i < a.chunks; i += NT) n += cs[i].count, m += mass_of(i);
    const uint64_t kept = sh.block.sum(n) + more_count, total = sh.block.sum(m);
    const double goal = goal_of(a.u[b], total);
    // the chunk in which the sum passes, in index order; the last with a mass where none does
    if (t == 0) sh.found = ~0ull, sh.n = 0;
    __syncthreads();
    uint64_t base = 0;
    for (int i0 = 0; i0 < a.chunks; i0 += NT) {
        const uint64_t c = mass_of(i0 + t);
        uint64_t all;
        const uint64_t before = base + sh.block.before(c, &all);
        if (c) {
            atomicMax(&sh.n, (uint32_t)(i0 + t));
            if ((double)(before + c) > goal) atomicMin((unsigned long long *)&sh.found, (unsigned long long)(i0 + t));
        }
        base += all;
    }
    __syncthreads();
    const int at = sh.found == ~0ull ? (int)sh.n : (int)sh.found;
    base = 0;
    for (int i = t; i < at; i += NT) base += mass_of(i);
    base = sh.block.sum(base);
    Chunk<T> ch;
    ch.load(a, b, at);
    draw_chunk(sh, a, b, ch, r, wt, end, base, total, kept, goal);
}

// Launch 2: the histogram of the row; for rows without top_k and top_p the
// chunk's mass.
template <typename T>
__global__ void __launch_bounds__(NT) sample_bins_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x, chunk = blockIdx.x % a.chunks;
    const int64_t slot = blockIdx.x / a.chunks, b = a.row0 + slot;
    RowSpace *const rs = row_space(a, slot);
    ChunkSpace *const cs = chunk_space(rs);
    fill_table(sh.table, t);
    clear(sh.hist);
    Chunk<T> ch;
    ch.load(a, b, chunk);
    uint32_t top, low;
    row_range(sh, a, cs, top, low);
    if (!top) return;
    const Row r(a, b);
    const Weigh wt{(double)value_of(top), r.c, a.shift, sh.table};
    if (r.keeps_all(a.M)) {
        uint64_t m, n;
        chunk_sums(sh, ch, r, wt, [](uint32_t, uint32_t) { return true; }, &m, &n);
        if (t == 0) cs[chunk].mass = m, cs[chunk].count = (uint32_t)n;
        return;
    }
    const Binning bins(value_of(top), value_of(low), r.temp);
    count_bins(sh, ch, r, wt, bins);
    __syncthreads();
    for (int i = t; i < BINS; i += NT) {
        if (!sh.hist.count[i]) continue;
        atomicAdd(&rs->hist.count[i], sh.hist.count[i]);
        if (sh.hist.mass[i]) atomicAdd((unsigned long long *)&rs->hist.mass[i], (unsigned long long)sh.hist.mass[i]);
    }
}

// What launches 3 and 4 begin with: the plan, read off the row's histogram by
// each work-group for itself.
__device__ __forceinline__ void row_plan(Shared &sh, const RowSpace *rs, const Row &r, int64_t M) {
    for (int i = threadIdx.x; i < BINS; i += NT) sh.hist.count[i] = rs->hist.count[i], sh.hist.mass[i] = rs->hist.mass[i];
    __syncthreads();
    make_plan(sh, r, M);
}

// Launch 3: entries of the bins in question listed, the mass of those before
// them summed.
template <typename T>
__global__ void __launch_bounds__(NT) sample_list_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x, chunk = blockIdx.x % a.chunks;
    const int64_t slot = blockIdx.x / a.chunks, b = a.row0 + slot;
    RowSpace *const rs = row_space(a, slot);
    ChunkSpace *const cs = chunk_space(rs);
    const Row r(a, b);
    if (r.keeps_all(a.M)) return;
    fill_table(sh.table, t);
    Chunk<T> ch;
    ch.load(a, b, chunk);
    uint32_t top, low;
    row_range(sh, a, cs, top, low);
    if (!top) return;
    row_plan(sh, rs, r, a.M);
    const Plan p = sh.plan;
    if (p.listed > CAP) return;
    const Weigh wt{(double)value_of(top), r.c, a.shift, sh.table};
    const Binning bins(value_of(top), value_of(low), r.temp);
    ch.each([&](uint32_t x, int q, int c) {
        if (p.asks(bins.bin(x))) rs->list[atomicAdd(&rs->listed, 1u)] = (uint64_t)~x << 32 | ch.at(q, c);
    });
    uint64_t m, n;
    const int sure = p.sure();
    chunk_sums(sh, ch, r, wt, [&](uint32_t x, uint32_t) { return bins.bin(x) < sure; }, &m, &n);
    if (t == 0) cs[chunk].mass = m, cs[chunk].count = (uint32_t)n;
}

// Launch 4, a work-group a row: the listed entries ranked, and the draw.
template <typename T>
__global__ void __launch_bounds__(NT) sample_draw_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x;
    const int64_t slot = blockIdx.x, b = a.row0 + slot;
    RowSpace *const rs = row_space(a, slot);
    ChunkSpace *const cs = chunk_space(rs);
    fill_table(sh.table, t);
    for (int i = t; i < MORE; i += NT) sh.more[i] = 0;
    uint32_t top, low;
    row_range(sh, a, cs, top, low);
    if (!top) {
        if (t == 0) put(a, b, -1, 0, 0, 0);
        return;
    }
    const Row r(a, b);
    const Weigh wt{(double)value_of(top), r.c, a.shift, sh.table};
    End end{1, 0xffffffffu};
    if (r.keeps_all(a.M)) {
        draw_row<T>(sh, a, b, cs, r, wt, end, 0);
        return;
    }
    row_plan(sh, rs, r, a.M);
    const Plan p = sh.plan;
    uint64_t count = 0;
    // (chunks past MORE: listed entries' masses would have no place)
    if (p.listed > CAP || (p.listed && a.chunks > MORE)) {
        if (p.listed > CAP) {
            end_by_passes<T>(sh, a, b, r, wt, top);
        } else {
            for (int i = t; i < (int)p.listed; i += NT) sh.list[i] = rs->list[i];
            __syncthreads();
            rank_list(sh, r, wt, Binning(value_of(top), value_of(low), r.temp), (int)p.listed);
        }
        end = sh.end;
        Chunk<T> ch;
        for (int i = 0; i < a.chunks; ++i) {
            ch.load(a, b, i);
            uint64_t m, n;
            chunk_sums(sh, ch, r, wt, [&](uint32_t x, uint32_t j) { return end.has(x, j); }, &m, &n);
            if (t == 0) cs[i].mass = m, cs[i].count = (uint32_t)n;
        }
        __threadfence_block();
        __syncthreads();
    } else if (p.listed) {
        const Binning bins(value_of(top), value_of(low), r.temp);
        for (int i = t; i < (int)p.listed; i += NT) sh.list[i] = rs->list[i];
        __syncthreads();
        rank_list(sh, r, wt, bins, (int)p.listed);
        end = sh.end;
        const int sure = p.sure();
        for (int i = t; i < (int)sh.n; i += NT) {
            const uint32_t x = ~(uint32_t)(sh.list[i] >> 32), j = (uint32_t)sh.list[i];
            if (bins.bin(x) < sure) continue;
            const double w = wt.weight(x);
            if (w < r.least) continue;
            ++count;
            atomicAdd((unsigned long long *)&sh.more[j / CHUNK], (unsigned long long)wt.mass_of(w));
        }
        count = sh.block.sum(count);
    }
    draw_row<T>(sh, a, b, cs, r, wt, end, count);
}

constexpr int64_t SLAB = 2048;      // rows of a large table in flight: their space is reused

size_t row_bytes(int64_t chunks) { return sizeof(RowSpace) + (size_t)chunks * sizeof(ChunkSpace); }
int64_t chunks_of(int64_t M) { return (M + CHUNK - 1) / CHUNK; }

template <typename T, int V, int Q> hipError_t launch_wave(const SampleArgs &a, hipStream_t s) {
    sample_wave_kernel<T, V, Q><<<dim3((unsigned)((a.B + 3) / 4)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, int P> hipError_t launch_thread(const SampleArgs &a, hipStream_t s) {
    sample_thread_kernel<T, P><<<dim3((unsigned)((a.B + 63) / 64)), dim3(64), 0, s>>>(a);
    return hipGetLastError();
}

template <typename T> hipError_t launch_typed(SampleArgs a, void *ws, hipStream_t s) {
    if (a.M <= 32 && a.B >= 4096) {
        if (a.M <= 8) return launch_thread<T, 8>(a, s);
        if (a.M <= 16) return launch_thread<T, 16>(a, s);
        return a.M <= 24 ? launch_thread<T, 24>(a, s) : launch_thread<T, 32>(a, s);
    }
    if (a.M <= 64) return launch_wave<T, 1, 1>(a, s);
    if (a.M <= 256) return launch_wave<T, 4, 1>(a, s);
    if (a.M <= 512) return launch_wave<T, 4, 2>(a, s);
    if (a.M <= 1024) return launch_wave<T, 4, 4>(a, s);
    if (a.M <= 2048) return launch_wave<T, 4, 8>(a, s);
    if (a.M <= CHUNK) {
        sample_group_kernel<T><<<dim3((unsigned)a.B), dim3(NT), 0, s>>>(a);
        return hipGetLastError();
    }
    a.chunks = (int)chunks_of(a.M);
    a.row_bytes = row_bytes(a.chunks);
    a.ws = ws;
    // one value for all rows that keeps everything: no row comes to the third launch
    const bool all = !a.top_k && !a.top_p && !a.temperature && a.temperature_all > 0.f &&
                     (a.top_k_all <= 0 || a.top_k_all >= a.M) && !(a.top_p_all < 1.f);
    for (a.row0 = 0; a.row0 < a.B; a.row0 += SLAB) {
        const int64_t rows = a.B - a.row0 < SLAB ? a.B - a.row0 : SLAB;
        const dim3 grid((unsigned)(rows * a.chunks));
        sample_top_kernel<T><<<grid, dim3(NT), 0, s>>>(a);
        sample_bins_kernel<T><<<grid, dim3(NT), 0, s>>>(a);
        if (!all) sample_list_kernel<T><<<grid, dim3(NT), 0, s>>>(a);
        sample_draw_kernel<T><<<dim3((unsigned)rows), dim3(NT), 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t sample_workspace(int64_t B, int64_t M) {
    if (M <= CHUNK) return 0;
    return (size_t)(B < SLAB ? B : SLAB) * row_bytes(chunks_of(M));
}

hipError_t launch_sample(gs_dtype st, SampleArgs a, void *ws, hipStream_t s) {
    int bits = 0;
    while (((int64_t)1 << bits) < a.M) ++bits;
    a.shift = 62 - bits < 52 ? 62 - bits : 52;
    return st == GS_F32 ? launch_typed<float>(a, ws, s) : launch_typed<bf16_t>(a, ws, s);
}

}  // namespace gs
