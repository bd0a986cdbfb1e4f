// Attention of a step's rows to their requests' states in a paged cache.
//
// The pass over the states is that of gs_xattn.hip: blocks of 32 rows a wave (the
// rows of the heads that share a key and value head side by side), tiles of keys
// and values through LDS, scores with the keys as rows, a running maximum and
// sum.  What differs is where a tile's rows lie (each state's page is looked up,
// a tile or two before its values are asked for) and what a row sees (states up
// to its own position, from its window's start on, and the first few).
//
// How the work is shared out follows the lengths in device memory.  Requests of
// few rows (up to 32 a key and value head: tokens, drafts): all tiles of all
// requests and heads lie in one line, of which every wave takes an equal part
// (few_kernel); a request cut by part ends is put together by few_join_kernel or,
// of many parts, few_join_many_kernel.
// More rows (prompts): a launch lists the blocks of 128 rows, longest first, cut
// where they are longer than a work-group's share (plan_kernel), and what was cut
// is put together by many_join_kernel.
//
// Few rows are bound by HBM: 48 requests of up to 7000 states, 32 heads over 8 of
// 128 values, bf16, 643 MB in 118 us, 5.5 TB/s (reads alone in such pages reach 6.2),
// and 5 us to join; one of 200001 states, 4 heads of keys, 410 MB in 79 + 7 us.  Equal
// parts of one line (rather than parts of each request) and all heads of a part side
// by side: 199 -> 161 us; neighbours on one XCD: 154.  Many rows are bound by the
// matrix cores, the exponentials and LDS in turn, as gs_xattn.hip's: 5 pieces of up to
// 1500 rows on up to 6000 states, 435 us, 840 TF/s.
//
// The form goes by the most rows of a request that the host names: one piece of a
// prompt in a step puts its tokens into blocks of 128 rows too.  (40 tokens over up to
// 7000 states and two pieces of 500 rows: 157 us in one call, 107 + 76 in two.)
#include <algorithm>

#include "gs_attn.h"
#include "gs_scan.h"

namespace gs {
namespace {
using namespace attn;

// ------------------------------------------------------------ what is seen

// Rows of request b: qoff clamped to the tensors' rows; `n` of them count for
// positions, the first `count` are computed.  A request that got no positions for
// its rows has them see nothing: they stand before state 0 of none.
struct Rows {
    int first, n, count, kl;
    __device__ __forceinline__ Rows(const PagedAttnArgs &a, int b) {
        const int got = a.added ? a.added[b] : 1;
        kl = clamped(a.klen, b, a.Lk);
        if (got <= 0) kl = 0;
        if (!a.qoff) {
            first = b;
            n = 1;
        } else {
            first = clamped(a.qoff, b, a.N);
            n = clamped(a.qoff, b + 1, a.N) - first;
        }
        if (n < 0) n = 0;
        count = n < a.Lq ? n : a.Lq;
    }
};

// States that rows i0 .. i1 of a request see: [0, sink) and [lo, hi), and the
// tiles of BN that hold them.
template <int BN> struct View {
    int hi, lo, sink, sink_tiles, first_tile, tiles;
    __device__ __forceinline__ View(const PagedAttnArgs &a, const Rows &r, int i0, int i1) {
        const int pmin = r.kl - r.n + i0, pmax = r.kl - r.n + i1;
        hi = pmax < 0 ? 0 : pmax + 1;
        lo = a.window && pmin >= a.window ? pmin - a.window + 1 : 0;
        sink = a.sinks < lo ? a.sinks : lo;
        sink_tiles = (sink + BN - 1) / BN;
        first_tile = lo / BN;
        if (first_tile < sink_tiles) first_tile = sink_tiles;
        const int end = (hi + BN - 1) / BN;
        tiles = sink_tiles + (end > first_tile ? end - first_tile : 0);
    }
    __device__ __forceinline__ int start(int x) const { return (x < sink_tiles ? x : first_tile + (x - sink_tiles)) * BN; }
    __device__ __forceinline__ bool holds(int j) const { return j < hi && (j < sink || j >= lo); }
};

// All keys of a tile at j0 are there (`on`), and seen by rows at positions from p to q.
template <int BN> __device__ __forceinline__ bool seen_by(const PagedAttnArgs &a, uint64_t on, int j0, int p, int q) {
    return on == ALL_LIVE<BN> && p >= j0 + BN - 1 && (!a.window || (int64_t)q - a.window < j0 || j0 + BN <= a.sinks);
}

// Bits 0 .. n - 1.
__device__ __forceinline__ uint64_t low_bits(int n) { return n <= 0 ? 0 : (n >= 64 ? ~0ull : (1ull << n) - 1); }

// Bit n: the row at position p sees key j0 + n.
__device__ __forceinline__ uint64_t seen_bits(const PagedAttnArgs &a, int p, int j0) {
    uint64_t seen = low_bits(p + 1 - j0);
    if (a.window) seen &= ~low_bits((p >= a.window ? p - a.window + 1 : 0) - j0) | low_bits(a.sinks - j0);
    return seen;
}

// ------------------------------------------------------------ tiles from pages

// The loop over tiles holds no branch with a load in it: the compiler counts the
// loads that are on their way, and behind such a branch it waits for all of them.
// So a tile behind the last one is "read" too, from the cache's first place.

// Where the keys of a tile lie: lane l knows key j0 + l.  Keys that are not
// there stand for page 0, place 0, which is in memory, and do not take part.
template <int BN> struct Places {
    const int32_t *table;       // the request's
    int l;
    int32_t id;
    int j;
    bool there;
    __device__ __forceinline__ int page_of(const PagedAttnArgs &a) const {
        return (int)(__umulhi((uint32_t)j, a.page_magic) >> a.page_shift) + (a.page == 1 ? j : 0);
    }
    // asks for the page of this lane's key of tile x (none from x1 on)
    __device__ __forceinline__ void ahead(const PagedAttnArgs &a, const View<BN> &v, int x, int x1) {
        j = v.start(x) + l;
        there = x < x1 && l < BN && v.holds(j);
        j = there ? j : 0;
        id = table[page_of(a)];
    }
    // Where lanes' keys and values lie, in values from the cache's first, and the
    // keys that are there (of the tile last asked for).
    __device__ __forceinline__ uint64_t take(const PagedAttnArgs &a, int64_t *k, int64_t *v) const {
        const bool on = there && id >= 0 && id < a.pages;
        const int g = on ? id : 0, i = on ? j - page_of(a) * a.page : 0;
        *k = g * a.k.b + i * a.k.l;
        *v = g * a.v.b + i * a.v.l;
        return __ballot(on);
    }
};
__device__ __forceinline__ int64_t from_lane(int64_t x, int lane) {
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)x, lane), hi = (uint32_t)__shfl((int)(x >> 32), lane);
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// A tile's place in LDS for blocks of 16 rows: as place() for bf16; in fp32 the
// rows 4 g + e of four groups of lanes g, read 16 values each, lie in different
// banks.
template <typename T, int DP> __device__ __forceinline__ int place16(int r, int c) {
    if constexpr (sizeof(T) == 2) return place<T, DP>(r, c);
    else return (r * (DP / 4) + (c ^ (((r >> 2) & 3) << 2 | (r & 3)))) * 16;
}

// A thread's part of a tile of K and of V on its way to LDS (as TileLoad, rows from
// pages).  Rows that are not there hold page 0's values until `clean`; pieces at
// and past dh are never written (threads that would carry them carry piece 0 as
// well), so what LDS holds there, zeros, stays.  ONCE: no other work-group reads the
// tile, so it is not kept in the caches (reads of 2048 waves in such tiles: 5.5 TB/s,
// with this 6.2).
template <typename T, int DP, int BN, int NT, bool VEC, bool ONCE> struct PagedLoad {
    static constexpr int PER = Op<T>::PER, CPR = DP / PER, N = BN * CPR / NT, RPI = NT / CPR;
    static_assert(BN * CPR % NT == 0 && NT % CPR == 0, "whole chunks per thread");
    u4v k[N], v[N];
    static __device__ __forceinline__ int piece(int t, int dh) { return t % CPR * PER < dh ? t % CPR : 0; }
    static __device__ __forceinline__ u4v load(const T *row, int c, int dh) {
        if constexpr (VEC && ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u4v *>(row + PER * c));
        else if constexpr (VEC) return *reinterpret_cast<const u4v *>(row + PER * c);
        else return load_chunk<T>(row, PER * c, dh, false);
    }
    // the rows at K + ks and V + vs of the lanes
    __device__ __forceinline__ void fetch(const PagedAttnArgs &a, const T *K, const T *V, int64_t ks, int64_t vs, int t) {
        const int c = piece(t, a.Dh), r0 = t / CPR;
        int64_t at[N];
#pragma unroll
        for (int q = 0; q < N; ++q) at[q] = from_lane(ks, r0 + q * RPI);
#pragma unroll
        for (int q = 0; q < N; ++q) k[q] = load(K + at[q], c, a.Dh);
        if (!a.alike)
#pragma unroll
            for (int q = 0; q < N; ++q) at[q] = from_lane(vs, r0 + q * RPI);
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = load(V + at[q], c, a.Dh);
    }
    // K's tile, and V's behind it; BLOCK16: for blocks of 16 rows
    template <bool BLOCK16> __device__ __forceinline__ void stash(char *tile, int dh, int t) const {
        const int c = piece(t, dh);
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int r = t / CPR + q * RPI, at = BLOCK16 ? place16<T, DP>(r, c) : place<T, DP>(r, c);
            *reinterpret_cast<u4v *>(tile + at) = k[q];
            *reinterpret_cast<u4v *>(tile + BN * DP * (int)sizeof(T) + at) = v[q];
        }
    }
    // zeros in V's rows that are not there
    __device__ __forceinline__ void clean(uint64_t live, int t) {
#pragma unroll
        for (int q = 0; q < N; ++q)
            if (!((live >> (t / CPR + q * RPI)) & 1)) v[q] = u4v{0, 0, 0, 0};
    }
    // Zeros in place of V's values that are not finite; says whether there were any.
    __device__ __forceinline__ bool finite() {
        bool any = false;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            bool bad = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t x = v[q][e];
                if constexpr (sizeof(T) == 4) {
                    const bool b = (x & 0x7f800000u) == 0x7f800000u;
                    if (b) v[q][e] = 0;
                    bad |= b;
                } else {
                    const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
                    v[q][e] = (lo ? 0 : x & 0xffffu) | (hi ? 0 : x & 0xffff0000u);
                    bad |= lo || hi;
                }
            }
            any |= bad;
        }
        return any;
    }
};

// o += the values of a state's row that are not finite.
template <typename T, int NJ> __device__ __forceinline__ void add_not_finite(f16v (&o)[NJ], const T *row, int dh, int l) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int d = 32 * j + 8 * (e / 4) + 4 * (l >> 5) + e % 4;
            const float x = d < dh ? ld_f32<T>(row, d) : 0.f;
            if (!(fabsf(x) < INFINITY)) o[j][e] += x;
        }
        asm volatile("" ::: "memory");      // (few registers matter more than time here)
    }
}

// Probabilities of bf16 tensors enter the second product as two bf16 terms where a
// wave works alone: the first 8 bits of each, and the rest rounded (off by 2^-15 of
// the probability at most).  Those kernels wait for memory, and a second product on
// the tile that is there takes little: 48 requests of up to 7000 states, 32 heads
// over 8 of 128, 121.5 -> 122.5 us, the error of O 0.0022 -> 0.0017 of its norm, which
// is its own rounding.  Blocks of 128 rows are bound by the products among others and
// keep one rounded term (Op::pack): 5 pieces of up to 1500 rows on up to 6000
// states, 444 us, with two terms 625, error 0.0023 and 0.0017.
template <typename T, int NW> constexpr bool TWO_TERMS = sizeof(T) == 2 && NW == 1;
__device__ __forceinline__ float first_term(float p) { return __uint_as_float(__float_as_uint(p) & 0xffff0000u); }
// (at least 2^-17 of p, so that an infinite value times both terms is infinite)
__device__ __forceinline__ float second_term(float p) { return fmaxf(p - first_term(p), 0x1p-17f * p); }

// ------------------------------------------------------------ the pass

// Waves a SIMD that registers are kept for.  (A wave on its own holds the whole tile
// that is on its way.  A value that found no register is read back from memory, and
// such a read waits for all loads before it, the next tile's too: 40 requests of up to
// 6000 states, 32 rows over 4 heads of 128, bf16, 94 us with two waves and 44 such
// values, 70 with one and none.)
template <typename T, int DC, int NW> constexpr int min_waves() {
    return NW == 1 ? (sizeof(T) == 4 || DC > 64 ? 1 : 2) : (sizeof(T) == 4 && DC > 64 ? 1 : 2);
}

// Heads whose values' places in LDS are too many (64 of four bytes) to be kept from
// tile to tile: they are worked out anew from a lane number of which the compiler
// does not know that it is the same.  (fp32 heads of 128, 32 rows: 167 -> 138 us,
// 8 rows 111 -> 105.)
template <typename T, int DC> constexpr bool MANY_PLACES = sizeof(T) == 4 && DC > 96;
__device__ __forceinline__ int anew(int l) {
    asm volatile("" : "+v"(l));
    return l;
}

// A block of 32 NW packed rows from m0 on of request b's head group hk against its
// tiles x0 .. x1 - 1.  Writes O and lse, or, with `part`, the rows' results of
// these tiles there.
template <typename T, int DC, int NW, int BN, bool VEC>
__device__ __forceinline__ void pass(const PagedAttnArgs &a, char *lds, int *marks, int b, int hk, const Rows &r, int m0, int x0, int x1,
                                     float *part, float *part_lse) {
    constexpr int DP = padded(DC), PER = Op<T>::PER, NS = DC / (2 * PER), NJ = DC / 32, NT = 64 * NW;
    constexpr int TILE = BN * DP * sizeof(T);
    // A wave on its own has read its tile before it writes the next one there: its
    // accesses to LDS take place in order.
    constexpr int BUFFERS = NW == 1 ? 1 : 2;
    const int t = threadIdx.x % NT, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int all = r.count * a.G, mw = m0 + 32 * w, m = mw + (l & 31);
    const bool on = m < all, wave_on = mw < all;
    const RowOf row(on ? m : 0, hk, a.G);
    const int64_t at = r.first + row.i;
    const int i0 = m0 / a.G, i1 = (m0 + 32 * NW < all ? m0 + 32 * NW - 1 : all - 1) / a.G;
    const View<BN> view(a, r, i0, i1);
    // positions: this lane's row's, and the first and last of the wave's rows
    const int p0 = r.kl - r.n, pos = p0 + row.i;
    const int pmin = p0 + mw / a.G, pmax = p0 + (mw + 32 < all ? mw + 31 : all - 1) / a.G;

    typename Op<T>::V q[NS];
    load_frags<T, DC>(q, on ? static_cast<const T *>(a.Q) + at * a.q.l + row.h * a.q.h : nullptr, a.Dh, VEC, l);
    const float c = fabsf(a.scale) * LOG2E;
    if (a.scale < 0) {
#pragma unroll
        for (int s = 0; s < NS; ++s) q[s] = -q[s];
    }
    const T *const K = static_cast<const T *>(a.K) + hk * a.k.h;
    const T *const V = static_cast<const T *>(a.V) + hk * a.v.h;
    Places<BN> keys{a.table + b * a.ldt, l, -1, 0, false};

    f16v o[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[j] = f16v{0};
    float mx = -INFINITY, sum = 0.f;

    PagedLoad<T, DP, BN, NT, VEC, NW == 1> way;
    uint64_t live = 0, next_live = 0;
    auto fetch = [&]() {
        int64_t ks, vs;
        const uint64_t on = keys.take(a, &ks, &vs);
        way.fetch(a, K, V, ks, vs, t);
        return on;
    };
    // Rows of the block see different states of the tile: a product takes 0 inf and 0
    // NaN for NaN, so values that are not finite are kept out of it, and added at
    // the end to the rows that see them.
    auto differ = [&](uint64_t on, int j0) { return i0 != i1 && !seen_by<BN>(a, on, j0, p0 + i0, p0 + i1); };
    auto stash = [&](int buffer, uint64_t on, int j0) {
        if (on != ALL_LIVE<BN>) way.clean(on, t);
        if (differ(on, j0)) marks[NW * buffer + w] = __any(way.finite());
        way.template stash<false>(lds + buffer * 2 * TILE, a.Dh, t);
    };
    int buffer = 0;             // the tile in use: K, then V
    int left_out = 0;           // some tile held values that were kept out
    if (x0 < x1) {
        if (a.Dh < DC) {
            lds_barrier();      // (an earlier block's tiles have been read)
            clear_lds<NT>(lds, BUFFERS * 2 * TILE, t);
            lds_barrier();
        }
        keys.ahead(a, view, x0, x1);
        live = fetch();
        keys.ahead(a, view, x0 + 1, x1);
        stash(0, live, view.start(x0));
        next_live = fetch();
        keys.ahead(a, view, x0 + 2, x1);
    }
    for (int x = x0; x < x1; ++x) {
        const int j0 = view.start(x);
        const char *const kt = lds + buffer * 2 * TILE, *const vt = kt + TILE;
        lds_barrier();
        const int lane = NW == 1 && MANY_PLACES<T, DC> ? anew(l) : l;
        if (wave_on) {
            f16v p[BN / 32];
#pragma unroll
            for (int n = 0; n < BN / 32; ++n) {
                p[n] = f16v{0};
#pragma unroll
                for (int s = 0; s < NS; ++s) p[n] = Op<T>::mma(row_frag<T, DP>(kt, 32 * n, s, l), q[s], p[n]);
            }
            if (!seen_by<BN>(a, live, j0, pmin, pmax)) {
                const uint64_t seen = seen_bits(a, pos, j0) & live;
#pragma unroll
                for (int n = 0; n < BN / 32; ++n) {
                    const uint32_t bits = (uint32_t)(seen >> (32 * n)) >> (4 * (l >> 5));
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (!((bits >> (8 * (e / 4) + e % 4)) & 1)) p[n][e] = -INFINITY;
                }
            }
            float top = p[0][0];
#pragma unroll
            for (int n = 0; n < BN / 32; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, p[n][e]);
            top = fmaxf(top, other_half(top)) * c;
            // (the reference of the exponents follows the maximum in steps of 2^8)
            if (__any(top > mx + 8.f)) {
                const float next = fmaxf(mx, top);
                const float turn = __builtin_amdgcn_exp2f(mx - (next == -INFINITY ? 0.f : next));
                mx = next;
                sum *= turn;
#pragma unroll
                for (int j = 0; j < NJ; ++j) o[j] *= turn;
            }
            const float ref = mx == -INFINITY ? 0.f : mx;
            float more = 0.f;
#pragma unroll
            for (int n = 0; n < BN / 32; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    p[n][e] = __builtin_amdgcn_exp2f(fmaf(p[n][e], c, -ref));
                    more += p[n][e];
                }
            sum += more;
#pragma unroll
            for (int n = 0; n < BN / 32; ++n)
#pragma unroll
                for (int s = 0; s < 16 / PER; ++s) {
                    if constexpr (TWO_TERMS<T, NW>) {
                        typename Op<T>::V first, second;
#pragma unroll
                        for (int e = 0; e < PER; ++e) {
                            first[e] = (__bf16)first_term(p[n][PER * s + e]);
                            second[e] = (__bf16)second_term(p[n][PER * s + e]);
                        }
#pragma unroll
                        for (int j = 0; j < NJ; ++j) {
                            const typename Op<T>::V v = col_frag<T, DP>(vt, 32 * n, s, j, lane);
                            o[j] = Op<T>::mma(v, first, o[j]);
                            o[j] = Op<T>::mma(v, second, o[j]);
                        }
                    } else {
                        const typename Op<T>::V pf = Op<T>::pack(p[n], s);
#pragma unroll
                        for (int j = 0; j < NJ; ++j) o[j] = Op<T>::mma(col_frag<T, DP>(vt, 32 * n, s, j, lane), pf, o[j]);
                    }
                }
        }
        if (differ(live, j0)) {
#pragma unroll
            for (int v = 0; v < NW; ++v) left_out |= __builtin_amdgcn_readfirstlane(marks[NW * buffer + v]);
        }
        if (BUFFERS == 2) buffer ^= 1;
        live = next_live;
        stash(buffer, live, view.start(x + 1));
        next_live = fetch();
        keys.ahead(a, view, x + 3, x1);
    }
    if (left_out) {             // they are added now, to the rows that see them
        for (int x = x0; x < x1; ++x) {
            const int j0 = view.start(x);
            int64_t ks, vs;
            keys.ahead(a, view, x, x1);
            const uint64_t there = keys.take(a, &ks, &vs);
            if (!differ(there, j0)) continue;
            for (uint64_t rest = there; rest; rest &= rest - 1) {
                const int k = __ffsll((unsigned long long)rest) - 1, j = j0 + k;
                const bool sees = j <= pos && (!a.window || pos - j < a.window || j < a.sinks);
                if (sees) add_not_finite<T, NJ>(o, V + lane_value(vs, k), a.Dh, l);
            }
        }
    }
    sum += other_half(sum);
    if (!on) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const float lse = sum != 0.f ? (mx + __builtin_amdgcn_logf(sum)) * LN2 : -INFINITY;
    if (part) {
        float *const po = part + (int64_t)(m - m0) * DP;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f4v v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = o[j][4 * g + e] * inv;
                *reinterpret_cast<f4v *>(po + 32 * j + 8 * g + 4 * (l >> 5)) = v;
            }
        if (l < 32) part_lse[m - m0] = lse;
        return;
    }
    T *const out = static_cast<T *>(a.O) + at * a.o.l + row.h * a.o.h;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f4v v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = o[j][4 * g + e] * inv;
            store4<T>(out, 32 * j + 8 * g + 4 * (l >> 5), a.Dh, VEC, v);
        }
    if (a.lse && l < 32) a.lse[at * a.Hq + row.h] = lse;
}

// ------------------------------------------------------------ up to 16 rows

// The same pass for one wave and up to 16 packed rows, with products of 16 x 16:
// lane l holds row l % 16 and of a block of 16 keys 4 (l / 16) + e.  Two such waves a
// SIMD, each with a tile on its way while it uses another, wait for memory alone.
// (One wave a SIMD with two tiles on their way: 122 us where this takes 119, 48
// requests of up to 7000 states, 32 heads over 8 of 128, bf16; three or four tiles
// 124 and 128.)
template <typename T> struct Op16;
template <> struct Op16<bf16_t> {
    static constexpr int BN = 32;       // keys a tile: the 32 terms of a product
    static __device__ __forceinline__ f4v mma(bf8v a, bf8v b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    // o += v p, the probabilities in two terms
    struct Terms {
        bf8v first, second;
        __device__ __forceinline__ explicit Terms(const f4v (&p)[2]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                first[e] = (__bf16)first_term(p[e / 4][e % 4]);
                second[e] = (__bf16)second_term(p[e / 4][e % 4]);
            }
        }
        __device__ __forceinline__ f4v add(bf8v v, f4v o) const { return mma(v, second, mma(v, first, o)); }
    };
    // values 16 j .. of the keys in the terms' order
    template <int DP> static __device__ __forceinline__ bf8v col(const char *tile, int j, int l) {
        const int a = l & 15, k = 4 * (l >> 4) + (a >> 2), n = 16 * j + 4 * (a & 3);
        const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GS_LDS s4v *)(tile + place16<bf16_t, DP>(k, n >> 3) + 2 * (n & 7)));
        const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GS_LDS s4v *)(tile + place16<bf16_t, DP>(k + 16, n >> 3) + 2 * (n & 7)));
        const s4v both[2] = {lo, hi};
        return *reinterpret_cast<const bf8v *>(both);
    }
};
template <> struct Op16<float> {
    static constexpr int BN = 16;
    static __device__ __forceinline__ f4v mma(f4v a, f4v b, f4v c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    struct Terms {
        f4v p;
        __device__ __forceinline__ explicit Terms(const f4v (&p)[1]) : p(p[0]) {}
        __device__ __forceinline__ f4v add(f4v v, f4v o) const { return mma(v, p, o); }
    };
    template <int DP> static __device__ __forceinline__ f4v col(const char *tile, int j, int l) {
        f4v r;
        const int n = 16 * j + (l & 15), k = 4 * (l >> 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = *reinterpret_cast<const float *>(tile + place16<float, DP>(k + e, n >> 2) + 4 * (n & 3));
        return r;
    }
};

template <typename T, int DC, bool VEC>
__device__ __forceinline__ void pass16(const PagedAttnArgs &a, char *lds, int b, int hk, const Rows &r, int x0, int x1,
                                       float *part, float *part_lse) {
    constexpr int BN = Op16<T>::BN, DP = padded(DC), PER = Op<T>::PER, NS = DC / (4 * PER), NJ = DC / 16, NB = BN / 16;
    constexpr int TILE = BN * DP * sizeof(T);
    const int l = threadIdx.x, m = l & 15;
    const int all = r.count * a.G;
    const bool on = m < all;
    const RowOf row(on ? m : 0, hk, a.G);
    const int64_t at = r.first + row.i;
    const View<BN> view(a, r, 0, r.count - 1);
    const int pmin = r.kl - r.n, pmax = pmin + r.count - 1, pos = pmin + row.i;

    typename Op<T>::V q[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        u4v v = {0, 0, 0, 0};
        if (on) v = load_chunk<T>(static_cast<const T *>(a.Q) + at * a.q.l + row.h * a.q.h, PER * (4 * s + (l >> 4)), a.Dh, VEC);
        q[s] = *reinterpret_cast<const typename Op<T>::V *>(&v);
    }
    const float c = fabsf(a.scale) * LOG2E;
    if (a.scale < 0) {
#pragma unroll
        for (int s = 0; s < NS; ++s) q[s] = -q[s];
    }
    const T *const K = static_cast<const T *>(a.K) + hk * a.k.h;
    const T *const V = static_cast<const T *>(a.V) + hk * a.v.h;

    f4v o[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[j] = f4v{0};
    float mx = -INFINITY, sum = 0.f;
    int left_out = 0;

    PagedLoad<T, DP, BN, 64, VEC, true> way;
    uint64_t live = 0;
    Places<BN> keys{a.table + b * a.ldt, l, -1, 0, false};
    auto differ = [&](uint64_t on, int j0) { return pmin != pmax && !seen_by<BN>(a, on, j0, pmin, pmax); };
    // the tile whose pages were asked for, and the pages of tile x
    auto fetch = [&](int x) {
        int64_t ks, vs;
        live = keys.take(a, &ks, &vs);
        way.fetch(a, K, V, ks, vs, l);
        keys.ahead(a, view, x, x1);
    };
    if (x0 < x1) {
        if (a.Dh < DC) {
            lds_barrier();
            clear_lds<64>(lds, 2 * TILE, l);
            lds_barrier();
        }
        keys.ahead(a, view, x0, x1);
        fetch(x0 + 1);
    }
    for (int x = x0; x < x1; ++x) {
        const int j0 = view.start(x);
        const uint64_t on = live;
        if (on != ALL_LIVE<BN>) way.clean(on, l);
        if (differ(on, j0)) left_out |= __any(way.finite());
        lds_barrier();          // (one wave: keeps the accesses in order)
        const int lane = MANY_PLACES<T, DC> ? anew(l) : l;
        way.template stash<true>(lds, a.Dh, l);
        fetch(x + 2);
        lds_barrier();
        f4v p[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            p[n] = f4v{0};
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const typename Op<T>::V k = *reinterpret_cast<const typename Op<T>::V *>(lds + place16<T, DP>(16 * n + m, 4 * s + (l >> 4)));
                p[n] = Op16<T>::mma(k, q[s], p[n]);
            }
        }
        if (!seen_by<BN>(a, on, j0, pmin, pmax)) {
            const uint32_t bits = (uint32_t)(seen_bits(a, pos, j0) & on) >> (4 * (l >> 4));
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!((bits >> (16 * n + e)) & 1)) p[n][e] = -INFINITY;
        }
        float top = p[0][0];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, p[n][e]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32)) * c;
        if (__any(top > mx + 8.f)) {        // (as in pass)
            const float next = fmaxf(mx, top);
            const float turn = __builtin_amdgcn_exp2f(mx - (next == -INFINITY ? 0.f : next));
            mx = next;
            sum *= turn;
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[j] *= turn;
        }
        const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[n][e] = __builtin_amdgcn_exp2f(fmaf(p[n][e], c, -ref));
                sum += p[n][e];
            }
        const typename Op16<T>::Terms terms(p);
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[j] = terms.add(Op16<T>::template col<DP>(lds + TILE, j, lane), o[j]);
    }
    if (left_out) {
        for (int x = x0; x < x1; ++x) {
            const int j0 = view.start(x);
            int64_t ks, vs;
            keys.ahead(a, view, x, x1);
            const uint64_t there = keys.take(a, &ks, &vs);
            if (!differ(there, j0)) continue;
            for (uint64_t rest = there; rest; rest &= rest - 1) {
                const int k = __ffsll((unsigned long long)rest) - 1;
                const T *const from = V + lane_value(vs, k);
                if (!((seen_bits(a, pos, j0) >> k) & 1)) continue;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int d = 16 * j + 4 * (l >> 4) + e;
                        const float v = d < a.Dh ? ld_f32<T>(from, d) : 0.f;
                        if (!(fabsf(v) < INFINITY)) o[j][e] += v;
                    }
            }
        }
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (!on) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const float lse = sum != 0.f ? (mx + __builtin_amdgcn_logf(sum)) * LN2 : -INFINITY;
    if (part) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) *reinterpret_cast<f4v *>(part + (int64_t)m * DP + 16 * j + 4 * (l >> 4)) = o[j] * inv;
        if (l < 16) part_lse[m] = lse;
        return;
    }
    T *const out = static_cast<T *>(a.O) + at * a.o.l + row.h * a.o.h;
#pragma unroll
    for (int j = 0; j < NJ; ++j) store4<T>(out, 16 * j + 4 * (l >> 4), a.Dh, VEC, o[j] * inv);
    if (a.lse && l < 16) a.lse[at * a.Hq + row.h] = lse;
}

// ------------------------------------------------------------ few rows

// Tiles of request b; one where there are rows, but no states.
template <int BN> __device__ __forceinline__ int few_tiles(const PagedAttnArgs &a, int b) {
    const Rows r(a, b);
    if (!r.count) return 0;
    const View<BN> v(a, r, 0, r.count - 1);
    return v.tiles > 1 ? v.tiles : 1;
}

__device__ __forceinline__ int few_share(const PagedAttnArgs &a, int total) {
    const int per = (int)((uint32_t)(total - 1) / (uint32_t)a.ranges) + 1;
    return per < a.least ? a.least : per;
}

// All requests' tiles lie in a line, requests in order.  Found by a wave: the
// share of the line that a range has, and for range i the request in which it
// begins and the tiles of those before that; b = a.B behind the end.
struct Line {
    int total, share, before, b;
    template <int BN> __device__ __forceinline__ void find(const PagedAttnArgs &a, int i) {
        const int l = threadIdx.x & 63;
        int s = 0, e = a.B;
        int64_t u = 0;
        before = 0;
        for (bool first = true; first || e - s > 1; first = false) {
            const int per = (e - s + 63) / 64;
            const int from = s + l * per, to = from + per < e ? from + per : e;
            int mine = 0;
#pragma unroll 4
            for (int k = from; k < to; ++k) mine += few_tiles<BN>(a, k);
            const int sums = wave_upto(mine);
            if (first) {
                total = lane_value(sums, 63);
                if (!total) break;
                share = few_share(a, total);
                u = (int64_t)i * share;
            }
            const uint64_t past = __ballot(before + sums > u);
            if (!past) {
                s = a.B;
                break;
            }
            const int at = __ffsll((unsigned long long)past) - 1;
            before += lane_value(sums - mine, at);
            s += at * per;
            e = s + per < e ? s + per : e;
        }
        b = total ? s : a.B;
    }
};

// Keys of a tile for up to R rows.
template <typename T> constexpr int few_keys(int R) { return R == 16 ? Op16<T>::BN : 32; }

// A range of the line, one head: a wave.  The heads of a range are read side by
// side, as their states lie in the cache.
template <typename T, int DC, int R, bool VEC>
__global__ void __launch_bounds__(64, (R == 16 ? 2 : min_waves<T, DC, 1>())) few_kernel(PagedAttnArgs a) {
    constexpr int BN = few_keys<T>(R);
    constexpr int DP = padded(DC);
    __shared__ __attribute__((aligned(16))) char lds[2 * BN * DP * sizeof(T)];
    __shared__ int marks[1];        // (32 rows)
    const int64_t place = logical_group((int64_t)a.ranges * a.Hkv);
    const int range = (int)(place / a.Hkv), hk = (int)(place % a.Hkv);
    if (range >= a.ranges) return;
    int b, before = 0, begin = 0, end;
    if (a.whole) {              // a request a range
        b = range;
        end = few_tiles<BN>(a, b);
    } else {
        Line line;
        line.find<BN>(a, range);
        b = line.b, before = line.before;
        if (b >= a.B) return;
        begin = range * line.share, end = line.total - begin < line.share ? line.total : begin + line.share;
        if (begin == 0 && hk == 0 && threadIdx.x == 0) a.line[a.B] = line.share;
    }
    for (int u = begin; u < end; ++b) {
        const Rows r(a, b);
        const int tiles = few_tiles<BN>(a, b);
        if (!tiles) continue;
        const int x0 = u - before, x1 = end - before < tiles ? end - before : tiles;
        const View<BN> v(a, r, 0, r.count - 1);
        float *part = nullptr, *part_lse = nullptr;
        if (x1 - x0 < tiles) {
            const int64_t slot = (int64_t)(2 * range + (before > begin)) * a.Hkv + hk;
            part = a.part + slot * a.rows * DP;
            part_lse = a.part_lse + slot * a.rows;
        }
        if (x0 == 0 && hk == 0 && threadIdx.x == 0 && !a.whole) a.line[b] = before;
        if constexpr (R == 16) pass16<T, DC, VEC>(a, lds, b, hk, r, x0, x1 < v.tiles ? x1 : v.tiles, part, part_lse);
        else pass<T, DC, 1, BN, VEC>(a, lds, marks, b, hk, r, 0, x0, x1 < v.tiles ? x1 : v.tiles, part, part_lse);
        u += x1 - x0;
        before += tiles;
    }
}

// Where the parts of a request and head that range ends cut lie.
struct Cut {
    int i0, i1;         // its ranges
    int64_t first, next, step;
    int before, share;
    // (asked for before anything is known of the request, which saves a wait)
    __device__ __forceinline__ Cut(const PagedAttnArgs &a, int b) : before(a.line[b]), share(a.line[a.B]) {}
    template <int BN> __device__ __forceinline__ void find(const PagedAttnArgs &a, int b, int hk) {
        const int tiles = few_tiles<BN>(a, b);
        i0 = before / share, i1 = (before + tiles - 1) / share;
        step = 2 * (int64_t)a.Hkv * a.rows;
        // the first part may be its range's second one
        first = ((int64_t)(2 * i0 + (before > i0 * share)) * a.Hkv + hk) * a.rows;
        next = ((int64_t)(2 * i0) * a.Hkv + hk) * a.rows;
    }
    __device__ __forceinline__ int64_t place(int i, int m) const { return (i == i0 ? first : next + (i - i0) * step) + m; }
};

__device__ __forceinline__ float joined_lse(float ref, float sum) {
    return sum != 0.f ? ref + __builtin_amdgcn_logf(sum) * LN2 : -INFINITY;
}

// Puts together rows of which there are a few parts: a thread for 4 values.
template <typename T, int DP, int BN> __global__ void __launch_bounds__(256) few_join_kernel(PagedAttnArgs a) {
    constexpr int LANES = DP / 4;
    const int hk = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv, d = 4 * (threadIdx.x % LANES);
    Cut c(a, b);
    const Rows r(a, b);
    const int m = blockIdx.y * (256 / LANES) + threadIdx.x / LANES;
    if (m >= r.count * a.G || d >= a.Dh) return;
    c.find<BN>(a, b, hk);
    if (c.i0 == c.i1) return;
    float top = -INFINITY, sum = 0.f;
    f4v o = {0.f, 0.f, 0.f, 0.f};
    // four parts at a time, their log-sums and values asked for together
    for (int i = c.i0; i <= c.i1; i += 4) {
        float lse[4];
        f4v v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t at = c.place(i + k <= c.i1 ? i + k : c.i1, m);
            lse[k] = a.part_lse[at];
            v[k] = *reinterpret_cast<const f4v *>(a.part + at * DP + d);
        }
        float next = top;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k <= c.i1) next = fmaxf(next, lse[k]);
        const float ref = next == -INFINITY ? 0.f : next;
        const float turn = __builtin_amdgcn_exp2f((top - ref) * LOG2E);
        top = next;
        sum *= turn;
        o *= turn;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i + k > c.i1) continue;
            const float e = __builtin_amdgcn_exp2f((lse[k] - ref) * LOG2E);
            sum += e;
            o += e * v[k];
        }
    }
    const float ref = top == -INFINITY ? 0.f : top;
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    const RowOf row(m, hk, a.G);
    const int64_t at = r.first + row.i;
    store4<T>(static_cast<T *>(a.O) + at * a.o.l + row.h * a.o.h, d, a.Dh, a.vec, o * inv);
    if (a.lse && d == 0) a.lse[at * a.Hq + row.h] = joined_lse(ref, sum);
}

// The same for many parts: a work-group for 4 LANES values of a row, parts shared out
// to its groups of so many lanes.
template <typename T, int DP, int BN, int NT, int LANES> __global__ void __launch_bounds__(NT) few_join_many_kernel(PagedAttnArgs a) {
    constexpr int GROUPS = NT / LANES, WAVES = NT / 64;
    __shared__ f4v sums[WAVES][LANES];
    __shared__ float weights[WAVES], tops[WAVES];
    const int t = threadIdx.x, l = t & 63, w = t >> 6, g = t / LANES, d = 4 * (blockIdx.z * LANES + t % LANES);
    const int hk = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
    Cut c(a, b);
    const Rows r(a, b);
    const int m = blockIdx.y;
    if (m >= r.count * a.G) return;
    c.find<BN>(a, b, hk);
    const int i0 = c.i0, i1 = c.i1;
    if (i0 == i1) return;
    auto place = [&](int i) { return c.place(i, m); };
    float top = -INFINITY;
    for (int i = i0 + t; i <= i1; i += NT) top = fmaxf(top, a.part_lse[place(i)]);
#pragma unroll
    for (int k = 32; k; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
    if (l == 0) tops[w] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < WAVES; ++k) top = fmaxf(top, tops[k]);
    const float ref = top == -INFINITY ? 0.f : top;
    f4v o = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll 4
    for (int i = i0 + g; i <= i1; i += GROUPS) {
        const int64_t at = place(i);
        const float e = __builtin_amdgcn_exp2f((a.part_lse[at] - ref) * LOG2E);
        sum += e;
        o += e * *reinterpret_cast<const f4v *>(a.part + at * DP + d);
    }
#pragma unroll
    for (int k = LANES; k < 64; k <<= 1) {
        sum += __shfl_xor(sum, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], k);
    }
    if (l < LANES) sums[w][l] = o;
    if (l == 0) weights[w] = sum;
    __syncthreads();
    if (t < LANES) {
#pragma unroll
        for (int k = 1; k < WAVES; ++k) o += sums[k][t], sum += weights[k];
        const float inv = sum != 0.f ? 1.f / sum : 0.f;
        const RowOf row(m, hk, a.G);
        const int64_t at = r.first + row.i;
        if (d < a.Dh) store4<T>(static_cast<T *>(a.O) + at * a.o.l + row.h * a.o.h, d, a.Dh, a.vec, o * inv);
        if (a.lse && d == 0) a.lse[at * a.Hq + row.h] = joined_lse(ref, sum);
    }
}

// ------------------------------------------------------------ many rows

constexpr int BLOCK = 128;      // packed rows of a work-group of four waves

// Requests' blocks lie in a line with a place for each: request b's from
// floor(qoff[b] G / BLOCK) + b on, which leaves room for all of them.
__device__ __forceinline__ int block_start(const PagedAttnArgs &a, int b) {
    return (a.qoff ? clamped(a.qoff, b, a.N) : b) * a.G / BLOCK + b;
}

// Lists the work: blocks of more than a share of the tiles in equal parts, and the
// longest first (in 64 steps), so that short ones fill the end.  Places within a
// step, and of parts in the workspace, go by the order of atomics; no result does.
template <int BN> __global__ void __launch_bounds__(1024) plan_kernel(PagedAttnArgs a) {
    constexpr int STEPS = 64, STAGED = 1024;
    __shared__ int64_t room[16];
    __shared__ int next[STEPS], longest, slots, joins;
    __shared__ int starts[STAGED];
    const int t = threadIdx.x;
    int b = 0, tile = 0;
    const bool staged = a.B <= STAGED;
    if (staged && t < a.B) starts[t] = block_start(a, t);
    auto tiles_of = [&](int i) {
        if (i >= a.blocks || a.B == 0) return 0;
        int lo = 0, hi = a.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if ((staged ? starts[mid] : block_start(a, mid)) <= i) lo = mid;
            else hi = mid;
        }
        const Rows r(a, lo);
        const int k = i - (staged ? starts[lo] : block_start(a, lo)), all = r.count * a.G;
        if (k < 0 || k * BLOCK >= all) return 0;
        b = lo, tile = k;
        const View<BN> v(a, r, k * BLOCK / a.G, ((k + 1) * BLOCK < all ? (k + 1) * BLOCK - 1 : all - 1) / a.G);
        return v.tiles > 1 ? v.tiles : 1;
    };
    if (t < STEPS) next[t] = 0;
    if (t == 0) longest = 1, slots = 0, joins = 0;
    __syncthreads();
    int64_t mine = 0, total;
    int n = 0, most = 0;
    for (int i = t; i < a.blocks; i += 1024) {
        n = tiles_of(i);
        mine += n;
        most = max(most, n);
    }
    (void)group_scan(mine, room, &total);
    total = (total * a.Hkv + a.waves - 1) / a.waves;
    const int share = total < a.least ? a.least : (int)(total < 0x40000000 ? total : 0x40000000);
#pragma unroll
    for (int d = 32; d; d >>= 1) most = max(most, __shfl_xor(most, d));
    if ((t & 63) == 0) atomicMax(&longest, min(most, share));
    __syncthreads();
    // parts of a block of n tiles, and their step by length
    const int top = longest;
    auto parts_of = [&](int n) { return n > share ? (n - 1) / share + 1 : (n ? 1 : 0); };
    auto step_of = [&](int n, int parts) { return (int)((STEPS - 1) - (int64_t)(n / parts) * (STEPS - 1) / top); };
    const bool again = a.blocks > 1024;         // more blocks than threads: looked up once more each time
    for (int i = t; i < a.blocks; i += 1024) {
        if (again) n = tiles_of(i);
        const int parts = parts_of(n);
        if (parts) atomicAdd(&next[step_of(n, parts)], parts);
    }
    __syncthreads();
    if (t < STEPS) {
        const int here = next[t], sum = wave_upto(here);
        next[t] = sum - here;
        if (t == STEPS - 1) a.head->items = sum;
    }
    __syncthreads();
    for (int i = t; i < a.blocks; i += 1024) {
        if (again) n = tiles_of(i);
        const int parts = parts_of(n);
        if (!parts) continue;
        const int item = atomicAdd(&next[step_of(n, parts)], parts);
        const int slot = parts > 1 ? atomicAdd(&slots, parts) : -1;
        for (int k = 0; k < parts; ++k)
            a.items[item + k] = PagedItem{b, tile, (int32_t)((int64_t)n * k / parts), (int32_t)((int64_t)n * (k + 1) / parts),
                                          parts > 1 ? slot + k : -1};
        if (parts > 1) a.joins[atomicAdd(&joins, 1)] = PagedJoin{b, tile, slot, parts};
    }
    __syncthreads();
    if (t == 0) a.head->joins = joins;
}

template <typename T, int DC, int BN, bool VEC>
__global__ void __launch_bounds__(256, (min_waves<T, DC, 4>())) many_kernel(PagedAttnArgs a) {
    constexpr int DP = padded(DC);
    __shared__ __attribute__((aligned(16))) char lds[4 * BN * DP * sizeof(T)];
    __shared__ int marks[8];
    const int item = blockIdx.x / a.Hkv, hk = blockIdx.x % a.Hkv;
    if (item >= a.head->items) return;
    const PagedItem p = a.items[item];
    const Rows r(a, p.b);
    const int m0 = p.tile * BLOCK, all = r.count * a.G;
    const View<BN> v(a, r, m0 / a.G, (m0 + BLOCK < all ? m0 + BLOCK - 1 : all - 1) / a.G);
    float *part = nullptr, *part_lse = nullptr;
    if (p.slot >= 0) {
        const int64_t slot = (int64_t)p.slot * a.Hkv + hk;
        part = a.part + slot * BLOCK * DP;
        part_lse = a.part_lse + slot * BLOCK;
    }
    pass<T, DC, 4, BN, VEC>(a, lds, marks, p.b, hk, r, m0, p.x0, p.x1 < v.tiles ? p.x1 : v.tiles, part, part_lse);
}

// Rows of blocks that were cut, DP / 4 lanes a row.
template <typename T, int DP> __global__ void __launch_bounds__(256) many_join_kernel(PagedAttnArgs a) {
    constexpr int LANES = DP / 4, PER = 256 / LANES, PIECES = BLOCK / PER;
    const int join = blockIdx.x / (a.Hkv * PIECES), hk = blockIdx.x / PIECES % a.Hkv;
    if (join >= a.head->joins) return;
    const PagedJoin p = a.joins[join];
    const int k = blockIdx.x % PIECES * PER + threadIdx.x / LANES, d = 4 * (threadIdx.x % LANES);
    const Rows r(a, p.b);
    const int m = p.tile * BLOCK + k;
    if (m >= r.count * a.G || d >= a.Dh) return;
    const float *const pl = a.part_lse + ((int64_t)p.slot * a.Hkv + hk) * BLOCK + k;
    const float *const po = a.part + (((int64_t)p.slot * a.Hkv + hk) * BLOCK + k) * DP + d;
    const int64_t step = (int64_t)a.Hkv * BLOCK;
    float top = -INFINITY, sum = 0.f;
#pragma unroll 8
    for (int s = 0; s < p.parts; ++s) top = fmaxf(top, pl[s * step]);
    const float ref = top == -INFINITY ? 0.f : top;
    f4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < p.parts; ++s) {
        const float e = __builtin_amdgcn_exp2f((pl[s * step] - ref) * LOG2E);
        sum += e;
        o += e * *reinterpret_cast<const f4v *>(po + s * step * DP);
    }
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    const RowOf row(m, hk, a.G);
    const int64_t at = r.first + row.i;
    store4<T>(static_cast<T *>(a.O) + at * a.o.l + row.h * a.o.h, d, a.Dh, a.vec, o * inv);
    if (a.lse && d == 0) a.lse[at * a.Hq + row.h] = joined_lse(ref, sum);
}

// ------------------------------------------------------------ dispatch

constexpr int FEW = 32;         // packed rows up to which waves work alone

constexpr int tile_keys(gs_dtype t) { return t == GS_F32 ? 32 : 64; }

// Sizes of the workspace's parts, by sizes that the host knows.
struct Layout {
    bool few, whole;
    int ranges, waves, least, rows;
    int64_t blocks, items, joins, slots;
    int dp;
    size_t list, bytes;
};
Layout layout(gs_dtype t, const PagedAttnArgs &a) {
    Layout z{};
    const int dc = computed(a.Dh);
    const int64_t rows = (int64_t)a.Lq * a.G;
    z.dp = padded(dc);
    z.few = rows <= FEW;
    if (z.few) {
        // as many waves as the CUs hold at once, by their registers (min_waves; 8 in pass16)
        const int held = rows > 16 && (t == GS_F32 || dc > 64) ? 4 : 8;
        z.rows = (int)rows;
        z.least = 4;
        const int64_t most = ((int64_t)a.Lk / 16 + 3) * a.B / z.least + 1, full = 256 * held / a.Hkv;
        z.ranges = (int)(most < full ? most : (full > 1 ? full : 1));
        // Short histories and windows are not cut: up to 8 tiles in a row take less
        // than a second launch.
        const int bn = t == GS_F32 && rows <= 16 ? 16 : 32;
        int64_t most_tiles = ((int64_t)a.Lk + bn - 1) / bn;
        if (a.window) most_tiles = std::min(most_tiles, ((int64_t)a.window + a.Lq - 2) / bn + 2 + ((int64_t)a.sinks + bn - 1) / bn);
        z.whole = most_tiles <= 8;
        if (z.whole) z.ranges = a.B;
        z.slots = z.whole ? 0 : 2 * (int64_t)z.ranges * a.Hkv;
    } else {
        const int64_t most = t == GS_F32 && dc > 64 ? 256 : 512;
        z.rows = BLOCK;
        z.least = 8;
        z.waves = (int)most;
        z.blocks = (int64_t)a.N * a.G / BLOCK + a.B;
        // a share is at least total Hkv / waves: blocks cut into parts have at most
        // waves / Hkv + 1 shares in all, and less than two parts a share
        z.slots = 2 * (most / a.Hkv + 1);
        z.items = z.blocks + z.slots;
        z.joins = z.slots / 2 + 1;
        z.slots *= a.Hkv;
    }
    z.list = z.whole ? 0 : z.few ? 4 * ((size_t)a.B + 1) : sizeof(PagedAttnHead) + (size_t)z.items * sizeof(PagedItem) + (size_t)z.joins * sizeof(PagedJoin);
    z.list = (z.list + 15) / 16 * 16;
    z.bytes = z.list + (size_t)z.slots * z.rows * (z.dp + 1) * 4;
    return z;
}

template <typename T, int DC, int R, bool VEC> hipError_t launch_few(const PagedAttnArgs &a, const Layout &z, hipStream_t s) {
    constexpr int DP = padded(DC), BN = few_keys<T>(R);
    few_kernel<T, DC, R, VEC><<<dim3((unsigned)((z.ranges * a.Hkv + 7) / 8 * 8)), dim3(64), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || z.whole || z.ranges == 1) return e;
    // Parts of a row are joined by a thread for 4 values, or shared out to a work-group:
    // from 16 a request on (the mean; one long history among short ones has more) to one
    // of 512 threads for a row, or, where they fit the CUs, to such of 1024 for 32 values.
    // Heads of 128 values, us by thread, by 512 and by 1024: 12 parts of 21 requests, 32
    // rows each 5.0, 5.5, 23; 16 of 16, 32 rows 5.5, 4.9, 17; 128 rows 6.4, 9.8, 61; 32 of
    // 8, 32 rows 7.7, 4.7, 10; 512 parts of one, 32 rows over 4 heads -, 8.6, 7.1; 782
    // parts, 8 rows -, 10.9, 7.4; 256 parts of one of 16 requests, 128 rows 42, 13, 47.
    const unsigned pairs = (unsigned)(a.B * a.Hkv);
    const int64_t parts = z.ranges / a.B, groups = (int64_t)pairs * a.rows * (DP / 32);
    if (parts >= 16 && groups <= 256) {
        few_join_many_kernel<T, DP, BN, 1024, 8><<<dim3(pairs, (unsigned)a.rows, DP / 32), dim3(1024), 0, s>>>(a);
    } else if (parts >= 16) {
        few_join_many_kernel<T, DP, BN, 512, DP / 4><<<dim3(pairs, (unsigned)a.rows, 1), dim3(512), 0, s>>>(a);
    } else {
        const unsigned pieces = (unsigned)((a.rows * (DP / 4) + 255) / 256);
        few_join_kernel<T, DP, BN><<<dim3(pairs, pieces), dim3(256), 0, s>>>(a);
    }
    return hipGetLastError();
}

template <typename T, int DC, bool VEC> hipError_t launch_sized(const PagedAttnArgs &a, const Layout &z, hipStream_t s) {
    constexpr int DP = padded(DC);
    constexpr gs_dtype t = sizeof(T) == 4 ? GS_F32 : GS_BF16;
    if (z.few) return z.rows <= 16 ? launch_few<T, DC, 16, VEC>(a, z, s) : launch_few<T, DC, 32, VEC>(a, z, s);
    constexpr int BN = tile_keys(t);
    plan_kernel<BN><<<dim3(1), dim3(1024), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    many_kernel<T, DC, BN, VEC><<<dim3((unsigned)(z.items * a.Hkv)), dim3(256), 0, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    many_join_kernel<T, DP><<<dim3((unsigned)(z.joins * a.Hkv * (BLOCK * DP / 1024))), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, bool VEC> hipError_t launch_typed(const PagedAttnArgs &a, const Layout &z, hipStream_t s) {
    const int dc = computed(a.Dh);
    if (dc == 64) return launch_sized<T, 64, VEC>(a, z, s);
    return dc == 96 ? launch_sized<T, 96, VEC>(a, z, s) : launch_sized<T, 128, VEC>(a, z, s);
}

}  // namespace

size_t paged_attn_workspace(gs_dtype t, const PagedAttnArgs &a) { return layout(t, a).bytes; }

hipError_t launch_paged_attn(gs_dtype t, PagedAttnArgs a, void *ws, hipStream_t s) {
    const Layout z = layout(t, a);
    a.rows = z.rows;
    a.blocks = (int)z.blocks;
    a.waves = z.waves;
    a.ranges = z.ranges;
    a.whole = z.whole;
    a.least = z.least;
    a.line = static_cast<int32_t *>(ws);
    a.head = static_cast<PagedAttnHead *>(ws);
    a.items = reinterpret_cast<PagedItem *>(a.head + 1);
    a.joins = reinterpret_cast<PagedJoin *>(a.items + z.items);
    a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + z.list);
    a.part_lse = a.part + z.slots * z.rows * z.dp;
    // j / page for j below 2^31: with 2^s >= page > 2^(s - 1) and m = ceil(2^(31 + s) / page)
    // < 2^32, floor(j m / 2^(31 + s)) is it (m page exceeds 2^(31 + s) by less than page <= 2^s)
    int shift = 0;
    while (((int64_t)1 << shift) < a.page) ++shift;
    a.page_magic = (uint32_t)((((unsigned __int128)1 << (31 + shift)) + a.page - 1) / a.page);
    a.page_shift = shift - 1;
    if (a.page == 1) a.page_magic = 0, a.page_shift = 0;
    a.alike = a.k.b == a.v.b && a.k.l == a.v.l;
    if (!a.pages) {             // what stands for the first place of a cache without pages
        a.K = a.V = a.Q;
        a.k = a.v = SeqStrides{0, 0, 0};
    }
    if (t == GS_F32) return a.vec ? launch_typed<float, true>(a, z, s) : launch_typed<float, false>(a, z, s);
    return a.vec ? launch_typed<bf16_t, true>(a, z, s) : launch_typed<bf16_t, false>(a, z, s);
}

}  // namespace gs
