// Cross attention: O = softmax(scale Q K^T) V over the live encoder states.
//
// One pass over the states with the running maximum and sum of the softmax:
// a work-group holds 32 query rows per wave (rows of the heads that share a
// key and value head lie side by side, so grouped heads read K and V once),
// streams tiles of K and V through LDS, and keeps scores, probabilities and
// the weighted sum in registers.  The scores are formed with the keys as rows
// and the queries as columns, so that a query's scores lie in two lanes, and
// the accumulators of the first product are, packed, an operand of the second.
//
// Many rows: bound by the matrix cores and, between their products, by the
// exponentials (4 x 32 heads over 8, 4096 x 4096 of 128 values, bf16: 1.12 ms,
// 980 TF/s, where a large library product runs at 1200; products and softmax of
// two tiles side by side in one wave needed registers that cost more, 1.34 ms).
// One position: bound by HBM (64 sequences of up to 4000 states, 32 heads over
// 8 of 128 values: 601 MB in 135 us, 4.45 TB/s, where a large copy reaches
// 4.77).  fp32 products take eight times as long as bf16 ones: 62 % of the
// library's rate at 1024 x 1024 of 64 values (the matrix cores are busy 69 % of
// the cycles) and of 128 (67 %).
#include "gs_attn.h"

namespace gs {
namespace {
using namespace attn;

// Waves a SIMD that registers are kept for: fp32 fragments take twice the
// registers of bf16 ones, and those with more than 64 values, or of a single wave (which
// carries whole tiles), would spill at two.
template <typename T, int DC, int NW> constexpr int min_waves() { return sizeof(T) == 4 && (DC > 64 || NW == 1) ? 1 : 2; }

// GR groups of NW waves take the tiles of keys in turn, each with LDS of its own
// and a weighted sum of its own, which are joined at the end.
template <typename T, int DC, int NW, int GR, int BN, bool VEC>
__global__ void __launch_bounds__(64 * NW * GR, (min_waves<T, DC, NW>())) xattn_kernel(CrossAttnArgs a) {
    constexpr int DP = padded(DC), PER = Op<T>::PER, NS = DC / (2 * PER), NJ = DC / 32, NT = 64 * NW;
    constexpr int TILE = BN * DP * sizeof(T), STEP = GR * BN;
    __shared__ __attribute__((aligned(16))) char lds[GR * 4 * TILE];        // two of K, two of V for each group
    const int t = threadIdx.x % NT, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int group = GR > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0, mine = group * BN;
    const int64_t L = logical_group(a.groups);
    if (L >= a.groups) return;
    const int rt = (int)(L % a.row_tiles);
    const int64_t rest = L / a.row_tiles;
    const int sp = (int)(rest % a.splits);
    const int bh = (int)(rest / a.splits);
    const int b = bh / a.Hkv, hk = bh % a.Hkv;
    const int ql = clamped(a.qlen, b, a.Lq), kl = clamped(a.klen, b, a.Lk);
    const int m = rt * 32 * NW + 32 * w + (l & 31);     // this lane's packed row
    const bool in = m < a.rows;
    const RowOf row(in ? m : 0, hk, a.G);
    const bool on = in && row.i < ql;

    int j0 = 0, kend = kl;
    if (a.splits > 1) {
        j0 = sp * a.split_keys;
        if (kl - j0 > a.split_keys) kend = j0 + a.split_keys;       // (the last part's end may lie beyond 2^31)
    }
    if ((rt * 32 * NW) / a.G >= ql) kend = 0;           // no row of the tile is there

    typename Op<T>::V q[NS];
    load_frags<T, DC>(q, on ? static_cast<const T *>(a.Q) + b * a.q.b + row.i * a.q.l + row.h * a.q.h : nullptr, a.Dh, VEC, l);
    // scores in units of log 2; a negative scale turns the queries round, so
    // that the largest product is the largest score
    const float c = fabsf(a.scale) * LOG2E;
    if (a.scale < 0) {
#pragma unroll
        for (int s = 0; s < NS; ++s) q[s] = -q[s];
    }
    const T *const K = static_cast<const T *>(a.K) + b * a.k.b + hk * a.k.h;
    const T *const V = static_cast<const T *>(a.V) + b * a.v.b + hk * a.v.h;
    LiveKeys<BN> keys{a.mask ? a.mask + b * a.mask_ld : nullptr, kend, l, 0};

    f16v o[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[j] = f16v{0};
    float mx = -INFINITY, sum = 0.f;

    TileLoad<T, DP, BN, NT, VEC> kr, vr;
    uint64_t live = 0, next_live = 0;
    auto fetch = [&](int j, uint64_t on) {
        kr.fetch(K + (int64_t)j * a.k.l, a.k.l, on, a.Dh, t);
        vr.fetch(V + (int64_t)j * a.v.l, a.v.l, on, a.Dh, t);
    };
    char *kt = lds + group * 4 * TILE, *vt = kt + TILE;       // the tile in use; the next goes 2 TILE on, or back
    int other = 2 * TILE;
    if (j0 < kend) {
        keys.ahead(j0 + mine);
        live = keys.take(j0 + mine);
        keys.ahead(j0 + STEP + mine);
        fetch(j0 + mine, live);
        kr.stash(kt, t);
        vr.stash(vt, t);
        if (j0 + STEP < kend) {
            next_live = keys.take(j0 + STEP + mine);
            keys.ahead(j0 + 2 * STEP + mine);
            fetch(j0 + STEP + mine, next_live);
        }
    }
    for (; j0 < kend; j0 += STEP) {
        lds_barrier();
        f16v p[BN / 32];
#pragma unroll
        for (int n = 0; n < BN / 32; ++n) {
            p[n] = f16v{0};
#pragma unroll
            for (int s = 0; s < NS; ++s) p[n] = Op<T>::mma(row_frag<T, DP>(kt, 32 * n, s, l), q[s], p[n]);
        }
        if (live != ALL_LIVE<BN>) {
#pragma unroll
            for (int n = 0; n < BN / 32; ++n) {
                const uint32_t bits = (uint32_t)(live >> (32 * n)) >> (4 * (l >> 5));
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!((bits >> (8 * (r / 4) + r % 4)) & 1)) p[n][r] = -INFINITY;
            }
        }
        float top = p[0][0];
#pragma unroll
        for (int n = 0; n < BN / 32; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, p[n][r]);
        top = fmaxf(top, other_half(top)) * c;          // -inf * 0 is NaN: c is not 0 (see the entry point)
        // The reference that exponents are taken from follows the maximum only
        // when that has risen by 2^8: sums and probabilities up to 2^8 times
        // larger cost no precision, and the weighted sum is rarely rescaled.
        if (__any(top > mx + 8.f)) {
            const float next = fmaxf(mx, top);
            const float turn = __builtin_amdgcn_exp2f(mx - (next == -INFINITY ? 0.f : next));
            mx = next;
            sum *= turn;
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[j] *= turn;
        }
        const float ref = mx == -INFINITY ? 0.f : mx;
        float part = 0.f;
#pragma unroll
        for (int n = 0; n < BN / 32; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                p[n][r] = __builtin_amdgcn_exp2f(fmaf(p[n][r], c, -ref));
                part += p[n][r];
            }
        sum += part;
#pragma unroll
        for (int n = 0; n < BN / 32; ++n)
#pragma unroll
            for (int s = 0; s < 16 / PER; ++s) {
                const typename Op<T>::V pf = Op<T>::pack(p[n], s);
#pragma unroll
                for (int j = 0; j < NJ; ++j) o[j] = Op<T>::mma(col_frag<T, DP>(vt, 32 * n, s, j, l), pf, o[j]);
            }
        kt += other;
        vt += other;
        other = -other;
        live = next_live;
        if (j0 + STEP < kend) {
            kr.stash(kt, t);
            vr.stash(vt, t);
            if (j0 + 2 * STEP < kend) {
                next_live = keys.take(j0 + 2 * STEP + mine);
                keys.ahead(j0 + 3 * STEP + mine);
                fetch(j0 + 2 * STEP + mine, next_live);
            }
        }
    }
    sum += other_half(sum);
    if constexpr (GR == 2) {        // the second group's share, through LDS
        f4v *const share = reinterpret_cast<f4v *>(lds) + w * NJ * 256 + l;
        f2v *const state = reinterpret_cast<f2v *>(lds + NW * NJ * 4096) + 64 * w + l;
        __syncthreads();
        if (group) {
            *state = f2v{mx, sum};
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    share[64 * (4 * j + g)] = f4v{o[j][4 * g], o[j][4 * g + 1], o[j][4 * g + 2], o[j][4 * g + 3]};
        }
        __syncthreads();
        if (group) return;
        const f2v theirs = *state;
        const float next = fmaxf(mx, theirs[0]), ref = next == -INFINITY ? 0.f : next;
        const float x = __builtin_amdgcn_exp2f(mx - ref), y = __builtin_amdgcn_exp2f(theirs[0] - ref);
        mx = next;
        sum = sum * x + theirs[1] * y;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f4v v = share[64 * (4 * j + g)];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][4 * g + e] = o[j][4 * g + e] * x + v[e] * y;
            }
    }
    if (!in) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const float lse = on && sum != 0.f ? (mx + __builtin_amdgcn_logf(sum)) * LN2 : -INFINITY;
    if (a.splits > 1) {
        const int64_t at = ((int64_t)bh * a.rows + m) * a.splits + sp;
        float *const po = a.part + at * DP;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f4v v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = o[j][4 * g + e] * inv;
                *reinterpret_cast<f4v *>(po + 32 * j + 8 * g + 4 * (l >> 5)) = v;
            }
        if (l < 32) a.part_lse[at] = lse;
        return;
    }
    T *const out = static_cast<T *>(a.O) + b * a.o.b + row.i * a.o.l + row.h * a.o.h;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f4v v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = on ? o[j][4 * g + e] * inv : 0.f;
            store4<T>(out, 32 * j + 8 * g + 4 * (l >> 5), a.Dh, VEC, v);
        }
    if (a.lse && l < 32) a.lse[((int64_t)b * a.Hq + row.h) * a.Lq + row.i] = lse;
}

// Joins the parts of a row: O = sum_s exp(lse_s - lse) O_s, DP / 4 lanes a row.
template <typename T, int DP>
__global__ void __launch_bounds__(256) xattn_join_kernel(CrossAttnArgs a) {
    constexpr int LANES = DP / 4;
    const int64_t at = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int d = 4 * (threadIdx.x % LANES);
    if (at >= (int64_t)a.B * a.Hkv * a.rows || d >= a.Dh) return;
    const int bh = (int)(at / a.rows), m = (int)(at % a.rows);
    const int b = bh / a.Hkv;
    const RowOf row(m, bh % a.Hkv, a.G);
    const bool on = row.i < clamped(a.qlen, b, a.Lq);
    const float *const pl = a.part_lse + at * a.splits;
    const float *const po = a.part + at * a.splits * DP + d;
    float top = -INFINITY, sum = 0.f;
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, pl[s]);
    const float ref = top == -INFINITY ? 0.f : top;
    f4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) {
        const float e = __builtin_amdgcn_exp2f((pl[s] - ref) * LOG2E);
        sum += e;
        o += e * *reinterpret_cast<const f4v *>(po + s * DP);
    }
    const float inv = on && sum != 0.f ? 1.f / sum : 0.f;
    f4v v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = on ? o[e] * inv : 0.f;
    store4<T>(static_cast<T *>(a.O) + b * a.o.b + row.i * a.o.l + row.h * a.o.h, d, a.Dh, a.vec, v);
    if (a.lse && d == 0)
        a.lse[((int64_t)b * a.Hq + row.h) * a.Lq + row.i] =
            on && sum != 0.f ? ref + __builtin_amdgcn_logf(sum) * LN2 : -INFINITY;
}

// Keys a tile: 16 KB each of K and V at 128 values for work-groups of four
// waves; half of that for single waves, of which more share a CU.
constexpr int tile_keys(gs_dtype t, int waves) { return t == GS_F32 || waves == 1 ? 32 : 64; }

// How the rows and keys are dealt out.  Up to 32 rows (a few positions) go to
// single waves, eight a CU in all if there are keys enough, in parts of at least
// 128 keys in bf16 and, as products take eight times as long there, 32 (one tile)
// in fp32 (4 sequences of 4 x 240, 4 heads of 96 values over one: 13 us, 31 in
// parts of 128).  More rows go to work-groups of four or eight waves (33
// sequences of 19 x 3741, 2 heads of 72 values over one: bf16 22 us, 28 in single
// waves; fp32 81 and 110).
struct Plan {
    int waves, splits, split_keys, row_tiles, dp;
};
Plan plan_for(gs_dtype t, int64_t B, int64_t Lq, int64_t Lk, int64_t Hq, int64_t Hkv, int64_t Dh) {
    Plan p{};
    const int64_t rows = Lq * (Hq / Hkv);
    const int dc = computed(Dh);
    const bool few = rows <= 32;
    p.dp = padded(dc);
    p.row_tiles = (int)((rows + (few ? 31 : 127)) / (few ? 32 : 128));
    const int64_t blocks = B * Hkv * p.row_tiles, tile = tile_keys(t, few ? 1 : 4);
    int64_t per;
    if (few) {
        p.waves = 1;
        const int64_t least = t == GS_F32 ? 32 : 128, want = 2048 / (blocks > 0 ? blocks : 1);
        per = (Lk + (want > 1 ? want : 1) - 1) / (want > 1 ? want : 1);
        if (per < least) per = least;
    } else {
        // (us a tile, measured: bf16 2.7 for heads of 128, 1.4 for 64; fp32 6.0 and 5.8)
        const bool single = t == GS_F32 && dc > 64;
        const double us = t == GS_F32 ? (single ? 0.047 * dc : 5.8) : 0.021 * dc;
        const Deal d = deal_out(blocks, (Lk + tile - 1) / tile, single, us, (double)(B * Hkv * rows) * (p.dp * 8) / 4.5e6);
        p.waves = d.waves;
        per = (Lk + d.parts - 1) / d.parts;
    }
    per = (per + tile - 1) / tile * tile;
    p.split_keys = (int)per;
    p.splits = per ? (int)((Lk + per - 1) / per) : 1;
    if (p.splits < 1) p.splits = 1;
    return p;
}

template <typename T, int DC, int NW, int GR, bool VEC>
hipError_t launch_rows(const CrossAttnArgs &a, hipStream_t s) {
    constexpr int DP = padded(DC), BN = tile_keys(sizeof(T) == 4 ? GS_F32 : GS_BF16, NW);
    xattn_kernel<T, DC, NW, GR, BN, VEC><<<dim3((unsigned)((a.groups + 7) / 8 * 8)), dim3(64 * NW * GR), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t rows = (int64_t)a.B * a.Hkv * a.rows, per = 256 / (DP / 4);
    xattn_join_kernel<T, DP><<<dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int DC, bool VEC> hipError_t launch_waves(const CrossAttnArgs &a, const Plan &p, hipStream_t s) {
    if (p.waves == 1) return launch_rows<T, DC, 1, 1, VEC>(a, s);
    if constexpr (sizeof(T) == 2 || DC == 64)
        if (p.waves == 8) return launch_rows<T, DC, 4, 2, VEC>(a, s);
    return launch_rows<T, DC, 4, 1, VEC>(a, s);
}
template <typename T, bool VEC> hipError_t launch_typed(const CrossAttnArgs &a, const Plan &p, hipStream_t s) {
    const int dc = computed(a.Dh);
    if (dc == 64) return launch_waves<T, 64, VEC>(a, p, s);
    return dc == 96 ? launch_waves<T, 96, VEC>(a, p, s) : launch_waves<T, 128, VEC>(a, p, s);
}

}  // namespace

size_t cross_attn_workspace(gs_dtype t, int64_t B, int64_t Lq, int64_t Lk, int64_t Hq, int64_t Hkv, int64_t Dh) {
    const Plan p = plan_for(t, B, Lq, Lk, Hq, Hkv, Dh);
    if (p.splits == 1) return 0;
    return (size_t)(B * Lq * Hq) * p.splits * (p.dp + 1) * 4;
}

hipError_t launch_cross_attn(gs_dtype t, CrossAttnArgs a, void *ws, hipStream_t s) {
    const Plan p = plan_for(t, a.B, a.Lq, a.Lk, a.Hq, a.Hkv, a.Dh);
    a.rows = a.Lq * a.G;
    a.row_tiles = p.row_tiles;
    a.splits = p.splits;
    a.split_keys = p.split_keys;
    a.groups = (int64_t)a.B * a.Hkv * p.row_tiles * p.splits;
    a.part = static_cast<float *>(ws);
    a.part_lse = a.part + (int64_t)a.B * a.Hkv * a.rows * p.splits * p.dp;
    // tiles are read with 32-bit offsets: rows of a tile within 2^31 bytes
    a.vec = a.vec && a.k.l < ATTN_VEC_STRIDE && a.v.l < ATTN_VEC_STRIDE;
    if (t == GS_F32) return a.vec ? launch_typed<float, true>(a, p, s) : launch_typed<float, false>(a, p, s);
    return a.vec ? launch_typed<bf16_t, true>(a, p, s) : launch_typed<bf16_t, false>(a, p, s);
}

}  // namespace gs
