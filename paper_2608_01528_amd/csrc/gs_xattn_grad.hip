// Gradient of cross attention.  With S = scale Q K^T, P = exp(S - lse) and
// D_i = sum_d dO_id O_id:
//   dV = P^T dO     dP = dO V^T     dS = P (dP - D)
//   dQ = scale dS K                 dK = scale dS^T Q
// Two passes form P again instead of storing it: one over the keys for each
// block of query rows (D and dQ), one over the query rows for each block of keys
// (dK and dV).  A joint pass would save two of the seven
// products, but one of its gradients would have to be summed across
// work-groups in an order that changes from run to run; here every sum has a
// fixed order.  Where there are few blocks, two halves of a work-group share
// the range that a block runs over, and it may be split into parts whose sums a
// last pass adds up.
//
// Bound by the matrix cores, the exponentials and the LDS reads between their
// products: 4 x 16 heads of 2048 x 2048, 128 values, bf16: dQ 225 us (three
// products, 920 TF/s), dK and dV 340 (four, 810 TF/s); fp32, 8 x 4 heads of
// 1024 x 1024, 64 values: dQ 125 us (103 TF/s of 152; the matrix cores are busy
// 75 % of its cycles), dK and dV 160 (107; 79 %).
#include "gs_attn.h"

namespace gs {
namespace {
using namespace attn;

// Adds the sums of a work-group's second four waves to those of its first four;
// true for the second, which have no more to do.
template <int N> __device__ __forceinline__ bool add_groups(f16v (&o)[N], char *lds, int group, int w, int l) {
    f4v *const share = reinterpret_cast<f4v *>(lds) + w * N * 256 + l;
    __syncthreads();
    if (group) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                share[64 * (4 * j + g)] = f4v{o[j][4 * g], o[j][4 * g + 1], o[j][4 * g + 2], o[j][4 * g + 3]};
    }
    __syncthreads();
    if (group) return true;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f4v v = share[64 * (4 * j + g)];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][4 * g + e] += v[e];
        }
    return false;
}

// 32 query rows a wave as columns, keys streamed through LDS, by GR groups of
// four waves in turn.
template <typename T, int DC, int GR, int BN, bool VEC>
__global__ void __launch_bounds__(256 * GR, (sizeof(T) == 4 && DC > 64 ? 1 : 2)) xattn_dq_kernel(CrossAttnGradArgs a) {
    constexpr int DP = padded(DC), PER = Op<T>::PER, NS = DC / (2 * PER), NJ = DC / 32, TILE = BN * DP * sizeof(T);
    constexpr int STEP = GR * BN;
    __shared__ __attribute__((aligned(16))) char lds[GR * 4 * TILE];
    const int t = threadIdx.x % 256, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int group = GR > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 256) : 0, mine = group * BN;
    const int64_t L = logical_group(a.q_groups);
    if (L >= a.q_groups) return;
    const int rt = (int)(L % a.row_tiles);
    const int64_t rest = L / a.row_tiles;
    const int sp = (int)(rest % a.q_parts), bh = (int)(rest / a.q_parts);
    const int b = bh / a.Hkv, hk = bh % a.Hkv;
    const int ql = clamped(a.qlen, b, a.Lq), kl = clamped(a.klen, b, a.Lk);
    const int m = rt * 128 + 32 * w + (l & 31);
    const bool in = m < a.rows;
    const RowOf row(in ? m : 0, hk, a.G);
    const bool on = in && row.i < ql;
    int j0 = sp * a.q_step, kend = kl - j0 > a.q_step ? j0 + a.q_step : kl;      // (the last part's end may lie beyond 2^31)
    if (rt * 128 / a.G >= ql) kend = 0;

    typename Op<T>::V q[NS], d[NS];
    load_frags<T, DC>(q, on ? static_cast<const T *>(a.Q) + b * a.q.b + row.i * a.q.l + row.h * a.q.h : nullptr, a.Dh, VEC, l);
    load_frags<T, DC>(d, on ? static_cast<const T *>(a.dO) + b * a.d.b + row.i * a.d.l + row.h * a.d.h : nullptr, a.Dh, VEC, l);
    // What both passes need of a row: -lse in units of log 2, the constant of the
    // exponent (minus infinity, so that exp2 gives 0, for rows that are not there
    // and rows without a live key), and D.
    const int64_t at_row = ((int64_t)b * a.Hq + row.h) * a.Lq + row.i;
    f2v st = {-INFINITY, 0.f};
    // Live states of the sequence, as far as `few` asks (the first 128 mask bytes
    // come with the rows above them: no time that shows).
    const uint8_t *const mask = a.mask ? a.mask + b * a.mask_ld : nullptr;
    int states = kl;
    if (mask && kl > BN) {
        states = 0;
        for (int j = 0; j < kl && states <= BN; j += 128) {
            const bool x = j + l < kl && mask[j + l], y = kl - j > 64 + l && mask[j + 64 + l];
            states += __popcll(__ballot(x)) + __popcll(__ballot(y));
        }
    }
    const bool few = states <= BN && j0 < kend;
    {
        typename Op<T>::V y[NS];
        load_frags<T, DC>(y, on ? static_cast<const T *>(a.O) + b * a.o.b + row.i * a.o.l + row.h * a.o.h : nullptr, a.Dh, VEC, l);
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int e = 0; e < PER; ++e) st[1] = fmaf((float)d[s][e], (float)y[s][e], st[1]);
        st[1] += other_half(st[1]);
        if (on) st[0] = -LOG2E * a.lse[at_row];
        if (st[0] == INFINITY) st[0] = -INFINITY;
    }
    const float c = a.scale * LOG2E;
    const T *const K = static_cast<const T *>(a.K) + b * a.k.b + hk * a.k.h;
    const T *const V = static_cast<const T *>(a.V) + b * a.v.b + hk * a.v.h;
    LiveKeys<BN> keys{mask, kend, l, 0};

    f16v o[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[j] = f16v{0};
    TileLoad<T, DP, BN, 256, VEC> kr, vr;
    uint64_t live = 0, next_live = 0;
    auto fetch = [&](int j, uint64_t alive) {
        kr.fetch(K + (int64_t)j * a.k.l, a.k.l, alive, a.Dh, t);
        vr.fetch(V + (int64_t)j * a.v.l, a.v.l, alive, a.Dh, t);
    };
    char *kt = lds + group * 4 * TILE, *vt = kt + TILE;
    int other = 2 * TILE;
    if (few) {
        // A tile's worth of states at most: D as the sum of P dP over them, in
        // fp32.  sum_d dO O has the rounding of O in it (half a step of T, 2^-8 in
        // bf16, of sum_d |dO O| at most), which dP - D keeps, and which is small
        // beside dP only where O is an average over many rows of V.  Every
        // work-group of the row and each of its groups goes over all of them.
        float D = 0.f;
        LiveKeys<BN> all{mask, kl, l, 0};
#pragma unroll 1
        for (int j = 0; j < kl; j += BN) {
            all.ahead(j);
            live = all.take(j);
            if (!live) continue;
            lds_barrier();
            fetch(j, live);
            kr.stash(kt, t);
            vr.stash(vt, t);
            lds_barrier();
#pragma unroll 1
            for (int n = 0; n < BN / 32; ++n) {
                f16v p = {0}, g = {0};
#pragma unroll
                for (int s = 0; s < NS; ++s) p = Op<T>::mma(row_frag<T, DP>(kt, 32 * n, s, l), q[s], p);
#pragma unroll
                for (int s = 0; s < NS; ++s) g = Op<T>::mma(row_frag<T, DP>(vt, 32 * n, s, l), d[s], g);
                // (a dead key's score is 0 here, which a row of very negative scores
                // makes an infinite probability)
                const uint32_t bits = (uint32_t)(live >> (32 * n)) >> (4 * (l >> 5));
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    D += (bits >> (8 * (r / 4) + r % 4)) & 1 ? __builtin_amdgcn_exp2f(fmaf(p[r], c, st[0])) * g[r] : 0.f;
            }
        }
        st[1] = D + other_half(D);
        lds_barrier();
    }
    if (on && l < 32 && !group && sp == 0) a.stat[at_row] = st;
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
#pragma unroll 1
        for (int n = 0; n < BN / 32; ++n) {
            f16v p = {0}, g = {0};
#pragma unroll
            for (int s = 0; s < NS; ++s) p = Op<T>::mma(row_frag<T, DP>(kt, 32 * n, s, l), q[s], p);
#pragma unroll
            for (int s = 0; s < NS; ++s) g = Op<T>::mma(row_frag<T, DP>(vt, 32 * n, s, l), d[s], g);
#pragma unroll
            for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], c, st[0])) * (g[r] - st[1]);
            if (live != ALL_LIVE<BN>) {
                // (dead keys are zeros in LDS: their score is 0, not minus infinity)
                const uint32_t bits = (uint32_t)(live >> (32 * n)) >> (4 * (l >> 5));
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!((bits >> (8 * (r / 4) + r % 4)) & 1)) p[r] = 0.f;
            }
#pragma unroll
            for (int s = 0; s < 16 / PER; ++s) {
                const typename Op<T>::V pf = Op<T>::pack(p, s);
#pragma unroll
                for (int j = 0; j < NJ; ++j) o[j] = Op<T>::mma(col_frag<T, DP>(kt, 32 * n, s, j, l), pf, o[j]);
            }
        }
        if constexpr (sizeof(T) == 4 && GR == 2) products_done(o);
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
    if constexpr (GR == 2) {
        if (add_groups<NJ>(o, lds, group, w, l)) return;
    }
    if (!in) return;
    float *const part = a.q_parts > 1 ? a.dq_part + (((int64_t)sp * a.B * a.Hkv + bh) * a.rows + m) * DP : nullptr;
    T *const out = static_cast<T *>(a.dQ) + b * a.dq.b + row.i * a.dq.l + row.h * a.dq.h;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f4v v;
            const int at = 32 * j + 8 * g + 4 * (l >> 5);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = on ? o[j][4 * g + e] * a.scale : 0.f;
            if (part) *reinterpret_cast<f4v *>(part + at) = v;
            else store4<T>(out, at, a.Dh, VEC, v);
        }
}

// 32 keys a wave as columns, query rows streamed through LDS: the positions of
// one head after those of another, for all heads that share the keys.
// The keys' rows of V stay in registers, and so do those of K where two waves
// a SIMD then still fit (256 registers each); bf16 rows of 128 values leave K
// in LDS, fp32 ones run one wave a SIMD.  (4 x 16 heads of 2048 x 2048, bf16: one
// wave a SIMD 443 us; two, with tiles through registers, which spill, 430; two,
// tiles straight to LDS, 348.)
template <typename T, int DC, int GR, bool VEC>
__global__ void __launch_bounds__(256 * GR, (sizeof(T) == 4 && DC > 64 ? 1 : 2)) xattn_dkv_kernel(CrossAttnGradArgs a) {
    constexpr int DP = padded(DC), PER = Op<T>::PER, NS = DC / (2 * PER), NJ = DC / 32, BM = 32, TILE = BM * DP * sizeof(T);
    constexpr bool KEEP_K = !(sizeof(T) == 2 && DC == 128);
    __shared__ __attribute__((aligned(16))) char lds[GR * 4 * TILE + (KEEP_K ? 0 : GR * 128 * DP * sizeof(T))];
    __shared__ __attribute__((aligned(16))) f2v stat[GR * 2 * BM];
    const int t = threadIdx.x % 256, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int group = GR > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 256) : 0;
    char *const own = lds + group * 4 * TILE, *const keys_lds = lds + GR * 4 * TILE + group * 128 * DP * sizeof(T);
    const int64_t L = logical_group(a.k_groups);
    if (L >= a.k_groups) return;
    const int kt = (int)(L % a.key_tiles);
    const int64_t rest = L / a.key_tiles;
    const int sp = (int)(rest % a.k_parts), bh = (int)(rest / a.k_parts);
    const int b = bh / a.Hkv, hk = bh % a.Hkv;
    const int ql = clamped(a.qlen, b, a.Lq), kl = clamped(a.klen, b, a.Lk);
    const int j = kt * 128 + 32 * w + (l & 31);         // this lane's key
    const bool in = j < a.Lk;
    bool on = j < kl;
    if (on && a.mask) on = a.mask[b * a.mask_ld + j] != 0;

    // tiles of 32 positions, `tiles` a head; this part's run of them, which the
    // groups of four waves take in turn
    const int tiles = kt * 128 < kl ? (ql + BM - 1) / BM : 0;
    // (below 2^31, as B Hq Lq is; divided once, kept in scalar registers)
    const int64_t total = (int64_t)tiles * a.G;
    const int first = __builtin_amdgcn_readfirstlane((int)(total * sp / a.k_parts));
    const int end = __builtin_amdgcn_readfirstlane((int)(total * (sp + 1) / a.k_parts));
    int n = first + group;
    int g = __builtin_amdgcn_readfirstlane(tiles ? n / tiles : 0), x = n - g * tiles;     // head and tile of the next fetch

    typename Op<T>::V k[NS], v[NS];
    load_frags<T, DC>(k, on ? static_cast<const T *>(a.K) + b * a.k.b + j * a.k.l + hk * a.k.h : nullptr, a.Dh, VEC, l);
    if constexpr (!KEEP_K) {    // (read back by the wave that writes them)
#pragma unroll
        for (int y = 0; y < NS; ++y)
            *reinterpret_cast<typename Op<T>::V *>(keys_lds + place<T, DP>(32 * w + (l & 31), 2 * y + (l >> 5))) = k[y];
    }
    load_frags<T, DC>(v, on ? static_cast<const T *>(a.V) + b * a.v.b + j * a.v.l + hk * a.v.h : nullptr, a.Dh, VEC, l);
    const float c = a.scale * LOG2E;
    f16v dk[NJ], dv[NJ];
#pragma unroll
    for (int y = 0; y < NJ; ++y) dk[y] = f16v{0}, dv[y] = f16v{0};

    // VEC: tiles go straight to LDS, the next while one is used; otherwise
    // through registers, each when it is needed
    TileLoad<T, DP, BM, 256, false> qr, dr;
    f2v st = {-INFINITY, 0.f};
    char *qt = own, *dt = own + TILE;
    f2v *ss = stat + group * 2 * BM;
    int other = 2 * TILE, other_s = BM;
    auto fetch = [&](char *to) {
        const int i0 = x * BM, h = hk * a.G + g;
        const T *const Q = static_cast<const T *>(a.Q) + b * a.q.b + (int64_t)i0 * a.q.l + h * a.q.h;
        const T *const O = static_cast<const T *>(a.dO) + b * a.d.b + (int64_t)i0 * a.d.l + h * a.d.h;
        if constexpr (VEC) {
            TileDma<T, DP, BM, 256>::issue(Q, a.q.l, ql - 1 - i0, a.Dh, to, t);
            TileDma<T, DP, BM, 256>::issue(O, a.d.l, ql - 1 - i0, a.Dh, to + TILE, t);
        } else {
            const uint64_t alive = ql - i0 >= BM ? ALL_LIVE<BM> : (1ull << (ql - i0)) - 1;
            qr.fetch(Q, a.q.l, alive, a.Dh, t);
            dr.fetch(O, a.d.l, alive, a.Dh, t);
        }
        if (t < BM) st = i0 + t < ql ? (a.stat + ((int64_t)b * a.Hq + h) * a.Lq + i0)[t] : f2v{-INFINITY, 0.f};
        for (x += GR; x >= tiles; x -= tiles) ++g;
    };
    clear_lds<256>(own, 4 * TILE, t);
    lds_barrier();
    if (VEC && n < end) fetch(qt);
    for (int n0 = first; n0 < end; n0 += GR, n += GR) {
        if constexpr (VEC) {
            wait_tiles();
        } else if (n < end) {
            fetch(qt);
            qr.stash(qt, t);
            dr.stash(dt, t);
        }
        if (t < BM) ss[t] = st;
        lds_barrier();
        if (n + GR < end) {
            if constexpr (VEC) fetch(qt + other);
        } else if (GR > 1) {
            // No tile is left for the next turn, if there is one (of the other
            // group): this one goes over what it has once more, at weight 0.
            st = f2v{-INFINITY, 0.f};
        }
        f16v p = {0}, s = {0};
#pragma unroll
        for (int y = 0; y < NS; ++y) {
            const typename Op<T>::V ky = KEEP_K ? k[y] : row_frag<T, DP>(keys_lds, 32 * w, y, l);
            p = Op<T>::mma(row_frag<T, DP>(qt, 0, y, l), ky, p);
        }
#pragma unroll
        for (int y = 0; y < NS; ++y) s = Op<T>::mma(row_frag<T, DP>(dt, 0, y, l), v[y], s);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const f4v *const sy = reinterpret_cast<const f4v *>(ss + 8 * y + 4 * (l >> 5));
            const f4v two[2] = {sy[0], sy[1]};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * y + e;
                p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], c, two[e / 2][2 * (e % 2)]));
                s[r] = p[r] * (s[r] - two[e / 2][2 * (e % 2) + 1]);
            }
        }
#pragma unroll
        for (int y = 0; y < 16 / PER; ++y) {
            const typename Op<T>::V pf = Op<T>::pack(p, y), sf = Op<T>::pack(s, y);
#pragma unroll
            for (int z = 0; z < NJ; ++z) dv[z] = Op<T>::mma(col_frag<T, DP>(dt, 0, y, z, l), pf, dv[z]);
#pragma unroll
            for (int z = 0; z < NJ; ++z) dk[z] = Op<T>::mma(col_frag<T, DP>(qt, 0, y, z, l), sf, dk[z]);
        }
        qt += other;
        dt += other;
        ss += other_s;
        other = -other;
        other_s = -other_s;
    }
    if constexpr (GR == 2) {
        add_groups<NJ>(dk, lds, group, w, l);
        if (add_groups<NJ>(dv, lds, group, w, l)) return;
    }
    if (!in) return;
    const int64_t keys = (int64_t)a.B * a.Hkv * a.Lk;
    float *const part = a.k_parts > 1 ? a.dkv_part + (2 * sp * keys + (int64_t)bh * a.Lk + j) * DP : nullptr;
    T *const ok = static_cast<T *>(a.dK) + b * a.dk.b + j * a.dk.l + hk * a.dk.h;
    T *const ov = static_cast<T *>(a.dV) + b * a.dv.b + j * a.dv.l + hk * a.dv.h;
#pragma unroll
    for (int z = 0; z < NJ; ++z)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            f4v kv, vv;
            const int at = 32 * z + 8 * y + 4 * (l >> 5);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                kv[e] = on ? dk[z][4 * y + e] * a.scale : 0.f;
                vv[e] = on ? dv[z][4 * y + e] : 0.f;
            }
            if (part) {
                *reinterpret_cast<f4v *>(part + at) = kv;
                *reinterpret_cast<f4v *>(part + keys * DP + at) = vv;
            } else {
                store4<T>(ok, at, a.Dh, VEC, kv);
                store4<T>(ov, at, a.Dh, VEC, vv);
            }
        }
}

// Adds up the parts of a row, DP / 4 lanes a row: rows of dQ first, then those
// of dK and of dV.
template <typename T, int DP, bool VEC>
__global__ void __launch_bounds__(256) xattn_parts_kernel(CrossAttnGradArgs a) {
    constexpr int LANES = DP / 4;
    const int d = 4 * (threadIdx.x % LANES);
    int64_t at = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int64_t qrows = (int64_t)a.B * a.Hkv * a.rows, keys = (int64_t)a.B * a.Hkv * a.Lk;
    if (d >= a.Dh) return;
    const float *p;
    T *out;
    int parts;
    int64_t step;
    if (at < a.join_q) {
        p = a.dq_part + at * DP;
        parts = a.q_parts;
        step = qrows * DP;
        const int bh = (int)(at / a.rows);
        const RowOf row((int)(at % a.rows), bh % a.Hkv, a.G);
        out = static_cast<T *>(a.dQ) + bh / a.Hkv * a.dq.b + row.i * a.dq.l + row.h * a.dq.h;
    } else {
        at -= a.join_q;
        if (at >= a.join_k) return;
        p = a.dkv_part + at * DP;
        parts = a.k_parts;
        step = 2 * keys * DP;
        const bool is_v = at >= keys;
        if (is_v) at -= keys;
        const int bh = (int)(at / a.Lk), j = (int)(at % a.Lk);
        const SeqStrides z = is_v ? a.dv : a.dk;
        out = static_cast<T *>(is_v ? a.dV : a.dK) + bh / a.Hkv * z.b + j * z.l + bh % a.Hkv * z.h;
    }
    f4v v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < parts; ++s) v += *reinterpret_cast<const f4v *>(p + s * step + d);
    store4<T>(out, d, a.Dh, VEC, v);
}

struct Plan {
    int dp, q_waves, q_parts, q_step, k_waves, k_parts;
};
Plan plan_for(gs_dtype t, int64_t B, int64_t Lq, int64_t Lk, int64_t Hq, int64_t Hkv, int64_t Dh) {
    Plan p{};
    const int dc = computed(Dh);
    const int64_t G = Hq / Hkv, unit = t == GS_F32 ? 32 : 64;
    const bool single = t == GS_F32 && dc > 64;
    p.dp = padded(dc);
    // us a tile, measured: dQ, 64 or 32 keys: bf16 3.4 for heads of 128, 1.9 for
    // 64; fp32 9.3 and 7.9.  dK and dV, 32 query rows: 2.7, 1.5; 12.5, 10.
    const double dq_us = t == GS_F32 ? (single ? 0.073 * dc : 7.9) : 0.027 * dc;
    const double dkv_us = t == GS_F32 ? (single ? 0.098 * dc : 10.) : 0.021 * dc;
    const double row_us = (double)(p.dp * 8) / 4.5e6;
    const Deal q = deal_out(B * Hkv * ((Lq * G + 127) / 128), (Lk + unit - 1) / unit, single, dq_us, (double)(B * Hq * Lq) * row_us);
    const Deal k = deal_out(B * Hkv * ((Lk + 127) / 128), (Lq + 31) / 32 * G, single, dkv_us, (double)(B * Hkv * Lk) * 2 * row_us);
    const int64_t step = ((Lk + q.parts - 1) / q.parts + unit - 1) / unit * unit;
    p.q_waves = q.waves;
    p.q_step = (int)(step ? step : unit);
    p.q_parts = Lk ? (int)((Lk + step - 1) / step) : 1;
    p.k_waves = k.waves;
    p.k_parts = k.parts;
    return p;
}

template <typename T, int DC, bool VEC> hipError_t launch_sized(const CrossAttnGradArgs &a, const Plan &p, hipStream_t s) {
    constexpr int DP = padded(DC), BN = sizeof(T) == 4 ? 32 : 64;
    constexpr bool EIGHT = sizeof(T) == 2 || DC == 64;
    const auto grid = [](int64_t n, int64_t per) { return dim3((unsigned)((n + per - 1) / per)); };
    hipError_t e = hipSuccess;
    if (a.q_groups) {
        const dim3 groups((unsigned)((a.q_groups + 7) / 8 * 8));
        if (EIGHT && p.q_waves == 8) xattn_dq_kernel<T, DC, EIGHT ? 2 : 1, BN, VEC><<<groups, dim3(512), 0, s>>>(a);
        else xattn_dq_kernel<T, DC, 1, BN, VEC><<<groups, dim3(256), 0, s>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.k_groups) {
        const dim3 groups((unsigned)((a.k_groups + 7) / 8 * 8));
        if (EIGHT && p.k_waves == 8) xattn_dkv_kernel<T, DC, EIGHT ? 2 : 1, VEC><<<groups, dim3(512), 0, s>>>(a);
        else xattn_dkv_kernel<T, DC, 1, VEC><<<groups, dim3(256), 0, s>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.join_q + a.join_k) {
        xattn_parts_kernel<T, DP, VEC><<<grid(a.join_q + a.join_k, 256 / (DP / 4)), dim3(256), 0, s>>>(a);
        e = hipGetLastError();
    }
    return e;
}

template <typename T, bool VEC> hipError_t launch_typed(const CrossAttnGradArgs &a, const Plan &p, hipStream_t s) {
    const int dc = computed(a.Dh);
    if (dc == 64) return launch_sized<T, 64, VEC>(a, p, s);
    return dc == 96 ? launch_sized<T, 96, VEC>(a, p, s) : launch_sized<T, 128, VEC>(a, p, s);
}

int64_t align4(int64_t n) { return (n + 3) / 4 * 4; }     // (16-byte rows of parts behind the rows' constants)

}  // namespace

size_t cross_attn_grad_workspace(gs_dtype t, int64_t B, int64_t Lq, int64_t Lk, int64_t Hq, int64_t Hkv, int64_t Dh) {
    const Plan p = plan_for(t, B, Lq, Lk, Hq, Hkv, Dh);
    size_t n = (size_t)align4(2 * B * Lq * Hq);
    if (p.q_parts > 1) n += (size_t)(B * Lq * Hq) * p.q_parts * p.dp;
    if (p.k_parts > 1) n += (size_t)(B * Lk * Hkv) * 2 * p.k_parts * p.dp;
    return n * 4;
}

hipError_t launch_cross_attn_grad(gs_dtype t, CrossAttnGradArgs a, void *ws, hipStream_t s) {
    const Plan p = plan_for(t, a.B, a.Lq, a.Lk, a.Hq, a.Hkv, a.Dh);
    a.rows = a.Lq * a.G;
    a.row_tiles = (int)(((int64_t)a.rows + 127) / 128);
    a.key_tiles = (int)(((int64_t)a.Lk + 127) / 128);
    a.q_parts = p.q_parts;
    a.q_step = p.q_step;
    a.k_parts = p.k_parts;
    a.q_groups = (int64_t)a.B * a.Hkv * a.row_tiles * p.q_parts;
    a.k_groups = (int64_t)a.B * a.Hkv * a.key_tiles * p.k_parts;
    const int64_t qrows = (int64_t)a.B * a.Hq * a.Lq, keys = (int64_t)a.B * a.Hkv * a.Lk;
    a.join_q = p.q_parts > 1 ? qrows : 0;
    a.join_k = p.k_parts > 1 ? 2 * keys : 0;
    a.stat = static_cast<f2v *>(ws);
    a.dq_part = static_cast<float *>(ws) + align4(2 * qrows);
    a.dkv_part = a.dq_part + a.join_q * p.q_parts * p.dp;
    // tiles are read with 32-bit offsets: rows of a tile within 2^31 bytes
    for (const SeqStrides *x : {&a.q, &a.k, &a.v, &a.d}) a.vec = a.vec && x->l < ATTN_VEC_STRIDE;
    if (t == GS_F32) return a.vec ? launch_typed<float, true>(a, p, s) : launch_typed<float, false>(a, p, s);
    return a.vec ? launch_typed<bf16_t, true>(a, p, s) : launch_typed<bf16_t, false>(a, p, s);
}

}  // namespace gs
