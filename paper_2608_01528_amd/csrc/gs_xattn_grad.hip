// Gradient of cross attention.  With S = scale Q K^T, P = exp(S - lse) and
// D_i = sum_d dO_id O_id:
//   dV = P^T dO     dP = dO V^T     dS = P (dP - D)
//   dQ = scale dS K                 dK = scale dS^T Q
// Two passes form P again instead of storing it: one over the keys for each
// block of query rows (dQ, and D on the way), one over the query rows for each
// block of keys (dK and dV).  A joint pass would save two of the seven
// products, but one of its gradients would have to be summed across
// work-groups, in an order that changes from run to run; here every sum has a
// fixed order.
#include "gs_attn.h"

namespace gs {
namespace {
using namespace attn;

struct RowOf {
    int i, h;
    __device__ __forceinline__ RowOf(int m, int hk, int G) : i(m / G), h(hk * G + m % G) {}
};

// 32 query rows a wave as columns, keys streamed through LDS.
template <typename T, int DP, int BN>
__global__ void __launch_bounds__(256) xattn_dq_kernel(CrossAttnGradArgs a) {
    constexpr int PER = Op<T>::PER, NS = DP / (2 * PER), NJ = DP / 32, CPR = DP / PER;
    __shared__ __attribute__((aligned(16))) char lds[2 * BN * DP * sizeof(T)];
    char *const kt = lds, *const vt = lds + BN * DP * sizeof(T);
    const int t = threadIdx.x, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t L = logical_group(a.q_groups);
    if (L >= a.q_groups) return;
    const int rt = (int)(L % a.row_tiles), bh = (int)(L / a.row_tiles);
    const int b = bh / a.Hkv, hk = bh % a.Hkv;
    const int ql = clamped(a.qlen, b, a.Lq), kl = clamped(a.klen, b, a.Lk);
    const int m = rt * 128 + 32 * w + (l & 31);
    const bool in = m < a.rows;
    const RowOf row(in ? m : 0, hk, a.G);
    const bool on = in && row.i < ql;
    const int kend = rt * 128 / a.G >= ql ? 0 : kl;

    typename Op<T>::V q[NS], d[NS];
    float D = 0.f, lse2 = INFINITY;     // exp2(s - inf) = 0: rows that are not there, rows without a live key
    const int64_t at = ((int64_t)b * a.Hq + row.h) * a.Lq + row.i;
    {
        load_frags<T, DP>(q, on ? static_cast<const T *>(a.O) + b * a.o.b + row.i * a.o.l + row.h * a.o.h : nullptr, a.Dh, a.vec, l);
        load_frags<T, DP>(d, on ? static_cast<const T *>(a.dO) + b * a.d.b + row.i * a.d.l + row.h * a.d.h : nullptr, a.Dh, a.vec, l);
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int e = 0; e < PER; ++e) D = fmaf((float)q[s][e], (float)d[s][e], D);
        D += other_half(D);
        load_frags<T, DP>(q, on ? static_cast<const T *>(a.Q) + b * a.q.b + row.i * a.q.l + row.h * a.q.h : nullptr, a.Dh, a.vec, l);
        if (on) {
            lse2 = a.lse[at] * LOG2E;
            if (lse2 == -INFINITY) lse2 = INFINITY;
        }
        if (in && l < 32) a.D[at] = D;
    }
    const float c = a.scale * LOG2E;
    const T *const K = static_cast<const T *>(a.K) + b * a.k.b + hk * a.k.h;
    const T *const V = static_cast<const T *>(a.V) + b * a.v.b + hk * a.v.h;
    const uint8_t *const mask = a.mask ? a.mask + b * a.mask_ld : nullptr;

    f16v o[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[j] = f16v{0};
    for (int j0 = 0; j0 < kend; j0 += BN) {
        __syncthreads();
        // (dead keys are zeros: their scores are 0 here, and a factor of a row
        // of K in dQ is 0 whatever dS is, as long as that is finite)
        for (int x = t; x < BN * CPR; x += 256) {
            const int r = x / CPR, j = j0 + r;
            const bool ok = j < kend && (!mask || mask[j]);
            u4v kv = {0, 0, 0, 0}, vv = {0, 0, 0, 0};
            if (ok) {
                kv = load_chunk<T>(K + (int64_t)j * a.k.l, PER * (x % CPR), a.Dh, a.vec);
                vv = load_chunk<T>(V + (int64_t)j * a.v.l, PER * (x % CPR), a.Dh, a.vec);
            }
            *reinterpret_cast<u4v *>(kt + place<T, DP>(r, x % CPR)) = kv;
            *reinterpret_cast<u4v *>(vt + place<T, DP>(r, x % CPR)) = vv;
        }
        bool alive = l < BN && j0 + l < kend;
        if (alive && mask) alive = mask[j0 + l] != 0;
        const uint64_t live = __ballot(alive);
        __syncthreads();
#pragma unroll
        for (int n = 0; n < BN / 32; ++n) {
            f16v p = {0}, g = {0};
#pragma unroll
            for (int s = 0; s < NS; ++s) p = Op<T>::mma(row_frag<T, DP>(kt, 32 * n, s, l), q[s], p);
#pragma unroll
            for (int s = 0; s < NS; ++s) g = Op<T>::mma(row_frag<T, DP>(vt, 32 * n, s, l), d[s], g);
            const uint32_t bits = (uint32_t)(live >> (32 * n)) >> (4 * (l >> 5));
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float e = __builtin_amdgcn_exp2f(fmaf(p[r], c, -lse2));
                p[r] = (bits >> (8 * (r / 4) + r % 4)) & 1 ? e * (g[r] - D) : 0.f;
            }
#pragma unroll
            for (int s = 0; s < 16 / PER; ++s) {
                const typename Op<T>::V pf = Op<T>::pack(p, s);
#pragma unroll
                for (int j = 0; j < NJ; ++j) o[j] = Op<T>::mma(col_frag<T, DP>(kt, 32 * n, s, j, l), pf, o[j]);
            }
        }
    }
    if (!in) return;
    T *const out = static_cast<T *>(a.dQ) + b * a.dq.b + row.i * a.dq.l + row.h * a.dq.h;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f4v v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = on ? o[j][4 * g + e] * a.scale : 0.f;
            store4<T>(out, 32 * j + 8 * g + 4 * (l >> 5), a.Dh, a.vec, v);
        }
}

// 32 keys a wave as columns, query rows (of all heads that share the keys)
// streamed through LDS.
template <typename T, int DP>
__global__ void __launch_bounds__(256, 1) xattn_dkv_kernel(CrossAttnGradArgs a) {
    constexpr int PER = Op<T>::PER, NS = DP / (2 * PER), NJ = DP / 32, CPR = DP / PER, BM = 32;
    __shared__ __attribute__((aligned(16))) char lds[2 * BM * DP * sizeof(T)];
    __shared__ __attribute__((aligned(16))) float stat[2 * BM];
    char *const qt = lds, *const dt = lds + BM * DP * sizeof(T);
    const int t = threadIdx.x, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t L = logical_group(a.k_groups);
    if (L >= a.k_groups) return;
    const int kt = (int)(L % a.key_tiles), bh = (int)(L / a.key_tiles);
    const int b = bh / a.Hkv, hk = bh % a.Hkv;
    const int ql = clamped(a.qlen, b, a.Lq), kl = clamped(a.klen, b, a.Lk);
    const int j = kt * 128 + 32 * w + (l & 31);         // this lane's key
    const bool in = j < a.Lk;
    bool on = j < kl;
    if (on && a.mask) on = a.mask[b * a.mask_ld + j] != 0;
    const int rows = kt * 128 < kl ? ql * a.G : 0;

    typename Op<T>::V k[NS], v[NS];
    load_frags<T, DP>(k, on ? static_cast<const T *>(a.K) + b * a.k.b + j * a.k.l + hk * a.k.h : nullptr, a.Dh, a.vec, l);
    load_frags<T, DP>(v, on ? static_cast<const T *>(a.V) + b * a.v.b + j * a.v.l + hk * a.v.h : nullptr, a.Dh, a.vec, l);
    const float c = a.scale * LOG2E;
    f16v dk[NJ], dv[NJ];
#pragma unroll
    for (int n = 0; n < NJ; ++n) dk[n] = f16v{0}, dv[n] = f16v{0};
    for (int m0 = 0; m0 < rows; m0 += BM) {
        __syncthreads();
        for (int x = t; x < BM * CPR; x += 256) {
            const int r = x / CPR, m = m0 + r;
            u4v qv = {0, 0, 0, 0}, ov = {0, 0, 0, 0};
            if (m < rows) {
                const RowOf row(m, hk, a.G);
                qv = load_chunk<T>(static_cast<const T *>(a.Q) + b * a.q.b + row.i * a.q.l + row.h * a.q.h, PER * (x % CPR), a.Dh, a.vec);
                ov = load_chunk<T>(static_cast<const T *>(a.dO) + b * a.d.b + row.i * a.d.l + row.h * a.d.h, PER * (x % CPR), a.Dh, a.vec);
            }
            *reinterpret_cast<u4v *>(qt + place<T, DP>(r, x % CPR)) = qv;
            *reinterpret_cast<u4v *>(dt + place<T, DP>(r, x % CPR)) = ov;
        }
        if (t < BM) {
            float lse2 = INFINITY, D = 0.f;
            if (m0 + t < rows) {
                const RowOf row(m0 + t, hk, a.G);
                const int64_t at = ((int64_t)b * a.Hq + row.h) * a.Lq + row.i;
                lse2 = a.lse[at] * LOG2E;
                if (lse2 == -INFINITY) lse2 = INFINITY;
                D = a.D[at];
            }
            stat[t] = lse2;
            stat[BM + t] = D;
        }
        __syncthreads();
        f16v p = {0}, g = {0};
#pragma unroll
        for (int s = 0; s < NS; ++s) p = Op<T>::mma(row_frag<T, DP>(qt, 0, s, l), k[s], p);
#pragma unroll
        for (int s = 0; s < NS; ++s) g = Op<T>::mma(row_frag<T, DP>(dt, 0, s, l), v[s], g);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const f4v lse2 = *reinterpret_cast<const f4v *>(stat + 8 * x + 4 * (l >> 5));
            const f4v D = *reinterpret_cast<const f4v *>(stat + BM + 8 * x + 4 * (l >> 5));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * x + e;
                p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], c, -lse2[e]));
                g[r] = p[r] * (g[r] - D[e]);
            }
        }
#pragma unroll
        for (int s = 0; s < 16 / PER; ++s) {
            const typename Op<T>::V pf = Op<T>::pack(p, s), gf = Op<T>::pack(g, s);
#pragma unroll
            for (int n = 0; n < NJ; ++n) dv[n] = Op<T>::mma(col_frag<T, DP>(dt, 0, s, n, l), pf, dv[n]);
#pragma unroll
            for (int n = 0; n < NJ; ++n) dk[n] = Op<T>::mma(col_frag<T, DP>(qt, 0, s, n, l), gf, dk[n]);
        }
    }
    if (!in) return;
    T *const ok = static_cast<T *>(a.dK) + b * a.dk.b + j * a.dk.l + hk * a.dk.h;
    T *const ov = static_cast<T *>(a.dV) + b * a.dv.b + j * a.dv.l + hk * a.dv.h;
#pragma unroll
    for (int n = 0; n < NJ; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            f4v kv, vv;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                kv[e] = on ? dk[n][4 * x + e] * a.scale : 0.f;
                vv[e] = on ? dv[n][4 * x + e] : 0.f;
            }
            store4<T>(ok, 32 * n + 8 * x + 4 * (l >> 5), a.Dh, a.vec, kv);
            store4<T>(ov, 32 * n + 8 * x + 4 * (l >> 5), a.Dh, a.vec, vv);
        }
}

template <typename T, int DP, int BN>
hipError_t launch_sized(const CrossAttnGradArgs &a, hipStream_t s) {
    if (a.q_groups) {
        xattn_dq_kernel<T, DP, BN><<<dim3((unsigned)((a.q_groups + 7) / 8 * 8)), dim3(256), 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!a.k_groups) return hipSuccess;
    xattn_dkv_kernel<T, DP><<<dim3((unsigned)((a.k_groups + 7) / 8 * 8)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

size_t cross_attn_grad_workspace(int64_t B, int64_t Lq, int64_t Hq) { return (size_t)(B * Lq * Hq) * 4; }

hipError_t launch_cross_attn_grad(gs_dtype t, CrossAttnGradArgs a, void *ws, hipStream_t s) {
    a.rows = a.Lq * a.G;
    a.row_tiles = (int)(((int64_t)a.rows + 127) / 128);
    a.key_tiles = (int)(((int64_t)a.Lk + 127) / 128);
    a.q_groups = (int64_t)a.B * a.Hkv * a.row_tiles;
    a.k_groups = (int64_t)a.B * a.Hkv * a.key_tiles;
    a.D = static_cast<float *>(ws);
    if (t == GS_F32) return a.Dh <= 64 ? launch_sized<float, 64, 32>(a, s) : launch_sized<float, 128, 32>(a, s);
    return a.Dh <= 64 ? launch_sized<bf16_t, 64, 64>(a, s) : launch_sized<bf16_t, 128, 64>(a, s);
}

}  // namespace gs
