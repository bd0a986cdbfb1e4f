// A paged cache's bookkeeping: pages and slots of a step (gs_paged_plan) and the
// states of its rows written into them (gs_paged_store).
//
// Plan.  Everything follows from prefix sums over the requests: of the pages
// given back, of the pages wanted and of the new rows.  One work-group forms
// them; then each page moved and each slot is found on its own, by a binary
// search of its index in those sums.  A page taken in this step may have been
// given back in this step: it is then read from the table of the request that
// gave it (which the step does not write), not from the free list, so that no
// part waits for another.  Latency bounds it: 250 requests of one more position
// each, some 3000 pages given back, 8.6 us in one work-group; 700 prompts of
// 702350 slots 4.2 us of sums and 10.4 of slots (a search of ten steps and a load,
// four times a thread, one after the other).
#include "gs_scan.h"

namespace gs {
namespace {

constexpr int SCAN = 1024;          // requests a round of the scan, and threads of its work-group
constexpr int STAGED = 2048;        // requests whose sums are searched in LDS

// One work-group does the whole step where requests, rows and the pages that may be
// given back are few.  (250 requests of 504 rows and 125000 pages at most, some 3000
// of them given back: 8.6 us, in two launches 4.2 + 4.0, their gap and 3 us of the host's.)
constexpr int64_t ONE_ROWS = 4096, ONE_PAGES = (int64_t)1 << 17;
bool in_one(int64_t B, int64_t rows, int64_t width) { return B <= SCAN && rows <= ONE_ROWS && B * width <= ONE_PAGES; }

typedef PagedPlanHead PlanHead;

// Pages of x positions (both below 2^31).
__device__ __forceinline__ int64_t up(int64_t x, int64_t page) {
    return x ? (int64_t)(((uint32_t)x - 1u) / (uint32_t)page + 1u) : 0;
}

// Sums over the requests as a step leaves them, side by side (B + 1 entries where
// there is a total).  left: positions before the new ones, or -1 - that where the
// request asked and got nothing.
struct PlanSums {
    int32_t *at;
    int64_t B;
    __device__ __forceinline__ int32_t *left() const { return at; }
    __device__ __forceinline__ int32_t *back() const { return at + B; }
    __device__ __forceinline__ int32_t *take() const { return at + 2 * B + 1; }
    __device__ __forceinline__ int32_t *qoff() const { return at + 3 * B + 2; }
    static constexpr int size(int B) { return 4 * B + 3; }
};

__device__ __forceinline__ int32_t below(int64_t x, int64_t most) { return (int32_t)(x < most ? x : most); }

// The sums, written to z and the outputs qoff, length_out, added and nfree_out.
__device__ void plan_sums(const PagedPlanArgs &a, const PlanSums &z, PlanHead *head) {
    int32_t *const left = z.left(), *const back = z.back(), *const take = z.take(), *const rows_at = z.qoff();
    __shared__ int64_t room[4][SCAN / 64];
    __shared__ unsigned long long first_short;
    const int t = threadIdx.x;
    const int64_t page = a.page, most = a.most_length;      // min(width page, 2^31 - 1)
    const int64_t nfree = min((int64_t)max(*a.nfree, 0), a.capacity), space = a.capacity - nfree;
    int64_t len = 0, add = 0;
    auto load = [&](int64_t b) {
        len = add = 0;
        if (b < a.B) {
            len = a.length[b];
            add = a.add[b];
            len = len < 0 ? 0 : (len > most ? most : len);
        }
    };
    if (t == 0) first_short = ~0ull;
    int64_t given = 0;
    int turn = 0;
    for (int64_t b0 = 0; b0 < a.B; b0 += SCAN) {
        const int64_t b = b0 + t;
        load(b);
        const int64_t rest = add < 0 ? max(len + add, (int64_t)0) : len;
        int64_t total;
        const int64_t at = group_scan(up(len, page) - up(rest, page), room[turn], &total);
        turn ^= 1;
        if (b < a.B) back[b] = below(given + at, space);
        given += total;
    }
    const int64_t returned = min(given, space), avail = nfree + returned;
    int64_t rows = 0, wanted = 0, taken = 0;
    if (a.B == 0) __syncthreads();      // (nfree has been read by all before it may be written)
    for (int64_t b0 = 0; b0 < a.B; b0 += SCAN) {
        const int64_t b = b0 + t;
        if (a.B > SCAN) load(b);
        const int64_t n = max(add, (int64_t)0), rest = add < 0 ? max(len + add, (int64_t)0) : len;
        int64_t row_total, want_total;
        const int64_t row = rows + group_scan(n, room[turn], &row_total);
        const bool fits = n > 0 && len + n <= most && row + n <= a.rows;
        const int64_t need = fits ? up(len + n, page) - up(len, page) : 0;
        const int64_t want = wanted + group_scan(need, room[2 + turn], &want_total);
        turn ^= 1;
        const bool served = fits && (need == 0 || want + need <= avail);
        // (`want` rises from lane to lane: a wave's first one is its least)
        const uint64_t wanting = __ballot(fits && !served);
        if (wanting && (t & 63) == __ffsll((unsigned long long)wanting) - 1) atomicMin(&first_short, (unsigned long long)want);
        rows += row_total;
        wanted += want_total;
        __syncthreads();
        // what was taken before the first request that found too few
        taken = first_short != ~0ull ? (int64_t)first_short : wanted;
        if (b < a.B) {
            take[b] = (int32_t)min(want, taken);
            left[b] = (int32_t)(n > 0 && !served ? -1 - rest : rest);
            a.length_out[b] = (int32_t)(served ? len + n : rest);
            a.added[b] = (int32_t)(served ? n : 0);
            a.qoff[b] = below(row, 0x7fffffff);
            rows_at[b] = below(row, 0x7fffffff);
        }
    }
    if (t == 0) {
        back[a.B] = (int32_t)returned;
        take[a.B] = (int32_t)taken;
        a.qoff[a.B] = below(rows, 0x7fffffff);
        rows_at[a.B] = below(rows, 0x7fffffff);
        *a.nfree_out = (int32_t)(avail - taken);
        *head = PlanHead{(int32_t)nfree, (int32_t)returned, (int32_t)taken, (int32_t)avail};
    }
}

// The last b with sums[b] <= i (sums[0] = 0, sums[B] > i).
__device__ __forceinline__ int owner(const int32_t *sums, int B, int i) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (int)((uint32_t)(lo + hi) >> 1);
        if (sums[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Pages given back, pages taken and slots lie in one line, of which this does
// number `first`, first + step, ...: one copy of the code for all three, which a
// launch reads from memory each time.  (What differs is chosen among numbers, not
// among places of numbers: such a choice lays them out in memory, which each thread
// wrote and read back.)
__device__ void plan_fill(const PagedPlanArgs &a, const PlanSums &z, const PlanHead &head, int64_t first, int64_t step) {
    const int B = (int)a.B;
    const int64_t end0 = head.back, end1 = end0 + head.taken, total = end1 + a.rows;
    const int rows = B ? z.qoff()[B] : 0;
    for (int64_t i = first; i < total; i += step) {
        const int kind = (i >= end0) + (i >= end1);
        const int k = (int)(i - (kind == 0 ? 0 : kind == 1 ? end0 : end1));
        const int32_t *const sums = z.at + (kind == 0 ? z.B : kind == 1 ? 2 * z.B + 1 : 3 * z.B + 2);   // back, take, qoff
        int32_t id = -1;
        int64_t left = -1, held = 0, at = 0;
        int b = 0;
        if (kind < 2 || k < rows) {
            b = owner(sums, B, k);
            left = z.left()[b];
        }
        if (left >= 0) {
            held = up(left, a.page);
            const int off = k - sums[b];
            int taken = -1;             // its number among the pages taken
            const int32_t *from = a.table + b * a.ldt;
            if (kind == 0) {
                from += held + off;
            } else if (kind == 1) {
                taken = k;
                at = held + off;
            } else {
                const int64_t p = left + off, g = (uint32_t)p / (uint32_t)a.page;
                at = p - g * a.page;
                if (g < held) from += g;
                else taken = z.take()[b] + (int)(g - held);
            }
            if (taken >= 0) {           // from the end of the free pages and the returned ones behind them
                const int pos = head.avail - 1 - taken;
                from = a.free_pages + pos;
                if (pos >= head.nfree) {
                    const int c = owner(z.back(), B, pos - head.nfree);
                    from = a.table + c * a.ldt + up(z.left()[c], a.page) + (pos - head.nfree - z.back()[c]);
                }
            }
            id = *from;
        }
        if (kind == 0) a.free_pages[(int64_t)head.nfree + k] = id;
        else if (kind == 1) a.table[b * a.ldt + at] = id;
        else a.slots[k] = id < 0 ? -1 : id * a.page + at;
    }
}

// The whole step in one work-group.  free_pages and table entries that are read
// are not those that are written, but for the free list's returned part, which is
// read from the tables.
__global__ void __launch_bounds__(SCAN) plan_kernel(PagedPlanArgs a) {
    __shared__ int32_t sums[PlanSums::size(SCAN)];
    __shared__ PlanHead head;
    const PlanSums z{sums, a.B};
    plan_sums(a, z, &head);
    __syncthreads();
    plan_fill(a, z, head, threadIdx.x, SCAN);
}

__global__ void __launch_bounds__(SCAN) plan_sums_kernel(PagedPlanArgs a) {
    plan_sums(a, PlanSums{a.sums, a.B}, a.head);
}

template <bool LDS> __global__ void __launch_bounds__(256) plan_fill_kernel(PagedPlanArgs a) {
    typedef int32_t i4v __attribute__((ext_vector_type(4)));
    __shared__ i4v staged[LDS ? STAGED + 1 : 1];
    const int B = (int)a.B;
    const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
    const PlanHead head = *a.head;
    if constexpr (LDS) {        // (asked for together: each load takes about a microsecond)
#pragma unroll 4
        for (int i = threadIdx.x; i < (PlanSums::size(B) + 3) / 4; i += 256) staged[i] = reinterpret_cast<const i4v *>(a.sums)[i];
        __syncthreads();
        plan_fill(a, PlanSums{reinterpret_cast<int32_t *>(staged), a.B}, head, first, step);
    } else {
        plan_fill(a, PlanSums{a.sums, a.B}, head, first, step);
    }
}

// ---------------------------------------------------------------- rows

// Eight values of a row from d on (read once: not kept in the caches).
template <typename T> __device__ __forceinline__ void read8(float (&v)[8], const T *row, int d, int dh, bool vec) {
    typedef uint32_t u4v __attribute__((ext_vector_type(4)));
    if (vec) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const u4v x = __builtin_nontemporal_load(reinterpret_cast<const u4v *>(row + d + 4 * q));
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * q + e] = __uint_as_float(x[e]);
            }
        } else {
            const u4v x = __builtin_nontemporal_load(reinterpret_cast<const u4v *>(row + d));
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = bf16_to_f32((uint16_t)(x[e / 2] >> (16 * (e & 1))));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = d + e < dh ? ld_f32<T>(row, d + e) : 0.f;
    }
}
template <typename T> __device__ __forceinline__ void write8(const float (&v)[8], T *row, int d, int dh, bool vec) {
    typedef uint32_t u4v __attribute__((ext_vector_type(4)));
    if (vec) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                u4v x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = __float_as_uint(v[4 * q + e]);
                *reinterpret_cast<u4v *>(row + d + 4 * q) = x;
            }
        } else {
            u4v x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = f32_to_bf16(v[2 * e]) | (uint32_t)f32_to_bf16(v[2 * e + 1]) << 16;
            *reinterpret_cast<u4v *>(row + d) = x;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (d + e < dh) st_f32<T>(row, d + e, v[e]);
    }
}

// A thread moves eight values of K and of V.  Bound by HBM: 16000 rows of 8 heads of
// 128 values, fp32 to bf16, of which 15000 have a slot, 185 MB in 34 us, 5.4 TB/s.
template <typename T, typename C> __global__ void __launch_bounds__(256) store_kernel(PagedStoreArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.N * a.pieces) return;
    const int64_t n = i / a.pieces;
    const int rest = (int)(i % a.pieces), h = rest / a.head_pieces, d = 8 * (rest % a.head_pieces);
    const int64_t slot = a.slots[n];
    if (slot < 0 || slot >= a.pages * a.page) return;
    const int64_t g = slot / a.page, at = slot % a.page;
    float k[8], v[8];
    read8<T>(k, static_cast<const T *>(a.K) + n * a.k.l + h * a.k.h, d, a.Dh, a.vec_in);
    read8<T>(v, static_cast<const T *>(a.V) + n * a.v.l + h * a.v.h, d, a.Dh, a.vec_in);
    write8<C>(k, static_cast<C *>(a.Kc) + g * a.kc.b + at * a.kc.l + h * a.kc.h, d, a.Dh, a.vec_out);
    write8<C>(v, static_cast<C *>(a.Vc) + g * a.vc.b + at * a.vc.l + h * a.vc.h, d, a.Dh, a.vec_out);
}

}  // namespace

size_t paged_plan_workspace(int64_t B, int64_t rows, int64_t width) {
    if (in_one(B, rows, width)) return 0;
    return (sizeof(PlanHead) + 4 * (size_t)(4 * B + 3) + 15) / 16 * 16;
}

hipError_t launch_paged_plan(PagedPlanArgs a, void *ws, hipStream_t s) {
    if (in_one(a.B, a.rows, a.width)) {
        plan_kernel<<<dim3(1), dim3(SCAN), 0, s>>>(a);
        return hipGetLastError();
    }
    a.head = static_cast<PlanHead *>(ws);
    a.sums = reinterpret_cast<int32_t *>(a.head + 1);
    plan_sums_kernel<<<dim3(1), dim3(SCAN), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t groups = (a.rows + 1023) / 1024, most = 1024;
    const dim3 grid((unsigned)(groups < 64 ? 64 : (groups < most ? groups : most)));
    if (a.B <= STAGED) plan_fill_kernel<true><<<grid, dim3(256), 0, s>>>(a);
    else plan_fill_kernel<false><<<grid, dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_paged_store(gs_dtype t, gs_dtype ct, PagedStoreArgs a, hipStream_t s) {
    a.head_pieces = (a.Dh + 7) / 8;
    a.pieces = (int64_t)a.Hkv * a.head_pieces;
    const dim3 grid((unsigned)((a.N * a.pieces + 255) / 256)), group(256);
    if (t == GS_F32 && ct == GS_F32) store_kernel<float, float><<<grid, group, 0, s>>>(a);
    else if (t == GS_F32) store_kernel<float, bf16_t><<<grid, group, 0, s>>>(a);
    else if (ct == GS_F32) store_kernel<bf16_t, float><<<grid, group, 0, s>>>(a);
    else store_kernel<bf16_t, bf16_t><<<grid, group, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace gs
