// Drafted entries taken or refused, and the entry after them drawn (gs_verify).
//
// Which drafts are taken needs two gathered numbers a draft; then one row of P
// (and of Q) is read for the draw.  A thread holds a few consecutive entries of it;
// one prefix sum over the threads gives the total and says which of them holds the
// entry.  Rows of up to ONE entries are a work-group's; longer ones take a launch in
// which each wave sums UNIT entries, and one that finds the unit and reads it once
// more.  Sums are fp64 in a fixed order.  What bounds it is a chain of dependent
// loads (offsets, drafts, their probabilities, the row) and, as each instruction
// runs once, the reading of the code: a thread holds no more than the row needs.
// One request, 131072 entries, fp32: 4.2 + 4.0 us; 120 of 50257, bf16, 23 MB: 9.8 +
// 5.0; 2000 of 1843, fp32: 8.6.  (Which lane's entry is the first goes by ballots:
// an atomic of many lanes on LDS, which the compiler runs lane by lane, cost 8 us a
// kernel.)
#include "gs_scan.h"

namespace gs {
namespace {

constexpr int WAVES = 4, GROUP = 64 * WAVES;
constexpr int ONE = 16 * GROUP;         // entries of a row that a work-group holds
constexpr int UNIT = 1024;              // entries that a wave sums, and a work-group searches

// Negative numbers, infinities and NaN have no weight.
__device__ __forceinline__ float weighed(float x) { return x > 0.f && x < INFINITY ? x : 0.f; }
template <typename T> __device__ __forceinline__ double weight(const T *p, int64_t i) { return weighed(ld_f32<T>(p, i)); }

__device__ __forceinline__ int64_t bounded(const int32_t *qoff, int64_t b, int64_t N) {
    const int64_t x = qoff[b];
    return x < 0 ? 0 : (x > N ? N : x);
}

struct Request {
    int64_t first;      // its first row
    int64_t n, taken;   // its rows, drafts taken
    int32_t refused;    // the draft that was not, -1 if all were
    int32_t drawn;      // its rows stand for positions: an entry is drawn
};

// Every wave finds this on its own, a draft a lane.
template <typename T> __device__ __forceinline__ Request request(const VerifyArgs &a, int64_t b) {
    const int l = threadIdx.x & 63;
    Request r{};
    r.first = bounded(a.qoff, b, a.N);
    r.n = bounded(a.qoff, b + 1, a.N) - r.first;
    r.refused = -1;
    if (r.n < 0) r.n = 0;
    r.drawn = r.n > 0 && (!a.added || a.added[b] > 0);
    if (!r.drawn) return r;
    for (int64_t i0 = 0; i0 < r.n - 1; i0 += 64) {
        const int64_t i = i0 + l, row = r.first + i;
        bool ok = true;
        int32_t x = -1;
        if (i < r.n - 1) {
            x = a.drafted[row];
            const float u = a.u[row];
            double p = 0., q = 0.;
            if (x >= 0 && x < a.M) {
                p = weight(static_cast<const T *>(a.P), row * a.ldp + x);
                q = a.Q ? weight(static_cast<const T *>(a.Q), row * a.ldq + x) : 1.;
            }
            ok = (u > 0.f ? (double)u : 0.) * q < p;
        }
        const uint64_t bad = ~__ballot(ok);
        if (bad) {
            const int at = __ffsll((unsigned long long)bad) - 1;
            r.taken = i0 + at;
            r.refused = __shfl(x, at);
            return r;
        }
    }
    r.taken = r.n - 1;
    return r;
}

// The weights of H consecutive entries.
template <typename T, int H> struct Part {
    float p[H], q[H];
    int64_t at;
    bool less;          // weights max(p - q, 0)
    // (rows start on any boundary: loads of 16 or 8 bytes need that of an entry)
    static __device__ __forceinline__ void fetch(float (&v)[H], const T *row, int64_t at, int64_t M) {
        constexpr int V = 4;
        typedef uint32_t word __attribute__((ext_vector_type(V * sizeof(T) / 4), aligned(sizeof(T))));
        if (at + H <= M) {
#pragma unroll
            for (int s = 0; s < H; s += V) {
                const word x = *reinterpret_cast<const word *>(row + at + s);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if constexpr (sizeof(T) == 4) v[s + e] = weighed(__uint_as_float(x[e]));
                    else v[s + e] = weighed(__uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16));
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < H; ++e) v[e] = 0.f;
            if (at < M)
#pragma unroll
                for (int e = 0; e < H; ++e)
                    if (at + e < M) v[e] = weighed(ld_f32<T>(row, at + e));
        }
    }
    __device__ __forceinline__ void load(const VerifyArgs &a, const Request &r, int64_t from) {
        const int64_t row = r.first + r.taken;
        at = from;
        less = r.taken < r.n - 1;
        fetch(p, static_cast<const T *>(a.P) + row * a.ldp, at, a.M);
        if (less && a.Q) {
            fetch(q, static_cast<const T *>(a.Q) + row * a.ldq, at, a.M);
        } else {
#pragma unroll
            for (int k = 0; k < H; ++k) q[k] = less && at + k == r.refused ? 1.f : 0.f;
        }
    }
    __device__ __forceinline__ double w(int k) const { return fmax((double)p[k] - (double)q[k], 0.); }
    __device__ __forceinline__ double sum() const {
        double x = 0.;
#pragma unroll
        for (int k = 0; k < H; ++k) x += w(k);
        return x;
    }
    __device__ __forceinline__ double sum_p() const {
        double x = 0.;
#pragma unroll
        for (int k = 0; k < H; ++k) x += (double)p[k];
        return x;
    }
    __device__ __forceinline__ void forget_q() {
        less = false;
#pragma unroll
        for (int k = 0; k < H; ++k) q[k] = 0.f;
    }
};

// Sums over the threads before this one and over all; room: NW values that are not
// in use.
template <int NW> __device__ __forceinline__ double sums_before(double mine, double *room, double *total) {
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const double upto = wave_upto(mine);
    if constexpr (NW == 1) {
        *total = lane_value(upto, 63);
        return upto - mine;
    }
    if (l == 63) room[w] = upto;
    __syncthreads();
    double before = 0., all = 0.;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
        if (v < w) before += room[v];
        all += room[v];
    }
    *total = all;
    return before + (upto - mine);
}

// The first number of a wave's lanes that have one, and the last.  (Lanes hold
// rising numbers, so no atomics are needed.)
struct Ends { int64_t first, last; };
__device__ __forceinline__ Ends ends_of(bool hit, int64_t at, bool any, int64_t top) {
    const uint64_t h = __ballot(hit), n = __ballot(any);
    return Ends{h ? lane_value(at, __ffsll((unsigned long long)h) - 1) : -1, n ? lane_value(top, 63 - __clzll((long long)n)) : -1};
}
// The same over the waves of a work-group; room: NW values that are not in use.
template <int NW> __device__ __forceinline__ Ends group_ends(Ends e, Ends *room) {
    if constexpr (NW == 1) return e;
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = e;
    __syncthreads();
    e = Ends{-1, -1};
#pragma unroll
    for (int v = 0; v < NW; ++v) {
        const Ends x = room[v];
        if (e.first < 0) e.first = x.first;
        if (x.last >= 0) e.last = x.last;
    }
    return e;
}

// The entry at which the sum of the weights passes `target`, which is below their
// total but for rounding (infinite: the last of any weight); -1 if none has any.
// before: the sum over the threads before this one.
template <int NW, typename T, int H>
__device__ __forceinline__ int64_t search(const Part<T, H> &part, double before, double target, Ends *room) {
    double c = before;
    int top = -1, hit = H;
#pragma unroll
    for (int k = 0; k < H; ++k) {
        const double x = part.w(k);
        c += x;
        if (x > 0.) {
            top = k;
            if (c > target && hit == H) hit = k;
        }
    }
    const Ends e = group_ends<NW>(ends_of(hit < H, part.at + hit, top >= 0, part.at + top), room);
    return e.first >= 0 ? e.first : e.last;
}

// target of a draw: v of the total, from 1 on beyond every sum
__device__ __forceinline__ double target_of(float v, double total) {
    return v >= 1.f ? (double)INFINITY : (v > 0.f ? (double)v * total : 0.);
}

__device__ __forceinline__ void write_out(const VerifyArgs &a, int64_t b, const Request &r, int64_t entry) {
    if (threadIdx.x == 0) {
        a.accepted[b] = (int32_t)r.taken;
        a.entry[b] = (int32_t)entry;
    }
    if (a.entries)
        for (int64_t i = threadIdx.x; i < r.n; i += blockDim.x)
            a.entries[r.first + i] = i < r.taken ? a.drafted[r.first + i] : (i == r.taken ? (int32_t)entry : -1);
}

// Rows of up to 64 NW H entries: a work-group of NW waves a request.
template <typename T, int NW, int H> __global__ void __launch_bounds__(64 * NW) verify_kernel(VerifyArgs a) {
    __shared__ double room[2][NW];
    __shared__ Ends ends[NW];
    const int64_t b = blockIdx.x;
    const float v = a.v[b];
    const Request r = request<T>(a, b);
    int64_t entry = -1;
    if (r.drawn) {
        Part<T, H> part;
        part.load(a, r, H * threadIdx.x);
        double mine = part.sum(), total;
        double before = sums_before<NW>(mine, room[0], &total);
        if (total == 0. && part.less) {
            part.forget_q();
            mine = part.sum_p();
            before = sums_before<NW>(mine, room[1], &total);
        }
        entry = search<NW>(part, before, target_of(v, total), ends);
    }
    write_out(a, b, r, entry);
}

// The sums of a wave's unit: of its weights, and of p.
template <typename T> __global__ void __launch_bounds__(GROUP) verify_sums_kernel(VerifyArgs a) {
    const int64_t groups = (a.parts + WAVES - 1) / WAVES;
    const int64_t b = blockIdx.x / groups, k = blockIdx.x % groups * WAVES + (threadIdx.x >> 6);
    const int l = threadIdx.x & 63;
    const Request r = request<T>(a, b);
    if (k == 0 && l == 0) a.requests[b] = VerifyRequest{r.first, r.n, r.taken, r.refused, r.drawn};
    if (!r.drawn || k >= a.parts) return;
    constexpr int H = UNIT / 64;
    Part<T, H> part;
    part.load(a, r, k * UNIT + H * l);
    const double w = wave_upto(part.sum()), p = wave_upto(part.sum_p());
    if (l == 63) {
        a.sums[2 * (b * a.parts + k)] = w;
        a.sums[2 * (b * a.parts + k) + 1] = p;
    }
}

template <typename T> __global__ void __launch_bounds__(GROUP) verify_draw_kernel(VerifyArgs a) {
    __shared__ double room[4][WAVES], before;
    __shared__ Ends ends[3][WAVES];
    const int t = threadIdx.x;
    const int64_t b = blockIdx.x;
    const VerifyRequest given = a.requests[b];
    const Request r{given.first, given.n, given.taken, given.refused, given.drawn};
    if (!r.drawn) {
        write_out(a, b, r, -1);
        return;
    }
    const float v = a.v[b];
    const double *const sums = a.sums + 2 * b * a.parts;
    double wt = 0., pt = 0.;
    for (int64_t k = t; k < a.parts; k += GROUP) wt += sums[2 * k], pt += sums[2 * k + 1];
    double mine = wt;
    (void)sums_before<WAVES>(mine, room[0], &wt);
    mine = pt;
    (void)sums_before<WAVES>(mine, room[1], &pt);
    const int from = wt > 0. ? 0 : 1;
    const double target = target_of(v, from ? pt : wt);
    // the unit in which the sum passes the target, GROUP units at a time
    double carry = 0.;
    int64_t k = -1, last = -1;
    int turn = 0;
    for (int64_t k0 = 0; k0 < a.parts && k < 0; k0 += GROUP, turn ^= 1) {
        const int64_t i = k0 + t;
        const double x = i < a.parts ? sums[2 * i + from] : 0.;
        double all;
        const double here = carry + sums_before<WAVES>(x, room[2 + turn], &all);
        carry += all;
        const bool hit = x > 0. && here + x > target;
        const Ends e = group_ends<WAVES>(ends_of(hit, i, x > 0., i), ends[turn]);
        k = e.first;
        if (e.last >= 0) last = e.last;
        if (k >= 0 && k == i) before = here;
    }
    __syncthreads();
    const double rest = k >= 0 ? target - before : (double)INFINITY;
    if (k < 0) k = last;
    int64_t entry = -1;
    if (k >= 0) {
        Part<T, UNIT / GROUP> part;
        part.load(a, r, k * UNIT + UNIT / GROUP * t);
        if (from) part.forget_q();
        double all;
        const double at = sums_before<WAVES>(part.sum(), room[0], &all);
        entry = search<WAVES>(part, at, rest, ends[2]);
    }
    write_out(a, b, r, entry);
}

int64_t parts_of(int64_t M) { return M <= ONE ? 1 : (M + UNIT - 1) / UNIT; }

template <typename T> hipError_t launch_typed(const VerifyArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)a.B);
    if (a.parts == 1) {
        if (a.M <= 256) verify_kernel<T, 1, 4><<<grid, dim3(64), 0, s>>>(a);
        else if (a.M <= GROUP * 4) verify_kernel<T, WAVES, 4><<<grid, dim3(GROUP), 0, s>>>(a);
        else if (a.M <= GROUP * 8) verify_kernel<T, WAVES, 8><<<grid, dim3(GROUP), 0, s>>>(a);
        else verify_kernel<T, WAVES, 16><<<grid, dim3(GROUP), 0, s>>>(a);
        return hipGetLastError();
    }
    verify_sums_kernel<T><<<dim3((unsigned)(a.B * ((a.parts + WAVES - 1) / WAVES))), dim3(GROUP), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    verify_draw_kernel<T><<<grid, dim3(GROUP), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

int64_t verify_groups(int64_t B, int64_t M) { return B * ((parts_of(M) + WAVES - 1) / WAVES); }

size_t verify_workspace(int64_t B, int64_t M) {
    const int64_t parts = parts_of(M);
    return parts == 1 ? 0 : (size_t)(B * parts) * 16 + (size_t)B * sizeof(VerifyRequest);
}

hipError_t launch_verify(gs_dtype pt, VerifyArgs a, void *ws, hipStream_t s) {
    a.parts = parts_of(a.M);
    a.sums = static_cast<double *>(ws);
    a.requests = reinterpret_cast<VerifyRequest *>(a.sums + 2 * a.B * a.parts);
    return pt == GS_F32 ? launch_typed<float>(a, s) : launch_typed<bf16_t>(a, s);
}

}  // namespace gs
