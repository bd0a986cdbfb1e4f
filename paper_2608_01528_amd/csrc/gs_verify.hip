// Drafted entries taken or refused, and the entry after them drawn (gs_verify).
//
// Which drafts are taken needs two gathered numbers a draft; then one row of P
// (and of Q) is read for the draw.  Its weights are summed and searched in parts
// of PART entries: a row of one part stays in registers, longer rows take a
// launch for the parts' sums and one that searches them and reads the part that
// the draw falls into once more.  Sums are fp64 in a fixed order (lanes, waves,
// pieces, parts): a draw depends on their last bits alone.
#include "gs_internal.h"

namespace gs {
namespace {

constexpr int GROUP = 256, WAVES = GROUP / 64;
constexpr int HELD = 16, PART = GROUP * HELD;       // entries a thread holds, a work-group holds

typedef uint32_t u4v __attribute__((ext_vector_type(4)));

// Negative numbers, infinities and NaN have no weight.
__device__ __forceinline__ double weight(float x) { return x > 0.f && x < INFINITY ? (double)x : 0.; }
template <typename T> __device__ __forceinline__ float widen(const T *p, int64_t i) { return ld_f32<T>(p, i); }

__device__ __forceinline__ int64_t bounded(const int32_t *qoff, int64_t b, int64_t N) {
    const int64_t x = qoff[b];
    return x < 0 ? 0 : (x > N ? N : x);
}

struct Request {
    int64_t first;      // its first row
    int64_t n, taken;   // its rows, drafts taken
    int32_t refused;    // the draft that was not, -1 if all were
};

// Every wave finds this on its own, a draft a lane.
template <typename T> __device__ __forceinline__ Request request(const VerifyArgs &a, int64_t b) {
    const int l = threadIdx.x & 63;
    Request r{};
    r.first = bounded(a.qoff, b, a.N);
    r.n = bounded(a.qoff, b + 1, a.N) - r.first;
    r.refused = -1;
    if (r.n < 0) r.n = 0;
    for (int64_t i0 = 0; i0 < r.n - 1; i0 += 64) {
        const int64_t i = i0 + l, row = r.first + i;
        bool ok = true;
        int32_t x = -1;
        if (i < r.n - 1) {
            x = a.drafted[row];
            const float u = a.u[row];
            double p = 0., q = 0.;
            if (x >= 0 && x < a.M) {
                p = weight(widen(static_cast<const T *>(a.P), row * a.ldp + x));
                q = a.Q ? weight(widen(static_cast<const T *>(a.Q), row * a.ldq + x)) : 1.;
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
    r.taken = r.n ? r.n - 1 : 0;
    return r;
}

// The weights of a part's entries that a thread holds: piece s, V consecutive
// entries at base + s GROUP V + V t.
template <typename T> struct Part {
    static constexpr int V = 16 / sizeof(T), PIECES = HELD / V;
    float p[HELD], q[HELD];
    int64_t at;
    bool less;          // weights max(p - q, 0)
    static __device__ __forceinline__ void fetch(float (&v)[HELD], const T *row, int64_t at, int64_t M, bool vec) {
#pragma unroll
        for (int s = 0; s < PIECES; ++s) {
            const int64_t j = at + (int64_t)s * GROUP * V;
            if (vec && j + V <= M) {
                const u4v x = *reinterpret_cast<const u4v *>(row + j);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if constexpr (sizeof(T) == 4) v[s * V + e] = __uint_as_float(x[e]);
                    else v[s * V + e] = bf16_to_f32((uint16_t)(x[e / 2] >> (16 * (e & 1))));
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) v[s * V + e] = j + e < M ? widen(row, j + e) : 0.f;
            }
        }
    }
    __device__ __forceinline__ void load(const VerifyArgs &a, const Request &r, int64_t part) {
        const int64_t row = r.first + r.taken;
        at = part * PART + (int64_t)V * threadIdx.x;
        less = r.taken < r.n - 1;
        fetch(p, static_cast<const T *>(a.P) + row * a.ldp, at, a.M, a.vec_p);
        if (!less) return;
        if (a.Q) {
            fetch(q, static_cast<const T *>(a.Q) + row * a.ldq, at, a.M, a.vec_q);
        } else {
#pragma unroll
            for (int k = 0; k < HELD; ++k) q[k] = at + (int64_t)(k / V) * GROUP * V + k % V == r.refused ? 1.f : 0.f;
        }
    }
    __device__ __forceinline__ double w(int k) const {
        const double x = weight(p[k]);
        return less ? fmax(x - weight(q[k]), 0.) : x;
    }
};

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// The entry at which the sum of the part's weights passes `target`, which is
// below their total but for rounding (infinite: the last of any weight); -1 if
// none has any.
template <typename T> __device__ __forceinline__ int64_t search(const Part<T> &part, double target) {
    constexpr int V = Part<T>::V, PIECES = Part<T>::PIECES;
    __shared__ double sums[PIECES][WAVES];
    __shared__ unsigned long long found, last;
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    if (t == 0) found = ~0ull, last = 0;
    double mine[PIECES];
    int64_t top = -1;
#pragma unroll
    for (int s = 0; s < PIECES; ++s) {
        mine[s] = 0.;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const double x = part.w(s * V + e);
            mine[s] += x;
            if (x > 0.) top = part.at + (int64_t)s * GROUP * V + e;
        }
        const double all = wave_sum(mine[s]);
        if (l == 0) sums[s][w] = all;
    }
    __syncthreads();
    double before = 0.;         // of the pieces and waves before this one
#pragma unroll
    for (int s = 0; s < PIECES; ++s) {
        double here = before;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            if (v < w) here += sums[s][v];
            before += sums[s][v];
        }
        if (!(target < here + sums[s][w])) continue;       // (wave-uniform)
        // exclusive sums of the lanes' weights
        double c = mine[s];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const double x = __shfl_up(c, d);
            if (l >= d) c += x;
        }
        c = here + c - mine[s];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const double x = part.w(s * V + e);
            c += x;
            if (x > 0. && c > target) {
                atomicMin(&found, (unsigned long long)(part.at + (int64_t)s * GROUP * V + e));
                break;
            }
        }
    }
    if (top >= 0) atomicMax(&last, (unsigned long long)(top + 1));
    __syncthreads();
    return found != ~0ull ? (int64_t)found : (int64_t)last - 1;
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
        for (int64_t i = threadIdx.x; i < r.n; i += GROUP)
            a.entries[r.first + i] = i < r.taken ? a.drafted[r.first + i] : (i == r.taken ? (int32_t)entry : -1);
}

// Sum over the work-group; room: WAVES values that are not in use.
__device__ __forceinline__ double group_sum(double x, double *room) {
    const double s = wave_sum(x);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = s;
    __syncthreads();
    double all = 0.;
#pragma unroll
    for (int v = 0; v < WAVES; ++v) all += room[v];
    return all;
}

// Rows of one part: a work-group a request.
template <typename T> __global__ void __launch_bounds__(GROUP) verify_kernel(VerifyArgs a) {
    __shared__ double room[2][WAVES];
    const int64_t b = blockIdx.x;
    const Request r = request<T>(a, b);
    int64_t entry = -1;
    if (r.n) {
        Part<T> part;
        part.load(a, r, 0);
        double mine = 0.;
#pragma unroll
        for (int k = 0; k < HELD; ++k) mine += part.w(k);
        double total = group_sum(mine, room[0]);
        if (total == 0. && part.less) {
            part.less = false;
            mine = 0.;
#pragma unroll
            for (int k = 0; k < HELD; ++k) mine += part.w(k);
            total = group_sum(mine, room[1]);
        }
        entry = search<T>(part, target_of(a.v[b], total));
    }
    write_out(a, b, r, entry);
}

// The sums of a part: of its weights, and of p.
template <typename T> __global__ void __launch_bounds__(GROUP) verify_sums_kernel(VerifyArgs a) {
    __shared__ double room[2][WAVES];
    const int64_t b = blockIdx.x / a.parts, k = blockIdx.x % a.parts;
    const Request r = request<T>(a, b);
    if (!r.n) return;
    Part<T> part;
    part.load(a, r, k);
    double w = 0., p = 0.;
#pragma unroll
    for (int i = 0; i < HELD; ++i) w += part.w(i), p += weight(part.p[i]);
    w = group_sum(w, room[0]);
    p = group_sum(p, room[1]);
    if (threadIdx.x == 0) {
        a.sums[2 * (b * a.parts + k)] = w;
        a.sums[2 * (b * a.parts + k) + 1] = p;
    }
}

template <typename T> __global__ void __launch_bounds__(GROUP) verify_draw_kernel(VerifyArgs a) {
    __shared__ double room[2][WAVES];
    __shared__ unsigned long long found, last;
    __shared__ double before;
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    const int64_t b = blockIdx.x;
    const Request r = request<T>(a, b);
    if (!r.n) {
        write_out(a, b, r, -1);
        return;
    }
    const double *const sums = a.sums + 2 * b * a.parts;
    double wt = 0., pt = 0.;
    for (int64_t k = t; k < a.parts; k += GROUP) wt += sums[2 * k], pt += sums[2 * k + 1];
    wt = group_sum(wt, room[0]);
    pt = group_sum(pt, room[1]);
    const int from = wt > 0. ? 0 : 1;
    const double total = from ? pt : wt, target = target_of(a.v[b], total);
    if (t == 0) found = ~0ull, last = 0;
    // the part in which the sum passes the target, GROUP parts at a time
    double carry = 0.;
    int64_t top = -1;
    for (int64_t k0 = 0; k0 < a.parts; k0 += GROUP) {
        const int64_t k = k0 + t;
        const double x = k < a.parts ? sums[2 * k + from] : 0.;
        double c = x;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const double y = __shfl_up(c, d);
            if (l >= d) c += y;
        }
        __syncthreads();
        if (l == 63) room[0][w] = c;
        __syncthreads();
        double all = 0., here = carry;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            if (v < w) here += room[0][v];
            all += room[0][v];
        }
        carry += all;
        if (x > 0.) {
            top = k;
            if (here + c > target) atomicMin(&found, (unsigned long long)k);
        }
        __syncthreads();
        if (found != ~0ull) {
            if (found == (unsigned long long)k) before = here + c - x;
            break;
        }
    }
    if (top >= 0) atomicMax(&last, (unsigned long long)(top + 1));
    __syncthreads();
    const bool hit = found != ~0ull;
    const int64_t k = hit ? (int64_t)found : (int64_t)last - 1;
    int64_t entry = -1;
    if (k >= 0) {
        Part<T> part;
        part.load(a, r, k);
        if (from) part.less = false;
        entry = search<T>(part, hit ? target - before : (double)INFINITY);
    }
    write_out(a, b, r, entry);
}

int64_t parts_of(int64_t M) { return (M + PART - 1) / PART; }

template <typename T> hipError_t launch_typed(const VerifyArgs &a, hipStream_t s) {
    if (a.parts == 1) {
        verify_kernel<T><<<dim3((unsigned)a.B), dim3(GROUP), 0, s>>>(a);
        return hipGetLastError();
    }
    verify_sums_kernel<T><<<dim3((unsigned)(a.B * a.parts)), dim3(GROUP), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    verify_draw_kernel<T><<<dim3((unsigned)a.B), dim3(GROUP), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

int64_t verify_groups(int64_t B, int64_t M) { return B * parts_of(M); }

size_t verify_workspace(int64_t B, int64_t M) {
    const int64_t parts = parts_of(M);
    return parts == 1 ? 0 : (size_t)(B * parts) * 16;
}

hipError_t launch_verify(gs_dtype pt, VerifyArgs a, void *ws, hipStream_t s) {
    a.parts = parts_of(a.M);
    a.sums = static_cast<double *>(ws);
    return pt == GS_F32 ? launch_typed<float>(a, s) : launch_typed<bf16_t>(a, s);
}

}  // namespace gs
