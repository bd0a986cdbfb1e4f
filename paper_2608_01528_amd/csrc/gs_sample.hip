// An entry drawn from a row of scores: temperature, top-k, top-p, min-p, and a
// given random number.
//
// Everything that decides is exact or in 64 bits.  Scores are ranked by an
// order-preserving integer key; weights are exp in fp64, then held as whole
// multiples of 2^-shift of the largest one, so sums are integer sums: the same
// in any order, whatever the split of a row over threads.
#include "gs_internal.h"

namespace gs {
namespace {

constexpr int NT = 256;

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

struct Weigh {
    double m, inv_t, unit;      // largest score, 1 / temperature, 2^shift
    __device__ __forceinline__ double weight(uint32_t key) const {
        if (!key) return 0.;
        const double x = value_of(key);
        return x == m ? 1. : exp((x - m) * inv_t);      // (an infinite m leaves 0 for the rest)
    }
    __device__ __forceinline__ uint64_t mass(uint32_t key) const {
        const double w = weight(key);
        return w > 0. ? (uint64_t)fmax(1., rint(w * unit)) : 0;
    }
};

template <typename V, typename F> __device__ __forceinline__ V block_reduce(V v, F f, V *tmp) {
#pragma unroll
    for (int x = 32; x; x >>= 1) v = f(v, (V)__shfl_xor(v, x));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    v = tmp[0];
    for (int i = 1; i < NT / 64; ++i) v = f(v, tmp[i]);
    return v;
}
template <typename V> __device__ __forceinline__ V block_sum(V v, V *tmp) {
    return block_reduce(v, [](V a, V b) { return a + b; }, tmp);
}
// sum over the threads before this one; total in *all
template <typename V> __device__ __forceinline__ V block_before(V v, V *tmp, V *all) {
    V x = v;
    for (int o = 1; o < 64; o <<= 1) {
        const V y = __shfl_up(x, o);
        if ((threadIdx.x & 63) >= o) x += y;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 63) tmp[threadIdx.x >> 6] = x;
    __syncthreads();
    V base = 0, sum = 0;
    for (int i = 0; i < NT / 64; ++i) {
        if (i < (int)(threadIdx.x >> 6)) base += tmp[i];
        sum += tmp[i];
    }
    *all = sum;
    return base + x - v;
}

template <typename T>
__global__ void __launch_bounds__(NT) sample_kernel(SampleArgs a) {
    __shared__ uint64_t tmp[NT / 64];
    __shared__ uint64_t found;
    const int64_t b = blockIdx.x;
    const T *const row = static_cast<const T *>(a.S) + b * a.lds;
    const int64_t M = a.M;
    const int t = threadIdx.x;
    auto key_at = [&](int64_t j) { return key_of(ld_f32<T>(row, j)); };

    uint32_t top = 0;
    for (int64_t j = t; j < M; j += NT) top = max(top, key_at(j));
    top = (uint32_t)block_reduce<uint64_t>(top, [](uint64_t x, uint64_t y) { return x > y ? x : y; }, tmp);
    if (!top) {
        if (t == 0) {
            a.idx[b] = -1;
            if (a.prob) a.prob[b] = 0.f;
            if (a.kept) a.kept[b] = 0;
        }
        return;
    }
    const float temp = a.temperature ? a.temperature[b] : a.temperature_all;
    int64_t k = a.top_k ? a.top_k[b] : a.top_k_all;
    const double p = a.top_p ? a.top_p[b] : a.top_p_all;
    const float min_p = a.min_p ? a.min_p[b] : a.min_p_all;
    const double least = min_p > 0.f ? fmin(1., (double)min_p) : 0.;
    if (k <= 0 || k > M) k = M;
    if (!(temp > 0.f)) k = 1;
    const Weigh wt{(double)value_of(top), temp > 0.f ? 1. / (double)temp : 1., a.unit};

    // kept by rank: keys above `cut`, and of those equal to it the first `ties` by index
    uint32_t cut = 1;
    int64_t ties = M;
    auto count_from = [&](uint32_t c) {
        uint64_t n = 0;
        for (int64_t j = t; j < M; j += NT) n += key_at(j) >= c;
        return block_sum(n, tmp);
    };
    auto mass_from = [&](uint32_t c) {
        uint64_t n = 0;
        for (int64_t j = t; j < M; j += NT) {
            const uint32_t x = key_at(j);
            if (x >= c) n += wt.mass(x);
        }
        return block_sum(n, tmp);
    };
    // the largest c in [lo, top] with enough(c), which holds for lo
    auto largest = [&](uint32_t lo, auto enough) {
        uint32_t hi = top;
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            if (enough(mid)) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    };
    if (k < M && (int64_t)count_from(1) > k) {
        cut = largest(1, [&](uint32_t c) { return (int64_t)count_from(c) >= k; });
        ties = k - (cut == top ? 0 : (int64_t)count_from(cut + 1));
    }
    if (p < 1.) {
        const uint64_t above_k = cut == top ? 0 : mass_from(cut + 1);
        const uint64_t w = wt.mass(cut);
        const uint64_t all = cut == 1 ? above_k : above_k + (uint64_t)ties * w;
        const double goal = fmax(p, 0.) * (double)all;
        const uint32_t at = (double)above_k >= goal && above_k ? largest(cut + 1, [&](uint32_t c) { return (double)mass_from(c) >= goal; }) : cut;
        if (at > cut) {
            cut = at;
            ties = M;
        }
        const uint64_t above = cut == top ? 0 : mass_from(cut + 1);
        const uint64_t one = wt.mass(cut);
        if (cut > 1 && one) {
            double n = ceil((goal - (double)above) / (double)one);
            n = n < 1. ? 1. : n;
            if (n < (double)ties) ties = (int64_t)n;
        }
    }
    // consecutive entries of a thread, so that sums run in index order
    const int64_t per = (M + NT - 1) / NT, j0 = t * per < M ? t * per : M, j1 = j0 + per < M ? j0 + per : M;
    int64_t equal = 0;
    for (int64_t j = j0; j < j1; ++j) equal += key_at(j) == cut;
    int64_t all_equal;
    const int64_t equal_before = block_before<int64_t>(equal, reinterpret_cast<int64_t *>(tmp), &all_equal);
    auto each = [&](auto use) {
        int64_t e = equal_before;
        for (int64_t j = j0; j < j1; ++j) {
            const uint32_t x = key_at(j);
            if (x < cut || !x) continue;
            if (x == cut && e++ >= ties) continue;
            if (wt.weight(x) < least) continue;
            use(j, wt.mass(x));
        }
    };
    uint64_t mine = 0, n = 0;
    each([&](int64_t, uint64_t w) { mine += w; ++n; });
    n = block_sum(n, tmp);
    uint64_t total;
    uint64_t sum = block_before<uint64_t>(mine, tmp, &total);
    const double u = (double)a.u[b];
    const double goal = u > 0. ? (u < 1. ? u * (double)total : (double)total) : 0.;
    __syncthreads();
    if (t == 0) found = ~0ull;
    __syncthreads();
    // the first entry whose sum passes the goal; the last one where none does
    // (u of 1 and more)
    int64_t hit = -1, last = -1;
    uint64_t hit_w = 0, last_w = 0;
    each([&](int64_t j, uint64_t w) {
        if (!w) return;
        sum += w;
        last = j, last_w = w;
        if (hit < 0 && (double)sum > goal) hit = j, hit_w = w;
    });
    if (hit >= 0) atomicMin((unsigned long long *)&found, (unsigned long long)hit);
    const uint64_t end = block_reduce<uint64_t>((uint64_t)(last + 1), [](uint64_t x, uint64_t y) { return x > y ? x : y; }, tmp);
    __syncthreads();
    const bool none = found == ~0ull;
    if (none ? (last >= 0 && (uint64_t)(last + 1) == end) : (hit >= 0 && (uint64_t)hit == found)) {
        a.idx[b] = (int32_t)(none ? last : hit);
        if (a.prob) a.prob[b] = (float)((double)(none ? last_w : hit_w) / (double)total);
        if (a.kept) a.kept[b] = (int32_t)n;
    }
}

}  // namespace

hipError_t launch_sample(gs_dtype st, SampleArgs a, hipStream_t s) {
    int bits = 0;
    while (((int64_t)1 << bits) < a.M) ++bits;
    a.unit = (double)((uint64_t)1 << (62 - bits < 52 ? 62 - bits : 52));
    if (st == GS_F32) sample_kernel<float><<<dim3((unsigned)a.B), dim3(NT), 0, s>>>(a);
    else sample_kernel<bf16_t><<<dim3((unsigned)a.B), dim3(NT), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace gs
