// Tiles shared by the cross-attention kernels (forward and gradient).
//
// A 32 x 32 score block is formed on the matrix cores with the side that a
// wave keeps in registers (32 query rows, or 32 keys in the gradient of K and
// V) as its columns: lane l holds column l % 32 and, of the block's rows,
// 8 g + 4 (l / 32) + e in accumulator register 4 g + e (g, e = 0..3).  The
// second product sums over those rows.  A contraction may take its terms in
// any order as long as both operands agree, so the accumulator registers are
// the second product's operand as they stand: register block PER s .. PER s +
// PER - 1 is the fragment of step s, and col_frag reads the other operand in
// the same order.  Scores never cross lanes, but for the two halves of a column.
#pragma once

#include "gs_internal.h"

namespace gs {
namespace attn {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef short s4v __attribute__((ext_vector_type(4)));
#define GS_LDS __attribute__((address_space(3)))

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Fragments: PER values a lane and step, 2 PER values of the contraction.
template <typename T> struct Op;
template <> struct Op<bf16_t> {
    static constexpr int PER = 8;
    typedef bf8v V;
    static __device__ __forceinline__ f16v mma(V a, V b, f16v c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    // registers PER s .. of an accumulator, rounded to bf16 (nearest even): the
    // probabilities and their gradients enter the second product in the inputs'
    // type, which costs each term half a step of that type, as the inputs' own
    // rounding did
    static __device__ __forceinline__ V pack(const f16v &p, int s) {
        V r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = (__bf16)p[8 * s + e];
        return r;
    }
};
template <> struct Op<float> {
    static constexpr int PER = 4;
    typedef f4v V;
    static __device__ __forceinline__ f16v mma(V a, V b, f16v c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ V pack(const f16v &p, int s) {
        V r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = p[4 * s + e];
        return r;
    }
};

// Heads of Dh values are computed with as DC = 64, 96 or 128 of them (zeros behind
// the last) and lie in LDS, and in parts of rows, as DP = 64 or 128.
constexpr int padded(int dc) { return dc <= 64 ? 64 : 128; }
inline int computed(int64_t dh) { return dh <= 64 ? 64 : (dh <= 96 ? 96 : 128); }

// How blocks of 128 rows (or keys), each of which runs over `pieces` tiles of the
// other side, are dealt out: to work-groups of four waves or of eight, whose two
// halves share the tiles, and every block's tiles to `parts` work-groups, whose
// results another launch adds up.
struct Deal {
    int waves, parts;
};
// The deal that should take least time.  piece_us: a tile's time in a work-group
// of four waves that shares its CU with another one (alone, it takes 0.65 of
// that; eight waves take two tiles in that time); a work-group takes about 3 us
// besides.  `single`: one work-group of four waves a CU.  part_us: the time to
// write and read one part of every block.  (Ten problems, both types, heads of 64
// to 128 values, in 1 to 16 parts with four and with eight waves: the deal was
// within 6 % of the best one in each, forward and gradient; where a block alone
// fills the CUs, two parts cost 1.3 to 1.8 times one, and 3 x 600 x 600, 6 heads
// of 128, fp32, 103 us in one part, 67 in the six dealt.)
inline Deal deal_out(int64_t blocks, int64_t pieces, bool single, double piece_us, double part_us) {
    Deal best = {4, 1};
    double least = 1e300;
    for (int64_t n = 1; n <= pieces && n <= 256 && (n == 1 || blocks * n <= 4096); n += n < 8 ? 1 : n / 4) {
        const int64_t groups = blocks * n;
        const double len = (double)((pieces + n - 1) / n), more = n > 1 ? 4. + (double)n * part_us : 0.;
        const double last = groups % 512 == 0 ? 0. : (groups % 512 <= 256 ? 0.65 : 1.);
        const double rounds = single ? (double)((groups + 255) / 256) : (double)(groups / 512) + last;
        const double four = rounds * (len * piece_us + 3.) + more;
        if (four < least) least = four, best = {4, (int)n};
        if (single || pieces < 2) continue;
        const double eight = (double)((groups + 255) / 256) * (ceil(len / 2.) * piece_us + 3.5) + more;
        if (eight < least) least = eight, best = {8, (int)n};
    }
    return best;
}

// A tile in LDS: rows of DP values in 16-byte chunks, chunk c of row r at
// position c ^ swizzle(r).  256 bytes of LDS (64 banks) are one row or several:
// 16 consecutive rows put the same chunk on 16 different places of those
// (row_frag reads one chunk of 32 rows), and four consecutive rows put four
// consecutive chunks on 16 different ones (what 32 lanes of col_frag's
// transpose reads take).
template <typename T, int DP> __device__ __forceinline__ int place(int r, int c) {
    constexpr int CPR = DP / Op<T>::PER;
    static_assert(CPR == 8 || CPR == 16 || CPR == 32, "rows of 128, 256 or 512 bytes");
    const int s = CPR == 8 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3);
    return (r * CPR + (c ^ s)) * 16;
}

// Operand whose rows are the tile's rows row0 + 0..31, step s of the
// contraction over a row's values.
template <typename T, int DP>
__device__ __forceinline__ typename Op<T>::V row_frag(const char *tile, int row0, int s, int l) {
    return *reinterpret_cast<const typename Op<T>::V *>(tile + place<T, DP>(row0 + (l & 31), 2 * s + (l >> 5)));
}

// Operand whose rows are the values 32 j + 0..31 of the tile's rows, step s of
// the contraction over the rows row0 + 0..31 in accumulator order.
template <typename T, int DP>
__device__ __forceinline__ typename Op<T>::V col_frag(const char *tile, int row0, int s, int j, int l) {
    if constexpr (sizeof(T) == 4) {
        f4v r;
        const int n = 32 * j + (l & 31), k = row0 + 8 * s + 4 * (l >> 5);
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = *reinterpret_cast<const float *>(tile + place<T, DP>(k + e, n >> 2) + 4 * (n & 3));
        return r;
    } else {
        // two transpose reads: 16 lanes read four rows of 16 values and each
        // gets one value of the four rows
        const int gq = l >> 4, a = l & 15;
        const int n = 32 * j + 16 * (gq & 1) + 4 * (a & 3);
        const int k = row0 + 16 * s + 4 * (gq >> 1) + (a >> 2);
        const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GS_LDS s4v *)(tile + place<T, DP>(k, n >> 3) + 2 * (n & 7)));
        const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GS_LDS s4v *)(tile + place<T, DP>(k + 8, n >> 3) + 2 * (n & 7)));
        const s4v both[2] = {lo, hi};
        return *reinterpret_cast<const bf8v *>(both);
    }
}

// 16 bytes (PER values) of a row from value d on; zeros at and past dh.  vec:
// rows start on 16-byte boundaries and dh is a multiple of PER.
template <typename T> __device__ __forceinline__ u4v load_chunk(const T *row, int d, int dh, bool vec) {
    u4v r = {0, 0, 0, 0};
    if (vec) {
        if (d < dh) r = *reinterpret_cast<const u4v *>(row + d);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (d + e < dh) r[e] = __float_as_uint(row[d + e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (d + e < dh) r[e >> 1] |= (uint32_t)row[d + e].bits << (16 * (e & 1));
    }
    return r;
}

// Four consecutive values of a row, rounded to T once.
template <typename T> __device__ __forceinline__ void store4(T *row, int d, int dh, bool vec, f4v v) {
    if (vec) {
        if (d >= dh) return;
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f4v *>(row + d) = v;
        } else {
            u2v p;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const __bf16 two[2] = {(__bf16)v[2 * e], (__bf16)v[2 * e + 1]};
                p[e] = *reinterpret_cast<const uint32_t *>(two);
            }
            *reinterpret_cast<u2v *>(row + d) = p;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (d + e < dh) st_f32<T>(row, d + e, v[e]);
    }
}

__device__ __forceinline__ int clamped(const int32_t *len, int b, int most) {
    if (!len) return most;
    const int n = len[b];
    return n < 0 ? 0 : (n > most ? most : n);
}

// Fragments of the side that stays in registers: row's values as the column
// l % 32 of a product; a null row gives zeros.
template <typename T, int DC>
__device__ __forceinline__ void load_frags(typename Op<T>::V (&f)[DC / (2 * Op<T>::PER)], const T *row, int dh, bool vec, int l) {
    constexpr int PER = Op<T>::PER;
#pragma unroll
    for (int s = 0; s < DC / (2 * PER); ++s) {
        u4v v = {0, 0, 0, 0};
        if (row) v = load_chunk<T>(row, PER * (2 * s + (l >> 5)), dh, vec);
        f[s] = *reinterpret_cast<const typename Op<T>::V *>(&v);
    }
}

// The part of a tile that a thread carries from memory to LDS: rows r of T
// values at base + r * stride; rows whose bit of `live` is off, and values at
// and past dh, are zeros.  VEC: 16-byte pieces, read through a buffer
// descriptor that returns zeros for the offset of a row that is off (base + BN
// rows within 2^31 bytes).
template <typename T, int DP, int BN, int NT, bool VEC> struct TileLoad {
    static constexpr int PER = Op<T>::PER, CPR = DP / PER, N = BN * CPR / NT, RPI = NT / CPR;
    static_assert(BN * CPR % NT == 0 && NT % CPR == 0, "whole chunks per thread");
    u4v v[N];
    __device__ __forceinline__ void fetch(const T *base, int64_t stride, uint64_t live, int dh, int t) {
        const int c = t % CPR, r0 = t / CPR;
        if constexpr (VEC) {
            const uint32_t row = (uint32_t)stride * (uint32_t)sizeof(T);
            const __amdgpu_buffer_rsrc_t rs =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(base), (short)0, 0x7fffffff, 0x00020000);
            const uint32_t at = (uint32_t)r0 * row + 16 * c;
            const uint64_t mine = c * PER < dh ? live >> r0 : 0;
#pragma unroll
            for (int q = 0; q < N; ++q)
                v[q] = __builtin_amdgcn_raw_buffer_load_b128(
                    rs, (int)((mine >> (q * RPI)) & 1 ? at + (uint32_t)(q * RPI) * row : 0x80000000u), 0, 0);
        } else {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                v[q] = u4v{0, 0, 0, 0};
                if ((live >> (r0 + q * RPI)) & 1) v[q] = load_chunk<T>(base + (r0 + q * RPI) * stride, PER * c, dh, false);
            }
        }
    }
    __device__ __forceinline__ void stash(char *tile, int t) const {
#pragma unroll
        for (int q = 0; q < N; ++q) *reinterpret_cast<u4v *>(tile + place<T, DP>(t / CPR + q * RPI, t % CPR)) = v[q];
    }
};

// The same tile brought straight to LDS, a piece of 16 bytes a lane: nothing is
// held in registers on the way.  The loads are written as assembly so that the
// compiler does not wait for them before unrelated LDS reads (it cannot tell
// the buffers apart); wait_tiles orders them.  Rows past the last one are read
// as that one (what is made of them has weight 0); pieces at and past dh are out
// of the resource's range and leave the zeros that clear_lds has put there, or
// zeros.
typedef int i4v __attribute__((ext_vector_type(4)));
template <typename T, int DP, int BN, int NT> struct TileDma {
    static constexpr int PER = Op<T>::PER, CPR = DP / PER, N = BN * CPR / NT;
    static_assert(BN * CPR % NT == 0, "whole pieces per thread");
    static __device__ __forceinline__ void issue(const T *base, int64_t stride, int last, int dh, const char *tile, int t) {
        const uint64_t a = reinterpret_cast<uint64_t>(base);
        i4v rs;
        rs[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
        rs[1] = __builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu));
        rs[2] = 0x7fffffff;
        rs[3] = 0x00020000;
        const uint32_t row = (uint32_t)stride * (uint32_t)sizeof(T);
        const int w = __builtin_amdgcn_readfirstlane(t >> 6);
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int r = (q * NT + t) / CPR, pos = (q * NT + t) % CPR;
            const int c = place<T, DP>(r, pos) / 16 - r * CPR;      // the piece that lies there
            const uint32_t off = c * PER < dh ? (uint32_t)(r < last ? r : last) * row + 16 * c : 0x80000000u;
            const int m0v = __builtin_amdgcn_readfirstlane((int)(size_t)(const GS_LDS char *)tile + (q * NT + 64 * w) * 16);
            asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds"
                         :
                         : "v"(off), "s"(m0v), "s"(rs)
                         : "memory", "m0");
        }
    }
};
template <int NT> __device__ __forceinline__ void clear_lds(char *p, int bytes, int t) {
    for (int i = 16 * t; i < bytes; i += 16 * NT) *reinterpret_cast<u4v *>(p + i) = u4v{0, 0, 0, 0};
}
// All of this wave's loads have landed (vmcnt 0).
__device__ __forceinline__ void wait_tiles() { __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8)); }

// Waits until matrix products have written their results (19 cycles at most).
// hipcc counts these waits itself, but where a branch lies between the products
// and the end of their loop it can (ROCm 7.2) count the longer way round the
// branch for both, and sums are read before they are written.  It did so in one
// instance, which calls this; a test looks at the code of all of them.
template <int N> __device__ __forceinline__ void products_done(f16v (&o)[N]) {
    static_assert(N == 2, "the results are named one by one");
    asm volatile("s_nop 15\n\ts_nop 3" : "+v"(o[0]), "+v"(o[1]));
}

// A row's position and head: packed row m = position G + head within the group.
struct RowOf {
    int i, h;
    __device__ __forceinline__ RowOf(int m, int hk, int G) : i(m / G), h(hk * G + m % G) {}
};

// Which keys of a tile take part.  The mask's bytes are asked for a tile before
// they are needed: the loads of K and V are issued by them, and would wait for
// them otherwise.
template <int BN> struct LiveKeys {
    const uint8_t *mask;
    int kend, l;
    uint8_t byte;
    __device__ __forceinline__ bool there(int j0) const { return l < BN && j0 + l < kend; }
    __device__ __forceinline__ void ahead(int j0) {
        byte = 1;
        if (mask && there(j0)) byte = mask[j0 + l];
    }
    // bit n: key j0 + n takes part (of the tile last asked for)
    __device__ __forceinline__ uint64_t take(int j0) const { return __ballot(there(j0) && byte != 0); }
};
template <int BN> constexpr uint64_t ALL_LIVE = BN == 64 ? ~0ull : (1ull << (BN & 63)) - 1;

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// Consecutive logical work-groups (which share what they read) on one XCD.
__device__ __forceinline__ int64_t logical_group(int64_t total) {
    const int64_t per = (total + 7) / 8;
    return (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
}

}  // namespace attn
}  // namespace gs
