// Shared by the kernels of the operators (norm, rotary, attention, cross entropy): element types, 16-byte groups, operands of the
// matrix instructions, lane exchanges, and the host's checks and launches.
#ifndef DDP_OPERATORS_H
#define DDP_OPERATORS_H

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <string>
#include <type_traits>

#include "ddp_internal.h"
#include "dreamddp_operators.h"

#pragma clang fp contract(fast)

namespace ddp {
namespace {

typedef __bf16 bf16;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define DDP_LDS __attribute__((address_space(3)))

constexpr float kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// A group of 16 bytes of T in memory, at any element: gfx950 takes 128-bit global accesses at any address.
template <class T>
struct Group {
    static constexpr int n = 16 / (int)sizeof(T);
    T v[n];
};
template <class T>
struct GroupIO;
template <>
struct GroupIO<float> {
    typedef f32x4 vec;
    typedef f32x4 any __attribute__((aligned(4)));
};
template <>
struct GroupIO<bf16> {
    typedef bf16x8 vec;
    typedef bf16x8 any __attribute__((aligned(2)));
};
template <class T>
using Vec = typename GroupIO<T>::vec;
template <class T>
__device__ __forceinline__ Vec<T> load_group(const T *p) {
    return *reinterpret_cast<const typename GroupIO<T>::any *>(p);
}
template <class T>
__device__ __forceinline__ void store_group(T *p, Vec<T> v) {
    *reinterpret_cast<typename GroupIO<T>::any *>(p) = v;
}
// the first n elements of a group, zeros for the rest
template <class T>
__device__ __forceinline__ Vec<T> load_part(const T *p, int n) {
    constexpr int N = Group<T>::n;
    if (n >= N) return load_group(p);
    Vec<T> v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = j < n ? p[j] : (T)0.0f;
    return v;
}
// STREAM: past the caches' usual way, for calls that move more than the last-level cache holds (streams_past).
template <bool STREAM = false, class T>
__device__ __forceinline__ void store_part(T *p, Vec<T> v, int n) {
    constexpr int N = Group<T>::n;
    if (n >= N) {
        if constexpr (STREAM)
            __builtin_nontemporal_store(v, reinterpret_cast<typename GroupIO<T>::any *>(p));
        else
            store_group(p, v);
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < n) p[j] = v[j];
}
// four consecutive elements from fp32, the first n of them
template <class T>
__device__ __forceinline__ void store4(T *p, f32x4 v, int n) {
    typedef T four __attribute__((ext_vector_type(4)));
    typedef four any __attribute__((aligned(sizeof(T))));
    if (n >= 4) {
        *reinterpret_cast<any *>(p) = __builtin_convertvector(v, four);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < n) p[j] = (T)v[j];
}

// ---- lanes -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

// a value that the wavefront's lanes share, known to be so
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// the value of the lane 32 further on, or back
__device__ __forceinline__ float other_half(float v) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);  // the lower half twice, the upper half twice
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? both[0] : both[1]);
}

// ---- matrix instructions ---------------------------------------------------------------------------------------
// C[32][32] += A[32][16] B[16][32].  Lane l gives eight elements of row (column) l % 32, k = (l / 32) * 8 + j.  Which k a place stands for
// is free as long as A and B agree.  Lane l gets column l % 32 and, in register r, row acc_row(l / 32, r).
//
// fp32 operands are three planes of bf16 each, x = a + b + c, what rounding to bf16 left over rounded again: 24 bits and fp32's range.  Six of
// their nine products, aa, ab, ba, bb, ac and ca, leave out terms of 2^-24 relative: as exact as an fp32 product with its sums in
// fp32, and six bf16 products take 0.4 of the time of the fp32 matrix instructions' one.
struct Triple {};
template <class T>
constexpr bool kTriple = std::is_same_v<T, Triple>;
template <class T>
constexpr int kPlanes = kTriple<T> ? 3 : 1;
template <class T>
using Out = std::conditional_t<kTriple<T>, float, T>;  // of tensors in memory
constexpr int kProducts = 6;
// the plane of operand A (B) in each of the six products, small terms first
__device__ __forceinline__ constexpr int plane_of(int product, bool b) { return (b ? 0x021010 : 0x201100) >> (4 * (kProducts - 1 - product)) & 3; }
// what rounding to bf16 leaves over (infinity and NaN are the first plane's alone)
__device__ __forceinline__ float left_over(float x) {
    const float y = (float)(bf16)x;
    return fabsf(y) < kInf ? x - y : 0.0f;
}

template <class T>
struct Operand8 {  // eight elements
    bf16x8 p[kPlanes<T>];
};
template <class T>
__device__ __forceinline__ void mma(f32x16 &c, const Operand8<T> &a, const Operand8<T> &b) {
    if constexpr (kTriple<T>) {
#pragma unroll
        for (int i = 0; i < kProducts; ++i) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[plane_of(i, false)], b.p[plane_of(i, true)], c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[0], b.p[0], c, 0, 0, 0);
    }
}
__device__ __forceinline__ constexpr int acc_row(int half, int r) { return 8 * (r / 4) + 4 * half + r % 4; }

// An accumulator's 32 rows to a lane's place in memory, x its first, times a factor, the first n of them.  bf16: the two lanes of a column
// exchange quads, so that each has eight rows next to each other, 16 bytes, and not two times four.
template <class T>
__device__ __forceinline__ void store_acc(T *x, const f32x16 &c, float factor, int n) {
    const int half = (threadIdx.x & 63) >> 5;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
            f32x4 a, b;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] = c[4 * q + e] * factor;
                b[e] = c[4 * q + 4 + e] * factor;
            }
            const u32x2 u = __builtin_bit_cast(u32x2, __builtin_convertvector(a, bf16x4)), v = __builtin_bit_cast(u32x2, __builtin_convertvector(b, bf16x4));
            const auto lo = __builtin_amdgcn_permlane32_swap(u.x, v.x, false, false), hi = __builtin_amdgcn_permlane32_swap(u.y, v.y, false, false);
            const u32x4 both = {lo[0], hi[0], lo[1], hi[1]};
            const int at = 8 * (q + half);
            if (at < n) store_part(x + at, __builtin_bit_cast(bf16x8, both), n - at);
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int at = acc_row(half, r);
            if (at < n) store4(x + at, f32x4{c[r], c[r + 1], c[r + 2], c[r + 3]} * factor, n - at);
        }
    }
}

// Rows of an accumulator as the next product's operand, whose k they are: rows 16 g .. 16 g + 15, in the order of acc_row.
template <class T>
__device__ __forceinline__ Operand8<T> acc_operand(const f32x16 &c, int g) {
    Operand8<T> v;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float x = c[g * 8 + j];
#pragma unroll
        for (int k = 0; k < kPlanes<T>; ++k) {
            v.p[k][j] = (bf16)x;
            if (k + 1 < kPlanes<T>) x = left_over(x);
        }
    }
    return v;
}

// ---- tiles in LDS ----------------------------------------------------------------------------------------------
// Rows of ROWB bytes (a power of two from 64 on) whose 16-byte groups are exchanged within each run of four (ROWB 64), eight (128) or sixteen by
// the row.  LDS has 64 banks, 256 bytes a cycle: one group of sixteen consecutive rows, and four groups next to each other of four consecutive
// rows, which are what a cycle of tile_row and of tile_col takes, then lie in different banks.  Linear in the row's bits.
template <int ROWB>
__device__ __forceinline__ constexpr int swizzle(int row) {
    return ROWB == 64 ? (row >> 2) & 3 : ROWB == 128 ? (row & 2) << 1 | ((row >> 2) & 3) : (row & 3) << 2 | ((row >> 2) & 3);
}
template <int ROWB>
__device__ __forceinline__ int tile_at(int row, int group) {
    return row * ROWB + ((group ^ swizzle<ROWB>(row)) << 4);
}
template <int ROWB>
__device__ __forceinline__ bf16x8 tile_row(const char *tile, int row, int group) {
    return *reinterpret_cast<const bf16x8 *>(tile + tile_at<ROWB>(row, group));
}
// The operand whose k runs down the tile's rows and whose 32 rows (columns) are the tile's columns from col0 on.  Column col0 + l % 32 at
// the rows k0 + acc_row(half, ..), the order of acc_operand, or with PLAIN k0 + half * 8 + .., that of tile_row.
template <int ROWB, bool PLAIN = false>
__device__ __forceinline__ bf16x8 tile_col(const char *tile, int k0, int col0, int lane) {
    const int half = lane >> 5;
    // each 16 lanes read four rows of 16 columns and get four rows of a column each
    const int row = k0 + (PLAIN ? 8 : 4) * half + ((lane & 15) >> 2), col = col0 + (lane & 16) + (lane & 3) * 4;
    s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DDP_LDS s16x4 *)(tile + tile_at<ROWB>(row, col >> 3) + (col & 7) * 2));
    s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DDP_LDS s16x4 *)(tile + tile_at<ROWB>(row + (PLAIN ? 4 : 8), col >> 3) + (col & 7) * 2));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, both);
}

// ---- host ------------------------------------------------------------------------------------------------------
inline int launched(const char *who) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return DDP_OK;
    return fail(nullptr, DDP_EHIP, std::string(who) + ": kernel launch failed: " + hipGetErrorString(e));
}
inline int bad(const char *who, int code, const char *what) { return fail(nullptr, code, std::string(who) + ": " + what); }
inline size_t element_size(int dtype) { return dtype == DDP_BF16 ? 2 : 4; }
inline bool typed(int dtype) { return dtype == DDP_F32 || dtype == DDP_BF16; }
inline bool misaligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
inline int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
// The most workgroups of a launch: a dimension of a grid has less than 2^32 threads.  Of one that has more a part runs, without an error.
constexpr int64_t most_groups(int threads) { return (((int64_t)1 << 32) - 1) / threads; }
// Whether a call that moves so many bytes writes its results with streaming stores.  From the 256 MB of the last-level cache on they take less:
// rotary positions of 16384 tokens, 40 heads of 128, 66 against 61 us, norm of 16384 x 4096 in bf16 forward 48 against 43, backward 83
// against 77.  Below, what they save is lost by the next reader of the results: norm of 2048 x 4096 1.7 us less, a copy of its result 1.4 more.
inline bool streams_past(int64_t bytes) { return bytes >= (int64_t)256 << 20; }
constexpr int64_t kMost = (int64_t)1 << 46;  // elements of a tensor: their bytes, and sums of a few such, fit 64 bits
// (n - 1) * stride, or -1 where it is more than kMost
inline int64_t reach(int64_t n, int64_t stride) {
    if (n <= 1) return 0;
    if (stride < 0 || stride > kMost / (n - 1)) return -1;
    return (n - 1) * stride;
}

}  // namespace
}  // namespace ddp

#endif
