// Building blocks of the kernels that read rows of logits in bf16, fp16 or fp32 (logprobs.hip,
// distill.hip): 16-byte loads of a row's part into registers, wave reductions, order keys.
// Internal to the library.
#pragma once

#include <climits>
#include <cmath>

#include "tt_internal.h"

namespace tt {
namespace rows {

constexpr int kWave = 64;
constexpr int kThreads = 256;        // threads of a workgroup that takes a part of a row, or a short row
constexpr int kWholeThreads = 1024;  // and of one that takes a longer row whole
constexpr float kLog2e = 0x1.715476p+0f;      // log2(e) rounded to fp32
constexpr double kLn2 = 0.693147180559945309;  // ln 2

// 16 bytes at an address aligned to an element only: rows of an odd stride start anywhere, and
// gfx950's 16-byte global accesses take any address.
typedef unsigned int u4u __attribute__((ext_vector_type(4), aligned(2)));

template <int DT>
struct Elem;
template <>
struct Elem<TT_BF16> {
    using T = uint16_t;
    static constexpr int kPer = 8;              // elements of 16 bytes
    static constexpr uint32_t kNone = 0xFF80u;  // minus infinity
};
template <>
struct Elem<TT_F16> {
    using T = uint16_t;
    static constexpr int kPer = 8;
    static constexpr uint32_t kNone = 0xFC00u;
};
template <>
struct Elem<TT_F32> {
    using T = uint32_t;
    static constexpr int kPer = 4;
    static constexpr uint32_t kNone = 0xFF800000u;
};

template <int DT>
__device__ __forceinline__ float decode(uint32_t bits) {
    if constexpr (DT == TT_BF16) return __uint_as_float(bits << 16);
    else if constexpr (DT == TT_F16) return (float)__builtin_bit_cast(_Float16, (unsigned short)bits);
    else return __uint_as_float(bits);
}

// element j of 16 bytes, as fp32
template <int DT>
__device__ __forceinline__ float value(const uint32_t (&w)[4], int j) {
    if constexpr (DT == TT_F32) return __uint_as_float(w[j]);
    else if constexpr (DT == TT_BF16) return __uint_as_float((j & 1) ? (w[j >> 1] & 0xFFFF0000u) : (w[j >> 1] << 16));
    else return decode<DT>((j & 1) ? (w[j >> 1] >> 16) : (w[j >> 1] & 0xFFFFu));
}

template <int DT>
__device__ __forceinline__ void set_bits(uint32_t (&w)[4], int j, uint32_t bits) {
    if constexpr (DT == TT_F32) w[j] = bits;
    else if (j & 1) w[j >> 1] = (w[j >> 1] & 0xFFFFu) | (bits << 16);
    else w[j >> 1] = (w[j >> 1] & 0xFFFF0000u) | bits;
}

// The address of an element of any type.
__device__ __forceinline__ const void *row_at(const void *p, int dtype, int64_t at) {
    return dtype == TT_F32 ? (const void *)(static_cast<const float *>(p) + at) : (const void *)(static_cast<const uint16_t *>(p) + at);
}

// One element of a row of any type, as fp32; NaN counts as minus infinity.
__device__ inline float load_logit(const void *row, int dtype, int64_t x) {
    float f;
    if (dtype == TT_F32) f = static_cast<const float *>(row)[x];
    else if (dtype == TT_F16) f = decode<TT_F16>(static_cast<const uint16_t *>(row)[x]);
    else f = decode<TT_BF16>(static_cast<const uint16_t *>(row)[x]);
    return f != f ? -INFINITY : f;
}

// Index of the first element of thread t's vector i in a part that starts at x_part.
template <int DT, int THREADS>
__device__ __forceinline__ int vector_at(int x_part, int i) {
    return x_part + (i * THREADS + (int)threadIdx.x) * Elem<DT>::kPer;
}

// A part of a row: NV vectors of 16 bytes a thread, each load instruction of a wave covering 1 KB
// of the row; minus infinity past v.  Nothing outside [0, v) is read: a vector that ends past v is
// replaced by the row's last whole one (a valid address) and then formed element by element.
template <int DT, int NV, int THREADS>
__device__ __forceinline__ void load_part(const typename Elem<DT>::T *row, int v, int x_part, uint32_t (&w)[NV][4]) {
    constexpr int kPer = Elem<DT>::kPer;
    if (x_part + NV * THREADS * kPer <= v) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const u4u t = *reinterpret_cast<const u4u *>(row + vector_at<DT, THREADS>(x_part, i));
            w[i][0] = t.x; w[i][1] = t.y; w[i][2] = t.z; w[i][3] = t.w;
        }
        return;
    }
    if (v >= kPer) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int x = vector_at<DT, THREADS>(x_part, i), last = v - kPer;
            const u4u t = *reinterpret_cast<const u4u *>(row + (x < last ? x : last));
            w[i][0] = t.x; w[i][1] = t.y; w[i][2] = t.z; w[i][3] = t.w;
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int x = vector_at<DT, THREADS>(x_part, i);
        if (x + kPer > v) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) set_bits<DT>(w[i], j, x + j < v ? (uint32_t)row[x + j] : Elem<DT>::kNone);
        }
    }
}

// An fp32 value rounded to the row's type, to nearest even.
template <int DT>
__device__ __forceinline__ uint32_t encode(float x) {
    if constexpr (DT == TT_F32) return __float_as_uint(x);
    else if constexpr (DT == TT_F16) return __builtin_bit_cast(unsigned short, (_Float16)x);
    else return __builtin_bit_cast(unsigned short, (__bf16)x);
}

template <int DT>
__device__ __forceinline__ void store_vector(typename Elem<DT>::T *row, int x, int v, const float (&d)[Elem<DT>::kPer]) {
    constexpr int kPer = Elem<DT>::kPer;
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (DT == TT_F32) w[q] = __float_as_uint(d[q]);
        else w[q] = encode<DT>(d[2 * q]) | (encode<DT>(d[2 * q + 1]) << 16);
    }
    if (x + kPer <= v) {
        u4u t;
        t.x = w[0]; t.y = w[1]; t.z = w[2]; t.w = w[3];
        *reinterpret_cast<u4u *>(row + x) = t;
    } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (x + j < v) row[x + j] = (typename Elem<DT>::T)(DT == TT_F32 ? w[j & 3] : (j & 1) ? (w[j >> 1] >> 16) : (w[j >> 1] & 0xFFFFu));
    }
}

__device__ __forceinline__ float scale_of(const float *inv_temp, int64_t row) {
    return inv_temp == nullptr ? 1.0f : inv_temp[row];
}

// With the IEEE bit of the MODE register set, v_max returns a signalling NaN operand quieted and loses
// the other one; with it clear, every NaN operand is passed over.  Cleared at a kernel's start, it
// makes fmaxf over raw logits the maximum of those that are no NaN, at no cost per element.
__device__ __forceinline__ void pass_over_nans() {
    constexpr int kModeIeee = 1 | (9 << 6);  // hardware register 1 (MODE), bit 9, one bit
    __builtin_amdgcn_s_setreg(kModeIeee, 0);
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d);
    return x;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d);
    return x;
}

// Unsigned keys in the order of the values (-0 as +0, minus infinity lowest, no NaN).
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

__device__ __forceinline__ float key_value(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}

// Running statistics of a set of logits at exponent scale c2 = beta * log2(e), relative to their
// largest: m, s = sum of 2^((x - m) c2), e = sum of 2^t t with t = (x - m) c2.
struct Sum {
    float m, s, e;
};

// Scaled exponents are held above this bound: 2^-200 is 0 in fp32, and 0 * -200 is 0 (0 * -inf is not).
constexpr float kLowest = -200.0f;

// The sums of a wave's vectors, the same in every lane; a wave without a finite logit has m = -inf, s = e = 0
// (exponents that are NaN, from NaN logits or from -inf - -inf, count 0).
template <int DT, int NV, bool ENTROPY>
__device__ __forceinline__ Sum wave_sums(const uint32_t (&w)[NV][4], float thread_max, float c2) {
    constexpr int kPer = Elem<DT>::kPer;
    const float m = wave_max(thread_max);
    float s[2] = {0.0f, 0.0f}, e[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            float t = (value<DT>(w[i], j) - m) * c2;
            if constexpr (ENTROPY) {
                t = fmaxf(t, kLowest);
                const float p = __builtin_amdgcn_exp2f(t);
                s[j & 1] += p;
                e[j & 1] = fmaf(p, t, e[j & 1]);
            } else {
                s[j & 1] += fminf(fmaxf(__builtin_amdgcn_exp2f(t), 0.0f), 1.0f);
            }
        }
    }
    Sum r;
    r.m = m;
    r.s = wave_sum(s[0] + s[1]);
    r.e = ENTROPY ? wave_sum(e[0] + e[1]) : 0.0f;
    return r;
}

// The union of two sets' sums.
__device__ __forceinline__ Sum join(const Sum &a, const Sum &b, float c2) {
    Sum r;
    r.m = fmaxf(a.m, b.m);
    const float da = fmaxf((a.m - r.m) * c2, kLowest), db = fmaxf((b.m - r.m) * c2, kLowest);
    const float pa = exp2f(da), pb = exp2f(db);
    r.s = a.s * pa + b.s * pb;
    r.e = (a.e + a.s * da) * pa + (b.e + b.s * db) * pb;
    return r;
}

// The kernels' choice of threads and vectors a thread.  A row is taken whole by one workgroup up to
// kThreads * kWideVectors vectors; longer ones by parts of that size, or smaller ones where they
// would not fill the GPU.
constexpr int kWideVectors = 8;
constexpr int kNarrowVectors = 2;
constexpr int kFullGrid = 1024;  // workgroups that fill the GPU: four a compute unit

inline int elements_per_vector(int dtype) { return dtype == TT_F32 ? 4 : 8; }
inline int element_bytes(int dtype) { return dtype == TT_F32 ? 4 : 2; }

struct Split {
    int threads, vectors;  // of a workgroup, of a thread
    int parts;             // of a row
};

inline Split split_rows(int64_t n_rows, int32_t v, int dtype) {
    const int64_t narrow = (int64_t)kNarrowVectors * kThreads * elements_per_vector(dtype);
    const int64_t wide = (int64_t)kWideVectors * kThreads * elements_per_vector(dtype);
    const int64_t whole = (int64_t)kWideVectors * kWholeThreads * elements_per_vector(dtype);
    if (v <= narrow) return {kThreads, kNarrowVectors, 1};
    if (v <= wide) return {kThreads, kWideVectors, 1};
    if (v <= whole) return {kWholeThreads, kWideVectors, 1};
    const int64_t parts = (v + wide - 1) / wide;
    if (n_rows * parts >= kFullGrid) return {kThreads, kWideVectors, (int)parts};
    return {kThreads, kNarrowVectors, (int)((v + narrow - 1) / narrow)};
}

inline size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

}  // namespace rows
}  // namespace tt
