// Matrix products of 16-bit floats and 8-bit integers on the matrix cores, by tiles: C[n][m] = sum_k A[m][k] B[n][k],
// both operands with k contiguous.  Internal to the library (head.hip, i8.hip).
//
// The operand with the rows m gives the result's contiguous index: a lane holds 4 consecutive m of one n for each 16 x 16
// block, so what goes on along a row of the result (a softmax over the vocabulary, a store) stays mostly within a lane.
#pragma once

#include "rows.h"

namespace tt {
namespace tiles {

constexpr int kI8 = 3;         // the 8-bit integers, beside TT_BF16 and TT_F16
constexpr int kStepBytes = 128;  // of k in a row of a tile: 64 elements of 16 bits, 128 of 8

typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef unsigned int u4 __attribute__((ext_vector_type(4)));
typedef unsigned int u4b __attribute__((ext_vector_type(4), aligned(1)));  // 16 bytes at any address

// One 16 x 16 block's product over 64 bytes of k: lane l holds row l % 16 of either operand, bytes 16 (l / 16) and up;
// the result's rows 4 (l / 16) .. + 3 (of the first operand) in column l % 16 (of the second).
template <int DT>
struct Mfma {
    typedef f4 Acc;
    static __device__ __forceinline__ f4 run(u4 a, u4 b, f4 c) {
        typedef __bf16 b8 __attribute__((ext_vector_type(8)));
        typedef _Float16 h8 __attribute__((ext_vector_type(8)));
        if constexpr (DT == TT_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    }
};
template <>
struct Mfma<kI8> {
    typedef i4 Acc;
    static __device__ __forceinline__ i4 run(u4 a, u4 b, i4 c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i4, a), __builtin_bit_cast(i4, b), c, 0, 0, 0);
    }
};

// A matrix with contiguous rows of `bytes` bytes; rows at and past `rows` count as zero.
struct Side {
    const char *p;
    int64_t ld;     // bytes from a row to the next
    int64_t plane;  // bytes from a part of an fp32 matrix to the next one
    int rows;
};

// The sequence of products of fp32 operands held as three bf16 parts each, largest part 0: those of parts i + j <= 2, the
// small ones first.  What is left out is below 2^-24 of the product.
constexpr int kParts = 3, kPasses = 6;
__device__ constexpr int kPartA[kPasses] = {2, 0, 1, 1, 0, 0}, kPartB[kPasses] = {0, 2, 1, 0, 1, 0};

// An fp32 value as three bf16 parts; what is not finite is all in the first.
__device__ __forceinline__ void split(float x, uint32_t (&part)[kParts]) {
    uint32_t hi = rows::encode<TT_BF16>(x);
    if ((hi & 0x7F80u) == 0x7F80u) {
        if ((__float_as_uint(x) & 0x7F800000u) != 0x7F800000u) hi = __float_as_uint(x) >> 16;  // rounded up to infinity
        else {
            part[0] = hi;
            part[1] = part[2] = 0;
            return;
        }
    }
    const float r = x - rows::decode<TT_BF16>(hi);
    const uint32_t mid = rows::encode<TT_BF16>(r);
    part[0] = hi;
    part[1] = mid;
    part[2] = rows::encode<TT_BF16>(r - rows::decode<TT_BF16>(mid));
}

// A tile of TM x TN by WM x WN waves.
template <int TM_, int TN_, int WM_, int WN_>
struct Shape {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_;
    static constexpr int THREADS = WM * WN * 64;
    static constexpr int FM = TM / WM / 16, FN = TN / WN / 16;  // blocks of a wave
    static constexpr int LDS = 2 * (TM + TN) * kStepBytes;
};

template <int ROWS, int THREADS>
struct Staged {
    static constexpr int N = ROWS * 8 / THREADS;  // 16-byte pieces of a thread
    u4 w[N];

    // Bytes k .. k + 127 of the rows from r0 on, into registers; zero outside the matrix.
    __device__ __forceinline__ void load(const Side &s, int64_t part, int r0, int64_t k, int64_t bytes) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * THREADS + (int)threadIdx.x, r = r0 + (c >> 3);
            const int64_t at = k + (c & 7) * 16;
            u4 v = {0, 0, 0, 0};
            if (r < s.rows && at < bytes) {
                const char *q = s.p + part + (int64_t)r * s.ld + at;
                if (at + 16 <= bytes) v = *reinterpret_cast<const u4b *>(q);
                else {
                    for (int j = 0; j < (int)(bytes - at); ++j) {
                        const uint32_t b = (uint32_t)(uint8_t)q[j] << (8 * (j & 3));
                        if (j < 4) v.x |= b;
                        else if (j < 8) v.y |= b;
                        else if (j < 12) v.z |= b;
                        else v.w |= b;
                    }
                }
            }
            w[i] = v;
        }
    }
    // Rows of 128 bytes, their 16-byte pieces in an order that differs between 8 rows in a row: the lanes that read
    // one piece of consecutive rows reach different banks.
    __device__ __forceinline__ void store(char *lds) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * THREADS + (int)threadIdx.x, r = c >> 3;
            *reinterpret_cast<u4 *>(lds + r * kStepBytes + ((c ^ r) & 7) * 16) = w[i];
        }
    }
};

// The tile at (m0, n0) of the product over bytes [k0, k1) of both sides' rows (multiples of 128, or the rows' end `bytes`).
template <int DT, typename S, int PASSES>
__device__ __forceinline__ void product(const Side &a, const Side &b, int m0, int n0, int64_t k0, int64_t k1, int64_t bytes, char *lds,
                                        typename Mfma<DT>::Acc (&acc)[S::FM][S::FN]) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int wm = wave % S::WM, wn = wave / S::WM;
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = {0, 0, 0, 0};
    const int steps = (int)((k1 - k0 + kStepBytes - 1) / kStepBytes), total = steps * PASSES;
    if (total <= 0) return;
    Staged<S::TM, S::THREADS> sa;
    Staged<S::TN, S::THREADS> sb;
    auto load = [&](int t) {
        const int pass = PASSES == 1 ? 0 : t / steps;
        const int64_t k = k0 + (int64_t)(t - pass * steps) * kStepBytes;
        sa.load(a, PASSES == 1 ? 0 : a.plane * kPartA[pass], m0, k, bytes);
        sb.load(b, PASSES == 1 ? 0 : b.plane * kPartB[pass], n0, k, bytes);
    };
    load(0);
    for (int t = 0; t < total; ++t) {
        char *at = lds + (t & 1) * (S::TM + S::TN) * kStepBytes, *bt = at + S::TM * kStepBytes;
        sa.store(at);
        sb.store(bt);
        __syncthreads();
        if (t + 1 < total) load(t + 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u4 fa[S::FM], fb[S::FN];
            auto read = [&](const char *tile, int r) {
                return *reinterpret_cast<const u4 *>(tile + r * kStepBytes + (((h * 4 + (lane >> 4)) ^ r) & 7) * 16);
            };
#pragma unroll
            for (int i = 0; i < S::FM; ++i) fa[i] = read(at, (wm * S::FM + i) * 16 + (lane & 15));
#pragma unroll
            for (int j = 0; j < S::FN; ++j) fb[j] = read(bt, (wn * S::FN + j) * 16 + (lane & 15));
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < S::FN; ++j) acc[i][j] = Mfma<DT>::run(fa[i], fb[j], acc[i][j]);
        }
    }
    __syncthreads();
}

// f(m, n, i, j) for every block of this thread's wave: m the first of its 4 rows, n its column.
template <typename S, typename F>
__device__ __forceinline__ void for_blocks(int m0, int n0, F f) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int wm = wave % S::WM, wn = wave / S::WM;
#pragma unroll
    for (int j = 0; j < S::FN; ++j)
#pragma unroll
        for (int i = 0; i < S::FM; ++i) f(m0 + (wm * S::FM + i) * 16 + (lane >> 4) * 4, n0 + (wn * S::FN + j) * 16 + (lane & 15), i, j);
}

// Four consecutive elements of a row that ends at `end`, rounded to the type.
template <int DT>
__device__ __forceinline__ void store4(typename rows::Elem<DT>::T *row, int m, int end, const float (&y)[4]) {
    typedef unsigned int u2e __attribute__((ext_vector_type(2), aligned(2)));
    typedef unsigned int u4e __attribute__((ext_vector_type(4), aligned(4)));
    if (m + 4 <= end) {
        if constexpr (DT == TT_F32) *reinterpret_cast<u4e *>(row + m) = u4e{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])};
        else *reinterpret_cast<u2e *>(row + m) = u2e{rows::encode_pair<DT>(y[0], y[1]), rows::encode_pair<DT>(y[2], y[3])};
        return;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (m + q < end) row[m + q] = (typename rows::Elem<DT>::T)rows::encode<DT>(y[q]);
}

// Largest value and sum of 2^((z - largest) c) of a set of logits z.  NaN passes through: the sum of a set with a NaN
// or plus infinity is NaN.
struct Part {
    float m, s;
};

__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.0f : m; }

// The parts of the tile's columns from z(i, j, q) (minus infinity where there is no logit), left in lds[n - n0] for
// threads below TN after the closing barrier.  scale(n): log2(e) times the row's inverse temperature.
template <typename S, typename Z, typename C>
__device__ __forceinline__ Part column_parts(int n0, char *lds, Z z, C scale) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int wm = wave % S::WM, wn = wave / S::WM;
    Part *part = reinterpret_cast<Part *>(lds);  // [WM][TN]
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int at = (wn * S::FN + j) * 16 + (lane & 15);
        float m = -INFINITY, s = 0.0f;
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) m = fmaxf(m, z(i, j, q));
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float c = scale(n0 + at), ref = reference(m);
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) s += __builtin_amdgcn_exp2f((z(i, j, q) - ref) * c);
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (lane < 16) part[wm * S::TN + at] = {m, s};
    }
    __syncthreads();
    Part r = {-INFINITY, 0.0f};
    if ((int)threadIdx.x < S::TN) {
        const float c = scale(n0 + (int)threadIdx.x);
#pragma unroll
        for (int w = 0; w < S::WM; ++w) r.m = fmaxf(r.m, part[w * S::TN + threadIdx.x].m);
        const float ref = reference(r.m);
#pragma unroll
        for (int w = 0; w < S::WM; ++w) {
            const Part p = part[w * S::TN + threadIdx.x];
            r.s += p.s * __builtin_amdgcn_exp2f((reference(p.m) - ref) * c);
        }
    }
    return r;
}

// What the parts of a row give, the same in every lane of the wave that holds the row: M, ln S.
__device__ __forceinline__ Part join_row(const Part *part, int n, float beta) {
    const int lane = (int)threadIdx.x & 63;
    float m = -INFINITY;
    for (int t = lane; t < n; t += 64) m = fmaxf(m, part[t].m);
    m = rows::wave_max(m);
    const float ref = reference(m), c = beta * rows::kLog2e;
    double s = 0.0;
    for (int t = lane; t < n; t += 64) {
        const Part p = part[t];
        s += (double)p.s * (double)exp2f((reference(p.m) - ref) * c);
    }
    s = rows::wave_sum(s);
    return {m, m == -INFINITY && s == 0.0 ? 0.0f : (float)log(s)};
}

}  // namespace tiles
}  // namespace tt
