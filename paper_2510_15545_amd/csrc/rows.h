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
constexpr int kThreads = 256;  // of a workgroup, unless said otherwise
constexpr float kLog2e = 0x1.715476p+0f;      // log2(e) rounded to fp32
constexpr double kLn2 = 0.693147180559945309;  // ln 2

// 16 bytes at an address aligned to an element only: rows of an odd stride start anywhere, and
// gfx950's 16-byte global accesses take any address.
typedef unsigned int u4u __attribute__((ext_vector_type(4), aligned(2)));

// A load known to the compiler as one from global memory, where a pointer's origin does not tell it (a flat
// load's wait would wait for every load in flight).
// LAST: this is the only or the last reading (the non-temporal hint keeps such lines from displacing others).
template <bool LAST>
__device__ __forceinline__ u4u load_global(const void *p) {
    const auto *g = reinterpret_cast<const __attribute__((address_space(1))) u4u *>(reinterpret_cast<uintptr_t>(p));
    if constexpr (LAST) return __builtin_nontemporal_load(g);
    else return *g;
}

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

// An fp32 value rounded to the row's type, to nearest even.
template <int DT>
__device__ __forceinline__ uint32_t encode(float x) {
    if constexpr (DT == TT_F32) return __float_as_uint(x);
    else if constexpr (DT == TT_F16) return __builtin_bit_cast(unsigned short, (_Float16)x);
    else return __builtin_bit_cast(unsigned short, (__bf16)x);
}

// Two values as the row holds them, the first in the lower half.
template <int DT>
__device__ __forceinline__ uint32_t encode_pair(float x, float y) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const f2 v = {x, y};
    if constexpr (DT == TT_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, h2));
}

// A vector's values in the row's type.
template <int DT>
__device__ __forceinline__ void encode_vector(const float (&d)[Elem<DT>::kPer], uint32_t (&w)[4]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (DT == TT_F32) w[q] = __float_as_uint(d[q]);
        else w[q] = encode_pair<DT>(d[2 * q], d[2 * q + 1]);
    }
}

// A vector's elements at 0 <= x < v, one by one.
template <int DT>
__device__ __forceinline__ void store_elements(typename Elem<DT>::T *row, int x, int v, const uint32_t (&w)[4]) {
#pragma unroll
    for (int j = 0; j < Elem<DT>::kPer; ++j)
        if (x + j >= 0 && x + j < v)
            row[x + j] = (typename Elem<DT>::T)(DT == TT_F32 ? w[j & 3] : (j & 1) ? (w[j >> 1] >> 16) : (w[j >> 1] & 0xFFFFu));
}

// A chunk's vectors, in the row's type, to the row; KEEP: without the non-temporal hint, which keeps lines that are
// not read here from displacing others.  (Not a value: of two stores that differ in the hint alone the compiler
// makes one without it.)
template <int DT, int NV, int THREADS, bool KEEP>
__device__ __forceinline__ void store_chunk(typename Elem<DT>::T *row, int v, int x_chunk, const uint32_t (&w)[NV][4]) {
    constexpr int kPer = Elem<DT>::kPer;
    auto store = [&](int i, int x) {
        u4u t;
        t.x = w[i][0]; t.y = w[i][1]; t.z = w[i][2]; t.w = w[i][3];
        if constexpr (KEEP) *reinterpret_cast<u4u *>(row + x) = t;
        else __builtin_nontemporal_store(t, reinterpret_cast<u4u *>(row + x));
    };
    if (x_chunk >= 0 && x_chunk + NV * THREADS * kPer <= v) {
#pragma unroll
        for (int i = 0; i < NV; ++i) store(i, vector_at<DT, THREADS>(x_chunk, i));
        return;
    }
    int end = v;  // where the thread's vector begins that the row ends in
    uint32_t part[4] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int x = vector_at<DT, THREADS>(x_chunk, i);
        if (x >= 0 && x + kPer <= v) {
            store(i, x);
        } else if (x >= 0 && x < v) {
            end = x;
#pragma unroll
            for (int q = 0; q < 4; ++q) part[q] = w[i][q];
        }
    }
    if (end < v) store_elements<DT>(row, end, v, part);
    if (x_chunk < 0 && threadIdx.x == 0) store_elements<DT>(row, x_chunk, v, w[0]);
}

__device__ __forceinline__ float scale_of(const float *inv_temp, int64_t row) {
    return inv_temp == nullptr ? 1.0f : inv_temp[row];
}

// Whether a row has a distribution at this inverse temperature: above 2^100 the scaled exponents of equal logits
// would no longer be numbers.
__device__ __forceinline__ bool sound(double beta) { return beta > 0.0 && beta <= 0x1p100; }

// With the IEEE bit of the MODE register set, v_max returns a signalling NaN operand quieted and loses
// the other one; with it clear, every NaN operand is passed over.  Cleared at a kernel's start, it
// makes fmaxf over raw logits the maximum of those that are no NaN, at no cost per element.
__device__ __forceinline__ void pass_over_nans() {
    constexpr int kModeIeee = 1 | (9 << 6);  // hardware register 1 (MODE), bit 9, one bit
    __builtin_amdgcn_s_setreg(kModeIeee, 0);
}

// x of other lanes by a DPP control; lanes without a source get `none`.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp(float x, float none) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(none), __float_as_uint(x), CTRL, ROW_MASK, 0xF, false));
}
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ double dpp(double x, double none) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x), o = __builtin_bit_cast(uint64_t, none);
    const uint32_t lo = __builtin_amdgcn_update_dpp((uint32_t)o, (uint32_t)b, CTRL, ROW_MASK, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp((uint32_t)(o >> 32), (uint32_t)(b >> 32), CTRL, ROW_MASK, 0xF, false);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ uint32_t dpp(uint32_t x, uint32_t none) {
    return __builtin_amdgcn_update_dpp(none, x, CTRL, ROW_MASK, 0xF, false);
}
__device__ __forceinline__ uint32_t last_lane(uint32_t x) { return __builtin_amdgcn_readlane(x, kWave - 1); }
__device__ __forceinline__ float last_lane(float x) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), kWave - 1)); }
__device__ __forceinline__ double last_lane(double x) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)b, kWave - 1), hi = __builtin_amdgcn_readlane((uint32_t)(b >> 32), kWave - 1);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

// A wave's reduction by f, the same in every lane (prefixes within rows of 16 lanes, then row broadcasts).
template <typename T, typename F>
__device__ __forceinline__ T wave_reduce(T x, T none, F f) {
    x = f(x, dpp<0x111, 0xF>(x, none));
    x = f(x, dpp<0x112, 0xF>(x, none));
    x = f(x, dpp<0x114, 0xF>(x, none));
    x = f(x, dpp<0x118, 0xF>(x, none));
    x = f(x, dpp<0x142, 0xA>(x, none));
    x = f(x, dpp<0x143, 0xC>(x, none));
    return last_lane(x);
}
__device__ __forceinline__ float wave_max(float x) {
    return wave_reduce(x, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    return wave_reduce(x, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint32_t wave_min(uint32_t x) {
    return wave_reduce(x, 0xFFFFFFFFu, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
template <typename T>
__device__ __forceinline__ T wave_sum(T x) {
    return wave_reduce(x, T(0), [](T a, T b) { return a + b; });
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

// Chunks of long rows begin at the row's address rounded down to 16 bytes (rows of an odd width begin
// anywhere): the row's first element is this many elements into its first chunk.  1,000 rows of 50,257 bf16
// and their gradients: 58.9 to 51.2 us (distillation), 43.6 to 40.7 (backward); rows of 60, whose first
// vectors would all be guarded: 50.9 to 71.4, so short rows begin where they begin.
constexpr int kLead = 7;           // at most
constexpr int kLeadRows = 4096;    // elements of a row from which on it has one

template <int DT>
__device__ __forceinline__ int lead_of(const void *row, int v) {
    return v < kLeadRows ? 0 : (int)(reinterpret_cast<uintptr_t>(row) % 16) / (int)sizeof(typename Elem<DT>::T);
}

// A chunk of a row: NV vectors of 16 bytes a thread.  The loads are unconditional, so that a chunk's loads
// stay in flight while the one before is worked on: a vector that would begin before the row or end past
// v is taken from the row's first or last elements instead (v >= kPer), and put right by fix_chunk once
// it has arrived.
template <int DT, int NV, int THREADS, bool LAST>
__device__ __forceinline__ void load_chunk(const typename Elem<DT>::T *row, int v, int x_chunk, uint32_t (&w)[NV][4]) {
    const int last = v - Elem<DT>::kPer;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        int x = vector_at<DT, THREADS>(x_chunk, i);
        x = x < last ? x : last;
        const u4u t = load_global<LAST>(row + (x > 0 ? x : 0));
        w[i][0] = t.x; w[i][1] = t.y; w[i][2] = t.z; w[i][3] = t.w;
    }
}

// Moves a vector's elements by 0 < n < kPer places towards the front (DOWN) or the back, minus infinity behind them.
template <int DT, bool DOWN>
__device__ __forceinline__ void shift_vector(uint32_t (&w)[4], int n) {
    constexpr uint32_t kNone = Elem<DT>::kNone, kNones = DT == TT_F32 ? kNone : kNone * 0x10001u;
    auto at = [&](const uint32_t(&o)[4], int q) { return q >= 0 && q < 4 ? o[q & 3] : kNones; };
    int words = n;
    if constexpr (DT != TT_F32) {
        if (n & 1) {
            const uint32_t o[4] = {w[0], w[1], w[2], w[3]};
#pragma unroll
            for (int q = 0; q < 4; ++q)
                w[q] = DOWN ? (o[q] >> 16) | (at(o, q + 1) << 16) : (o[q] << 16) | (at(o, q - 1) >> 16);
        }
        words = n >> 1;
    }
#pragma unroll
    for (int step = 1; step <= 2; step <<= 1) {
        if (words & step) {
            const uint32_t o[4] = {w[0], w[1], w[2], w[3]};
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = at(o, DOWN ? q + step : q - step);
        }
    }
}

// Minus infinity before the row and past v: the vectors that load_chunk took from the row's ends lose the elements
// that are other vectors', the rest move to their places.
template <int DT, int NV, int THREADS>
__device__ __forceinline__ void fix_chunk(int v, int x_chunk, uint32_t (&w)[NV][4]) {
    constexpr int kPer = Elem<DT>::kPer;
    if (x_chunk < 0 && threadIdx.x == 0) shift_vector<DT, false>(w[0], -x_chunk);  // the row's lead
    if (x_chunk + NV * THREADS * kPer <= v) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int over = vector_at<DT, THREADS>(x_chunk, i) - (v - kPer);  // elements to drop
        if (over >= kPer) w[i][0] = w[i][1] = w[i][2] = w[i][3] = DT == TT_F32 ? Elem<DT>::kNone : Elem<DT>::kNone * 0x10001u;
        else if (over > 0) shift_vector<DT, true>(w[i], over);
    }
}

// A thread's sums with its vectors of one more chunk; vm: the largest values of these.  NaN logits and
// those of a thread without a finite one count 0 (their exponents are NaN: held at kLowest, or clamped).
template <int DT, int NV, bool ENTROPY>
__device__ __forceinline__ void add_chunk(const uint32_t (&w)[NV][4], float c2, Sum &a, float (&vm)[NV]) {
    constexpr int kPer = Elem<DT>::kPer;
    float m = a.m;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        vm[i] = -INFINITY;
#pragma unroll
        for (int j = 0; j < kPer; ++j) vm[i] = fmaxf(vm[i], value<DT>(w[i], j));
        m = fmaxf(m, vm[i]);
    }
    const float d = fmaxf((a.m - m) * c2, kLowest), f = __builtin_amdgcn_exp2f(d);
    float s[2] = {}, e[2] = {};
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
    // the chunk's sums by themselves, then to the others': one rounding a chunk at the size of the whole sum
    if constexpr (ENTROPY) a.e = fmaf(fmaf(a.s, d, a.e), f, e[0] + e[1]);
    a.s = fmaf(a.s, f, s[0] + s[1]);
    a.m = m;
}

// The wave's sums from its threads', the same in every lane.
template <bool ENTROPY>
__device__ __forceinline__ Sum wave_join(const Sum &a, float c2) {
    Sum r;
    r.m = wave_max(a.m);
    const float d = fmaxf((a.m - r.m) * c2, kLowest), f = __builtin_amdgcn_exp2f(d);
    r.s = wave_sum(a.s * f);
    r.e = ENTROPY ? wave_sum(fmaf(a.s, d, a.e) * f) : 0.0f;
    return r;
}

// What rows shorter than a vector are loaded from (their elements are then read one by one).
static __device__ const uint32_t kNoRow[4] = {};

// Calls f(vectors, first element) for every chunk from x0 to x1 (x0: whole chunks from the row's lead before it),
// minus infinity before the row and past v, while the next chunk's loads are in flight; before() once the first chunk's are.
// BACK: from the last chunk to the first.  AHEAD false: a chunk's loads only when it is its turn (for a workgroup
// of one chunk, or now and then two).
template <int DT, int NV, int THREADS, bool LAST, bool BACK, bool AHEAD, int UNROLL, typename B, typename F>
__device__ __forceinline__ void for_chunks(const typename Elem<DT>::T *row, int v, int x0, int x1, B before, F f) {
    using T = typename Elem<DT>::T;
    constexpr int kPer = Elem<DT>::kPer, kChunk = NV * THREADS * kPer;
    const bool tiny = v < kPer;
    const T *from = tiny ? reinterpret_cast<const T *>(kNoRow) : row;
    const int width = tiny ? kPer : v;
    const int n = (x1 - x0 + kChunk - 1) / kChunk, step = BACK ? -kChunk : kChunk;
    int x = BACK ? x0 + (n - 1) * kChunk : x0;
    uint32_t w[NV][4];
    load_chunk<DT, NV, THREADS, LAST>(from, width, x, w);
    if (tiny) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) set_bits<DT>(w[0], j, j < v ? (uint32_t)row[j] : Elem<DT>::kNone);
    }
    before();
#pragma unroll UNROLL
    for (int c = 1; c <= n; ++c, x += step) {
        uint32_t next[NV][4];
        if constexpr (AHEAD) load_chunk<DT, NV, THREADS, LAST>(from, width, c < n ? x + step : width, next);  // past the end: one line
        fix_chunk<DT, NV, THREADS>(width, x, w);
        f(w, x);
        if constexpr (AHEAD) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) w[i][q] = next[i][q];
        } else if (c < n) {
            load_chunk<DT, NV, THREADS, LAST>(from, width, x + step, w);
        }
    }
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

constexpr int kFullGrid = 1024;  // workgroups of kThreads that fill the GPU: four a compute unit
inline int elements_per_vector(int dtype) { return dtype == TT_F32 ? 4 : 8; }
inline int element_bytes(int dtype) { return dtype == TT_F32 ? 4 : 2; }

inline size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

}  // namespace rows
}  // namespace tt
