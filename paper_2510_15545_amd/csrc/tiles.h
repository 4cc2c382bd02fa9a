// Matrix products of bf16, fp16, fp32 and 8-bit integers on the matrix cores, by tiles: C[n][m] = sum_k A[m][k] B[n][k].
// Internal to the library (head.hip, i8.hip).
//
// The operand with the rows m gives the result's contiguous index: a lane holds 4 consecutive m of one n for each 16 x 16
// block, so what goes on along a row of the result (a softmax over the vocabulary, a store) stays mostly within a lane.
#pragma once

#include <type_traits>

#include "rows.h"

namespace tt {
namespace tiles {

constexpr int kI8 = 3;           // the 8-bit integers, beside TT_BF16, TT_F16 and TT_F32
constexpr int kStepBytes = 128;  // of k that a step takes of every row: 64 elements of 16 bits, 32 of 32, 128 of 8

typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef unsigned int u4 __attribute__((ext_vector_type(4)));
typedef unsigned int u4b __attribute__((ext_vector_type(4), aligned(1)));  // 16 bytes at any address

constexpr __host__ __device__ int bytes_of(int dt) { return dt == TT_F32 ? 4 : dt == kI8 ? 1 : 2; }

// One 16 x 16 block's product over 64 bytes of k: lane l holds row l % 16 of either operand, bytes 16 (l / 16) and up;
// the result's rows 4 (l / 16) .. + 3 (of the first operand) in column l % 16 (of the second).  fp32: four products over 4
// elements each, the j-th over elements j of the four lanes' 16 bytes.
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
struct Mfma<TT_F32> {
    typedef f4 Acc;
    static __device__ __forceinline__ f4 run(u4 a, u4 b, f4 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
        return c;
    }
};
template <>
struct Mfma<kI8> {
    typedef i4 Acc;
    static __device__ __forceinline__ i4 run(u4 a, u4 b, i4 c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i4, a), __builtin_bit_cast(i4, b), c, 0, 0, 0);
    }
};

// A matrix of `rows` rows of `bytes` bytes, `ld` bytes from one to the next.
struct Side {
    const char *p;
    int64_t ld;
    int rows;
    int bytes;
};

// A tile of TM x TN by WM x WN waves, wave w at (w / WN, w % WN).
template <int TM_, int TN_, int WM_, int WN_>
struct Shape {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_;
    static constexpr int THREADS = WM * WN * 64;
    static constexpr int FM = TM / WM / 16, FN = TN / WN / 16;  // blocks of a wave
    static constexpr int LDS = 2 * (TM + TN) * kStepBytes;
    // The blocks of 16 rows and columns that a wave's blocks (i, j) lie in.
    static __device__ __forceinline__ int row_block(int wave, int i) { return wave / WN * FM + i; }
    static __device__ __forceinline__ int column_block(int wave, int j) { return wave % WN * FN + j; }
};

// 16 bytes at any global address that are read once (the non-temporal hint keeps such lines from displacing others).
__device__ __forceinline__ u4 load_once(const char *p) {
    return __builtin_nontemporal_load(reinterpret_cast<const __attribute__((address_space(1))) u4b *>(reinterpret_cast<uintptr_t>(p)));
}

// The first n (below 16) bytes at q, one by one; zeros behind them.
__device__ inline u4 load_some(const char *q, int n) {
    u4 v = {0, 0, 0, 0};
    for (int j = 0; j < n; ++j) {
        const uint32_t b = (uint32_t)(uint8_t)q[j] << (8 * (j & 3));
        if (j < 4) v.x |= b;
        else if (j < 8) v.y |= b;
        else if (j < 12) v.z |= b;
        else v.w |= b;
    }
    return v;
}

template <int ROWS, int THREADS>
struct Staged {
    static constexpr int N = ROWS * 8 / THREADS;  // 16-byte pieces of a thread
    u4 w[N];

    // Bytes k .. k + 127 of the rows from r0 on, into registers; zero outside the matrix.
    __device__ __forceinline__ void load(const Side &s, int r0, int k) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * THREADS + (int)threadIdx.x, r = r0 + (c >> 3);
            const int at = k + (c & 7) * 16;
            u4 v = {0, 0, 0, 0};
            if (r < s.rows && at < s.bytes) {
                const char *q = s.p + (int64_t)r * s.ld + at;
                v = at + 16 <= s.bytes ? (u4)*reinterpret_cast<const u4b *>(q) : load_some(q, s.bytes - at);
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

// The tile at (m0, n0) of the product of two matrices with k contiguous, staged through registers: any alignment, any width.
template <int DT, typename S>
__device__ __forceinline__ void product_any(const Side &a, const Side &b, int m0, int n0, char *lds, typename Mfma<DT>::Acc (&acc)[S::FM][S::FN]) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int wm = wave / S::WN, wn = wave % S::WN;
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = {0, 0, 0, 0};
    const int total = (a.bytes + kStepBytes - 1) / kStepBytes;
    Staged<S::TM, S::THREADS> sa;
    Staged<S::TN, S::THREADS> sb;
    auto load = [&](int t) {
        sa.load(a, m0, t * kStepBytes);
        sb.load(b, n0, t * kStepBytes);
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

// ------------------------------------------------------------------------------------------------ tiles by loads to LDS
typedef __attribute__((address_space(3))) void *lds_ptr;

// Tiles of 64 C columns (rows of the second operand).  Wide: 256 rows of the first operand, 8 waves of 128 x 16 C, one
// workgroup to a compute unit.  Half: 128 rows, 4 waves of 64 x 32 C, two workgroups.  A wave's blocks of 16 lie apart, in
// groups of four: block 4 i + c of a side for a few c.
template <int C>
struct Wide {
    static constexpr int TM = 256, TN = 64 * C, COLUMNS = C, WAVES = 8, WM = 2, WN = 4, THREADS = 512, FM = 8, FN = C;
    static __device__ __forceinline__ int row_c(int wave, int i) { return (wave >> 2) * 2 + (i >> 2); }
    static __device__ __forceinline__ int column_c(int wave, int) { return wave & 3; }
    static constexpr __device__ int row_i(int i) { return i & 3; }
    static constexpr __device__ int column_i(int j) { return j; }
    static __device__ __forceinline__ int row_block(int wave, int i) { return row_i(i) * 4 + row_c(wave, i); }
    static __device__ __forceinline__ int column_block(int wave, int j) { return column_i(j) * 4 + column_c(wave, j); }
};
template <int C>
struct Half {
    static constexpr int TM = 128, TN = 64 * C, COLUMNS = C, WAVES = 4, WM = 2, WN = 2, THREADS = 256, FM = 4, FN = 2 * C;
    static __device__ __forceinline__ int row_c(int wave, int i) { return (wave >> 1) * 2 + (i >> 1); }
    static __device__ __forceinline__ int column_c(int wave, int j) { return (wave & 1) * 2 + (j & 1); }
    static constexpr __device__ int row_i(int i) { return i & 1; }
    static constexpr __device__ int column_i(int j) { return j >> 1; }
    static __device__ __forceinline__ int row_block(int wave, int i) { return row_i(i) * 4 + row_c(wave, i); }
    static __device__ __forceinline__ int column_block(int wave, int j) { return column_i(j) * 4 + column_c(wave, j); }
};

// 16 bytes a lane from the memory's start + `at`, to LDS at `to` and on, in the order of the lanes.  Written as an instruction
// because the compiler, which cannot tell the two steps' buffers apart across a loop, would have every read of LDS wait for all
// loads; here they are waited for where a step begins (vmcnt).  Nothing is returned to registers, and addresses are read at issue.
__device__ __forceinline__ void load_to_lds(u4 memory, uint32_t at, uint32_t to) {
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(at), "s"(memory), "{m0}"(to) : "memory");
}

// One operand's tile of a step: ROWS rows of the result by 128 bytes of k, brought to LDS by loads that go past the
// registers (a wave's 64 lanes fill 1 KB), from memory with k contiguous, or (KM) with the rows of the result contiguous.
// k contiguous: rows of 128 bytes, the 16-byte pieces of row r at place piece ^ (r & 7).  KM: lines of one k; the 16
// elements of a block at place block ^ s(k), s different for the eight lines that 32 lanes read together; the 16-bit elements are
// transposed by the reading (ds_read_b64_tr_b16: lane l of 16 gets element l of the four lines that their lanes' 8 bytes
// lie in), the 32-bit ones read one by one.  All of LDS's banks are reached evenly in every case.
template <int DT, bool KM, int ROWS, int WAVES>
struct Operand {
    static constexpr int E = DT == TT_F32 ? 4 : 2;         // KM: bytes of an element
    static constexpr int LINE = ROWS * E, BLOCK = 16 * E;  // KM: bytes of a line and of a block in it
    static constexpr int K = kStepBytes / E;               // KM: lines of a step
    static constexpr int N = ROWS / 8 / WAVES;             // loads of a wave
    const char *p;
    int64_t ld;
    uint32_t at[N];
    int lane, wave, lines;  // KM: lines from the first step's first to the end

    static_assert(!KM || ROWS == 128 || ROWS == 256, "places of whole groups of 8 blocks");
    static __device__ __forceinline__ int place(int k) { return E == 2 ? (k & 3) | (k >> 3 & 1) << 2 : k >> 2 & 3; }
    // r0: the tile's first row; step0: steps to leave out.  Rows past the matrix's end are those of its last row, bytes
    // past a line's end those of its end.
    __device__ __forceinline__ void begin(const Side &s, int r0, int step0) {
        lane = (int)threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        if constexpr (!KM) {
            p = s.p + r0 * s.ld + (int64_t)step0 * kStepBytes;
#pragma unroll
            for (int i = 0; i < N; ++i)
                at[i] = __umul24(min((wave * N + i) * 8 + (lane >> 3), s.rows - 1 - r0), (int)s.ld) + ((lane & 7) ^ (lane >> 3)) * 16;
        } else {
            p = s.p + (int64_t)step0 * K * s.ld + r0 * E;
            ld = s.ld;
            lines = s.rows - step0 * K;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int b = (wave * N + i) * 1024 + lane * 16, k = b / LINE, c = (b % LINE / BLOCK ^ place(k)) * BLOCK + b % BLOCK;
                at[i] = __umul24(k, (int)s.ld) + min(c, s.bytes - 16 - r0 * E);
            }
        }
    }
    // more: bytes to a matrix of the same form.
    __device__ __forceinline__ void fetch(char *tile, int t, int64_t more = 0) const {
        const uint64_t from = reinterpret_cast<uint64_t>(p) + (KM ? (int64_t)t * K * ld : (int64_t)t * kStepBytes) + more;
        const u4 memory = {(uint32_t)from, (uint32_t)(from >> 32), 0xFFFFFFFFu, 0x00027000u};
        const uint32_t to = (uint32_t)reinterpret_cast<uintptr_t>((lds_ptr)tile) + wave * N * 1024;
        if (KM && (t + 1) * K > lines) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                load_to_lds(memory, at[i] - __umul24(max(0, ((wave * N + i) * 1024 + lane * 16) / LINE - (lines - 1 - t * K)), (int)ld), to + i * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) load_to_lds(memory, at[i], to + i * 1024);
        }
    }
    // Half h (64 bytes of k) of a step for the rows of block 4 i + c (c below 4: one or two addresses serve all i).
    __device__ __forceinline__ u4 read(const char *tile, int c, int i, int h) const {
        if constexpr (!KM) {
            return *reinterpret_cast<const u4 *>(tile + c * 2048 + i * 8192 + (lane & 15) * kStepBytes + ((h * 4 + (lane >> 4)) ^ (lane & 7)) * 16);
        } else if constexpr (E == 2) {
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef short s8 __attribute__((ext_vector_type(8)));
            typedef __attribute__((address_space(3))) s4 *s4_ptr;
            const int k = (lane >> 4) * 8 + (lane >> 2 & 3);
            const char *q = tile + k * LINE + (lane & 3) * 8 + ((i * 4 + c) ^ place(k)) * BLOCK + h * 32 * LINE;
            const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s4_ptr)q), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s4_ptr)(q + 4 * LINE));
            return __builtin_bit_cast(u4, (s8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const int k = (lane >> 4) * 4;
            const char *q = tile + k * LINE + (lane & 15) * 4 + (c ^ place(k)) * BLOCK + i * 4 * BLOCK + h * 16 * LINE;
            u4 f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = *reinterpret_cast<const uint32_t *>(q + j * LINE);
            return f;
        }
    }
};

// LDS of a tile's product: three steps of the first operand, two of the second.
#define TT_TILE_LDS(S) __shared__ __attribute__((aligned(1024))) char lds[(3 * S::TM + 2 * S::TN) * kStepBytes]

// The tile at (m0, n0) of the product over the steps [step0, step0 + steps).  Needs 16-byte aligned rows; k contiguous: whole
// steps of 128 bytes.  twice = 1: the second operand is a sum of two matrices, `rest` bytes apart; each step of the first is
// multiplied with the one's, then the other's.
//
// Wide tiles: waves 0-3 hold half of the blocks of 16 rows, 4-7 the other half; every SIMD runs one of each.  A step is two
// halves of k: reads from LDS, barrier, matrix instructions, barrier.  The second half's waves are one barrier behind, so
// that on every SIMD one wave's reads lie beside the other's matrix instructions.  The second operand (hidden states, tokens: it
// comes from the L2) is loaded a step ahead, the first one (the weights, from HBM) two: one was too short for it (8-bit 288 x
// 128,256 x 2,048 132 us against 127, the gradient of 391 x 50,257 x 1,024 201 against 191).
// 8,192^3 with plain stores: bf16 790 us, 1,390 TFLOP/s, 8 bits 420 us, 2,600 TOP/s.  The matrix instructions take 63% of the cycles
// of 4,096 x 151,936 x 2,048 bf16, 55% of 2,304 x 151,936 x 4,096 in 8 bits, and the clock falls to 1.8 GHz under them: fewer cycles
// (a twenty-fifth less by even halves) gain little in bf16.
// Blocks of 32 x 32 are slower (1,330 and 2,460).
//
// Half tiles: two workgroups to a compute unit, whose reads, matrix instructions, beginnings and ends lie beside each other as
// they come.
template <int DT, bool AKM, bool BKM, typename S>
struct Product {
static __device__ __forceinline__ void run(const Side &a, const Side &b, int m0, int n0, int step0, int steps, char *lds,
                                           typename Mfma<DT>::Acc (&acc)[S::FM][S::FN], int twice = 0, int64_t rest = 0) {
    Operand<DT, AKM, S::TM, S::WAVES> oa;
    Operand<DT, BKM, S::TN, S::WAVES> ob;
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = {0, 0, 0, 0};
    if (steps <= 0) return;
    oa.begin(a, m0, step0);
    ob.begin(b, n0, step0);
    u4 fa[S::FM], fb[S::FN];
    const auto read = [&](const char *at, const char *bt, int h) {
#pragma unroll
        for (int j = 0; j < S::FN; ++j) fb[j] = ob.read(bt, S::column_c(ob.wave, j), S::column_i(j), h);
#pragma unroll
        for (int i = 0; i < S::FM; ++i) fa[i] = oa.read(at, S::row_c(oa.wave, i), S::row_i(i), h);
    };
    const auto multiply = [&]() {
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j) acc[i][j] = Mfma<DT>::run(fa[i], fb[j], acc[i][j]);
    };
    const auto wait_reads = [] { __builtin_amdgcn_s_waitcnt(0xc07f); };
    const auto wait_loads = [](bool but_first) {  // the first operand's loads of the step after next may be on their way
        if (but_first) __builtin_amdgcn_s_waitcnt(0x0f70 | Operand<DT, AKM, S::TM, S::WAVES>::N);
        else __builtin_amdgcn_s_waitcnt(0x0f70);
    };
    const auto barrier = [] {  // which to the compiler touches no memory: nothing is to be moved across it
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" : : : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int A = S::TM * kStepBytes, B = S::TN * kStepBytes;
    char *const bs = lds + 3 * A;
    steps <<= twice;
    oa.fetch(lds, 0);
    ob.fetch(bs, 0);
    if (steps > 1) oa.fetch(lds + A, 1 >> twice);
    const char *at = lds, *bt = bs;
    char *to = lds + 2 * A;  // of the step after next
    const auto ahead = [&](int t) {
        if (t + 1 < steps) ob.fetch(bt == bs ? bs + B : bs, (t + 1) >> twice, (t + 1) & twice ? rest : 0);
        if (t + 2 < steps) oa.fetch(to, (t + 2) >> twice);
    };
    const auto next = [&] {
        to = const_cast<char *>(at);
        at = at == lds + 2 * A ? lds : at + A;
        bt = bt == bs ? bs + B : bs;
    };
    if constexpr (S::WAVES == 8) {
        const bool late = oa.wave >= 4;
        wait_loads(steps > 1);
        barrier();
        if (late) barrier();
        for (int t = 0; t < steps; ++t) {
            read(at, bt, 0);
            ahead(t);
            wait_reads();
            barrier();
            __builtin_amdgcn_s_setprio(1);
            multiply();
            __builtin_amdgcn_s_setprio(0);
            barrier();
            read(at, bt, 1);
            wait_reads();
            if (late) wait_loads(t + 2 < steps);
            barrier();
            __builtin_amdgcn_s_setprio(1);
            multiply();
            __builtin_amdgcn_s_setprio(0);
            if (!late) wait_loads(t + 2 < steps);
            barrier();
            next();
        }
        if (!late) barrier();
    } else {
        for (int t = 0; t < steps; ++t) {
            wait_loads(t + 1 < steps);
            barrier();  // the step is there, and the memory of the one before is read
            ahead(t);
            read(at, bt, 0);
            multiply();
            read(at, bt, 1);
            multiply();
            wait_reads();
            next();
        }
    }
    __syncthreads();
}
};

// ------------------------------------------------------------------------------------------------ few rows
// Products with few rows of the second operand, bound by the reading of the first: it goes from memory to registers once, 16
// rows to a wave, 8 loads of 16 bytes a lane ahead (4 where the columns' sums need the registers); the second operand waits in
// LDS (all of it, or a chunk of k at a time).  Any alignment, any width.  128,256 x 2,048 bf16, 17 / 32 / 48 / 64 rows: 130 / 122
// / 130 / 130 us (4.0 to 4.3 TB/s), by tiles 131 / 127 / 121 / 128; 8 bits, 17 / 32 / 64: 59 / 64 / 80, by tiles 66 / 65 / 66; fp32, 64
// x 128,256 x 1,024: 192, by tiles 156.  So tiles would gain at 48 to 64 rows and with fp32; few tokens gain here (64 x 32,000 x 512: 20, 21).
constexpr int kThinThreads = 512, kThinRows = kThinThreads / 64 * 16;  // rows of the first operand that a workgroup takes at a time
constexpr int kThinLds = 65536;                                      // two workgroups to a compute unit
constexpr int kThinGroups = 512;                                     // workgroups at most: as many as run at once
constexpr int kThinMost = 64;                                        // rows of the second operand at most

// Bytes of k that fit LDS for n rows.
__host__ __device__ inline int thin_chunk(int n, int bytes) { return min((bytes + 127) / 128 * 128, kThinLds / n / 128 * 128); }

// finish(m, acc): results of rows m .. m + 3 (16-row block of the wave, a quarter of it to 16 lanes) and columns 16 j + lane % 16.
template <int DT, int FN, typename F>
__device__ __forceinline__ void product_thin(const Side &w, const Side &x, char *lds, F finish) {
    constexpr int U = FN == 4 ? 4 : 8;
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, quarter = lane >> 4;
    const int chunk = thin_chunk(x.rows, w.bytes), groups = (w.rows + kThinRows - 1) / kThinRows;
    const char *column[FN];  // of LDS: the lane's row of the second operand
    int turn[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int r = min(j * 16 + (lane & 15), x.rows - 1);
        column[j] = lds + r * chunk;
        turn[j] = (quarter ^ (r & 7)) * 16;
    }
    bool staged = false;
    for (int g = (int)blockIdx.x; g < groups; g += (int)gridDim.x) {
        const int m0 = g * kThinRows + wave * 16;
        const char *row = w.p + (int64_t)min(m0 + (lane & 15), w.rows - 1) * w.ld + quarter * 16;
        typename Mfma<DT>::Acc acc[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[j] = {0, 0, 0, 0};
        for (int k0 = 0; k0 < w.bytes; k0 += chunk) {
            const int bytes = min(chunk, w.bytes - k0), full = bytes / 64;
            u4 a[U], b[U];
            const auto load = [&](u4 (&f)[U], int s) {
#pragma unroll
                for (int u = 0; u < U; ++u) f[u] = load_once(row + k0 + min(s + u, full - 1) * 64);
            };
            const auto multiply = [&](const u4 &f, int s) {
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    acc[j] = Mfma<DT>::run(f, *reinterpret_cast<const u4 *>(column[j] + (s >> 1) * 128 + (turn[j] ^ (s & 1) * 64)), acc[j]);
            };
            if (full > 0) load(a, 0);
            if (!staged) {
                __syncthreads();  // the chunk before is done with
                const int pieces = chunk / 16;
                for (int i = (int)threadIdx.x; i < x.rows * pieces; i += kThinThreads) {
                    const int r = i / pieces, c = i % pieces, left = x.bytes - (k0 + c * 16);
                    const char *q = x.p + (int64_t)r * x.ld + k0 + c * 16;
                    const u4 v = left >= 16 ? (u4)*reinterpret_cast<const u4b *>(q) : left > 0 ? load_some(q, left) : u4{0, 0, 0, 0};
                    *reinterpret_cast<u4 *>(lds + r * chunk + (c & ~7) * 16 + ((c ^ r) & 7) * 16) = v;
                }
                __syncthreads();
                staged = chunk >= w.bytes;
            }
            for (int s = 0; s < full; s += 2 * U) {
                if (s + U < full) load(b, s + U);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (s + u < full) multiply(a[u], s + u);
                if (s + 2 * U < full) load(a, s + 2 * U);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (s + U + u < full) multiply(b[u], s + U + u);
            }
            if (full * 64 < bytes) {
                const int left = bytes - full * 64 - quarter * 16;
                const char *q = row + k0 + full * 64;
                multiply(left >= 16 ? (u4)*reinterpret_cast<const u4b *>(q) : left > 0 ? load_some(q, left) : u4{0, 0, 0, 0}, full);
            }
        }
        finish(m0 + quarter * 4, acc);
    }
}

// Up to 16 rows of the second operand: 16 rows of the first to a workgroup, whose 8 waves lie side by side along k, 128 bytes of a
// row each, so that 1 KB of a row is read at a time (the same bytes 16 rows by 64 bytes a wave come at 5.2 TB/s, these at 5.9 to
// 6.1, read in order at 6.8).  Loads roll through four such KBs: what has been multiplied makes room for the one four further on,
// in this row or the next.  The waves' sums are joined in LDS; then thread t (of 256) has row t % 16 and column t / 16.  8 x
// 151,936 x 2,048 bf16 (622 MB) 108 us, 5.8 TB/s.  128,256 x 2,048, 4 / 8 / 12 / 16 rows: 98 us each, product_thin 108 to 110; fp32, 16 x
// 1,024: 101, 117; 8 bits, 4 / 16 rows: 55 / 61, 55 / 58.  Rows that do not fit LDS as a whole are staged again for every 16 tokens: 8 x
// 4,096 bf16 (64 KB) 182, product_thin 203, but 9 and 16 x 4,096 241 and 256, product_thin 210 and 216.
constexpr int kFewMost = 16, kFewRows = 16, kFewBytes = 1024;

// finish(m, n, y): one result.  WHOLE: rows of whole KBs, loaded without a branch (past the last row the last one again).
template <int DT, bool WHOLE, typename F>
__device__ __forceinline__ void product_few(const Side &w, const Side &x, char *lds, float (*sums)[256], F finish) {
    typedef typename Mfma<DT>::Acc Acc;
    constexpr int AHEAD = 4;
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, quarter = lane >> 4;
    const int chunk = min((w.bytes + 127) / 128 * 128, kThinLds / x.rows / kFewBytes * kFewBytes);
    const int groups = (w.rows + kFewRows - 1) / kFewRows, pieces = (w.bytes + kFewBytes - 1) / kFewBytes;  // of a row
    const int r = min(lane & 15, x.rows - 1), inside = wave * 128 + quarter * 16;                        // a piece
    const char *column = lds + r * chunk + wave * 128;
    const int turn = (quarter ^ (r & 7)) * 16;
    u4 f[AHEAD][2];
    // the place that is loaded next: row group, piece
    int load_g = (int)blockIdx.x, load_c = 0;
    const char *load_row = w.p + (int64_t)min(load_g * kFewRows + (lane & 15), w.rows - 1) * w.ld + inside;
    const auto load = [&](u4 (&to)[2]) {
        const int at = load_c * kFewBytes;
        if (WHOLE || at + kFewBytes <= w.bytes) {
#pragma unroll
            for (int h = 0; h < 2; ++h) to[h] = load_once(load_row + at + h * 64);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int left = w.bytes - at - inside - h * 64;
                const char *q = load_row + at + h * 64;
                to[h] = left >= 16 ? (u4)*reinterpret_cast<const u4b *>(q) : left > 0 ? load_some(q, left) : u4{0, 0, 0, 0};
            }
        }
        if (++load_c == pieces) {
            load_c = 0;
            load_g += (int)gridDim.x;
            load_row = w.p + (int64_t)min(load_g * kFewRows + (lane & 15), w.rows - 1) * w.ld + inside;
        }
    };
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) load(f[s]);
    int staged = -1, c = 0;  // the chunk in LDS; the piece that is multiplied next
    Acc acc = {0, 0, 0, 0};
    for (int g = (int)blockIdx.x; g < groups;) {
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            if (g >= groups) break;
            const int at = c * kFewBytes, k0 = at / chunk * chunk;
            if (staged != k0) {
                __syncthreads();  // the chunk before is done with
                const int n_pieces = chunk / 16;
                for (int i = (int)threadIdx.x; i < x.rows * n_pieces; i += kThinThreads) {
                    const int n = i / n_pieces, p = i % n_pieces, left = x.bytes - (k0 + p * 16);
                    const char *q = x.p + (int64_t)n * x.ld + k0 + p * 16;
                    const u4 v = left >= 16 ? (u4)*reinterpret_cast<const u4b *>(q) : left > 0 ? load_some(q, left) : u4{0, 0, 0, 0};
                    *reinterpret_cast<u4 *>(lds + n * chunk + (p & ~7) * 16 + ((p ^ n) & 7) * 16) = v;
                }
                __syncthreads();
                staged = k0;
            }
            // a wave whose 128 bytes lie past the row's end has nothing to add
            if (WHOLE || at - k0 + wave * 128 < chunk)
#pragma unroll
                for (int h = 0; h < 2; ++h) acc = Mfma<DT>::run(f[s][h], *reinterpret_cast<const u4 *>(column + (at - k0) + (turn ^ h * 64)), acc);
            load(f[s]);
            if (++c < pieces) continue;
            c = 0;
            // [wave][row][column], row r's columns turned by r
            __syncthreads();  // the sums before are read
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int m = quarter * 4 + q, to = m * 16 + ((lane + m) & 15);
                if constexpr (DT == kI8) sums[wave][to] = __int_as_float(acc[q]);
                else sums[wave][to] = acc[q];
            }
            acc = {0, 0, 0, 0};
            __syncthreads();
            if (threadIdx.x < 256) {
                const int m = (int)threadIdx.x & 15, n = (int)threadIdx.x >> 4, from = m * 16 + ((n + m) & 15);
                if constexpr (DT == kI8) {
                    int y = 0;
#pragma unroll
                    for (int v = 0; v < 8; ++v) y += __float_as_int(sums[v][from]);
                    finish(g * kFewRows + m, n, y);
                } else {
                    float y = 0.0f;
#pragma unroll
                    for (int v = 0; v < 8; ++v) y += sums[v][from];
                    finish(g * kFewRows + m, n, y);
                }
            }
            g += (int)gridDim.x;
        }
    }
}

// Rows that tiles of 64, 128, 192 or 256 columns reach where n rows are wanted.
__host__ __device__ inline int64_t padded_rows(int64_t n) {
    const int64_t by_256 = (n + 255) / 256 * 256, by_192 = (n + 191) / 192 * 192;
    return by_256 > by_192 ? by_256 : by_192;
}

// f(shape) for the tiles of a product of m rows of the first operand with n of the second.
// As few tiles as 256 columns give, no wider than they need (333 rows: 2 x 192): every tile of columns is a reading of the
// first operand.  Half tiles up to 128 rows (forward, 128,256 x 1,024 bf16: 72 rows 65 us, wide 87; 128: 66, 81; 144: wide 69, half 95;
// 256: 79, 97), and where their smaller ones leave less undone: the gradient's logits of up to 512 rows (how many carry a weight is not
// known here) and its short sums over them (256 x 50,257 x 1,024: 205 us, wide for both 219; 512: 329, 359; 576: wide 382, half for
// all 412; 1,024: 650, 660), and fp32, which the matrix cores bound.  The smallest where even 128 x 128 would not fill the compute
// units (500 rows of 600 x 4,096 fp32: 152 us, not 272; bf16 34, not 84; 300 x 8,000 x 1,024 bf16 20, not 30; 300 x 11,000 x 1,024,
// 258 tiles, 29, which smaller ones would do in 22; 70 x 64,000: 30, smaller ones 35).
enum Use { kForward, kGradLogits, kGradHidden, kGradWeight };
template <int DT, Use U, typename F>
void with_shape(int64_t m, int64_t n, F f) {
    const int64_t tiles = (n + 255) / 256;
    const int columns = (int)(((n + tiles - 1) / tiles + 63) / 64);
    if constexpr (U != kGradWeight) {
        if ((U != kGradHidden && (m + 127) / 128 * ((n + 127) / 128) <= 256) || ((DT == TT_F32 || U == kGradLogits) && n <= 64)) return f(Half<1>());
    }
    if constexpr (DT == TT_F32) f(Half<2>());
    else if (n <= (U == kGradLogits || U == kGradWeight ? 512 : 128)) f(Half<2>());
    else if constexpr (U == kGradWeight) f(Wide<4>());
    else if (columns == 3) f(Wide<3>());
    else f(Wide<4>());
}

// Workgroups of a product with few rows, for n rows of the second operand and m of the first: a part each of every row.
inline int thin_groups(int64_t n, int64_t m) {
    const int64_t rows = n <= kFewMost ? kFewRows : kThinRows, groups = (m + rows - 1) / rows;
    return (int)(groups < kThinGroups ? groups : kThinGroups);
}

// Parts that up to n rows of m results leave at most, by whichever product they are formed.
inline size_t most_parts(int64_t n, int64_t m) {
    const int64_t tiles = n * ((m + 127) / 128), few = (n < kFewMost ? n : kFewMost) * thin_groups(1, m);
    return (size_t)(tiles > few ? tiles : few);
}

// The tile of workgroup `id` of mt x nt: neighbours in time on one XCD (every eighth workgroup) share rows of both operands in
// its L2: they go through 8 tiles of the first operand by all of the second's.
__device__ __forceinline__ void tile_of(int id, int total, int mt, int nt, int &m, int &n) {
    constexpr int kXcds = 8, kGroup = 8;
    const int xcd = id % kXcds, per = total / kXcds, more = total % kXcds;
    const int at = xcd * per + min(xcd, more) + id / kXcds, group = at / (kGroup * nt), in = at % (kGroup * nt);
    const int wide = min(kGroup, mt - group * kGroup);
    m = group * kGroup + in % wide;
    n = in / wide;
}

// Whether a matrix's rows can go to LDS as they are, with k contiguous: whole steps, 16-byte aligned.
inline bool whole_steps(const Side &s) {
    return reinterpret_cast<uintptr_t>(s.p) % 16 == 0 && s.ld % 16 == 0 && s.bytes % kStepBytes == 0 && s.ld < (1 << 22);
}

// f(n, j) for the columns n that this thread holds parts of, f(m, i) for its blocks' first rows m.
template <typename S, typename F>
__device__ __forceinline__ void for_columns(int n0, F f) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) f(n0 + S::column_block(wave, j) * 16 + (lane & 15), j);
}
template <typename S, typename F>
__device__ __forceinline__ void for_rows(int m0, F f) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < S::FM; ++i) f(m0 + S::row_block(wave, i) * 16 + (lane >> 4) * 4, i);
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

// Stores a tile's results, values(n, j, m, i, y) giving four of a column n, to row(n): 16-bit results go through LDS, 64
// columns at a time, so that every row gets 512 or 256 bytes at once (from the registers it would be 32 at a time); the columns' 16-byte
// pieces at place piece ^ column there.  m_end, n_end: where the result ends.  For one after another of the columns' groups
// each thread calls values() for its blocks.  REST (16 bits): what the rounding of a result takes off it is stored `rest`
// elements further on (0 beside an infinity); four of such LDS pieces are needed, two from a0 on and two more.
template <int DT, typename S, bool REST = false, typename V, typename R>
__device__ __forceinline__ void store_tile(int m0, int m_end, int n0, int n_end, char *a0, char *a1, V values, R row, int64_t rest = 0) {
    typedef unsigned int u2 __attribute__((ext_vector_type(2)));
    constexpr int PIECES = S::TM / 8, SAME = S::FN / S::COLUMNS;  // of a row; blocks of a wave in 64 columns
    constexpr int SECOND = 2 * S::TM * kStepBytes;                // from a result's place in LDS to its rest's
    static_assert(!REST || 2 * SECOND <= (3 * S::TM + 2 * S::TN) * kStepBytes, "four pieces in a tile's memory");
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
#pragma unroll
    for (int g = 0; g < S::COLUMNS; ++g) {
        char *lds = g & 1 ? a1 : a0;
#pragma unroll
        for (int j = g * SAME; j < (g + 1) * SAME; ++j) {
            const int in = S::column_block(wave, j) * 16 + (lane & 15), n = n0 + in;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int at = S::row_block(wave, i) * 16 + (lane >> 4) * 4;
                float y[4];
                values(n, j, m0 + at, i, y);
                if constexpr (DT == TT_F32) {
                    if (n < n_end && m0 + at < m_end) store4<DT>(row(n), m0 + at, m_end, y);
                } else {
                    char *to = lds + ((in & 63) * PIECES + ((at >> 3) ^ (in & (PIECES - 1)))) * 16 + (at & 4) * 2;
                    const u2 v = {rows::encode_pair<DT>(y[0], y[1]), rows::encode_pair<DT>(y[2], y[3])};
                    *reinterpret_cast<u2 *>(to) = v;
                    if constexpr (REST) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float stored = rows::decode<DT>(v[q >> 1] >> (q & 1) * 16 & 0xFFFFu);
                            y[q] = fabsf(stored) < INFINITY ? y[q] - stored : 0.0f;
                        }
                        *reinterpret_cast<u2 *>(to + SECOND) = u2{rows::encode_pair<DT>(y[0], y[1]), rows::encode_pair<DT>(y[2], y[3])};
                    }
                }
            }
        }
        if constexpr (DT != TT_F32) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < (REST ? 2 : 1) * 64 * PIECES / S::THREADS; ++k) {
                const int second = k / (64 * PIECES / S::THREADS), in = k % (64 * PIECES / S::THREADS) * S::THREADS + (int)threadIdx.x;
                const int r = in / PIECES, c = in % PIECES, m = m0 + c * 8, to = n0 + g * 64 + r;
                const u4 v = *reinterpret_cast<const u4 *>(lds + second * SECOND + (r * PIECES + (c ^ (r & (PIECES - 1)))) * 16);
                if (to >= n_end) continue;
                typename rows::Elem<DT>::T *out = row(to) + second * rest;
                if (m + 8 <= m_end) *reinterpret_cast<u4b *>(out + m) = v;
                else {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (m + q < m_end) out[m + q] = (typename rows::Elem<DT>::T)(v[q >> 1] >> (q & 1) * 16);
                }
            }
        }
    }
}

// Largest value m of a set of logits z, and the sum s of 2^((z - m) c) over the set without one of its largest (a set without logits:
// minus infinity and 0).  That term is 1, and what the others give beside it is all that ln (1 + s) holds where a token is almost
// certain: in a sum with the 1 fp32 would keep steps of 2^-24 of it (1 x 640 logits, a log probability of -4e-5: 1.4e-3 off).
// NaN passes through: s of a set with a NaN or plus infinity is NaN.
struct Part {
    float m, s;
};

__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.0f : m; }

// The factor of a sum relative to m when it becomes relative to ref, which is at least m, or 0 in the place of minus infinity
// (a set without logits has the sum 0, which no factor may make NaN).
__device__ __forceinline__ float factor(float m, float ref, float c) { return __builtin_amdgcn_exp2f(fminf((reference(m) - ref) * c, 0.0f)); }

constexpr float kNear = 1.03125f;  // a sum from here on leaves 2^-18 of its rest when the 1 is taken off

__device__ __forceinline__ float term(float z, float ref, float c) { return __builtin_amdgcn_exp2f((z - ref) * c); }

// What makes a set's s of those of its parts and logits.  FINE: the terms below 1, and how many are 1; otherwise all of them together,
// for a log-sum-exp that is wanted beside its largest logit alone.
template <typename F, bool FINE>
struct Terms {
    F s = 0, ones = 0;

    __device__ __forceinline__ void logit(float z, float ref, float c) {
        const float t = term(z, ref, c), below = FINE ? __builtin_amdgcn_fractf(t) : t;  // 1 to 0, what is below as it is, NaN as well
        s += below;
        if (FINE) ones += t - below;
    }
    // A set whose largest value may be the whole's, m.
    __device__ __forceinline__ void part(const Part &p, float m, float c) {
        const bool top = FINE && p.m == m && m != -INFINITY;
        const F f = factor(p.m, reference(m), c), one = p.m == -INFINITY ? 0.0f : 1.0f;
        s += top ? (F)p.s : (one + (F)p.s) * f;
        if (FINE) ones += top ? 1.0f : 0.0f;
    }
    // f(value) for each value that lanes or waves add up.
    template <typename A>
    __device__ __forceinline__ void join(A f) {
        s = f(s);
        if (FINE) ones = f(ones);
    }
    __device__ __forceinline__ F rest(float m) const {
        if (FINE) return s + (ones > 0 ? ones - 1 : (F)0);
        return m == -INFINITY ? s : s - 1;
    }
};

// The parts of the tile's columns from z(i, j, q) (minus infinity where there is no logit), left in lds[n - n0] for
// threads below TN after the closing barrier.  scale(n): log2(e) times the row's inverse temperature.
template <typename S, bool FINE, typename Z, typename C>
__device__ __forceinline__ Part column_parts(int n0, char *lds, Z z, C scale) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int wm = wave / S::WN;
    Part *part = reinterpret_cast<Part *>(lds);  // [WM][TN]
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int at = S::column_block(wave, j) * 16 + (lane & 15);
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) m = fmaxf(m, z(i, j, q));
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float c = scale(n0 + at), ref = reference(m);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) s += term(z(i, j, q), ref, c);
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        float rest = m == -INFINITY ? s : s - 1.0f;
        // Up to kNear the subtraction would cost digits: the terms again, without the 1 (the terms below 1 beside all of them for every
        // set: 4,096 x 151,936 x 2,048 36 us more instead of 10 or less, 1,000 x 50,257 x 256 5.4 instead of 1.4)
        if (FINE && __any(m != -INFINITY && s < kNear)) {
            s = 0.0f;
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) s += __builtin_amdgcn_fractf(term(z(i, j, q), ref, c));
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            rest = m != -INFINITY && rest < kNear - 1.0f ? s : rest;  // there is but one 1 below 2
        }
        if (lane < 16) part[wm * S::TN + at] = {m, rest};
    }
    __syncthreads();
    Part r = {-INFINITY, 0.0f};
    if ((int)threadIdx.x < S::TN) {
        const float c = scale(n0 + (int)threadIdx.x);
#pragma unroll
        for (int w = 0; w < S::WM; ++w) r.m = fmaxf(r.m, part[w * S::TN + threadIdx.x].m);
        Terms<float, FINE> terms;
#pragma unroll
        for (int w = 0; w < S::WM; ++w) terms.part(part[w * S::TN + threadIdx.x], r.m, c);
        r.s = terms.rest(r.m);
    }
    return r;
}

// Adds four logits to a lane's running part.
template <bool FINE>
__device__ __forceinline__ void add_part(Part &p, const float (&z)[4], float c) {
    const float m = fmaxf(fmaxf(p.m, fmaxf(z[0], z[1])), fmaxf(z[2], z[3]));
    Terms<float, FINE> terms;
    terms.part(p, m, c);
#pragma unroll
    for (int q = 0; q < 4; ++q) terms.logit(z[q], reference(m), c);
    p = {m, terms.rest(m)};
}

template <bool FINE>
__device__ __forceinline__ void add_part(Part &p, float z, float c) {
    const float m = fmaxf(p.m, z);
    Terms<float, FINE> terms;
    terms.part(p, m, c);
    terms.logit(z, reference(m), c);
    p = {m, terms.rest(m)};
}

// The part of 16 lanes that hold one column's.
template <bool FINE>
__device__ __forceinline__ Part join_quarter(Part p, float c) {
    float m = p.m;
#pragma unroll
    for (int d = 1; d < 16; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    Terms<float, FINE> terms;
    terms.part(p, m, c);
#pragma unroll
    for (int d = 1; d < 16; d *= 2) terms.join([&](float x) { return x + __shfl_xor(x, d); });
    return {m, terms.rest(m)};
}

// The workgroup's part of column threadIdx.x (below n) from its lanes' running parts of columns 16 j + lane % 16.
template <int FN, bool FINE, typename C>
__device__ __forceinline__ Part join_lanes(const Part (&p)[FN], int n, char *lds, C scale) {
    Part *all = reinterpret_cast<Part *>(lds);  // [wave][16 FN]
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, waves = (int)blockDim.x / 64, at = (int)threadIdx.x;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const float m = fmaxf(p[j].m, __shfl_xor(p[j].m, 16)), top = fmaxf(m, __shfl_xor(m, 32));
        Terms<float, FINE> terms;
        terms.part(p[j], top, scale(j * 16 + (lane & 15)));
#pragma unroll
        for (int d = 16; d < 64; d *= 2) terms.join([&](float x) { return x + __shfl_xor(x, d); });
        if (lane < 16) all[wave * 16 * FN + j * 16 + lane] = {top, terms.rest(top)};
    }
    __syncthreads();
    Part r = {-INFINITY, 0.0f};
    if (at >= n) return r;
    for (int w = 0; w < waves; ++w) r.m = fmaxf(r.m, all[w * 16 * FN + at].m);
    Terms<float, FINE> terms;
    for (int w = 0; w < waves; ++w) terms.part(all[w * 16 * FN + at], r.m, scale(at));
    r.s = terms.rest(r.m);
    return r;
}

// What the n parts of a row give, M and L = ln (1 + s), to the first of its 256 threads.
__device__ __forceinline__ Part join_row(const Part *part, int n, float beta) {
    __shared__ float tops[4];
    __shared__ double sums[4], ones[4];
    constexpr int kHeld = 4;
    const int t = (int)threadIdx.x, wave = t >> 6;
    Part held[kHeld];  // read once, all at a time
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = i * 256 + t < n ? part[i * 256 + t] : Part{-INFINITY, 0.0f};
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) m = fmaxf(m, held[i].m);
    for (int i = kHeld * 256 + t; i < n; i += 256) m = fmaxf(m, part[i].m);
    m = rows::wave_max(m);
    if ((t & 63) == 0) tops[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float c = beta * rows::kLog2e;
    Terms<double, true> terms;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) terms.part(held[i], m, c);
    for (int i = kHeld * 256 + t; i < n; i += 256) terms.part(part[i], m, c);
    terms.join([](double x) { return rows::wave_sum(x); });
    if ((t & 63) == 0) {
        sums[wave] = terms.s;
        ones[wave] = terms.ones;
    }
    __syncthreads();
    terms.s = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    terms.ones = (ones[0] + ones[1]) + (ones[2] + ones[3]);
    return {m, m == -INFINITY && terms.s == 0.0 ? 0.0f : (float)log1p(terms.rest(m))};
}

}  // namespace tiles
}  // namespace tt
