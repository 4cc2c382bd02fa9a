// Log probabilities of given tokens with log-sum-exp, entropy and top alternatives, and their
// gradient, from rows of bf16, fp16 or fp32 logits on gfx950.
//
// With x the row's logits (NaN counts as minus infinity), beta the row's inverse temperature:
//   M = max x,  S = sum exp(beta (x - M)),  L = ln S,  lse = beta M + L
//   lp_j = beta (x_j - M) - L,  p_j = exp(lp_j),  H = -sum p_j lp_j = L - sum beta (x_j - M) p_j
//   alternatives: the largest x, ties by the lower index, minus infinity never listed
//   d_j = beta (g ([j = id] - p_j) - h p_j (lp_j + H)), upstream gradients g of lp_id and h of H
//
// One pass over the row.  A workgroup holds a part of a row in registers, forms its largest value
// first and then its sums (base 2, v_exp_f32), and, for the alternatives, a lower bound of its k-th
// largest value: the k-th largest of 256 groups' largest values (a lane's, or four lanes'), found by
// 16 ballots on the upper 16 bits of their order keys.  k distinct elements reach it, so the k largest
// do, and about 1.2 to 2 k in all: these become 64-bit keys (value, then lower index).
// row_parts: parts of 16 KB to 32 KB, their sums and keys to the workspace; row_finish: a workgroup
// per row joins the sums in fp64 and selects the k largest keys in the same way, ordered by counting.
// row_whole: a workgroup per row that takes the row as one part and finishes it itself.
#include "rows.h"

namespace tt {
namespace {

using namespace rows;

constexpr int kMaxTop = 128;
constexpr int kSelect = 1024;                       // keys that are ordered in LDS
constexpr int kGroups = 256;                        // lane groups whose largest values give the bound
constexpr size_t kMaxKeyBytes = size_t(128) << 20;  // workspace: rows are taken in groups beyond
constexpr int64_t kMaxGrid = int64_t(1) << 18;      // workgroups of one launch

// Keys that a part may hand over.  Where fewer than k lanes hold a finite value, all their elements may
// reach the bound (a lane has 8 then); more are ties, and the part selects its k largest exactly.
inline int part_capacity(int n_top) { return 8 * n_top + 64; }

struct RowArgs {
    const void *logits;
    int64_t ld, row0;  // row0: the first row of this launch
    int v, dtype, parts, n_top, capacity;
    const float *inv_temp;
    const int32_t *ids;
    float4 *sums;    // per part: m, s, e, number of keys (bits)
    uint64_t *keys;  // per part: capacity
    float *logprob, *lse, *entropy, *stats;
    int32_t *top_ids;
    float *top_logprobs;
};

// LDS of the selection; a wave stages its keys in a segment of its own.
template <int THREADS>
struct TopLds {
    static constexpr int kStage = THREADS == kThreads ? 512 : 128;
    uint32_t largest[THREADS];
    uint64_t stage[THREADS / kWave][kStage];
    int count[THREADS / kWave], slots[64], total;
};

// Largest bound P on 16-bit keys that at least k of the kGroups groups reach (each wave for itself).
template <int THREADS>
__device__ __forceinline__ uint32_t kth_key16(const uint32_t *sh_largest, int k) {
    constexpr int kPerLane = kGroups / kWave;
    const int lane = threadIdx.x % kWave;
    uint32_t q[kPerLane];
#pragma unroll
    for (int u = 0; u < kPerLane; ++u) {
        q[u] = sh_largest[u * kWave + lane];
#pragma unroll
        for (int g = 1; g < THREADS / kGroups; ++g) {
            const uint32_t o = sh_largest[g * kGroups + u * kWave + lane];
            q[u] = o > q[u] ? o : q[u];
        }
    }
    uint32_t p = 0;
#pragma unroll
    for (int b = 15; b >= 0; --b) {
        const uint32_t c = p | (1u << b);
        int n = 0;
#pragma unroll
        for (int u = 0; u < kPerLane; ++u) n += __popcll(__ballot(q[u] >= c));
        if (n >= k) p = c;
    }
    return p;
}

// The lowest finite value whose key's upper half reaches p.
__device__ __forceinline__ float bound_value(uint32_t p) {
    return p <= 0x007Fu ? -0x1.fffffep+127f : key_value(p << 16);
}

__device__ __forceinline__ uint64_t full_key(float x, int index) {
    return ((uint64_t)order_key(x) << 32) | (0xFFFFFFFFu - (uint32_t)index);
}

// Lanes below this one among those of a mask.
__device__ __forceinline__ int lanes_below(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Sum over the workgroup of a count, through a zeroed LDS slot of its own.
__device__ __forceinline__ int block_count(int n, int *slot) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) n += __shfl_xor(n, d);
    if (threadIdx.x % kWave == 0) atomicAdd(slot, n);
    __syncthreads();
    return *slot;
}

// Hides from the compiler that a value has not changed: what follows is formed from it again instead of
// being held in registers from before.
__device__ __forceinline__ void form_again(uint32_t &x) { asm volatile("" : "+v"(x)); }

template <int NV>
__device__ __forceinline__ void form_again(uint32_t (&w)[NV][4]) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) form_again(w[i][q]);
}

// Elements of a part that satisfy f(order key, index in the part), counted by this thread.
template <int DT, int NV, int THREADS, typename F>
__device__ __forceinline__ int count_if(uint32_t (&w)[NV][4], F f) {
    constexpr int kPer = Elem<DT>::kPer;
    int n = 0;
    uint32_t first = threadIdx.x * kPer;
    form_again(w);
    form_again(first);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float x = value<DT>(w[i], j);
            n += (x > -INFINITY && f(order_key(x), (int)first + i * THREADS * kPer + j)) ? 1 : 0;
        }
    }
    return n;
}

// The part's k largest elements exactly, where too many reach the bound (many equal values): the k-th
// largest value by binary search on its order key, then the last index among the elements equal to
// it.  At least k elements are finite.  49 counts, each over the registers.
template <int DT, int NV, int THREADS>
__device__ __forceinline__ void select_exactly(uint32_t (&w)[NV][4], int x_part, int k, uint64_t *keys, int *sh_slots,
                                               int *sh_total) {
    if (threadIdx.x < 64) sh_slots[threadIdx.x] = 0;
    if (threadIdx.x == 0) *sh_total = 0;
    __syncthreads();
    int slot = 0;
    uint32_t kth = 0;
    for (int b = 31; b >= 0; --b) {
        const uint32_t c = kth | (1u << b);
        const int n = count_if<DT, NV, THREADS>(w, [c](uint32_t o, int) { return o >= c; });
        if (block_count(n, &sh_slots[slot++]) >= k) kth = c;
    }
    const int above = count_if<DT, NV, THREADS>(w, [kth](uint32_t o, int) { return o > kth; });
    const int need = k - block_count(above, &sh_slots[slot++]);
    int last = 0;  // the largest index bound with fewer than `need` equal elements below it
    for (int b = 15; b >= 0; --b) {  // indices in a part are below 2^16
        const int c = last | (1 << b);
        const int n = count_if<DT, NV, THREADS>(w, [kth, c](uint32_t o, int at) { return o == kth && at < c; });
        if (block_count(n, &sh_slots[slot++]) < need) last = c;
    }
    count_if<DT, NV, THREADS>(w, [=](uint32_t o, int at) {
        if (o > kth || (o == kth && at <= last))
            keys[atomicAdd(sh_total, 1)] = ((uint64_t)o << 32) | (0xFFFFFFFFu - (uint32_t)(x_part + at));
        return false;
    });
}

// Keys of a part's elements that reach the bound, to dst (LDS or global); returns their number, at least
// the part's finite elements or k, at most capacity (>= k).  sh.largest is written and a barrier passed.
template <int DT, int NV, int THREADS>
__device__ __forceinline__ int collect(uint32_t (&w)[NV][4], const float (&vm)[NV], int x_part, int k, uint64_t *dst, int capacity,
                                       TopLds<THREADS> &sh) {
    constexpr int kWaves = THREADS / kWave, kStage = TopLds<THREADS>::kStage;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const float bound = bound_value(kth_key16<THREADS>(sh.largest, k));
    int n = 0;
    form_again(w);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (__ballot(vm[i] >= bound) == 0) continue;
#pragma unroll
        for (int j = 0; j < Elem<DT>::kPer; ++j) {
            const float x = value<DT>(w[i], j);
            const uint64_t hit = __ballot(x >= bound);
            if (hit == 0) continue;
            const int at = n + lanes_below(hit);
            if (x >= bound && at < kStage) sh.stage[wave][at] = full_key(x, vector_at<DT, THREADS>(x_part, i) + j);
            n += __popcll(hit);
        }
    }
    if (lane == 0) sh.count[wave] = n;
    __syncthreads();
    int total = 0, before = 0;
    bool over = false;
#pragma unroll
    for (int u = 0; u < kWaves; ++u) {
        const int c = sh.count[u];
        before += u < wave ? c : 0;
        total += c;
        over = over || c > kStage;
    }
    if (over || total > capacity) {
        select_exactly<DT, NV, THREADS>(w, x_part, k, dst, sh.slots, &sh.total);
        return k;
    }
    for (int i = lane; i < n; i += kWave) dst[before + i] = sh.stage[wave][i];
    return total;
}

// The largest k (all, if fewer) of c <= kSelect distinct keys in LDS, descending, in sh_out; returns their number.
template <int THREADS>
__device__ __forceinline__ int order_keys(uint64_t *sh_sel, int c, int k, uint32_t *sh_largest, int *sh_total, uint64_t *sh_out) {
    const int lane = threadIdx.x % kWave;
    if (c > kGroups) {  // counting is quadratic: the bound once more, a key or a few a lane
        constexpr int kEach = kSelect / THREADS;
        uint64_t mine[kEach];
        uint32_t most = 0;
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const int i = u * THREADS + (int)threadIdx.x;
            mine[u] = i < c ? sh_sel[i] : 0;
            const uint32_t o = (uint32_t)(mine[u] >> 48);
            most = o > most ? o : most;
        }
        sh_largest[threadIdx.x] = most;
        if (threadIdx.x == 0) *sh_total = 0;
        __syncthreads();
        const uint64_t from = (uint64_t)kth_key16<THREADS>(sh_largest, k) << 48;
        int n = 0;
#pragma unroll
        for (int u = 0; u < kEach; ++u) n += __popcll(__ballot(mine[u] != 0 && mine[u] >= from));
        int base = 0;
        if (lane == 0) base = atomicAdd(sh_total, n);
        base = __builtin_amdgcn_readfirstlane(base);
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const uint64_t hit = __ballot(mine[u] != 0 && mine[u] >= from);
            if (mine[u] != 0 && mine[u] >= from) sh_sel[base + lanes_below(hit)] = mine[u];
            base += __popcll(hit);
        }
        __syncthreads();
        c = *sh_total;
    }
    for (int i = threadIdx.x; i < c; i += THREADS) {
        const uint64_t key = sh_sel[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < c; ++j) rank += sh_sel[j] > key ? 1 : 0;
        if (rank < k) sh_out[rank] = key;
    }
    __syncthreads();
    return c < k ? c : k;
}

// What the alternatives need of a row's statistics.
struct RowStats {
    double m, beta, log_sum;
    bool bad;
};

// A row's results but the alternatives, by one thread: m, s and e as in Sum, in natural units and fp64.
__device__ __forceinline__ RowStats write_row(const RowArgs &a, int64_t row, double beta, float m, double s, double e) {
    // m = -inf: nothing is finite (s = 0); m = +inf or an unsound temperature: NaN
    RowStats q;
    q.m = m;
    q.beta = beta;
    q.bad = !(beta > 0.0 && beta < INFINITY) || m == INFINITY;
    const bool empty = m == -INFINITY;
    q.log_sum = q.bad ? NAN : (empty ? 0.0 : log(s));
    if (a.stats != nullptr) {
        a.stats[2 * row] = q.bad ? NAN : m;
        a.stats[2 * row + 1] = (float)q.log_sum;
    }
    if (a.lse != nullptr) a.lse[row] = (float)(q.bad ? NAN : q.m * beta + q.log_sum);
    if (a.entropy != nullptr) a.entropy[row] = (float)(q.bad ? NAN : (empty ? 0.0 : q.log_sum - e / s));
    if (a.logprob != nullptr) {
        const int32_t id = a.ids[row];
        double lp = NAN;
        if (!q.bad && id >= 0 && id < a.v) {
            const float x = load_logit(row_at(a.logits, a.dtype, row * a.ld), a.dtype, id);
            lp = x == -INFINITY ? -INFINITY : ((double)x - q.m) * beta - q.log_sum;
        }
        a.logprob[row] = (float)lp;
    }
    return q;
}

__device__ __forceinline__ void write_top(const RowArgs &a, int64_t row, const RowStats &q, const uint64_t *sh_out, int n, int i) {
    int32_t id = -1;
    double lp = q.bad ? NAN : -INFINITY;
    if (i < n && !q.bad) {
        id = (int32_t)(0xFFFFFFFFu - (uint32_t)sh_out[i]);
        lp = ((double)key_value((uint32_t)(sh_out[i] >> 32)) - q.m) * q.beta - q.log_sum;
    }
    a.top_ids[row * a.n_top + i] = id;
    a.top_logprobs[row * a.n_top + i] = (float)lp;
}

// Largest values of a thread's vectors, and of the thread.
template <int DT, int NV>
__device__ __forceinline__ float vector_maxima(const uint32_t (&w)[NV][4], float (&vm)[NV]) {
    float tm = -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        vm[i] = -INFINITY;
#pragma unroll
        for (int j = 0; j < Elem<DT>::kPer; ++j) vm[i] = fmaxf(vm[i], value<DT>(w[i], j));
        tm = fmaxf(tm, vm[i]);
    }
    return tm;
}

template <int DT, int NV, bool TOP, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void row_parts(RowArgs a) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ Sum sh_sum[kWaves];
    __shared__ TopLds<TOP ? kThreads : kWave> sh;
    pass_over_nans();
    const int64_t r = blockIdx.x / (uint32_t)a.parts;
    const int part = blockIdx.x % (uint32_t)a.parts;
    const int x_part = part * NV * kThreads * Elem<DT>::kPer;
    uint32_t w[NV][4];
    load_part<DT, NV, kThreads>(static_cast<const typename Elem<DT>::T *>(a.logits) + (a.row0 + r) * a.ld, a.v, x_part, w);
    const float c2 = scale_of(a.inv_temp, a.row0 + r) * kLog2e;
    float vm[NV];
    const float tm = vector_maxima<DT, NV>(w, vm);
    if constexpr (TOP) {
        sh.largest[threadIdx.x] = order_key(tm) >> 16;
        form_again(w);
    }
    const Sum ws = wave_sums<DT, NV, ENTROPY>(w, tm, c2);
    if (threadIdx.x % kWave == 0) sh_sum[threadIdx.x / kWave] = ws;
    __syncthreads();
    const size_t slot = (size_t)r * a.parts + part;
    int count = 0;
    if constexpr (TOP)
        count = collect<DT, NV, kThreads>(w, vm, x_part, a.n_top, a.keys + slot * a.capacity, a.capacity, sh);
    if (threadIdx.x == 0) {
        Sum s = sh_sum[0];
#pragma unroll
        for (int u = 1; u < kWaves; ++u) s = join(s, sh_sum[u], c2);
        a.sums[slot] = make_float4(s.m, s.s, s.e, __int_as_float(count));
    }
}

template <int DT, int NV, int THREADS, bool TOP, bool ENTROPY>
__global__ __launch_bounds__(THREADS) void row_whole(RowArgs a) {
    constexpr int kWaves = THREADS / kWave;
    __shared__ Sum sh_sum[kWaves];
    __shared__ TopLds<TOP ? THREADS : kWave> sh;
    __shared__ uint64_t sh_sel[TOP ? kSelect : 1], sh_out[TOP ? kMaxTop : 1];
    __shared__ RowStats sh_stats;
    pass_over_nans();
    const int64_t row = a.row0 + blockIdx.x;
    uint32_t w[NV][4];
    load_part<DT, NV, THREADS>(static_cast<const typename Elem<DT>::T *>(a.logits) + row * a.ld, a.v, 0, w);
    const float beta = scale_of(a.inv_temp, row), c2 = beta * kLog2e;
    float vm[NV];
    const float tm = vector_maxima<DT, NV>(w, vm);
    if constexpr (TOP) {
        sh.largest[threadIdx.x] = order_key(tm) >> 16;
        form_again(w);
    }
    const Sum ws = wave_sums<DT, NV, ENTROPY>(w, tm, c2);
    if (threadIdx.x % kWave == 0) sh_sum[threadIdx.x / kWave] = ws;
    __syncthreads();
    if (threadIdx.x < kWave) {  // one wave joins the waves' sums
        float m = -INFINITY;
        const Sum mine = (int)threadIdx.x < kWaves ? sh_sum[threadIdx.x] : Sum{-INFINITY, 0.0f, 0.0f};
        m = wave_max(mine.m);
        double s = 0.0, e = 0.0;
        if (mine.s > 0.0f) {
            const double t = ((double)mine.m - (double)m) * (double)beta, f = exp(t);
            s = mine.s * f;
            e = (mine.e * kLn2 + mine.s * fmax(t, -1000.0)) * f;
        }
        s = wave_sum(s);
        e = ENTROPY ? wave_sum(e) : 0.0;
        if (threadIdx.x == 0) sh_stats = write_row(a, row, beta, m, s, e);
    }
    if constexpr (TOP) {
        int n = collect<DT, NV, THREADS>(w, vm, 0, a.n_top, sh_sel, kSelect, sh);
        __syncthreads();
        n = order_keys<THREADS>(sh_sel, n, a.n_top, sh.largest, &sh.total, sh_out);
        if ((int)threadIdx.x < a.n_top) write_top(a, row, sh_stats, sh_out, n, threadIdx.x);
    }
}

constexpr int kHeld = 16;  // keys that a lane of row_finish holds

// Calls f(key) for every key of a row, 0 where a lane has none: waves take runs of 64 keys of a part.
template <typename F>
__device__ __forceinline__ void for_each_key(const RowArgs &a, const float4 *sums, const uint64_t *keys, F f) {
    const int lane = threadIdx.x % kWave;
    for (int p = threadIdx.x / kWave; p < a.parts; p += kThreads / kWave) {
        const int n = __float_as_int(sums[p].w);
        for (int i = lane; i < n + (-n & (kWave - 1)); i += kWave) f(i < n ? keys[(size_t)p * a.capacity + i] : 0);
    }
}

// A row's keys that reach the bound on the k-th, in sh_sel; returns their number (<= kSelect).
__device__ __forceinline__ int gather_keys(const RowArgs &a, const float4 *sums, const uint64_t *keys, uint64_t *sh_sel, uint32_t *sh_largest,
                           int *sh_slots, int *sh_total) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    constexpr int kWaves = kThreads / kWave;
    // the largest number of keys that a part has, for the layout of runs of 64 keys over the waves
    int longest = 0;
    for (int p = lane; p < a.parts; p += kWave) {
        const int n = __float_as_int(sums[p].w);
        longest = n > longest ? n : longest;
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_xor(longest, d);
        longest = o > longest ? o : longest;
    }
    const int runs = (longest + kWave - 1) / kWave;
    const bool held = a.parts * runs <= kHeld * kWaves;  // all keys in registers, their loads in flight together
    uint64_t mine[kHeld];
    uint32_t most = 0;
    if (held) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const int c = u * kWaves + wave, p = runs > 0 ? c / runs : a.parts, i = (c - p * runs) * kWave + lane;
            mine[u] = 0;
            if (p < a.parts && i < __float_as_int(sums[p].w)) mine[u] = keys[(size_t)p * a.capacity + i];
        }
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const uint32_t o = (uint32_t)(mine[u] >> 48);
            most = o > most ? o : most;
        }
    } else {
        for_each_key(a, sums, keys, [&](uint64_t key) {
            const uint32_t o = (uint32_t)(key >> 48);
            most = o > most ? o : most;
        });
    }
    sh_largest[threadIdx.x] = most;
    if (threadIdx.x == 0) *sh_total = 0;
    __syncthreads();
    uint64_t from = (uint64_t)kth_key16<kThreads>(sh_largest, a.n_top) << 48;
    from = from > 1 ? from : 1;
    for (;;) {
        auto put = [&](uint64_t key) {
            const uint64_t hit = __ballot(key >= from);
            if (hit == 0) return;
            int base = 0;
            if (lane == 0) base = atomicAdd(sh_total, __popcll(hit));
            base = __builtin_amdgcn_readfirstlane(base) + lanes_below(hit);
            if (key >= from && base < kSelect) sh_sel[base] = key;
        };
        if (held) {
#pragma unroll
            for (int u = 0; u < kHeld; ++u) put(mine[u]);
        } else {
            for_each_key(a, sums, keys, put);
        }
        __syncthreads();
        if (*sh_total <= kSelect) return *sh_total;
        // many equal values: the k-th largest key itself (keys are distinct, so k reach it), by binary search
        uint64_t kth = 0;
        for (int b = 63; b >= 0; --b) {
            const uint64_t c = kth | (1ull << b);
            int n = 0;
            for_each_key(a, sums, keys, [&](uint64_t key) { n += key >= c ? 1 : 0; });
            __syncthreads();
            if (threadIdx.x == 0) sh_slots[0] = 0;
            __syncthreads();
            if (block_count(n, sh_slots) >= a.n_top) kth = c;
        }
        from = kth;
        __syncthreads();
        if (threadIdx.x == 0) *sh_total = 0;
        __syncthreads();
    }
}

template <bool TOP>
__global__ __launch_bounds__(kThreads) void row_finish(RowArgs a) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ float sh_m[kWaves];
    __shared__ double sh_s[kWaves], sh_e[kWaves];
    __shared__ uint64_t sh_sel[TOP ? kSelect : 1], sh_out[TOP ? kMaxTop : 1];
    __shared__ uint32_t sh_largest[TOP ? kThreads : 1];
    __shared__ int sh_slots[1], sh_total;
    __shared__ RowStats sh_stats;
    const int64_t r = blockIdx.x, row = a.row0 + r;
    const float4 *sums = a.sums + (size_t)r * a.parts;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const double beta = scale_of(a.inv_temp, row);
    int n = 0;
    if constexpr (TOP) n = gather_keys(a, sums, a.keys + (size_t)r * a.parts * a.capacity, sh_sel, sh_largest, sh_slots, &sh_total);
    float m = -INFINITY;
    for (int p = threadIdx.x; p < a.parts; p += kThreads) m = fmaxf(m, sums[p].x);
    m = wave_max(m);
    if (lane == 0) sh_m[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(sh_m[0], sh_m[1]), fmaxf(sh_m[2], sh_m[3]));
    double s = 0.0, e = 0.0;  // e in natural units
    for (int p = threadIdx.x; p < a.parts; p += kThreads) {
        const float4 q = sums[p];
        if (q.y > 0.0f) {
            const double t = ((double)q.x - (double)m) * beta, f = exp(t);
            s += q.y * f;
            e += (q.z * kLn2 + q.y * fmax(t, -1000.0)) * f;
        }
    }
    s = wave_sum(s);
    e = wave_sum(e);
    if (lane == 0) {
        sh_s[wave] = s;
        sh_e[wave] = e;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        s = sh_s[0] + sh_s[1] + sh_s[2] + sh_s[3];
        e = sh_e[0] + sh_e[1] + sh_e[2] + sh_e[3];
        sh_stats = write_row(a, row, beta, m, s, e);
    }
    if constexpr (TOP) {
        n = order_keys<kThreads>(sh_sel, n, a.n_top, sh_largest, &sh_total, sh_out);
        if ((int)threadIdx.x < a.n_top) write_top(a, row, sh_stats, sh_out, n, threadIdx.x);
    }
}

struct Plan {
    Split split;   // split.parts == 1: row_whole
    int64_t rows;  // rows of one launch
    size_t sums, total;
};

Plan plan_of(int64_t n_rows, int32_t v, int dtype, int n_top) {
    Plan p;
    p.split = split_rows(n_rows, v, dtype);
    int64_t most = kMaxGrid / p.split.parts;
    const size_t per_row = (size_t)p.split.parts * part_capacity(n_top) * sizeof(uint64_t);
    if (p.split.parts > 1 && n_top > 0 && (int64_t)(kMaxKeyBytes / per_row) < most) most = (int64_t)(kMaxKeyBytes / per_row);
    if (most < 1) most = 1;
    const int64_t groups = (n_rows + most - 1) / most;
    p.rows = groups == 0 ? 0 : (n_rows + groups - 1) / groups;
    p.sums = p.split.parts > 1 ? round256((size_t)p.rows * p.split.parts * sizeof(float4)) : 0;
    p.total = p.sums + (p.split.parts > 1 && n_top > 0 ? (size_t)p.rows * per_row : 0);
    return p;
}

template <int DT, int NV, int THREADS, bool TOP, bool ENTROPY>
void launch_rows(const RowArgs &a, int64_t n, hipStream_t stream) {
    if (a.parts == 1) row_whole<DT, NV, THREADS, TOP, ENTROPY><<<(unsigned)n, THREADS, 0, stream>>>(a);
    else if constexpr (THREADS == kThreads) row_parts<DT, NV, TOP, ENTROPY><<<(unsigned)(n * a.parts), THREADS, 0, stream>>>(a);
}

template <int DT, int NV, int THREADS>
void launch_rows(const RowArgs &a, int64_t n, hipStream_t stream) {
    if (a.n_top > 0) {
        if (a.entropy != nullptr) launch_rows<DT, NV, THREADS, true, true>(a, n, stream);
        else launch_rows<DT, NV, THREADS, true, false>(a, n, stream);
    } else {
        if (a.entropy != nullptr) launch_rows<DT, NV, THREADS, false, true>(a, n, stream);
        else launch_rows<DT, NV, THREADS, false, false>(a, n, stream);
    }
}

template <int DT>
void launch_rows(const RowArgs &a, const Split &s, int64_t n, hipStream_t stream) {
    if (s.threads == kWholeThreads) launch_rows<DT, kWideVectors, kWholeThreads>(a, n, stream);
    else if (s.vectors == kWideVectors) launch_rows<DT, kWideVectors, kThreads>(a, n, stream);
    else launch_rows<DT, kNarrowVectors, kThreads>(a, n, stream);
}

// ---------------------------------------------------------------- gradient
constexpr int kGradVectors = 4;

struct GradArgs {
    const void *logits;
    int64_t ld, row0;
    int v, parts;
    const float *inv_temp;
    const int32_t *ids;
    const float *stats, *entropy, *g, *h;
    void *out;
    int64_t out_ld;
};

template <int DT, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void logprob_grad(GradArgs a) {
    using T = typename Elem<DT>::T;
    constexpr int kPer = Elem<DT>::kPer;
    const int64_t r = a.row0 + blockIdx.x / (uint32_t)a.parts;
    const int x_part = (int)(blockIdx.x % (uint32_t)a.parts) * kGradVectors * kThreads * kPer;
    const T *row = static_cast<const T *>(a.logits) + r * a.ld;
    T *out = static_cast<T *>(a.out) + r * a.out_ld;
    const int32_t id = a.ids == nullptr ? -1 : a.ids[r];
    const bool given = id >= 0 && id < a.v;
    const float g = given && a.g != nullptr ? a.g[r] : 0.0f;
    const float h = ENTROPY ? a.h[r] : 0.0f;
    const float m = a.stats[2 * r], log_sum = a.stats[2 * r + 1];
    float d[kPer];
    if ((g == 0.0f && h == 0.0f) || m == -INFINITY) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) d[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < kGradVectors; ++i) store_vector<DT>(out, vector_at<DT, kThreads>(x_part, i), a.v, d);
        return;
    }
    const float beta = scale_of(a.inv_temp, r), c2 = beta * kLog2e, l2 = log_sum * kLog2e;
    const float ent = ENTROPY ? a.entropy[r] : 0.0f;
    // d = p (first + second t), t = lp / ln 2 held above -200 (p is 0 there); NaN statistics make it NaN
    const float first = -beta * (g + h * ent) + (log_sum - log_sum), second = ENTROPY ? -beta * h * (float)kLn2 : 0.0f;
    uint32_t w[kGradVectors][4];
    load_part<DT, kGradVectors, kThreads>(row, a.v, x_part, w);
#pragma unroll
    for (int i = 0; i < kGradVectors; ++i) {
        const int x = vector_at<DT, kThreads>(x_part, i);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float t = fmaxf((value<DT>(w[i], j) - m) * c2 - l2, kLowest);
            const float p = __builtin_amdgcn_exp2f(t);
            d[j] = p * (ENTROPY ? fmaf(second, t, first) : first);
        }
        if (given && id >= x && id < x + kPer) {  // the token itself: 1 - p from its log probability
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                if (id == x + j) {
                    const float y = value<DT>(w[i], j);
                    const float lp = y == y ? (y - m) * beta - log_sum : -INFINITY;
                    const float rest = -expm1f(lp);
                    d[j] = beta * (g * rest - (ENTROPY ? h * expf(lp) * (fmaxf(lp, kLowest) + ent) : 0.0f)) + (log_sum - log_sum);
                }
            }
        }
        store_vector<DT>(out, x, a.v, d);
    }
}

template <int DT>
void launch_grad(const GradArgs &a, unsigned grid, hipStream_t stream) {
    if (a.h != nullptr) logprob_grad<DT, true><<<grid, kThreads, 0, stream>>>(a);
    else logprob_grad<DT, false><<<grid, kThreads, 0, stream>>>(a);
}

}  // namespace

size_t logprobs_workspace_bytes(int32_t n_rows, int32_t v, int dtype, int n_top) { return plan_of(n_rows, v, dtype, n_top).total; }

int launch_logprobs(const LogprobsArgs &l, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const Plan p = plan_of(l.n_rows, l.v, l.dtype, l.n_top);
    if (p.total > 0 && (workspace == nullptr || workspace_bytes < p.total)) return TT_EWORKSPACE;
    if (p.total > 0 && reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return TT_EINVAL;
    RowArgs a;
    a.logits = l.logits;
    a.ld = l.ld;
    a.v = l.v;
    a.dtype = l.dtype;
    a.parts = p.split.parts;
    a.n_top = l.n_top;
    a.capacity = part_capacity(l.n_top);
    a.inv_temp = l.inv_temp;
    a.ids = l.ids;
    a.sums = static_cast<float4 *>(workspace);
    a.keys = p.total > 0 ? reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + p.sums) : nullptr;
    a.logprob = l.logprob;
    a.lse = l.lse;
    a.entropy = l.entropy;
    a.stats = l.stats;
    a.top_ids = l.top_ids;
    a.top_logprobs = l.top_logprobs;
    for (int64_t row0 = 0; row0 < l.n_rows; row0 += p.rows) {
        const int64_t n = l.n_rows - row0 < p.rows ? l.n_rows - row0 : p.rows;
        a.row0 = row0;
        if (l.dtype == TT_BF16) launch_rows<TT_BF16>(a, p.split, n, stream);
        else if (l.dtype == TT_F16) launch_rows<TT_F16>(a, p.split, n, stream);
        else launch_rows<TT_F32>(a, p.split, n, stream);
        if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
        if (a.parts == 1) continue;
        if (l.n_top > 0) row_finish<true><<<(unsigned)n, kThreads, 0, stream>>>(a);
        else row_finish<false><<<(unsigned)n, kThreads, 0, stream>>>(a);
        if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
    }
    return TT_OK;
}

int launch_logprobs_backward(const LogprobsGradArgs &l, hipStream_t stream) {
    GradArgs a;
    a.logits = l.logits;
    a.ld = l.ld;
    a.v = l.v;
    const int64_t per = (int64_t)kGradVectors * kThreads * elements_per_vector(l.dtype);
    a.parts = (int)((l.v + per - 1) / per);
    a.inv_temp = l.inv_temp;
    a.ids = l.ids;
    a.stats = l.stats;
    a.entropy = l.entropy;
    a.g = l.grad_logprob;
    a.h = l.grad_entropy;
    a.out = l.dlogits;
    a.out_ld = l.out_ld;
    const int64_t most = kMaxGrid / a.parts;
    for (int64_t row0 = 0; row0 < l.n_rows; row0 += most) {
        const int64_t n = l.n_rows - row0 < most ? l.n_rows - row0 : most;
        const unsigned grid = (unsigned)(n * a.parts);
        a.row0 = row0;
        if (l.dtype == TT_BF16) launch_grad<TT_BF16>(a, grid, stream);
        else if (l.dtype == TT_F16) launch_grad<TT_F16>(a, grid, stream);
        else launch_grad<TT_F32>(a, grid, stream);
        if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
    }
    return TT_OK;
}

}  // namespace tt
