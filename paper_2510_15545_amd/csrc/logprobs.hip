// Log probabilities of given tokens with log-sum-exp, entropy and top alternatives, and their
// gradient, from rows of bf16, fp16 or fp32 logits on gfx950.
//
// With x the row's logits (NaN counts as minus infinity), beta the row's inverse temperature:
//   M = max x,  S = sum exp(beta (x - M)),  L = ln S,  lse = beta M + L
//   lp_j = beta (x_j - M) - L,  p_j = exp(lp_j),  H = -sum p_j lp_j = L - sum beta (x_j - M) p_j
//   alternatives: the largest x, ties by the lower index, minus infinity never listed
//   d_j = beta (g ([j = id] - p_j) - h p_j (lp_j + H)), upstream gradients g of lp_id and h of H
//
// One pass over the row: row_stream, a workgroup for a row or a part of it, by chunks of 4 to 32 KB whose
// loads are in flight while the chunk before is worked on.  Each thread keeps the largest value and the sums
// (base 2, v_exp_f32) of what it has seen: in fp32 over a thread's elements, chunk by chunk, in fp64
// from the waves' sums on (from the workgroups', where they share a row).  The token's logit is read behind
// the first chunk's loads.
//
// Alternatives, in the same pass: each thread keeps the place of its largest value as well.  k of the
// workgroup's 64 or 256 groups of threads hold a largest value that reaches the k-th largest of the groups',
// so every one of the k largest elements does.  That bound is formed after chunks 1, 2, 4, 8, ..., and elements
// that reach it are staged in LDS as 64-bit keys (value, then lower index), over a row of N chunks about
// k (1 + log2 N) of them (of long rows their whole vectors, told apart at the end); then the keys are ordered by
// counting.  Rows of which more are staged than there is room for (TopSet::finish) are read again.  A row's only
// workgroup finishes it; with several, each hands its sums and keys to row_finish.
//
// What bounds it: the reading of the logits, at 6.4 to 6.9 TB/s on a row set beyond the Infinity Cache (4,096
// rows of 151,936 bf16: 187 us a pass, 6.7 TB/s; a kernel that only reads gets no more), and the VALU where the
// alternatives are wanted (about 9 issue slots an element for the statistics, the exponential four of them; 1,024
// rows of 262,144 with 64 alternatives: 94 us against 80 to read them; the VALU is busy 77% of the cycles).  Few rows
// are latency: one row of 640 takes 5 us on the GPU, one of 151,936 with 20 alternatives 6 for its 19 parts and 7 to
// join them.
#include "rows.h"

namespace tt {
namespace {

using namespace rows;

constexpr int kMaxTop = 128;
constexpr int kSelect = 1024;                       // keys that are ordered in LDS
constexpr int kGroups = 256;                        // lane groups whose largest values give the bound
constexpr int kChunkVectors = 4;                     // 20 alternatives of 1,000 rows of 50,257: 26.7 us; by 6: 29.5; 8: 34.2
constexpr int64_t kShortBytes = 8 << 10;            // rows up to these bytes are taken by one vector a thread
// For rows of over one chunk taken whole where they are few (20 alternatives of one row of 16,000 bf16: 7.2 us, 9.3 by
// kThreads; of 200: 8.2 and 10.4; of 50,257 of one to 64: 11.9 to 13.3, 11.9 to 15.2 split).
constexpr int kLongThreads = 1024, kLongVectors = 2;
// Rows of more bytes stage whole vectors where they are taken by kThreads, or have many alternatives (20 of 1,000 rows
// of 24,000 bf16: 19.0 us so, 19.4 by elements; of 50,257: 26.9 and 29.4, 128: 38.4 and 47.3; 20 of 2,000 of 16,000: 27.8
// and 26.0; by 1,024 threads, 128 of 64 rows of 50,257: 19.7 and 21.4, 20: 13.3 and 12.7).
constexpr int64_t kVectorBytes = 32 << 10;
// Rows up to these bytes are taken whole, by 1,024 threads each, however few they are; longer ones from few_rows
// on; fewer are split over more workgroups and joined by a second kernel (20 alternatives of one row of 151,936 bf16:
// 12.9 us, 21.9 whole; of 48 of 128,256: 15.5 and 19.4; of 128: 21.2 and 18.7; of 96 of 262,200: 26 and 31, of 128: 31.5
// and 31.7, of 160: 33.7 and 32.0, of 191: 37 and 32, without alternatives 24 and 24; of 96 of 500,000: 36 and 45, of 160:
// 45 and 46, of 191: 51 and 46; of 96 of a million: 52 and 77, of 160: 70 and 78, of 191: 82 and 78).
constexpr int64_t kLongBytes = 128 << 10;
int64_t few_rows(int64_t row_bytes) { return row_bytes <= (512 << 10) ? 96 : 192; }

// Rows from which on a workgroup of kThreads each keeps the GPU busy; fewer are better taken by 1,024 threads
// each (alternatives of 333 rows of 201 KB: 18.9 us by 256 threads, 20.9 by 1,024; of 400 rows of 304 KB: 36.4
// and 32.7; of 1,000: 54.5 and 62.0).
int64_t many_rows(int64_t row_bytes) { return row_bytes <= (256 << 10) ? 256 : 512; }
constexpr int64_t kMaxGrid = int64_t(1) << 18;      // workgroups of one launch

// Keys that a part may hand over; a part with more that reach its bound selects its k largest exactly.
inline int part_capacity(int n_top) { return 8 * n_top + 64; }

struct RowArgs {
    const void *logits;
    int64_t ld, row0;  // row0: the first row of this launch
    int v, dtype, parts, part_width, n_top, capacity;
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
    static constexpr int kStage = THREADS == kThreads ? 512 : 256;
    uint32_t group[2][kGroups];  // in turn, so that one barrier does
    uint32_t largest[THREADS];
    int where[THREADS];
    uint64_t stage[THREADS / kWave][kStage];
    int slots[64], total;
};

// An element reaches the bound if its order key is larger than `key`, or equal and its index at most `index`.
struct Bound {
    uint32_t key;
    int index;
    __device__ __forceinline__ float lowest() const { return key_value(key); }
    __device__ __forceinline__ uint64_t full() const { return ((uint64_t)key << 32) | (0xFFFFFFFFu - (uint32_t)index); }
};

constexpr uint32_t kLowestFinite = 0x00800000u;  // order key of -FLT_MAX

__device__ __forceinline__ uint64_t full_key(uint32_t order, int index) {
    return ((uint64_t)order << 32) | (0xFFFFFFFFu - (uint32_t)index);
}

// Lanes below this one among those of a mask.
__device__ __forceinline__ int lanes_below(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// The largest of the keys of GROUP lanes (1, 4 or 16 in a row of 16), in each of them.
template <int GROUP>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
    auto with = [&](uint32_t y) { x = y > x ? y : x; };
    if constexpr (GROUP >= 4) {
        with(__builtin_amdgcn_update_dpp(0u, x, 0xB1, 0xF, 0xF, true));  // quad_perm 1,0,3,2
        with(__builtin_amdgcn_update_dpp(0u, x, 0x4E, 0xF, 0xF, true));  // quad_perm 2,3,0,1
    }
    if constexpr (GROUP >= 16) {
        with(__builtin_amdgcn_update_dpp(0u, x, 0x124, 0xF, 0xF, true));  // row_ror 4
        with(__builtin_amdgcn_update_dpp(0u, x, 0x128, 0xF, 0xF, true));  // row_ror 8
    }
    return x;
}

// A key that at least k of the wave's keys reach, G a lane, and how many do: not more than `enough`, unless that many
// are equal to it (then it is the k-th largest itself).  kLowestFinite where fewer than k are finite.
struct Kth {
    uint32_t key;
    int n;
    bool tied;
};

template <int G>
__device__ __forceinline__ Kth kth_key(const uint32_t (&q)[G], int k, int enough) {
    auto reach = [&](uint32_t c) {
        int n = 0;
#pragma unroll
        for (int u = 0; u < G; ++u) n += __popcll(__ballot(q[u] >= c));
        return n;
    };
    uint32_t most = 0, least = 0xFFFFFFFFu;  // of the finite ones: a close range to search
#pragma unroll
    for (int u = 0; u < G; ++u) {
        most = q[u] > most ? q[u] : most;
        least = q[u] >= kLowestFinite && q[u] < least ? q[u] : least;
    }
    uint32_t lo = wave_min(least), hi = wave_max(most);
    int n = reach(lo);
    if (n < k) return {kLowestFinite, n, false};
    const int m = reach(hi);
    if (m >= k) return {hi, m, m > enough};
    while (n > enough && hi - lo > 1) {  // n reach lo, fewer than k reach hi
        const uint32_t c = lo + (hi - lo) / 2;
        const int r = reach(c);
        if (r >= k) {
            lo = c;
            n = r;
        } else {
            hi = c;
        }
    }
    return {lo, n, n > enough};
}

// The same for the workgroup's keys, one a thread: by 64 groups of threads for small k (a group counts once), 256 else.
// sh_group: kGroups words that nobody reads until the barrier in here.
constexpr int kFewTop = 32;

template <int THREADS>
__device__ __forceinline__ Kth kth_of_threads(uint32_t key, int k, uint32_t *sh_group) {
    constexpr int kFew = THREADS / kWave, kMany = THREADS / kGroups;  // threads of a group
    const int lane = threadIdx.x % kWave, enough = k + k / 4 + 2;
    if (k <= kFewTop) {
        key = group_max<kFew>(key);
        if (lane % kFew == 0) sh_group[threadIdx.x / kFew] = key;
        __syncthreads();
        const uint32_t q[1] = {sh_group[lane]};
        return kth_key<1>(q, k, enough);
    }
    key = group_max<kMany>(key);
    if (lane % kMany == 0) sh_group[threadIdx.x / kMany] = key;
    __syncthreads();
    uint32_t q[kGroups / kWave];
#pragma unroll
    for (int u = 0; u < kGroups / kWave; ++u) q[u] = sh_group[u * kWave + lane];
    return kth_key<kGroups / kWave>(q, k, enough);
}

// The same by the threads themselves: a closer bound.  (Not for every row: 1,100 rows of 640 with 20 alternatives take
// 8.8 us, 10.5 with it.)  sh_each: THREADS words.
template <int THREADS>
__device__ __forceinline__ Kth kth_of_each(uint32_t key, int k, int enough, uint32_t *sh_each) {
    constexpr int kEach = THREADS / kWave;
    __syncthreads();
    sh_each[threadIdx.x] = key;
    __syncthreads();
    uint32_t q[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) q[u] = sh_each[u * kWave + threadIdx.x % kWave];
    return kth_key<kEach>(q, k, enough);
}

// Sum over the workgroup of a count, through a zeroed LDS slot of its own.
__device__ __forceinline__ int block_count(int n, int *slot) {
    n = (int)wave_sum((uint32_t)n);
    if (threadIdx.x % kWave == 0) atomicAdd(slot, n);
    __syncthreads();
    return *slot;
}

// Elements x0 .. x1 - 1 of a row that satisfy f(order key, index), counted by this thread.
template <int DT, int THREADS, typename F>
__device__ __forceinline__ int count_if(const typename Elem<DT>::T *row, int x0, int x1, F f) {
    int n = 0;
#pragma unroll 4
    for (int x = x0 + (int)threadIdx.x; x < x1; x += THREADS) {
        const float y = decode<DT>(row[x]);
        n += (y > -INFINITY && f(order_key(y), x)) ? 1 : 0;
    }
    return n;
}

// The k largest of a part's elements exactly, where too many reach the closest bound, too (only rows made for it do
// that: large values all in the same lanes): the k-th largest value by binary search on its order key, then the last
// index among the elements equal to it, each step a count over the part, read again element by element (57 of them: 400
// us for a row of 50,257).  At least k elements are finite.
template <int DT, int THREADS>
__device__ __noinline__ void select_exactly(const typename Elem<DT>::T *row, int x0, int x1, int k, uint64_t *keys, int *sh_slots,
                                            int *sh_total) {
    if (threadIdx.x < 64) sh_slots[threadIdx.x] = 0;
    if (threadIdx.x == 0) *sh_total = 0;
    __syncthreads();
    int slot = 0;
    uint32_t kth = 0;
    for (int b = 31; b >= 0; --b) {
        const uint32_t c = kth | (1u << b);
        const int n = count_if<DT, THREADS>(row, x0, x1, [c](uint32_t o, int) { return o >= c; });
        if (block_count(n, &sh_slots[slot++]) >= k) kth = c;
    }
    const int above = count_if<DT, THREADS>(row, x0, x1, [kth](uint32_t o, int) { return o > kth; });
    const int need = k - block_count(above, &sh_slots[slot++]);
    int last = 0;  // the largest index with fewer than `need` equal elements below it
    for (int b = 23; b >= 0; --b) {
        const int c = last | (1 << b);
        const int n = count_if<DT, THREADS>(row, x0, x1, [kth, c](uint32_t o, int x) { return o == kth && x < c; });
        if (block_count(n, &sh_slots[slot++]) < need) last = c;
    }
    count_if<DT, THREADS>(row, x0, x1, [=](uint32_t o, int x) {
        if (o > kth || (o == kth && x <= last)) keys[atomicAdd(sh_total, 1)] = full_key(o, x);
        return false;
    });
    __syncthreads();
}

// The keys of a part that reach a bound, to dst (as many as fit), the part read again; returns their number.
template <int DT, int THREADS>
__device__ __noinline__ int read_again(const typename Elem<DT>::T *row, int v, int x0, int x1, Bound bound, uint64_t *dst, int capacity,
                                       int *sh_total) {
    constexpr int kPer = Elem<DT>::kPer, NV = 2;
    const int lane = threadIdx.x % kWave;
    const float lowest = bound.lowest();
    __syncthreads();
    if (threadIdx.x == 0) *sh_total = 0;
    __syncthreads();
    for_chunks<DT, NV, THREADS, true, false, true, 1>(row, v, x0, x1, [] {}, [&](uint32_t(&w)[NV][4], int x_chunk) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const float x = value<DT>(w[i], j);
                const int at = vector_at<DT, THREADS>(x_chunk, i) + j;
                const bool in = at < x1 && (x > lowest || (x == lowest && at <= bound.index));
                const uint64_t hit = __ballot(in);
                if (hit == 0) continue;
                int base = 0;
                if (lane == 0) base = atomicAdd(sh_total, __popcll(hit));
                base = __builtin_amdgcn_readfirstlane(base) + lanes_below(hit);
                if (in && base < capacity) dst[base] = full_key(order_key(x), at);
            }
        }
    });
    __syncthreads();
    const int n = *sh_total;
    __syncthreads();
    return n;
}

// Many keys are equal to a bound (a row of capped or of few different logits): of the elements equal to it, those up to
// an index that enough threads' elements do not pass.  largest, last: of each thread, in LDS.
template <int THREADS>
__device__ __forceinline__ void break_tie(Bound &bound, int k, uint32_t key, int last, TopLds<THREADS> &sh) {
    const int lane = threadIdx.x % kWave;
    __syncthreads();
    sh.largest[threadIdx.x] = key;
    sh.where[threadIdx.x] = last;
    __syncthreads();
    auto count = [&](auto f) {
        int n = 0;
        for (int u = 0; u < THREADS / kWave; ++u) n += __popcll(__ballot(f(sh.largest[u * kWave + lane], sh.where[u * kWave + lane])));
        return n;
    };
    const uint32_t kth = bound.key;
    const int need = k - count([=](uint32_t o, int) { return o > kth; });
    if (need <= 0) {
        ++bound.key;  // enough lie above it
        return;
    }
    bound.index = 0;  // the largest index with fewer than `need` equal ones below it
    for (int b = 23; b >= 0; --b) {
        const int c = bound.index | (1 << b);
        if (count([=](uint32_t o, int at) { return o == kth && at < c; }) < need) bound.index = c;
    }
}

// The bound from the threads' own largest values.
template <int THREADS>
__device__ __forceinline__ Bound closer_bound(uint32_t key, int last, int k, int enough, TopLds<THREADS> *sh) {
    const Kth q = kth_of_each<THREADS>(key, k, enough, sh->largest);
    Bound bound = {q.key, INT_MAX};
    if (q.tied) break_tie<THREADS>(bound, k, key, last, *sh);
    return bound;
}

// The elements of a row that may be among its k largest, chunk by chunk.  VECTORS: whole vectors are staged, with
// their largest value, and those that reach the last bound are read again for their elements: fewer instructions in
// a long row's stream, but another round trip at its end.
template <int DT, int NV, int THREADS, bool VECTORS>
struct TopSet {
    static constexpr int kPer = Elem<DT>::kPer, kStage = TopLds<THREADS>::kStage;
    TopLds<THREADS> &sh;
    int k;
    Bound bound = {kLowestFinite, INT_MAX};
    float most = -INFINITY;     // the thread's largest value
    int where = 0;              // first index of its vector
    int staged = 0, chunks = 0; // of this wave; of the row
    int turn = 0;
    bool current = false;       // the bound is that of all chunks so far

    // The bound from the threads' largest values.
    __device__ __forceinline__ void raise() {
        const uint32_t key = order_key(most);
        turn ^= 1;
        const Kth q = kth_of_threads<THREADS>(key, k, sh.group[turn]);
        bound = {q.key, INT_MAX};
        if (q.tied) break_tie<THREADS>(bound, k, key, where + kPer - 1, sh);
        current = true;
    }

    __device__ __forceinline__ void add(const uint32_t (&w)[NV][4], const float (&vm)[NV], int x_chunk) {
        const int wave = threadIdx.x / kWave;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (vm[i] > most) {
                most = vm[i];
                where = vector_at<DT, THREADS>(x_chunk, i);
            }
        }
        current = false;
        ++chunks;
        if ((chunks & (chunks - 1)) == 0) raise();
        const float lowest = bound.lowest();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (__ballot(vm[i] >= lowest) == 0) continue;
            auto put = [&](float x, int at) {
                const bool in = x > lowest || (x == lowest && at <= bound.index);
                const uint64_t hit = __ballot(in);
                const int slot = staged + lanes_below(hit);
                if (in && slot < kStage) sh.stage[wave][slot] = full_key(order_key(x), at);
                staged += __popcll(hit);
            };
            const int at = vector_at<DT, THREADS>(x_chunk, i);
            if constexpr (VECTORS) {
                put(vm[i], at);
                continue;
            }
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const float x = value<DT>(w[i], j);
                if (__ballot(x >= lowest) != 0) put(x, at + j);
            }
        }
    }

    // The elements of the staged vectors, read again, that reach the bound, to dst; their number goes to sh.total.
    __device__ __forceinline__ void expand(const typename Elem<DT>::T *row, int x1, uint64_t *dst, int capacity) {
        const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
        const uint64_t from = bound.full();
        for (int i = lane; i - lane < staged; i += kWave) {
            const uint64_t key = i < staged ? sh.stage[wave][i] : 0;
            const bool in = i < staged && (uint32_t)(key >> 32) >= bound.key;
            const int at = (int)(0xFFFFFFFFu - (uint32_t)key);
            uint64_t mine[kPer];
            int n = 0;
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const float x = in && at + j >= 0 && at + j < x1 ? decode<DT>(row[at + j]) : -INFINITY;
                mine[j] = x > -INFINITY ? full_key(order_key(x), at + j) : 0;  // no NaN
                n += __popcll(__ballot(mine[j] >= from));
            }
            int base = 0;
            if (lane == 0) base = atomicAdd(&sh.total, n);
            base = __builtin_amdgcn_readfirstlane(base);
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const uint64_t hit = __ballot(mine[j] >= from);
                const int slot = base + lanes_below(hit);
                if (mine[j] >= from && slot < capacity) dst[slot] = mine[j];
                base += __popcll(hit);
            }
        }
    }

    // The staged keys that reach the bound, to dst (as many as `capacity`, or none); returns their number, or more than
    // `capacity` where a wave's did not fit.
    __device__ __forceinline__ int gather(const typename Elem<DT>::T *row, int x1, uint64_t *dst, int capacity) {
        const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
        const uint64_t from = bound.full();
        if (threadIdx.x == 0) sh.total = 0;
        __syncthreads();
        const bool over = staged > kStage;
        int n = 0;
        if (over) {
            n = capacity + 1;
        } else if constexpr (VECTORS) {
            expand(row, x1, dst, capacity);
        } else {
            for (int i = lane; i - lane < staged; i += kWave) n += __popcll(__ballot(i < staged && sh.stage[wave][i] >= from));
        }
        int base = 0;
        if (lane == 0) base = atomicAdd(&sh.total, n);
        base = __builtin_amdgcn_readfirstlane(base);
        __syncthreads();
        const int total = sh.total;
        if (VECTORS || total > capacity) return total;
        for (int i = lane; i - lane < staged; i += kWave) {
            const uint64_t key = i < staged ? sh.stage[wave][i] : 0;
            const bool in = i < staged && key >= from;
            const uint64_t hit = __ballot(in);
            if (in) dst[base + lanes_below(hit)] = key;
            base += __popcll(hit);
        }
        return total;
    }

    // The keys that reach the bound of the whole part, to dst (LDS or global, `capacity` >= k of them); returns their
    // number: at least k, or all of the part's finite elements.  Where more were staged than there is room for, the
    // running bounds were too low (a mask has left a run of tokens, or the part is short, and hardly more groups of
    // threads than k hold one) or came too late (what precedes the likely tokens is masked or low, or the row rises): the
    // part is read again by the threads' own bound (20 alternatives of one row of 50,257 held to 500 tokens: 22 us, other
    // rows 12.6; 64 of 1,024 rows of 262,144 whose first half is masked: 245 and 108).
    __device__ __forceinline__ int finish(const typename Elem<DT>::T *row, int v, int x0, int x1, uint64_t *dst, int capacity) {
        if (!current) raise();
        const uint32_t key = order_key(most);
        const int last = where + kPer - 1;
        const int total = gather(row, x1, dst, capacity);
        if (total <= capacity) return total;
        for (int enough = k + k / 4 + 2;; enough = k) {  // the second time exactly: of tokens that rise 8 k reach it
            bound = closer_bound<THREADS>(key, last, k, enough, &sh);
            const int n = read_again<DT, THREADS>(row, v, x0, x1, bound, dst, capacity, &sh.total);
            if (n <= capacity) return n;
            if (enough == k) break;
        }
        select_exactly<DT, THREADS>(row, x0 > 0 ? x0 : 0, x1, k, dst, sh.slots, &sh.total);
        return k;
    }
};

// The largest k (all, if fewer) of c <= kSelect distinct keys in LDS, descending, in sh_out; returns their number.
template <int THREADS>
__device__ __forceinline__ int order_keys(uint64_t *sh_sel, int c, int k, uint32_t *sh_group, int *sh_total, uint64_t *sh_out) {
    const int lane = threadIdx.x % kWave;
    if (c > kGroups) {  // counting is quadratic: the bound once more, a few keys a lane
        constexpr int kEach = kSelect / THREADS;
        uint64_t mine[kEach];
        uint32_t most = 0;
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const int i = u * THREADS + (int)threadIdx.x;
            mine[u] = i < c ? sh_sel[i] : 0;
            const uint32_t o = (uint32_t)(mine[u] >> 32);
            most = o > most ? o : most;
        }
        __syncthreads();
        if (threadIdx.x == 0) *sh_total = 0;
        const uint64_t from = (uint64_t)kth_of_threads<THREADS>(most, k, sh_group).key << 32;
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

// A row's token, -1 where there is none, and its logit: both read long before they are wanted.
__device__ __forceinline__ int32_t token_of(const RowArgs &a, int64_t row) {
    const int32_t id = a.logprob == nullptr ? -1 : a.ids[row];
    return id < a.v ? id : -1;
}
__device__ __forceinline__ float token_logit(const RowArgs &a, int64_t row, int32_t id) {
    return id >= 0 ? load_logit(row_at(a.logits, a.dtype, row * a.ld), a.dtype, id) : 0.0f;
}

// From the row's largest logit m and the sum s relative to it.
__device__ __forceinline__ RowStats row_stats(double beta, float m, double s) {
    // m = -inf: nothing is finite (s = 0); m = +inf or an unsound temperature: NaN
    RowStats q;
    q.m = m;
    q.beta = beta;
    q.bad = !sound(beta) || m == INFINITY;
    q.log_sum = q.bad ? NAN : (m == -INFINITY ? 0.0 : log(s));
    return q;
}

// A row's results but the alternatives, by one thread: s and e as in Sum, in natural units; the token and its logit.
__device__ __forceinline__ void write_row(const RowArgs &a, int64_t row, const RowStats &q, double s, double e, int32_t id, float x_id) {
    if (a.stats != nullptr) {
        a.stats[2 * row] = q.bad ? NAN : (float)q.m;
        a.stats[2 * row + 1] = (float)q.log_sum;
    }
    if (a.lse != nullptr) a.lse[row] = (float)(q.bad ? NAN : q.m * q.beta + q.log_sum);
    if (a.entropy != nullptr) a.entropy[row] = (float)(q.bad ? NAN : (q.m == -INFINITY ? 0.0 : q.log_sum - e / s));
    if (a.logprob != nullptr) {
        double lp = NAN;
        if (!q.bad && id >= 0) lp = x_id == -INFINITY ? -INFINITY : ((double)x_id - q.m) * q.beta - q.log_sum;
        a.logprob[row] = (float)lp;
    }
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

// A part of a row by a workgroup; FINISH: the row is one part, and finished here.  VECTORS: as in TopSet.
template <int DT, int THREADS, int NV, bool TOP, bool ENTROPY, bool FINISH, bool VECTORS>
__global__ __launch_bounds__(THREADS, THREADS == kThreads ? 1 : 8) void row_stream(RowArgs a) {
    constexpr int kWaves = THREADS / kWave;
    __shared__ Sum sh_sum[kWaves];
    __shared__ TopLds<THREADS> sh;
    __shared__ uint64_t sh_sel[kSelect], sh_out[kMaxTop];
    __shared__ RowStats sh_stats;
    pass_over_nans();
    const int64_t r = FINISH ? blockIdx.x : blockIdx.x / (uint32_t)a.parts, row_i = a.row0 + r;
    const int part = FINISH ? 0 : blockIdx.x % (uint32_t)a.parts, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const auto *row = static_cast<const typename Elem<DT>::T *>(a.logits) + row_i * a.ld;
    const int x0 = part * a.part_width - lead_of<DT>(row, a.v), x1 = FINISH || part + 1 == a.parts ? a.v : x0 + a.part_width;
    const float beta = scale_of(a.inv_temp, row_i), c2 = beta * kLog2e;
    const int32_t id = FINISH ? token_of(a, row_i) : -1;
    float x_id = 0.0f;  // read behind the first chunk's loads, or where registers are few behind the sums
    constexpr bool kLate = TOP && THREADS == kLongThreads;
    int count = 0;
    Sum mine = {-INFINITY, 0.0f, 0.0f};
    TopSet<DT, NV, THREADS, VECTORS> top{sh, a.n_top};
    for_chunks<DT, NV, THREADS, true, false, true, TOP ? 1 : 2>(row, a.v, x0, x1, [&] { if (!kLate) x_id = token_logit(a, row_i, id); }, [&](uint32_t(&w)[NV][4], int x) {
        float vm[NV];
        add_chunk<DT, NV, ENTROPY>(w, c2, mine, vm);
        if constexpr (TOP) top.add(w, vm, x);
    });
    if (kLate) x_id = token_logit(a, row_i, id);
    mine = wave_join<ENTROPY>(mine, c2);
    if (lane == 0) sh_sum[wave] = mine;
    if constexpr (TOP)
        count = top.finish(row, a.v, x0, x1, FINISH ? sh_sel : a.keys + ((size_t)r * a.parts + part) * a.capacity, FINISH ? kSelect : a.capacity);
    __syncthreads();
    if constexpr (!FINISH) {
        if (threadIdx.x == 0) {
            Sum s = sh_sum[0];
#pragma unroll
            for (int u = 1; u < kWaves; ++u) s = join(s, sh_sum[u], c2);
            a.sums[(size_t)r * a.parts + part] = make_float4(s.m, s.s, s.e, __int_as_float(count));
        }
        return;
    }
    if (wave == 0) {  // one wave joins the waves' sums
        const Sum q = lane < kWaves ? sh_sum[lane] : Sum{-INFINITY, 0.0f, 0.0f};
        const float m = wave_max(q.m);
        double s = 0.0, e = 0.0;
        if (q.s > 0.0f) {
            const double t = ((double)q.m - (double)m) * (double)beta, f = exp(t);
            s = q.s * f;
            e = (q.e * kLn2 + q.s * fmax(t, -1000.0)) * f;
        }
        s = wave_sum(s);
        e = ENTROPY ? wave_sum(e) : 0.0;
        const RowStats stats = row_stats(beta, m, s);
        if (lane == 0) {
            sh_stats = stats;
            write_row(a, row_i, stats, s, e, id, x_id);
        }
    }
    if constexpr (TOP && FINISH) {
        count = order_keys<THREADS>(sh_sel, count, a.n_top, sh.group[0], &sh.total, sh_out);
        if ((int)threadIdx.x < a.n_top) write_top(a, row_i, sh_stats, sh_out, count, threadIdx.x);
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

template <bool TOP>
__global__ __launch_bounds__(kThreads) void row_finish(RowArgs a) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ float sh_m[kWaves];
    __shared__ double sh_s[kWaves], sh_e[kWaves];
    __shared__ uint64_t sh_sel[kSelect], sh_out[kMaxTop];
    __shared__ uint32_t sh_group[kGroups];
    __shared__ int sh_count[kThreads], sh_longest[kWaves], sh_slots[1], sh_total;
    const int64_t r = blockIdx.x, row = a.row0 + r;
    const float4 *sums = a.sums + (size_t)r * a.parts;
    const uint64_t *keys = a.keys + (size_t)r * a.parts * a.capacity;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int32_t id = token_of(a, row);
    const double beta = scale_of(a.inv_temp, row);
    float4 q = {-INFINITY, 0.0f, 0.0f, 0.0f};  // the thread's first part
    if ((int)threadIdx.x < a.parts) q = sums[threadIdx.x];
    float m = q.x;
    uint32_t longest = __float_as_uint(q.w);
    for (int p = threadIdx.x + kThreads; p < a.parts; p += kThreads) {
        m = fmaxf(m, sums[p].x);
        const uint32_t n = __float_as_uint(sums[p].w);
        longest = n > longest ? n : longest;
    }
    m = wave_max(m);
    if (lane == 0) sh_m[wave] = m;
    if constexpr (TOP) {
        sh_count[threadIdx.x] = __float_as_int(q.w);
        longest = wave_max(longest);
        if (lane == 0) sh_longest[wave] = (int)longest;
    }
    if (threadIdx.x == 0) sh_total = 0;
    __syncthreads();
    const float x_id = token_logit(a, row, id);
    // the keys: where they are few, all of them in registers, a run of 64 of a part's a load, in flight together
    uint64_t mine[kHeld];
    bool held = false;
    if constexpr (TOP) {
        int most = sh_longest[0];
#pragma unroll
        for (int u = 1; u < kWaves; ++u) most = sh_longest[u] > most ? sh_longest[u] : most;
        const int runs = (most + kWave - 1) / kWave;
        held = a.parts <= kThreads && a.parts * runs <= kHeld * kWaves;
        if (held) {
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                const int c = u * kWaves + wave, p = runs > 0 ? c / runs : a.parts, i = (c - p * runs) * kWave + lane;
                mine[u] = 0;
                if (p < a.parts && i < sh_count[p]) mine[u] = keys[(size_t)p * a.capacity + i];
            }
        }
    }
    m = fmaxf(fmaxf(sh_m[0], sh_m[1]), fmaxf(sh_m[2], sh_m[3]));
    double s = 0.0, e = 0.0;  // e in natural units
    for (int p = threadIdx.x; p < a.parts; p += kThreads) {
        if (p >= kThreads) q = sums[p];
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
    uint64_t from = 0;
    uint32_t most = 0;  // of the thread's keys
    if constexpr (TOP) {
        auto larger = [&](uint64_t key) {
            const uint32_t o = (uint32_t)(key >> 32);
            most = o > most ? o : most;
        };
        if (held) {
#pragma unroll
            for (int u = 0; u < kHeld; ++u) larger(mine[u]);
        } else {
            for_each_key(a, sums, keys, larger);
        }
        from = (uint64_t)kth_of_threads<kThreads>(most, a.n_top, sh_group).key << 32;  // (a barrier)
    } else {
        __syncthreads();
    }
    s = sh_s[0] + sh_s[1] + sh_s[2] + sh_s[3];
    e = sh_e[0] + sh_e[1] + sh_e[2] + sh_e[3];
    const RowStats stats = row_stats(beta, m, s);
    if (threadIdx.x == kThreads - 1) write_row(a, row, stats, s, e, id, x_id);
    if constexpr (TOP) {
        for (bool closer = true;; closer = false) {
            auto put = [&](uint64_t key) {
                const uint64_t hit = __ballot(key >= from);
                if (hit == 0) return;
                int base = 0;
                if (lane == 0) base = atomicAdd(&sh_total, __popcll(hit));
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
            if (sh_total <= kSelect) break;
            if (closer) {
                // many equal values, or hardly more groups than k hold a key (a wave's lanes past the parts' keys have
                // none): the k-th largest of the threads' largest keys, lower tokens first (64 alternatives of 48
                // rows of 151,936 zeros: 67 us, 482 by the search below; other rows 19.6)
                uint64_t own = 0, q[kWaves];
                auto larger = [&](uint64_t key) { own = key > own ? key : own; };
                if (held) {
#pragma unroll
                    for (int u = 0; u < kHeld; ++u) larger(mine[u]);
                } else {  // a part's keys over all threads: of equal values those of the row's first parts decide
                    for (int p = 0; p < a.parts; ++p)
                        for (int i = threadIdx.x, n = __float_as_int(sums[p].w); i < n; i += kThreads) larger(keys[(size_t)p * a.capacity + i]);
                }
                __syncthreads();
                sh_sel[threadIdx.x] = own;
                __syncthreads();
#pragma unroll
                for (int u = 0; u < kWaves; ++u) q[u] = sh_sel[u * kWave + lane];
                from = 0;
                for (int b = 63; b >= 0; --b) {
                    const uint64_t c = from | (1ull << b);
                    int n = 0;
#pragma unroll
                    for (int u = 0; u < kWaves; ++u) n += __popcll(__ballot(q[u] >= c));
                    if (n >= a.n_top) from = c;
                }
                from = from > 0 ? from : 1;  // fewer threads have one: all keys
            } else {  // the k-th largest key itself (keys are distinct, so k reach it), by binary search
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
            }
            __syncthreads();
            if (threadIdx.x == 0) sh_total = 0;
            __syncthreads();
        }
        const int n = order_keys<kThreads>(sh_sel, sh_total, a.n_top, sh_group, &sh_total, sh_out);
        if ((int)threadIdx.x < a.n_top) write_top(a, row, stats, sh_out, n, threadIdx.x);
    }
}

struct Plan {
    int parts, part_width;  // of a row; one part: a row's workgroup finishes it
    int threads;
    int64_t rows;           // of one launch
    size_t sums, total;
};

// Rows whole, a workgroup each, where they are enough or short; else in as many parts as fill the GPU.
Plan plan_of(int64_t n_rows, int32_t v, int dtype, int n_top) {
    Plan p;
    const int chunk = kChunkVectors * kThreads * elements_per_vector(dtype), chunks = (v + chunk - 1) / chunk;
    int64_t parts = 1;
    p.threads = kThreads;
    const int64_t bytes = (int64_t)v * element_bytes(dtype);
    if (chunks > 1 && n_rows < many_rows(bytes)) {
        if (n_rows >= few_rows(bytes) || bytes <= kLongBytes) p.threads = kLongThreads;
        else parts = n_rows > 0 ? (kFullGrid + n_rows - 1) / n_rows : 1;
        if (parts > chunks) parts = chunks;
    }
    const int each = (int)((chunks + parts - 1) / parts);
    p.part_width = each * chunk;
    p.parts = (chunks + each - 1) / each;
    const int64_t most = kMaxGrid / p.parts;
    const int64_t groups = (n_rows + most - 1) / most;
    p.rows = groups == 0 ? 0 : (n_rows + groups - 1) / groups;
    p.sums = p.parts > 1 ? round256((size_t)p.rows * p.parts * sizeof(float4)) : 0;
    p.total = p.sums + (p.parts > 1 && n_top > 0 ? (size_t)p.rows * p.parts * part_capacity(n_top) * sizeof(uint64_t) : 0);
    return p;
}

template <int DT, bool TOP, bool ENTROPY>
void launch_rows(const RowArgs &a, int threads, int64_t n, hipStream_t stream) {
    const unsigned grid = (unsigned)(n * a.parts);
    const int64_t bytes = (int64_t)a.v * element_bytes(DT);
    const bool vectors = TOP && bytes > kVectorBytes && (threads == kThreads || a.n_top > kFewTop);
    if (threads == kLongThreads) {
        if (vectors) row_stream<DT, kLongThreads, kLongVectors, TOP, ENTROPY, true, TOP><<<grid, kLongThreads, 0, stream>>>(a);
        else row_stream<DT, kLongThreads, kLongVectors, TOP, ENTROPY, true, false><<<grid, kLongThreads, 0, stream>>>(a);
    } else if (a.parts > 1) {
        row_stream<DT, kThreads, kChunkVectors, TOP, ENTROPY, false, false><<<grid, kThreads, 0, stream>>>(a);
    } else if (bytes <= kShortBytes) {
        // 4,000 rows of 2,000 (5 alternatives): 19.4 us by one vector, 22.8 by four; 333 of 50,257 fp32: 33.4 and 19.1
        row_stream<DT, kThreads, 1, TOP, ENTROPY, true, false><<<grid, kThreads, 0, stream>>>(a);
    } else if (vectors) {
        row_stream<DT, kThreads, kChunkVectors, TOP, ENTROPY, true, TOP><<<grid, kThreads, 0, stream>>>(a);
    } else {
        row_stream<DT, kThreads, kChunkVectors, TOP, ENTROPY, true, false><<<grid, kThreads, 0, stream>>>(a);
    }
}

template <int DT>
void launch_rows(const RowArgs &a, int threads, int64_t n, hipStream_t stream) {
    if (a.n_top > 0) {
        if (a.entropy != nullptr) launch_rows<DT, true, true>(a, threads, n, stream);
        else launch_rows<DT, true, false>(a, threads, n, stream);
    } else {
        if (a.entropy != nullptr) launch_rows<DT, false, true>(a, threads, n, stream);
        else launch_rows<DT, false, false>(a, threads, n, stream);
    }
}

// ---------------------------------------------------------------- gradient
// One reading and one writing of the row, nothing kept between elements: p from the row's statistics, one
// exponential each.  A workgroup takes one part of two vectors a thread, so that very many are at different
// points of load and store, which mixes reads and writes best; loads ahead of the stores gain nothing.  Bound by
// HBM: 2,048 rows of 128,256 bf16 take 166 us, 6.3 TB/s read and written (a large copy gets 5.1).
constexpr int kGradVectors = 2;

// Gradients up to the Infinity Cache's size are left in it for what reads them next, which costs nothing here (600 rows
// of 128,256, 154 MB: 50 us, 49 with the non-temporal hint; 1,000 rows, 256 MB: 79 and 82); larger ones would only pass
// through it (1,200 rows: 104 and 98; 2,048: 172 and 166).
constexpr int64_t kKeptBytes = int64_t(256) << 20;

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

template <int DT, bool ENTROPY, bool KEEP>
__global__ __launch_bounds__(kThreads) void logprob_grad(GradArgs a) {
    using T = typename Elem<DT>::T;
    constexpr int kPer = Elem<DT>::kPer, kPart = kGradVectors * kThreads * kPer;
    const int64_t r = a.row0 + blockIdx.x / (uint32_t)a.parts;
    const int part = (int)(blockIdx.x % (uint32_t)a.parts);
    const T *row = static_cast<const T *>(a.logits) + r * a.ld;
    T *out = static_cast<T *>(a.out) + r * a.out_ld;
    const int32_t id = a.ids == nullptr ? -1 : a.ids[r];
    const bool given = id >= 0 && id < a.v;
    const float g = given && a.g != nullptr ? a.g[r] : 0.0f;
    const float h = ENTROPY ? a.h[r] : 0.0f;
    const float m = a.stats[2 * r], log_sum = a.stats[2 * r + 1];
    const int x0 = part * kPart - lead_of<DT>(out, a.v), x1 = part + 1 == a.parts ? a.v : x0 + kPart;
    if ((g == 0.0f && h == 0.0f) || m == -INFINITY) {
        const uint32_t none[kGradVectors][4] = {};
        for (int x = x0; x < x1; x += kPart) store_chunk<DT, kGradVectors, kThreads, KEEP>(out, a.v, x, none);
        return;
    }
    const float beta = scale_of(a.inv_temp, r), c2 = beta * kLog2e, l2 = log_sum * kLog2e;
    const float ent = ENTROPY ? a.entropy[r] : 0.0f;
    // d = p (first + second t), t = lp / ln 2 held above -200 (p is 0 there); NaN statistics make it NaN
    const float first = -beta * (g + h * ent) + (log_sum - log_sum), second = ENTROPY ? -beta * h * (float)kLn2 : 0.0f;
    for_chunks<DT, kGradVectors, kThreads, true, false, false, 1>(row, a.v, x0, x1, [] {}, [&](uint32_t(&w)[kGradVectors][4], int x_chunk) {
#pragma unroll
        for (int i = 0; i < kGradVectors; ++i) {
            const int x = vector_at<DT, kThreads>(x_chunk, i);
            float d[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const float t = fmaxf((value<DT>(w[i], j) - m) * c2 - l2, kLowest);
                const float p = __builtin_amdgcn_exp2f(t);
                d[j] = p * (ENTROPY ? fmaf(second, t, first) : first);
            }
            if (given && id >= x && id < x + kPer) {  // the token itself: 1 - p from its log probability
                float y = 0.0f;
#pragma unroll
                for (int j = 0; j < kPer; ++j) y = id == x + j ? value<DT>(w[i], j) : y;
                const float lp = y == y ? (y - m) * beta - log_sum : -INFINITY, rest = -expm1f(lp);
                const float own = beta * (g * rest - (ENTROPY ? h * expf(lp) * (fmaxf(lp, kLowest) + ent) : 0.0f)) + (log_sum - log_sum);
#pragma unroll
                for (int j = 0; j < kPer; ++j) d[j] = id == x + j ? own : d[j];
            }
            encode_vector<DT>(d, w[i]);
        }
        store_chunk<DT, kGradVectors, kThreads, KEEP>(out, a.v, x_chunk, w);
    });
}

template <int DT, bool ENTROPY>
void launch_grad(const GradArgs &a, bool keep, unsigned grid, hipStream_t stream) {
    if (keep) logprob_grad<DT, ENTROPY, true><<<grid, kThreads, 0, stream>>>(a);
    else logprob_grad<DT, ENTROPY, false><<<grid, kThreads, 0, stream>>>(a);
}

template <int DT>
void launch_grad(const GradArgs &a, bool keep, unsigned grid, hipStream_t stream) {
    if (a.h != nullptr) launch_grad<DT, true>(a, keep, grid, stream);
    else launch_grad<DT, false>(a, keep, grid, stream);
}

}  // namespace

size_t logprobs_workspace_used(int32_t n_rows, int32_t v, int dtype, int n_top) { return plan_of(n_rows, v, dtype, n_top).total; }

// The most that any number of rows up to n_rows uses: more rows are split less, and from few_rows on not at all.
size_t logprobs_workspace_bytes(int32_t n_rows, int32_t v, int dtype, int n_top) {
    const int64_t few = few_rows((int64_t)v * element_bytes(dtype));
    size_t most = 0;
    for (int64_t n = 1; n <= n_rows && n < few; ++n) {
        const size_t used = plan_of(n, v, dtype, n_top).total;
        most = used > most ? used : most;
    }
    return most;
}

int launch_logprobs(const LogprobsArgs &l, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const Plan p = plan_of(l.n_rows, l.v, l.dtype, l.n_top);
    if (p.total > 0 && (workspace == nullptr || workspace_bytes < p.total)) return TT_EWORKSPACE;
    if (p.total > 0 && reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return TT_EINVAL;
    RowArgs a;
    a.logits = l.logits;
    a.ld = l.ld;
    a.v = l.v;
    a.dtype = l.dtype;
    a.parts = p.parts;
    a.part_width = p.part_width;
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
        if (l.dtype == TT_BF16) launch_rows<TT_BF16>(a, p.threads, n, stream);
        else if (l.dtype == TT_F16) launch_rows<TT_F16>(a, p.threads, n, stream);
        else launch_rows<TT_F32>(a, p.threads, n, stream);
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
    const bool keep = (int64_t)l.n_rows * l.v * element_bytes(l.dtype) <= kKeptBytes;
    const int64_t most = kMaxGrid / a.parts;
    for (int64_t row0 = 0; row0 < l.n_rows; row0 += most) {
        const int64_t n = l.n_rows - row0 < most ? l.n_rows - row0 : most;
        const unsigned grid = (unsigned)(n * a.parts);
        a.row0 = row0;
        if (l.dtype == TT_BF16) launch_grad<TT_BF16>(a, keep, grid, stream);
        else if (l.dtype == TT_F16) launch_grad<TT_F16>(a, keep, grid, stream);
        else launch_grad<TT_F32>(a, keep, grid, stream);
        if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
    }
    return TT_OK;
}

}  // namespace tt
