// Log probabilities of given tokens with log-sum-exp, entropy and top alternatives, and their
// gradient, from rows of bf16, fp16 or fp32 logits on gfx950.
//
// With x the row's logits (NaN counts as minus infinity), beta the row's inverse temperature:
//   M = max x,  S = sum exp(beta (x - M)),  L = ln S,  lse = beta M + L
//   lp_j = beta (x_j - M) - L,  p_j = exp(lp_j),  H = -sum p_j lp_j = L - sum beta (x_j - M) p_j
//   alternatives: the largest x, ties by the lower index, minus infinity never listed
//   d_j = beta (g ([j = id] - p_j) - h p_j (lp_j + H)), upstream gradients g of lp_id and h of H
//
// One pass over the row.  row_parts: a workgroup holds a part of a row in registers, forms its
// largest value first and then its sums (base 2, v_exp_f32), and, for the alternatives, a lower
// bound of its k-th largest value: the k-th largest of its 256 lanes' largest values, found by 16
// ballots on the upper 16 bits of their order keys (k distinct elements reach it, so the k largest
// do).  Elements that reach the bound go to the workspace as 64-bit keys (value, then lower index),
// about 1.2 to 2 k of them.  row_finish: a workgroup per row joins the parts' sums in fp64 and
// selects the k largest keys the same way, ordered by counting.
#include "rows.h"

namespace tt {
namespace {

using namespace rows;

constexpr int kMaxTop = 128;
constexpr int kSelect = 1024;                        // keys that row_finish orders in LDS
constexpr size_t kMaxKeyBytes = size_t(128) << 20;   // workspace: rows are taken in groups beyond
constexpr int64_t kMaxGrid = int64_t(1) << 18;       // workgroups of one launch

// Keys that a part may hand over: 8 k where fewer than k lanes hold a finite value (each lane then
// 8 elements a vector or fewer), ties otherwise; a part with more selects its k largest exactly.
inline int part_capacity(int n_top) { return 8 * n_top + 64; }

struct PartArgs {
    const void *logits;
    int64_t ld, row0;  // first row of this launch
    int v, parts, n_top, capacity;
    const float *inv_temp;
    float4 *sums;     // per part: m, s, e, number of keys (bits)
    uint64_t *keys;   // per part: capacity
};

// Largest bound P on 16-bit keys that at least k of the 256 in LDS reach (each wave for itself).
__device__ __forceinline__ uint32_t kth_key16(const uint32_t *sh_keys, int k) {
    const int lane = threadIdx.x % kWave;
    uint32_t q[kWaves];
#pragma unroll
    for (int u = 0; u < kWaves; ++u) q[u] = sh_keys[u * kWave + lane];
    uint32_t p = 0;
#pragma unroll
    for (int b = 15; b >= 0; --b) {
        const uint32_t c = p | (1u << b);
        int n = 0;
#pragma unroll
        for (int u = 0; u < kWaves; ++u) n += __popcll(__ballot(q[u] >= c));
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

// Sum over the workgroup of a count, through a zeroed LDS slot of its own.
__device__ __forceinline__ int block_count(int n, int *slot) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) n += __shfl_xor(n, d);
    if (threadIdx.x % kWave == 0) atomicAdd(slot, n);
    __syncthreads();
    return *slot;
}

// The part's k largest elements exactly, where more than the capacity reach the bound (many equal
// values): the k-th largest value by binary search on its order key, then the last index among the
// elements equal to it.  At least k elements are finite.  54 counts, each over the registers.
template <int DT, int NV>
__device__ __forceinline__ void select_exactly(const uint32_t (&w)[NV][4], int x_part, int k, uint64_t *keys, int *sh_slots,
                                            int *sh_count) {
    constexpr int kPer = Elem<DT>::kPer;
    for (int i = threadIdx.x; i < 64; i += kThreads) sh_slots[i] = 0;
    if (threadIdx.x == 0) *sh_count = 0;
    __syncthreads();
    int slot = 0;
    uint32_t kth = 0;
    for (int b = 31; b >= 0; --b) {
        const uint32_t c = kth | (1u << b);
        int n = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const float x = value<DT>(w[i], j);
                n += (x > -INFINITY && order_key(x) >= c) ? 1 : 0;
            }
        if (block_count(n, &sh_slots[slot++]) >= k) kth = c;
    }
    int above = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float x = value<DT>(w[i], j);
            above += (x > -INFINITY && order_key(x) > kth) ? 1 : 0;
        }
    const int need = k - block_count(above, &sh_slots[slot++]);
    int last = 0;  // the largest index bound with fewer than `need` equal elements below it
    for (int b = 15; b >= 0; --b) {  // indices relative to the part: below 2^15
        const int c = last | (1 << b);
        int n = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const float x = value<DT>(w[i], j);
                n += (x > -INFINITY && order_key(x) == kth && vector_at<DT>(0, i) + j < c) ? 1 : 0;
            }
        if (block_count(n, &sh_slots[slot++]) < need) last = c;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float x = value<DT>(w[i], j);
            if (!(x > -INFINITY)) continue;
            const uint32_t o = order_key(x);
            const int at = vector_at<DT>(0, i) + j;
            if (o > kth || (o == kth && at <= last)) keys[atomicAdd(sh_count, 1)] = full_key(x, x_part + at);
        }
    __syncthreads();
}

template <int DT, int NV, bool TOP, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void row_parts(PartArgs a) {
    using T = typename Elem<DT>::T;
    constexpr int kPer = Elem<DT>::kPer;
    __shared__ Sum sh_sum[kWaves];
    __shared__ uint32_t sh_keys[TOP ? kThreads : 1];
    __shared__ int sh_count, sh_slots[TOP ? 64 : 1];
    pass_over_nans();
    const int64_t r = blockIdx.x / (uint32_t)a.parts;
    const int part = blockIdx.x % (uint32_t)a.parts;
    const int x_part = part * NV * kThreads * kPer;
    const T *row = static_cast<const T *>(a.logits) + (a.row0 + r) * a.ld;
    uint32_t w[NV][4];
    load_part<DT, NV>(row, a.v, x_part, w);
    const float c2 = scale_of(a.inv_temp, a.row0 + r) * kLog2e;
    float vm[NV], tm = -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        vm[i] = -INFINITY;
#pragma unroll
        for (int j = 0; j < kPer; ++j) vm[i] = fmaxf(vm[i], value<DT>(w[i], j));
        tm = fmaxf(tm, vm[i]);
    }
    if constexpr (TOP) {
        sh_keys[threadIdx.x] = order_key(tm) >> 16;
        if (threadIdx.x == 0) sh_count = 0;
    }
    const Sum ws = wave_sums<DT, NV, ENTROPY>(w, tm, c2);
    if (threadIdx.x % kWave == 0) sh_sum[threadIdx.x / kWave] = ws;
    __syncthreads();
    const size_t slot = (size_t)r * a.parts + part;
    int count = 0;
    if constexpr (TOP) {
        const float bound = bound_value(kth_key16(sh_keys, a.n_top));
        uint64_t *keys = a.keys + slot * a.capacity;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (vm[i] >= bound) {
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const float x = value<DT>(w[i], j);
                    if (x >= bound) {
                        const int at = atomicAdd(&sh_count, 1);
                        if (at < a.capacity) keys[at] = full_key(x, vector_at<DT>(x_part, i) + j);
                    }
                }
            }
        }
        __syncthreads();
        count = sh_count;
        if (count > a.capacity) {
            __syncthreads();
            select_exactly<DT, NV>(w, x_part, a.n_top, keys, sh_slots, &sh_count);
            count = a.n_top;
        }
    }
    if (threadIdx.x == 0) {
        Sum s = sh_sum[0];
#pragma unroll
        for (int u = 1; u < kWaves; ++u) s = join(s, sh_sum[u], c2);
        a.sums[slot] = make_float4(s.m, s.s, s.e, __int_as_float(count));
    }
}

struct FinishArgs {
    const void *logits;
    int64_t ld, row0;
    int v, dtype, parts, n_top, capacity;
    const float *inv_temp;
    const int32_t *ids;
    const float4 *sums;
    const uint64_t *keys;
    float *logprob, *lse, *entropy, *stats;
    int32_t *top_ids;
    float *top_logprobs;
};

// The k largest of a row's keys, descending, in sh_sel[0 .. min(k, keys)); returns their number.
__device__ int select_keys(const FinishArgs &a, const float4 *sums, const uint64_t *keys, uint64_t *sh_sel, uint32_t *sh_keys,
                           int *sh_slots, int *sh_count, uint64_t *sh_out) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    uint32_t most = 0;
    int mine = 0;
    for (int p = wave; p < a.parts; p += kWaves) {
        const int n = __float_as_int(sums[p].w);
        for (int i = lane; i < n; i += kWave) {
            const uint32_t o = (uint32_t)(keys[(size_t)p * a.capacity + i] >> 32);
            most = o > most ? o : most;
            ++mine;
        }
    }
    sh_keys[threadIdx.x] = most >> 16;
    if (threadIdx.x < 64) sh_slots[threadIdx.x] = 0;
    if (threadIdx.x == 64) *sh_count = 0;
    __syncthreads();
    const int total = block_count(mine, &sh_slots[0]);
    uint64_t from = total <= kWave ? 0 : (uint64_t)(kth_key16(sh_keys, a.n_top) << 16) << 32;
    for (int round = 0; round < 2; ++round) {
        for (int p = wave; p < a.parts; p += kWaves) {
            const int n = __float_as_int(sums[p].w);
            for (int i = lane; i < n; i += kWave) {
                const uint64_t key = keys[(size_t)p * a.capacity + i];
                if (key >= from) {
                    const int at = atomicAdd(sh_count, 1);
                    if (at < kSelect) sh_sel[at] = key;
                }
            }
        }
        __syncthreads();
        if (*sh_count <= kSelect) break;
        // many equal values: the k-th largest key itself (keys are distinct, so k reach it)
        uint64_t kth = 0;
        for (int b = 63; b >= 0; --b) {
            const uint64_t c = kth | (1ull << b);
            int n = 0;
            for (int p = wave; p < a.parts; p += kWaves) {
                const int m = __float_as_int(sums[p].w);
                for (int i = lane; i < m; i += kWave) n += keys[(size_t)p * a.capacity + i] >= c ? 1 : 0;
            }
            __syncthreads();
            if (threadIdx.x == 0) sh_slots[1] = 0;
            __syncthreads();
            if (block_count(n, &sh_slots[1]) >= a.n_top) kth = c;
        }
        from = kth;
        __syncthreads();
        if (threadIdx.x == 0) *sh_count = 0;
        __syncthreads();
    }
    const int c = *sh_count;
    for (int i = threadIdx.x; i < c; i += kThreads) {
        const uint64_t key = sh_sel[i];
        int rank = 0;
        for (int j = 0; j < c; ++j) rank += sh_sel[j] > key ? 1 : 0;
        if (rank < a.n_top) sh_out[rank] = key;
    }
    __syncthreads();
    return c < a.n_top ? c : a.n_top;
}

template <bool TOP>
__global__ __launch_bounds__(kThreads) void row_finish(FinishArgs a) {
    __shared__ float sh_m[kWaves];
    __shared__ double sh_s[kWaves], sh_e[kWaves];
    __shared__ uint64_t sh_sel[TOP ? kSelect : 1], sh_out[TOP ? kMaxTop : 1];
    __shared__ uint32_t sh_keys[TOP ? kThreads : 1];
    __shared__ int sh_slots[64], sh_count;
    const int64_t r = blockIdx.x, row = a.row0 + r;
    const float4 *sums = a.sums + (size_t)r * a.parts;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const double beta = scale_of(a.inv_temp, row);
    const bool sound = beta > 0.0 && beta < INFINITY;
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
    s = sh_s[0] + sh_s[1] + sh_s[2] + sh_s[3];
    e = sh_e[0] + sh_e[1] + sh_e[2] + sh_e[3];
    // m = -inf: nothing is finite (s = 0); m = +inf or an unsound temperature: NaN
    const bool bad = !sound || m == INFINITY, empty = m == -INFINITY;
    const double log_sum = bad ? NAN : (empty ? 0.0 : log(s));
    if (threadIdx.x == 0) {
        if (a.stats != nullptr) {
            a.stats[2 * row] = bad ? NAN : m;
            a.stats[2 * row + 1] = (float)log_sum;
        }
        if (a.lse != nullptr) a.lse[row] = (float)(bad ? NAN : (double)m * beta + log_sum);
        if (a.entropy != nullptr) a.entropy[row] = (float)(bad ? NAN : (empty ? 0.0 : log_sum - e / s));
        if (a.logprob != nullptr) {
            const int32_t id = a.ids[row];
            double lp = NAN;
            if (!bad && id >= 0 && id < a.v) {
                const int64_t at = row * a.ld;
                const float x = load_logit(a.dtype == TT_F32 ? (const void *)(static_cast<const float *>(a.logits) + at)
                                                             : (const void *)(static_cast<const uint16_t *>(a.logits) + at),
                                           a.dtype, id);
                lp = x == -INFINITY ? -INFINITY : ((double)x - (double)m) * beta - log_sum;
            }
            a.logprob[row] = (float)lp;
        }
    }
    if constexpr (TOP) {
        const int n = select_keys(a, sums, a.keys + (size_t)r * a.parts * a.capacity, sh_sel, sh_keys, sh_slots, &sh_count, sh_out);
        for (int i = threadIdx.x; i < a.n_top; i += kThreads) {
            int32_t id = -1;
            double lp = bad ? NAN : -INFINITY;
            if (i < n && !bad) {
                id = (int32_t)(0xFFFFFFFFu - (uint32_t)sh_out[i]);
                lp = ((double)key_value((uint32_t)(sh_out[i] >> 32)) - (double)m) * beta - log_sum;
            }
            a.top_ids[row * a.n_top + i] = id;
            a.top_logprobs[row * a.n_top + i] = (float)lp;
        }
    }
}

struct Plan {
    Split split;
    int64_t rows;  // rows of one launch
    size_t sums, total;
};

Plan plan_of(int64_t n_rows, int32_t v, int dtype, int n_top) {
    Plan p;
    p.split = split_rows(n_rows, v, dtype);
    const size_t per_row = (size_t)p.split.parts * part_capacity(n_top) * sizeof(uint64_t);
    int64_t most = kMaxGrid / p.split.parts;
    if (n_top > 0 && (int64_t)(kMaxKeyBytes / per_row) < most) most = (int64_t)(kMaxKeyBytes / per_row);
    if (most < 1) most = 1;
    const int64_t groups = (n_rows + most - 1) / most;
    p.rows = groups == 0 ? 0 : (n_rows + groups - 1) / groups;
    p.sums = round256((size_t)p.rows * p.split.parts * sizeof(float4));
    p.total = p.sums + (n_top > 0 ? (size_t)p.rows * per_row : 0);
    return p;
}

template <int DT, int NV>
void launch_parts(const PartArgs &a, bool entropy, unsigned grid, hipStream_t stream) {
    if (a.n_top > 0) {
        if (entropy) row_parts<DT, NV, true, true><<<grid, kThreads, 0, stream>>>(a);
        else row_parts<DT, NV, true, false><<<grid, kThreads, 0, stream>>>(a);
    } else {
        if (entropy) row_parts<DT, NV, false, true><<<grid, kThreads, 0, stream>>>(a);
        else row_parts<DT, NV, false, false><<<grid, kThreads, 0, stream>>>(a);
    }
}

template <int DT>
void launch_parts(const PartArgs &a, int vectors, bool entropy, unsigned grid, hipStream_t stream) {
    if (vectors == kWideVectors) launch_parts<DT, kWideVectors>(a, entropy, grid, stream);
    else launch_parts<DT, kNarrowVectors>(a, entropy, grid, stream);
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
        for (int i = 0; i < kGradVectors; ++i) store_vector<DT>(out, vector_at<DT>(x_part, i), a.v, d);
        return;
    }
    const float beta = scale_of(a.inv_temp, r), c2 = beta * kLog2e, l2 = log_sum * kLog2e;
    const float ent = ENTROPY ? a.entropy[r] : 0.0f;
    // d = p (first + second t), t = lp / ln 2 held above -200 (p is 0 there); NaN statistics make it NaN
    const float first = -beta * (g + h * ent) + (log_sum - log_sum), second = ENTROPY ? -beta * h * (float)kLn2 : 0.0f;
    uint32_t w[kGradVectors][4];
    load_part<DT, kGradVectors>(row, a.v, x_part, w);
#pragma unroll
    for (int i = 0; i < kGradVectors; ++i) {
        const int x = vector_at<DT>(x_part, i);
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
    if (workspace == nullptr || workspace_bytes < p.total) return TT_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return TT_EINVAL;
    PartArgs a;
    a.logits = l.logits;
    a.ld = l.ld;
    a.v = l.v;
    a.parts = p.split.parts;
    a.n_top = l.n_top;
    a.capacity = part_capacity(l.n_top);
    a.inv_temp = l.inv_temp;
    a.sums = static_cast<float4 *>(workspace);
    a.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + p.sums);
    FinishArgs f;
    f.logits = l.logits;
    f.ld = l.ld;
    f.v = l.v;
    f.dtype = l.dtype;
    f.parts = a.parts;
    f.n_top = l.n_top;
    f.capacity = a.capacity;
    f.inv_temp = l.inv_temp;
    f.ids = l.ids;
    f.sums = a.sums;
    f.keys = a.keys;
    f.logprob = l.logprob;
    f.lse = l.lse;
    f.entropy = l.entropy;
    f.stats = l.stats;
    f.top_ids = l.top_ids;
    f.top_logprobs = l.top_logprobs;
    for (int64_t row0 = 0; row0 < l.n_rows; row0 += p.rows) {
        const int64_t n = l.n_rows - row0 < p.rows ? l.n_rows - row0 : p.rows;
        const unsigned grid = (unsigned)(n * a.parts);
        a.row0 = f.row0 = row0;
        const bool entropy = l.entropy != nullptr;
        if (l.dtype == TT_BF16) launch_parts<TT_BF16>(a, p.split.vectors, entropy, grid, stream);
        else if (l.dtype == TT_F16) launch_parts<TT_F16>(a, p.split.vectors, entropy, grid, stream);
        else launch_parts<TT_F32>(a, p.split.vectors, entropy, grid, stream);
        if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
        if (l.n_top > 0) row_finish<true><<<(unsigned)n, kThreads, 0, stream>>>(f);
        else row_finish<false><<<(unsigned)n, kThreads, 0, stream>>>(f);
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
