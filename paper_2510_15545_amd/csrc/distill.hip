// Distillation from a teacher's top tokens: the loss of every row and, if wanted, its gradient, from
// rows of bf16, fp16 or fp32 student logits on gfx950.
//
// Row i lists the teacher's tokens (through the id map, if the vocabularies differ) with log
// probabilities a_k; entries outside the student's vocabulary or of probability 0 are left out.
//   w_k = exp(a_k) (with the tail) or exp(a_k) / sum over the entries kept;  P_j = sum of w_k with id_k = j
//   r = max(0, 1 - sum P) (with the tail, if an unlisted token has a logit above -inf) or 0
//   Q = softmax(beta x),  R = sum of Q over the unlisted tokens,  u_j = Q_j / R for them
//   loss = sum P_j (ln P_j - ln Q_j) + r (ln r - ln R)
//   dloss/dx_j = beta (T Q_j - P_j) for listed j, beta (T R - r) u_j otherwise, T = sum P + r
// The unlisted tokens' sums are formed without the listed ones (a difference of the two totals would
// lose R where the student, too, puts nearly all its mass on the list), and so is their softmax u.
//
// list_parts: a workgroup holds a part of a row in registers, takes the listed tokens out by a bitmap
// in LDS and forms the rest's largest value and sum.  list_rows: a workgroup per row joins them,
// gathers the listed logits, merges equal tokens and forms the loss in fp64, and what the gradient
// needs: the unlisted softmax's reference and factor, the listed tokens' gradients.  list_grad: reads
// the row again and writes its gradient.  The three run for groups of rows small enough that the
// second reading comes out of the Infinity Cache.
#include "rows.h"

namespace tt {
namespace {

using namespace rows;

constexpr int kMaxTop = 128;
constexpr int kWaves = kThreads / kWave;
constexpr int kListThreads = 128;  // one thread an entry
constexpr int64_t kMaxGrid = int64_t(1) << 18;
constexpr size_t kCachedBytes = size_t(96) << 20;  // logits of one group of rows, with the gradient

struct Entry {
    int32_t id;  // -1: none (left out, or an earlier entry has the token)
    float grad;
};

// What the gradient of a row's unlisted tokens needs: factor * 2^((x - m) c2 - shift).
struct RowGrad {
    float m, c2, shift, factor;
};

struct ListArgs {
    const void *logits;
    int64_t ld, row0;
    int v, dtype, parts, n_top, tail;
    const float *inv_temp;
    const int32_t *ids;
    const float *logprobs;
    const int32_t *id_map;
    int n_map;
    float2 *sums;  // per part: m, s of the unlisted tokens
    float *loss;
    const float *grad_loss;
    RowGrad *row_grad;
    Entry *entries;
    void *out;
    int64_t out_ld;
};

// Student token of list entry k, -1 if it is left out.
__device__ __forceinline__ int32_t entry_id(const ListArgs &a, int64_t row, int k) {
    const float lp = a.logprobs[row * a.n_top + k];
    int32_t id = a.ids[row * a.n_top + k];
    if (!(lp > -INFINITY)) return -1;  // probability 0, NaN
    if (a.id_map != nullptr) {
        if (id < 0 || id >= a.n_map) return -1;
        id = a.id_map[id];
    }
    return id >= 0 && id < a.v ? id : -1;
}

template <int DT, int NV>
__global__ __launch_bounds__(kThreads) void list_parts(ListArgs a) {
    using T = typename Elem<DT>::T;
    constexpr int kPer = Elem<DT>::kPer;
    constexpr int kPart = NV * kThreads * kPer;
    __shared__ uint32_t sh_bits[kPart / 32];
    __shared__ Sum sh_sum[kWaves];
    pass_over_nans();
    const int64_t r = blockIdx.x / (uint32_t)a.parts, row_i = a.row0 + r;
    const int part = blockIdx.x % (uint32_t)a.parts, x_part = part * kPart;
    const T *row = static_cast<const T *>(a.logits) + row_i * a.ld;
    uint32_t w[NV][4];
    load_part<DT, NV, kThreads>(row, a.v, x_part, w);
    for (int i = threadIdx.x; i < kPart / 32; i += kThreads) sh_bits[i] = 0;
    const float c2 = scale_of(a.inv_temp, row_i) * kLog2e;
    __syncthreads();
    if ((int)threadIdx.x < a.n_top) {
        const int at = entry_id(a, row_i, threadIdx.x) - x_part;
        if (at >= 0 && at < kPart) atomicOr(&sh_bits[at / 32], 1u << (at % 32));
    }
    __syncthreads();
    float tm = -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = vector_at<DT, kThreads>(0, i);
        const uint32_t hit = (sh_bits[at / 32] >> (at % 32)) & ((1u << kPer) - 1u);
        if (hit != 0) {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if ((hit >> j) & 1u) set_bits<DT>(w[i], j, Elem<DT>::kNone);
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) tm = fmaxf(tm, value<DT>(w[i], j));
    }
    const Sum ws = wave_sums<DT, NV, false>(w, tm, c2);
    if (threadIdx.x % kWave == 0) sh_sum[threadIdx.x / kWave] = ws;
    __syncthreads();
    if (threadIdx.x == 0) {
        Sum s = sh_sum[0];
#pragma unroll
        for (int u = 1; u < kWaves; ++u) s = join(s, sh_sum[u], c2);
        a.sums[(size_t)r * a.parts + part] = make_float2(s.m, s.s);
    }
}

// Reductions over the two waves of list_rows, the result in every thread.
__device__ __forceinline__ float pair_max(float x, float *sh) {
    x = wave_max(x);
    __syncthreads();
    if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = x;
    __syncthreads();
    return fmaxf(sh[0], sh[1]);
}
__device__ __forceinline__ double pair_sum(double x, double *sh) {
    x = wave_sum(x);
    __syncthreads();
    if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = x;
    __syncthreads();
    return sh[0] + sh[1];
}

template <bool GRAD>
__global__ __launch_bounds__(kListThreads) void list_rows(ListArgs a) {
    __shared__ float sh_f[2];
    __shared__ double sh_d[2], sh_w[kMaxTop];
    __shared__ int32_t sh_id[kMaxTop];
    const int64_t r = blockIdx.x, row = a.row0 + r;
    const int k = threadIdx.x;
    const float2 *sums = a.sums + (size_t)r * a.parts;
    const double beta = scale_of(a.inv_temp, row);
    const bool sound = beta > 0.0 && beta < INFINITY;
    // the unlisted tokens: largest logit m_out, sum s_out relative to it
    float m_out = -INFINITY;
    for (int p = k; p < a.parts; p += kListThreads) m_out = fmaxf(m_out, sums[p].x);
    m_out = pair_max(m_out, sh_f);
    double s_out = 0.0;
    for (int p = k; p < a.parts; p += kListThreads) {
        const float2 q = sums[p];
        if (q.y > 0.0f) s_out += q.y * exp(((double)q.x - (double)m_out) * beta);
    }
    s_out = pair_sum(s_out, sh_d);
    // the list
    const int32_t id = k < a.n_top ? entry_id(a, row, k) : -1;
    const float lp = id >= 0 ? a.logprobs[row * a.n_top + k] : -INFINITY;
    const float lp_most = pair_max(lp, sh_f);
    double w = id >= 0 ? exp(a.tail ? (double)lp : (double)lp - (double)lp_most) : 0.0;
    if (!a.tail) {
        const double all = pair_sum(w, sh_d);
        w = id >= 0 ? w / all : 0.0;
    }
    sh_id[k] = id;
    sh_w[k] = w;
    __syncthreads();
    bool first = id >= 0;  // the entry that stands for its token
    double mass = 0.0;     // the teacher's probability of that token
    for (int i = 0; i < a.n_top; ++i) {
        if (sh_id[i] == id) {
            mass += sh_w[i];
            first = first && i >= k;
        }
    }
    if (!first) mass = 0.0;
    float x = -INFINITY;
    if (first) {
        const int64_t at = row * a.ld;
        const void *base = a.dtype == TT_F32 ? (const void *)(static_cast<const float *>(a.logits) + at)
                                             : (const void *)(static_cast<const uint16_t *>(a.logits) + at);
        x = load_logit(base, a.dtype, id);
    }
    const float m = fmaxf(m_out, pair_max(x, sh_f));
    const double t = ((double)x - (double)m) * beta;  // -inf (or NaN, in a row without a finite logit) where x is
    const double e = x > -INFINITY ? exp(t) : 0.0;
    const double t_out = ((double)m_out - (double)m) * beta;  // ln of the unlisted sum's scale
    const double s_in = pair_sum(e, sh_d);
    const double s = s_in + (s_out > 0.0 ? s_out * exp(t_out) : 0.0);
    const double listed = pair_sum(mass, sh_d);
    const bool any = pair_sum(first ? 1.0 : 0.0, sh_d) > 0.0;
    const double rest = a.tail && s_out > 0.0 ? fmax(0.0, 1.0 - listed) : 0.0;
    // nothing listed, or no finite logit: 0; a logit or list value of +inf, or an unsound temperature: NaN
    const bool bad = !sound || m == INFINITY || lp_most == INFINITY;
    const bool zero = !bad && (!any || m == -INFINITY);
    const double log_s = log(s);
    double term = 0.0;
    if (mass > 0.0) term = x > -INFINITY ? mass * (log(mass) - (t - log_s)) : INFINITY;
    double loss = pair_sum(term, sh_d);
    const double log_rest = t_out + log(s_out) - log_s;  // ln R
    if (rest > 0.0) loss += rest * (log(rest) - log_rest);
    if (bad) loss = NAN;
    if (zero) loss = 0.0;
    if (k == 0) a.loss[row] = (float)loss;
    if constexpr (GRAD) {
        const double g = a.grad_loss[row];
        const double scale = g == 0.0 || zero ? 0.0 : (bad ? NAN : g * beta), total = listed + rest;
        if (k < a.n_top) {
            Entry out;
            out.id = first ? id : -1;
            out.grad = scale == 0.0 ? 0.0f : (float)(scale * (total * (e / s) - mass));
            a.entries[(size_t)r * a.n_top + k] = out;
        }
        if (k == 0) {
            RowGrad q;
            q.m = m_out;
            q.c2 = (float)beta * kLog2e;
            q.shift = s_out > 0.0 ? (float)log2(s_out) : 0.0f;
            const double share = s_out > 0.0 ? exp(log_rest) : 0.0;
            q.factor = scale == 0.0 ? 0.0f : (float)(scale * (total * share - rest));
            a.row_grad[r] = q;
        }
    }
}

constexpr int kGradVectors = 4;

template <int DT>
__global__ __launch_bounds__(kThreads) void list_grad(ListArgs a, int parts) {
    using T = typename Elem<DT>::T;
    constexpr int kPer = Elem<DT>::kPer;
    constexpr int kPart = kGradVectors * kThreads * kPer;
    const int64_t r = blockIdx.x / (uint32_t)parts, row_i = a.row0 + r;
    const int x_part = (int)(blockIdx.x % (uint32_t)parts) * kPart;
    const T *row = static_cast<const T *>(a.logits) + row_i * a.ld;
    T *out = static_cast<T *>(a.out) + row_i * a.out_ld;
    const RowGrad q = a.row_grad[r];
    Entry mine = {-1, 0.0f};
    if ((int)threadIdx.x < a.n_top) mine = a.entries[(size_t)r * a.n_top + threadIdx.x];
    float d[kPer];
    if (q.factor == 0.0f) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) d[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < kGradVectors; ++i) store_vector<DT>(out, vector_at<DT, kThreads>(x_part, i), a.v, d);
    } else {
        uint32_t w[kGradVectors][4];
        load_part<DT, kGradVectors, kThreads>(row, a.v, x_part, w);
#pragma unroll
        for (int i = 0; i < kGradVectors; ++i) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const float t = fmaxf((value<DT>(w[i], j) - q.m) * q.c2 - q.shift, kLowest);
                d[j] = q.factor * __builtin_amdgcn_exp2f(t);
            }
            store_vector<DT>(out, vector_at<DT, kThreads>(x_part, i), a.v, d);
        }
    }
    // the listed tokens over what was just written: after the workgroup's stores have been made
    __threadfence_block();
    __syncthreads();
    if (mine.id >= x_part && mine.id < x_part + kPart) out[mine.id] = (T)encode<DT>(mine.grad);
}

struct Plan {
    Split split;
    int64_t rows;
    size_t row_grad, entries, total;
};

Plan plan_of(int64_t n_rows, int32_t v, int dtype, int n_top, bool grad) {
    Plan p;
    p.split = split_rows(n_rows, v, dtype);
    if (p.split.threads != kThreads) p.split = {kThreads, kWideVectors, (int)((v + 8 * 256 * elements_per_vector(dtype) - 1) / (8 * 256 * elements_per_vector(dtype)))};
    int64_t most = kMaxGrid / p.split.parts;
    if (grad) {
        const int64_t per = (int64_t)kGradVectors * kThreads * elements_per_vector(dtype);
        const int64_t grid = kMaxGrid / ((v + per - 1) / per);
        const int64_t cached = (int64_t)(kCachedBytes / ((size_t)v * element_bytes(dtype)));
        most = most < grid ? most : grid;
        most = most < cached ? most : cached;
    }
    if (most < 1) most = 1;
    const int64_t groups = (n_rows + most - 1) / most;
    p.rows = groups == 0 ? 0 : (n_rows + groups - 1) / groups;
    p.row_grad = round256((size_t)p.rows * p.split.parts * sizeof(float2));
    p.entries = p.row_grad + (grad ? round256((size_t)p.rows * sizeof(RowGrad)) : 0);
    p.total = p.entries + (grad ? (size_t)p.rows * n_top * sizeof(Entry) : 0);
    return p;
}

template <int DT>
void launch_list_parts(const ListArgs &a, int vectors, unsigned grid, hipStream_t stream) {
    if (vectors == kWideVectors) list_parts<DT, kWideVectors><<<grid, kThreads, 0, stream>>>(a);
    else list_parts<DT, kNarrowVectors><<<grid, kThreads, 0, stream>>>(a);
}

}  // namespace

size_t distill_workspace_bytes(int32_t n_rows, int32_t v, int dtype, int n_top, bool grad) {
    return plan_of(n_rows, v, dtype, n_top, grad).total;
}

int launch_distill(const DistillArgs &l, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const bool grad = l.dlogits != nullptr;
    const Plan p = plan_of(l.n_rows, l.v, l.dtype, l.n_top, grad);
    if (workspace == nullptr || workspace_bytes < p.total) return TT_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return TT_EINVAL;
    char *ws = static_cast<char *>(workspace);
    ListArgs a;
    a.logits = l.logits;
    a.ld = l.ld;
    a.v = l.v;
    a.dtype = l.dtype;
    a.parts = p.split.parts;
    a.n_top = l.n_top;
    a.tail = l.tail;
    a.inv_temp = l.inv_temp;
    a.ids = l.top_ids;
    a.logprobs = l.top_logprobs;
    a.id_map = l.id_map;
    a.n_map = l.n_map;
    a.sums = reinterpret_cast<float2 *>(ws);
    a.loss = l.loss;
    a.grad_loss = l.grad_loss;
    a.row_grad = reinterpret_cast<RowGrad *>(ws + p.row_grad);
    a.entries = reinterpret_cast<Entry *>(ws + p.entries);
    a.out = l.dlogits;
    a.out_ld = l.out_ld;
    const int64_t per = (int64_t)kGradVectors * kThreads * elements_per_vector(l.dtype);
    const int grad_parts = (int)((l.v + per - 1) / per);
    for (int64_t row0 = 0; row0 < l.n_rows; row0 += p.rows) {
        const int64_t n = l.n_rows - row0 < p.rows ? l.n_rows - row0 : p.rows;
        a.row0 = row0;
        const unsigned grid = (unsigned)(n * a.parts);
        if (l.dtype == TT_BF16) launch_list_parts<TT_BF16>(a, p.split.vectors, grid, stream);
        else if (l.dtype == TT_F16) launch_list_parts<TT_F16>(a, p.split.vectors, grid, stream);
        else launch_list_parts<TT_F32>(a, p.split.vectors, grid, stream);
        if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
        if (grad) list_rows<true><<<(unsigned)n, kListThreads, 0, stream>>>(a);
        else list_rows<false><<<(unsigned)n, kListThreads, 0, stream>>>(a);
        if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
        if (!grad) continue;
        const unsigned grad_grid = (unsigned)(n * grad_parts);
        if (l.dtype == TT_BF16) list_grad<TT_BF16><<<grad_grid, kThreads, 0, stream>>>(a, grad_parts);
        else if (l.dtype == TT_F16) list_grad<TT_F16><<<grad_grid, kThreads, 0, stream>>>(a, grad_parts);
        else list_grad<TT_F32><<<grad_grid, kThreads, 0, stream>>>(a, grad_parts);
        if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
    }
    return TT_OK;
}

}  // namespace tt
