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
// list_whole: a workgroup per row.  It takes the listed tokens out by a bitmap in LDS and streams the row
// by chunks for the rest's largest value and sum; one wave merges equal tokens, gathers the listed
// logits (while the first loads are in flight) and forms the loss in fp64, and what the gradient needs:
// the unlisted softmax's reference and factor, the listed tokens' gradients; then the row is streamed
// again for its gradient.  512 rows at most are worked on at once (two workgroups a compute unit), so that the second
// reading comes out of the Infinity Cache where these fit (156 MB of rows of 151,936 bf16).  Wider ones take the same
// time a byte: 1,024 rows of 151,936 fp32, 311 MB at once, 290 us, 2,048 in bf16 289; 1,024 of 262,144 bf16 252.
// Where the rows are too few to fill the GPU they are split: list_parts forms the sums of parts (in fp32 within a
// workgroup), list_rows joins them and does the one wave's work, list_grad writes the gradient of parts.
//
// What bounds it: the loss alone reads at 5.1 TB/s with 512 rows of 151,936 bf16 (30.5 us; two workgroups a compute
// unit, whose start and end are 7 of them).  The gradient of 2,048 such rows takes 275 us: 4.5 TB/s of the 1.24 GB
// that HBM has to carry, where a large copy gets 5.1, and 6.8 TB/s of the 1.87 GB with the second reading, which
// HBM alone would not give.  Between the two readings a workgroup writes nothing, and both want an exponential
// an element (the VALU is busy 60% of the cycles).
#include "rows.h"

namespace tt {
namespace {

using namespace rows;

constexpr int kMaxTop = 128;
constexpr int kSlots = kMaxTop / kWave;  // list entries of a lane
constexpr int64_t kMaxGrid = int64_t(1) << 18;
constexpr int kChunkVectors = 4;  // of a thread, for a part of a row
constexpr int kMaxBits = 1 << 18;  // tokens of a bitmap: 32 KB

// What the gradient of a row's unlisted tokens needs: factor * 2^t, t = x c2 - shift <= 0 (m = 0), or
// (x - m) c2 - shift where x c2 may be so large that its own steps would show.
struct RowGrad {
    float m, c2, shift, factor;
};
constexpr double kNear = 0x1p14;

// A listed token and its gradient; id -1: none (left out, or an earlier entry has the token).
struct Entry {
    int32_t id;
    float grad;
};

struct ListArgs {
    const void *logits;
    int64_t ld, row0;
    int v, dtype, parts, part_width, n_top, tail;
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
__device__ __forceinline__ int32_t entry_id(const ListArgs &a, int64_t row, int k, float lp) {
    int32_t id = a.ids[row * a.n_top + k];
    if (a.id_map != nullptr) id = id >= 0 && id < a.n_map ? a.id_map[id] : -1;
    return id >= 0 && id < a.v && lp > -INFINITY ? id : -1;  // no entry of probability 0 or NaN
}

// A row's list as one wave holds it, kSlots entries a lane: entry u * 64 + lane.
struct List {
    int32_t id[kSlots];    // -1: left out, or an earlier entry has the token
    float x[kSlots];       // the token's logit
    double mass[kSlots];   // the teacher's probability of the token
    double log_mass[kSlots];
    double listed;         // sum of the masses
    float most;            // largest of the list's log probabilities
    bool any;
};

// Entry e of a value held as a list, for every lane (e is the same in all of them).
__device__ __forceinline__ int32_t entry_of(const int32_t (&x)[kSlots], int e) {
    return __builtin_amdgcn_readlane(e < kWave ? x[0] : x[1], e % kWave);
}
__device__ __forceinline__ double entry_of(const double (&x)[kSlots], int e) {
    const uint64_t b = __builtin_bit_cast(uint64_t, e < kWave ? x[0] : x[1]);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)b, e % kWave), hi = __builtin_amdgcn_readlane((uint32_t)(b >> 32), e % kWave);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
static_assert(kSlots == 2, "entry_of chooses between two slots");

// The list's tokens, log probabilities (-inf for an entry that is left out) and logits.
__device__ __forceinline__ void read_list(const ListArgs &a, int64_t row, List &q, float (&lp)[kSlots]) {
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
        const int k = u * kWave + lane;
        q.id[u] = -1;
        lp[u] = -INFINITY;
        if (k < a.n_top) {
            lp[u] = a.logprobs[row * a.n_top + k];
            q.id[u] = entry_id(a, row, k, lp[u]);
        }
        if (q.id[u] < 0) lp[u] = -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < kSlots; ++u)
        q.x[u] = q.id[u] >= 0 ? load_logit(row_at(a.logits, a.dtype, row * a.ld), a.dtype, q.id[u]) : -INFINITY;
}

// Whether a token is listed twice.
__device__ __forceinline__ bool repeats(const List &q, int n_top) {
    int same[kSlots] = {};
    for (int e = 0; e < n_top; ++e) {
        const int32_t id = entry_of(q.id, e);
#pragma unroll
        for (int u = 0; u < kSlots; ++u) same[u] += q.id[u] == id ? 1 : 0;
    }
    return __ballot((q.id[0] >= 0 && same[0] > 1) || (q.id[1] >= 0 && same[1] > 1)) != 0;
}

// The list's masses; equal tokens are merged into their first entry.
__device__ __forceinline__ void weigh_list(const ListArgs &a, List &q, const float (&lp)[kSlots], bool repeated) {
    const int lane = threadIdx.x % kWave;
    q.most = wave_max(fmaxf(lp[0], lp[1]));
    q.any = q.most > -INFINITY;
    double all = 0.0;
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
        q.log_mass[u] = a.tail ? (double)lp[u] : (double)lp[u] - (double)q.most;
        q.mass[u] = q.id[u] >= 0 ? exp(q.log_mass[u]) : 0.0;
        all += q.mass[u];
    }
    if (!a.tail) {
        all = wave_sum(all);
        const double log_all = log(all);
#pragma unroll
        for (int u = 0; u < kSlots; ++u) {
            q.mass[u] = q.id[u] >= 0 ? q.mass[u] / all : 0.0;
            q.log_mass[u] -= log_all;
        }
    }
    if (repeated) {
        double mass[kSlots] = {};
        int first[kSlots] = {kMaxTop, kMaxTop};
        for (int e = a.n_top - 1; e >= 0; --e) {
            const int32_t id = entry_of(q.id, e);
            const double w = entry_of(q.mass, e);
#pragma unroll
            for (int u = 0; u < kSlots; ++u) {
                if (q.id[u] == id) {
                    mass[u] += w;
                    first[u] = e;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kSlots; ++u) {
            if (q.id[u] < 0) continue;
            if (first[u] < u * kWave + lane) {
                q.id[u] = -1;
                q.x[u] = -INFINITY;
                q.mass[u] = 0.0;
            } else {
                q.mass[u] = mass[u];
                q.log_mass[u] = log(mass[u]);
            }
        }
    }
    q.listed = wave_sum(q.mass[0] + q.mass[1]);
}

// A row's loss (written by lane 0) and, with GRAD, what its gradient needs, from its list and its unlisted
// tokens' largest logit m_out and sum s_out relative to it.  One wave.
template <bool GRAD>
__device__ __forceinline__ RowGrad finish_row(const ListArgs &a, int64_t row, const List &q, float m_out, double s_out,
                                              double (&grad)[kSlots]) {
    const double beta = scale_of(a.inv_temp, row);
    const float m = fmaxf(m_out, wave_max(fmaxf(q.x[0], q.x[1])));
    double t[kSlots], e[kSlots];  // -inf (or NaN, in a row without a finite logit) and 0 where x is -inf
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
        t[u] = ((double)q.x[u] - (double)m) * beta;
        e[u] = q.x[u] > -INFINITY ? exp(t[u]) : 0.0;
    }
    const double t_out = ((double)m_out - (double)m) * beta;  // ln of the unlisted sum's scale
    const double s = wave_sum(e[0] + e[1]) + (s_out > 0.0 ? s_out * exp(t_out) : 0.0), log_s = log(s);
    const double rest = a.tail && s_out > 0.0 ? fmax(0.0, 1.0 - q.listed) : 0.0;
    // nothing listed, or no finite logit: 0; a logit or list value of +inf, or an unsound temperature: NaN
    const bool bad = !sound(beta) || m == INFINITY || q.most == INFINITY;
    const bool zero = !bad && (!q.any || m == -INFINITY);
    double loss = 0.0;
#pragma unroll
    for (int u = 0; u < kSlots; ++u)
        if (q.mass[u] > 0.0) loss += q.x[u] > -INFINITY ? q.mass[u] * (q.log_mass[u] - (t[u] - log_s)) : INFINITY;
    loss = wave_sum(loss);
    const double log_out = log(s_out), log_rest = t_out + log_out - log_s;  // ln R
    if (rest > 0.0) loss += rest * (log(rest) - log_rest);
    if (bad) loss = NAN;
    if (zero) loss = 0.0;
    if (threadIdx.x % kWave == 0) a.loss[row] = (float)loss;
    RowGrad r = {};
    if constexpr (GRAD) {
        const double g = a.grad_loss[row];
        const double scale = g == 0.0 || zero ? 0.0 : (bad ? NAN : g * beta), total = q.listed + rest;
#pragma unroll
        for (int u = 0; u < kSlots; ++u) grad[u] = scale == 0.0 ? 0.0 : scale * (total * (e[u] / s) - q.mass[u]);
        // u_j = 2^((x_j - m_out) c2 - log2 s_out); the exponent is kept one below, so that its power can be
        // held in [0, 1] (which makes a NaN 0), and what rounding its offset loses goes into the factor
        r.c2 = (float)beta * kLog2e;
        const double log2_out = s_out > 0.0 ? log_out * (1.0 / kLn2) : 0.0, offset = (double)m_out * (double)r.c2;
        const bool near = fabs(offset) <= kNear;
        r.m = near ? 0.0f : m_out;
        const double shift = log2_out + (near ? offset : 0.0);
        r.shift = (float)(shift + 1.0);
        const double factor = total * (s_out > 0.0 ? exp(log_rest) : 0.0) - rest;
        r.factor = scale == 0.0 ? 0.0f : (float)(scale * factor * exp2((double)r.shift - shift));
    }
    return r;
}

// Takes the listed tokens out of a chunk: bits of the part that starts at x_part.
template <int DT, int NV, int THREADS>
__device__ __forceinline__ void take_out(uint32_t (&w)[NV][4], const uint32_t *sh_bits, int x_chunk, int x_part) {
    constexpr int kPer = Elem<DT>::kPer;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = vector_at<DT, THREADS>(x_chunk - x_part, i);
        const uint32_t hit = (sh_bits[at / 32] >> (at % 32)) & ((1u << kPer) - 1u);
        if (hit != 0) {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if ((hit >> j) & 1u) set_bits<DT>(w[i], j, Elem<DT>::kNone);
        }
    }
}

// Words of a bitmap over `width` tokens, after a row's lead, that whole chunks may ask for.
template <int DT, int NV, int THREADS>
__host__ __device__ __forceinline__ int bitmap_words(int width) {
    constexpr int kChunk = NV * THREADS * Elem<DT>::kPer;
    return (width + kLead + kChunk - 1) / kChunk * (kChunk / 32);
}

// Gradients of the unlisted tokens of elements x0 .. x1 - 1, from what get() returns (called once the first loads
// are in flight); zeros where the factor is 0.
template <int DT, int NV, int THREADS, bool AHEAD, typename G>
__device__ __forceinline__ void write_grad(const ListArgs &a, int64_t row_i, int x0, int x1, G get) {
    using T = typename Elem<DT>::T;
    constexpr int kPer = Elem<DT>::kPer;
    const T *row = static_cast<const T *>(a.logits) + row_i * a.ld;
    T *out = static_cast<T *>(a.out) + row_i * a.out_ld;
    RowGrad q;
    for_chunks<DT, NV, THREADS, true, true, AHEAD, 1>(row, a.v, x0, x1, [&] { q = get(); }, [&](uint32_t(&w)[NV][4], int x) {
        auto form = [&](auto exponent) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float d[kPer];
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    d[j] = q.factor * fminf(fmaxf(__builtin_amdgcn_exp2f(exponent(value<DT>(w[i], j))), 0.0f), 1.0f);
                encode_vector<DT>(d, w[i]);
            }
        };
        if (q.m == 0.0f) form([&](float y) { return fmaf(y, q.c2, -q.shift); });
        else form([&](float y) { return (y - q.m) * q.c2 - q.shift; });
        // kept, they would displace logits that are yet to be read again (2,048 rows of 151,936: 371 us, not 301)
        store_chunk<DT, NV, THREADS, false>(out, a.v, x, w);
    });
}

template <int DT, int NV, int THREADS, bool GRAD>
__global__ __launch_bounds__(THREADS) void list_whole(ListArgs a) {
    using T = typename Elem<DT>::T;
    constexpr int kWaves = THREADS / kWave;
    extern __shared__ uint32_t sh_bits[];
    __shared__ Sum sh_sum[kWaves];
    __shared__ Entry sh_entry[kMaxTop];
    __shared__ RowGrad sh_grad;
    pass_over_nans();
    const int64_t row_i = a.row0 + blockIdx.x;
    const T *row = static_cast<const T *>(a.logits) + row_i * a.ld;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const float c2 = scale_of(a.inv_temp, row_i) * kLog2e;
    const int x0 = -lead_of<DT>(GRAD ? static_cast<const void *>(static_cast<T *>(a.out) + row_i * a.out_ld) : row, a.v);
    List list;
    Sum mine = {-INFINITY, 0.0f, 0.0f};
    auto read = [&] {
        for (int i = threadIdx.x; i < bitmap_words<DT, NV, THREADS>(a.v); i += THREADS) sh_bits[i] = 0;
        __syncthreads();
        float lp[kSlots];
        bool repeated = false;
        if (wave == 0) {
            read_list(a, row_i, list, lp);
#pragma unroll
            for (int u = 0; u < kSlots; ++u) {
                if (list.id[u] < 0) continue;
                const int at = list.id[u] - x0;
                const uint32_t bit = 1u << (at % 32);
                repeated = (atomicOr(&sh_bits[at / 32], bit) & bit) != 0 || repeated;
            }
        }
        __syncthreads();
        if (wave == 0) weigh_list(a, list, lp, __ballot(repeated) != 0);
    };
    for_chunks<DT, NV, THREADS, !GRAD, false, true, 1>(row, a.v, x0, a.v, read, [&](uint32_t(&w)[NV][4], int x) {
        float vm[NV];
        take_out<DT, NV, THREADS>(w, sh_bits, x, x0);
        add_chunk<DT, NV, false>(w, c2, mine, vm);
    });
    mine = wave_join<false>(mine, c2);
    if (lane == 0) sh_sum[wave] = mine;
    auto finish = [&] {
        __syncthreads();
        if (wave == 0) {
            const Sum q = lane < kWaves ? sh_sum[lane] : Sum{-INFINITY, 0.0f, 0.0f};
            const float m_out = wave_max(q.m);
            double s_out = 0.0, grad[kSlots];
            if (q.s > 0.0f) s_out = q.s * exp(((double)q.m - (double)m_out) * (double)scale_of(a.inv_temp, row_i));
            s_out = wave_sum(s_out);
            const RowGrad r = finish_row<GRAD>(a, row_i, list, m_out, s_out, grad);
            if constexpr (GRAD) {
#pragma unroll
                for (int u = 0; u < kSlots; ++u) sh_entry[u * kWave + lane] = {list.id[u], (float)grad[u]};
                if (lane == 0) sh_grad = r;
            }
        }
        if constexpr (GRAD) __syncthreads();
        return sh_grad;
    };
    if constexpr (GRAD) {
        write_grad<DT, NV, THREADS, true>(a, row_i, x0, a.v, finish);
        // the listed tokens over what was just written: after the workgroup's stores
        __syncthreads();
        if ((int)threadIdx.x < a.n_top) {
            const Entry e = sh_entry[threadIdx.x];
            if (e.id >= 0) (static_cast<T *>(a.out) + row_i * a.out_ld)[e.id] = (T)encode<DT>(e.grad);
        }
    } else {
        finish();
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void list_parts(ListArgs a) {
    using T = typename Elem<DT>::T;
    constexpr int kWaves = kThreads / kWave, NV = kChunkVectors;
    extern __shared__ uint32_t sh_bits[];
    __shared__ Sum sh_sum[kWaves];
    pass_over_nans();
    const int64_t r = blockIdx.x / (uint32_t)a.parts, row_i = a.row0 + r;
    const int part = blockIdx.x % (uint32_t)a.parts;
    const T *row = static_cast<const T *>(a.logits) + row_i * a.ld;
    const int x0 = part * a.part_width - lead_of<DT>(row, a.v), x1 = part + 1 == a.parts ? a.v : x0 + a.part_width;
    const float c2 = scale_of(a.inv_temp, row_i) * kLog2e;
    auto read = [&] {
        for (int i = threadIdx.x; i < bitmap_words<DT, NV, kThreads>(x1 - x0); i += kThreads) sh_bits[i] = 0;
        __syncthreads();
        if ((int)threadIdx.x < a.n_top) {
            const int id = entry_id(a, row_i, threadIdx.x, a.logprobs[row_i * a.n_top + threadIdx.x]), at = id - x0;
            if (id >= 0 && at >= 0 && at < x1 - x0) atomicOr(&sh_bits[at / 32], 1u << (at % 32));
        }
        __syncthreads();
    };
    Sum mine = {-INFINITY, 0.0f, 0.0f};
    for_chunks<DT, NV, kThreads, false, false, true, 1>(row, a.v, x0, x1, read, [&](uint32_t(&w)[NV][4], int x) {
        float vm[NV];
        take_out<DT, NV, kThreads>(w, sh_bits, x, x0);
        add_chunk<DT, NV, false>(w, c2, mine, vm);
    });
    mine = wave_join<false>(mine, c2);
    if (threadIdx.x % kWave == 0) sh_sum[threadIdx.x / kWave] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        Sum s = sh_sum[0];
#pragma unroll
        for (int u = 1; u < kWaves; ++u) s = join(s, sh_sum[u], c2);
        a.sums[(size_t)r * a.parts + part] = make_float2(s.m, s.s);
    }
}

// One wave a row.
template <bool GRAD>
__global__ __launch_bounds__(kWave) void list_rows(ListArgs a) {
    const int64_t r = blockIdx.x, row = a.row0 + r;
    const int lane = threadIdx.x;
    const float2 *sums = a.sums + (size_t)r * a.parts;
    List list;
    float lp[kSlots];
    read_list(a, row, list, lp);
    weigh_list(a, list, lp, repeats(list, a.n_top));
    float m_out = -INFINITY;
    for (int p = lane; p < a.parts; p += kWave) m_out = fmaxf(m_out, sums[p].x);
    m_out = wave_max(m_out);
    const double beta = scale_of(a.inv_temp, row);
    double s_out = 0.0, grad[kSlots];
    for (int p = lane; p < a.parts; p += kWave) {
        const float2 q = sums[p];
        if (q.y > 0.0f) s_out += q.y * exp(((double)q.x - (double)m_out) * beta);
    }
    s_out = wave_sum(s_out);
    const RowGrad q = finish_row<GRAD>(a, row, list, m_out, s_out, grad);
    if constexpr (GRAD) {
#pragma unroll
        for (int u = 0; u < kSlots; ++u)
            if (u * kWave + lane < a.n_top) a.entries[(size_t)r * a.n_top + u * kWave + lane] = {list.id[u], (float)grad[u]};
        if (lane == 0) a.row_grad[r] = q;
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void list_grad(ListArgs a, int parts) {
    using T = typename Elem<DT>::T;
    constexpr int kPart = kChunkVectors * kThreads * Elem<DT>::kPer;
    const int64_t r = blockIdx.x / (uint32_t)parts, row_i = a.row0 + r;
    const int part = (int)(blockIdx.x % (uint32_t)parts);
    T *out = static_cast<T *>(a.out) + row_i * a.out_ld;
    const int x0 = part * kPart - lead_of<DT>(out, a.v), x1 = part + 1 == parts ? a.v : x0 + kPart;
    Entry mine = {-1, 0.0f};
    if ((int)threadIdx.x < a.n_top) mine = a.entries[(size_t)r * a.n_top + threadIdx.x];
    write_grad<DT, kChunkVectors, kThreads, false>(a, row_i, x0, x1, [&] { return a.row_grad[r]; });
    // the listed tokens over what was just written: after the workgroup's stores
    __syncthreads();
    if (mine.id >= 0 && mine.id >= x0 && mine.id < x1) out[mine.id] = (T)encode<DT>(mine.grad);
}

// list_whole takes rows by 1,024 threads each, or by kThreads: up to kTinyRow bytes, and from many_rows on up to
// kShortRow bytes with the gradient and of any length without (gradients of one row of 16,000 bf16 take 7.3 us by 1,024
// threads and 10.0 by kThreads, of 2,000 of them 38.7 and 31.7, of 500 of 8,000 11.6 and 9.8; losses of 1,000 of 50,257
// 25.0 and 21.9, of 512 of 151,936 30.3 and 34.2, of 700 40.6 and 37.7).
constexpr int kLongThreads = 1024, kLongVectors = 2;
constexpr int64_t kTinyRow = 12 << 10;
constexpr int64_t kShortRow = 32 << 10;
int64_t many_rows(int64_t row_bytes) { return row_bytes <= (256 << 10) ? 256 : 640; }
// Rows of more than kSplitRow bytes are split where there are fewer than kFewRows of them: too many compute units
// would be without one (gradients of 16 rows of 151,936: 15.5 us split, 24.2 whole; of 96: 27.5 and 26.0; of 128: 33
// and 26.8; of 96 rows of 32,000 fp32, 128,000 bytes: 15.7 and 10.9).
constexpr int64_t kSplitRow = 128 << 10;
constexpr int64_t kFewRows = 96;
// Logits of a group of split rows whose gradient is wanted: list_grad reads them again, from the Infinity Cache
// (256 MB) if the group and its gradients fit.
constexpr size_t kCachedBytes = size_t(96) << 20;

struct Plan {
    int parts, part_width;  // parts == 0: list_whole
    int threads;
    int64_t rows, most;  // of one launch; at most
    size_t row_grad, entries, total;
};

Plan plan_of(int64_t n_rows, int32_t v, int dtype, int n_top, bool grad) {
    Plan p = {};
    const int64_t bytes = (int64_t)v * element_bytes(dtype);
    const int chunk = kChunkVectors * kThreads * elements_per_vector(dtype), chunks = (v + chunk - 1) / chunk;
    int64_t most = kMaxGrid;
    if (v <= kMaxBits && (n_rows >= kFewRows || bytes <= kSplitRow)) {
        p.threads = bytes <= kTinyRow || (n_rows >= many_rows(bytes) && (!grad || bytes <= kShortRow)) ? kThreads : kLongThreads;
    } else {
        int64_t parts = n_rows > 0 ? (kFullGrid + n_rows - 1) / n_rows : 1;
        const int64_t least = (v + kMaxBits - 1) / kMaxBits;
        if (parts < least) parts = least;
        if (parts > chunks) parts = chunks;
        const int each = (int)((chunks + parts - 1) / parts);
        p.part_width = each * chunk;
        p.parts = (chunks + each - 1) / each;
        most = kMaxGrid / (grad ? chunks : p.parts);
        if (grad && (int64_t)(kCachedBytes / bytes) < most) most = (int64_t)(kCachedBytes / bytes);  // 3 or more: v <= 2^23
    }
    const int64_t groups = (n_rows + most - 1) / most;
    p.rows = groups == 0 ? 0 : (n_rows + groups - 1) / groups;
    p.most = most;
    if (p.parts > 0) {
        p.row_grad = round256((size_t)p.rows * p.parts * sizeof(float2));
        p.entries = p.row_grad + (grad ? round256((size_t)p.rows * sizeof(RowGrad)) : 0);
        p.total = p.entries + (grad ? (size_t)p.rows * n_top * sizeof(Entry) : 0);
    }
    return p;
}

template <int DT, bool GRAD>
void launch_whole(const ListArgs &a, int threads, int64_t n, hipStream_t stream) {
    if (threads == kThreads) {
        // short rows with the gradient, rows of any length without: 17,000 of 60 and 2,000 of 700 take 58 and 10.6 us
        // with the gradient by one vector, 69 and 12.5 by two; 800 of 128,256 without it 44.0 and 39.3
        constexpr int kVectors = GRAD ? 1 : 2;
        const size_t lds = bitmap_words<DT, kVectors, kThreads>(a.v) * sizeof(uint32_t);
        list_whole<DT, kVectors, kThreads, GRAD><<<(unsigned)n, kThreads, lds, stream>>>(a);
    } else {
        const size_t lds = bitmap_words<DT, kLongVectors, kLongThreads>(a.v) * sizeof(uint32_t);
        list_whole<DT, kLongVectors, kLongThreads, GRAD><<<(unsigned)n, kLongThreads, lds, stream>>>(a);
    }
}

template <int DT>
int launch_rows(const ListArgs &a, const Plan &p, int64_t n, hipStream_t stream) {
    const bool grad = a.out != nullptr;
    if (p.parts == 0) {
        if (grad) launch_whole<DT, true>(a, p.threads, n, stream);
        else launch_whole<DT, false>(a, p.threads, n, stream);
        return hipGetLastError() == hipSuccess ? TT_OK : TT_ELAUNCH;
    }
    const size_t lds = bitmap_words<DT, kChunkVectors, kThreads>(a.part_width) * sizeof(uint32_t);
    list_parts<DT><<<(unsigned)(n * p.parts), kThreads, lds, stream>>>(a);
    if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
    if (grad) list_rows<true><<<(unsigned)n, kWave, 0, stream>>>(a);
    else list_rows<false><<<(unsigned)n, kWave, 0, stream>>>(a);
    if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
    if (grad) {
        const int chunk = kChunkVectors * kThreads * Elem<DT>::kPer, parts = (a.v + chunk - 1) / chunk;
        list_grad<DT><<<(unsigned)(n * parts), kThreads, 0, stream>>>(a, parts);
        if (hipGetLastError() != hipSuccess) return TT_ELAUNCH;
    }
    return TT_OK;
}

}  // namespace

size_t distill_workspace_used(int32_t n_rows, int32_t v, int dtype, int n_top, bool grad) {
    return plan_of(n_rows, v, dtype, n_top, grad).total;
}

// The most that any number of rows up to n_rows uses.  From kFullGrid rows on their parts are as few as the bitmap
// allows, and a group of them is largest where it is the only one.
size_t distill_workspace_bytes(int32_t n_rows, int32_t v, int dtype, int n_top, bool grad) {
    size_t most = 0;
    auto add = [&](int64_t n) {
        const size_t used = plan_of(n, v, dtype, n_top, grad).total;
        most = used > most ? used : most;
    };
    for (int64_t n = 1; n <= n_rows && n <= kFullGrid; ++n) add(n);
    const int64_t group = n_rows > kFullGrid ? plan_of(n_rows, v, dtype, n_top, grad).most : 0;
    if (group > kFullGrid) add(group < n_rows ? group : n_rows);
    return most;
}

int launch_distill(const DistillArgs &l, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const Plan p = plan_of(l.n_rows, l.v, l.dtype, l.n_top, l.dlogits != nullptr);
    if (p.total > 0 && (workspace == nullptr || workspace_bytes < p.total)) return TT_EWORKSPACE;
    if (p.total > 0 && reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return TT_EINVAL;
    char *ws = static_cast<char *>(workspace);
    ListArgs a;
    a.logits = l.logits;
    a.ld = l.ld;
    a.v = l.v;
    a.dtype = l.dtype;
    a.parts = p.parts;
    a.part_width = p.part_width;
    a.n_top = l.n_top;
    a.tail = l.tail;
    a.inv_temp = l.inv_temp;
    a.ids = l.top_ids;
    a.logprobs = l.top_logprobs;
    a.id_map = l.id_map;
    a.n_map = l.n_map;
    a.sums = p.total > 0 ? reinterpret_cast<float2 *>(ws) : nullptr;
    a.loss = l.loss;
    a.grad_loss = l.grad_loss;
    a.row_grad = p.total > 0 ? reinterpret_cast<RowGrad *>(ws + p.row_grad) : nullptr;
    a.entries = p.total > 0 ? reinterpret_cast<Entry *>(ws + p.entries) : nullptr;
    a.out = l.dlogits;
    a.out_ld = l.out_ld;
    for (int64_t row0 = 0; row0 < l.n_rows; row0 += p.rows) {
        const int64_t n = l.n_rows - row0 < p.rows ? l.n_rows - row0 : p.rows;
        a.row0 = row0;
        int st;
        if (l.dtype == TT_BF16) st = launch_rows<TT_BF16>(a, p, n, stream);
        else if (l.dtype == TT_F16) st = launch_rows<TT_F16>(a, p, n, stream);
        else st = launch_rows<TT_F32>(a, p, n, stream);
        if (st != TT_OK) return st;
    }
    return TT_OK;
}

}  // namespace tt
