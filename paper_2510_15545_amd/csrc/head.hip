// The output head without its logits: log probabilities of given tokens from hidden states x [n, h] and the head's
// weights W [v, h] (tt_head_logprobs), and their gradient (tt_head_logprobs_backward).
//
//   z = x W^T,  M = max z,  L = ln sum exp(beta (z - M)),  logprob = beta (z_t - M) - L
//   dz_j = beta (g ([j = t] - p_j) + q p_j),  dx = dz W,  dW = dz^T x
//
// Forward: one product by tiles (tiles.h), whose epilogue leaves each tile's largest logit and sum of exponentials for
// every row, and a second kernel that joins a row's parts.  Backward: the rows that carry a weight are gathered; then, for
// one piece of the vocabulary after another, the product again, by the same sums, with an epilogue that makes dz of it, rounded to
// the operands' type twice, itself and what that takes off it (relative to the largest row weight; kBeside), and two more products:
// dx += dz W (in fp32, over all pieces) and the piece's rows of dW, written once.  Of these three products' operands dz, W and x each is kept
// as it is, whichever of its indices is summed over (tiles.h).  No atomics: results do not depend on scheduling.
#include <algorithm>

#include "tiles.h"

namespace tt {
namespace {

using namespace tiles;
using rows::round256;

constexpr int kTile = 256;   // tokens (or hidden elements) of a wide tile
constexpr int kAlign = 256;  // pieces of the vocabulary come in multiples of this
typedef Shape<128, 128, 2, 2> Any;  // of the products of matrices that lie in any way

constexpr int64_t kSplitTiles = 256;  // workgroups that the sum over a piece's tokens is split into at most
constexpr int64_t kPieceBytes = int64_t(256) << 20;  // what a piece of the vocabulary may take of the workspace
constexpr int64_t kCus = 256;
constexpr int kRowsPerLaunch = 1 << 14;  // 2^23 tokens of so many rows stay below 2^32 threads

__host__ __device__ inline int64_t round_to(int64_t x, int64_t n) { return (x + n - 1) / n * n; }
__host__ __device__ constexpr int step_elements(int dtype) { return kStepBytes / bytes_of(dtype); }
inline int64_t tiles_of(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }
// A row that carries a weight, for the gradient's epilogue: p = 2^((z - m) c - l), dz = (w - g) p, and g (1 - p) + w p at
// its token.  What pads the list is its first row again with g = w = 0: hidden states of zeros would make a NaN of an infinite
// weight, and 0 times it another of dz, which reaches that token's row of dW.
struct Row {
    float c, m, l, g, w;
    int32_t id;
};
// In 16 bits what rounding takes off dz is kept beside it, so that dz has twice the type's digits and the gradients' error is that
// of rounding the result once (1.00 times; without it 1.3 to 1.5).  Up to kBeside rows as rows of their own, this many or half
// as many further on, beside the same hidden states again: the tiles have room (64 x
// 32,000 x 1,024: 88 us, 76 without).  From there on as a second matrix behind the first, and both products go through both (66 x
// 32,000 x 1,024: 102 us, 83 without; 391 x 50,257 x 1,024 fp16 276, 198 without; 2,048 x 128,256 x 2,048 4.55 to 4.8 ms, 2.9 without).
constexpr int kBeside = 64;

struct Totals {
    int32_t rows;  // that carry a weight
    float scale;   // of the stored dz: the true one is scale times as large
};

// ------------------------------------------------------------------------------------------------ copies
// Rows of `bytes` bytes at any address, at a stride of `ld` bytes, into rows of `out_bytes` (a multiple of 16), filled up with zeros.
// list: the rows by their index in it, totals->rows of them, padded with the first of them (again: to that many, which are
// written twice; zeros where there is none); or null.
__global__ __launch_bounds__(256) void lay_out(const char *src, int64_t ld, int n_rows, int bytes, const int32_t *list, const Totals *totals,
                                               int again, char *out, int out_bytes) {
    const int count = totals ? totals->rows : n_rows, pieces = out_bytes / 16;
    const int64_t end = (again ? 2 * again : totals ? padded_rows(count) : n_rows) * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < end; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces;
        const int c = (int)(i % pieces) * 16;
        u4 v = {0, 0, 0, 0};
        int64_t from = again && r >= again ? r - again : r;
        if (from >= count) from = 0;
        if (count > 0 && c < bytes) {
            const char *q = src + (list ? (int64_t)list[from] : from) * ld + c;
            v = c + 16 <= bytes ? (u4)*reinterpret_cast<const u4b *>(q) : load_some(q, bytes - c);
        }
        *reinterpret_cast<u4 *>(out + r * out_bytes + c) = v;
    }
}

// ------------------------------------------------------------------------------------------------ forward
// Parts of the rows' distributions from a tile's tokens, and the given tokens' logits.
template <int DT, typename S>
__device__ __forceinline__ void parts_of_tile(const Side &w, const Side &x, int m0, int n0, f4 (&acc)[S::FM][S::FN], const float *inv_temp,
                                              const int32_t *ids, Part *parts, int n_tiles, float *token, char *lds) {
    const int n_rows = x.rows;
    if (ids)
        for_columns<S>(n0, [&](int n, int j) {
            const int at = n < n_rows ? ids[n] : -1;
            if (__any(at >= m0 && at < m0 + S::TM && at < w.rows))
                for_rows<S>(m0, [&](int m, int i) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (at == m + q && at < w.rows) token[n] = acc[i][j][q];
                });
        });
    if (m0 + S::TM > w.rows)
        for_columns<S>(n0, [&](int, int j) {
            for_rows<S>(m0, [&](int m, int i) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (m + q >= w.rows) acc[i][j][q] = -INFINITY;
            });
        });
    const Part p = column_parts<S, true>(
        n0, lds, [&](int i, int j, int q) { return acc[i][j][q]; },
        [&](int n) { return (n < n_rows ? rows::scale_of(inv_temp, n) : 1.0f) * rows::kLog2e; });
    const int n = n0 + (int)threadIdx.x;
    if ((int)threadIdx.x < S::TN && n < n_rows) parts[(int64_t)n * n_tiles + m0 / S::TM] = p;
}

template <int DT, typename S>
__global__ __launch_bounds__(S::THREADS, 2) void head_parts(Side w, Side x, int mt, int nt, const float *inv_temp, const int32_t *ids, Part *parts,
                                                            float *token) {
    TT_TILE_LDS(S);
    f4 acc[S::FM][S::FN];
    int m, n;
    tile_of((int)blockIdx.x, (int)gridDim.x, mt, nt, m, n);
    Product<DT, false, false, S>::run(w, x, m * S::TM, n * S::TN, 0, w.bytes / kStepBytes, lds, acc);
    parts_of_tile<DT, S>(w, x, m * S::TM, n * S::TN, acc, inv_temp, ids, parts, mt, token, lds);
}

template <int DT>
__global__ __launch_bounds__(Any::THREADS) void head_parts_any(Side w, Side x, const float *inv_temp, const int32_t *ids, Part *parts, float *token) {
    __shared__ __attribute__((aligned(16))) char lds[Any::LDS];
    f4 acc[Any::FM][Any::FN];
    const int m0 = (int)blockIdx.x * Any::TM, n0 = (int)blockIdx.y * Any::TN;
    product_any<DT, Any>(w, x, m0, n0, lds, acc);
    parts_of_tile<DT, Any>(w, x, m0, n0, acc, inv_temp, ids, parts, gridDim.x, token, lds);
}

// Up to 16 rows.
template <int DT, bool WHOLE>
__global__ __launch_bounds__(kThinThreads, 4) void head_parts_few(Side w, Side x, const float *inv_temp, const int32_t *ids, Part *parts, float *token) {
    __shared__ __attribute__((aligned(16))) char lds[kThinLds];
    __shared__ float sums[8][256];
    const int n = (int)threadIdx.x >> 4;
    const float c = (n < x.rows ? rows::scale_of(inv_temp, n) : 1.0f) * rows::kLog2e;
    const int id = ids && n < x.rows ? ids[n] : -1;
    Part p = {-INFINITY, 0.0f};
    product_few<DT, WHOLE>(w, x, lds, sums, [&](int m, int, float z) {
        if (m >= w.rows) return;
        if (m == id) token[n] = z;
        add_part<true>(p, z, c);
    });
    p = join_quarter<true>(p, c);
    if (((int)threadIdx.x & 15) == 0 && n < x.rows) parts[(int64_t)n * gridDim.x + blockIdx.x] = p;
}

// Few rows: every workgroup's part of them.
template <int DT, int FN>
__global__ __launch_bounds__(kThinThreads, 4) void head_parts_thin(Side w, Side x, const float *inv_temp, const int32_t *ids, Part *parts, float *token) {
    __shared__ __attribute__((aligned(16))) char lds[kThinLds];
    const int column = (int)threadIdx.x & 15;
    const auto scale = [&](int n) { return (n < x.rows ? rows::scale_of(inv_temp, n) : 1.0f) * rows::kLog2e; };
    Part p[FN];
    float c[FN];
    int id[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        p[j] = {-INFINITY, 0.0f};
        c[j] = scale(j * 16 + column);
        id[j] = ids && j * 16 + column < x.rows ? ids[j * 16 + column] : -1;
    }
    product_thin<DT, FN>(w, x, lds, [&](int m, f4 (&acc)[FN]) {
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            float z[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                z[q] = m + q < w.rows ? acc[j][q] : -INFINITY;
                if (m + q == id[j] && m + q < w.rows) token[j * 16 + column] = acc[j][q];
            }
            add_part<true>(p[j], z, c[j]);
        }
    });
    const Part r = join_lanes<FN, true>(p, x.rows, lds, scale);
    if ((int)threadIdx.x < x.rows) parts[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = r;
}

// A workgroup a row.
__global__ __launch_bounds__(256) void head_join(const Part *parts, int n_tiles, int v, const float *inv_temp, const int32_t *ids,
                                                 const float *token, float *logprob, float *lse, float *stats) {
    const int n = (int)blockIdx.x;
    const float beta = rows::scale_of(inv_temp, n);
    Part r = join_row(parts + (int64_t)n * n_tiles, n_tiles, beta);
    if (threadIdx.x != 0) return;
    if (!rows::sound(beta)) r.m = r.s = NAN;
    if (r.s != r.s) r.m = NAN;
    if (lse) lse[n] = fmaf(beta, r.m, r.s);
    if (stats) {
        stats[2 * (int64_t)n] = r.m;
        stats[2 * (int64_t)n + 1] = r.s;
    }
    if (logprob) {
        const int id = ids[n];
        float y = NAN;
        if (id >= 0 && id < v) y = r.m == -INFINITY ? -INFINITY : (token[n] - r.m) * beta - r.s;
        logprob[n] = y;
    }
}

// ------------------------------------------------------------------------------------------------ backward
// The rows that carry a weight, in order, the scale of their gradients, and what the epilogue takes of them; the
// place of every row in the list, -1 for none.  One workgroup.
__global__ __launch_bounds__(1024) void head_select(int n, int v, const float *inv_temp, const int32_t *ids, const float *stats, const float *grad,
                                                    const float *grad_lse, float store_scale, int32_t *place, int32_t *list, Row *out, Totals *totals) {
    __shared__ int32_t counts[16];
    __shared__ float tops[16];
    const int t = (int)threadIdx.x, wave = t >> 6, lane = t & 63;
    const auto weights = [&](int i, float &g, float &w) {
        const int id = ids ? ids[i] : -1;
        g = grad && id >= 0 && id < v ? grad[i] : 0.0f;
        w = grad_lse ? grad_lse[i] : 0.0f;
        const bool some = (g != 0.0f || w != 0.0f) && stats[2 * (int64_t)i] != -INFINITY;
        if (!some) g = w = 0.0f;
        return some;
    };
    float top = 0.0f;
    for (int i = t; i < n; i += 1024) {
        float g, w;
        weights(i, g, w);
        const float beta = rows::scale_of(inv_temp, i), y = beta * (fabsf(g) + fabsf(w));
        if (rows::sound(beta) && y < INFINITY) top = fmaxf(top, y);  // a row that will be NaN does not count
    }
    top = rows::wave_max(top);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    for (int k = 0; k < 16; ++k) top = fmaxf(top, tops[k]);
    if (!(top > 0.0f)) top = 1.0f;
    int before = 0;
    for (int i0 = 0; i0 < n; i0 += 1024) {
        const int i = i0 + t;
        float g = 0.0f, w = 0.0f;
        const bool some = i < n && weights(i, g, w);
        const uint64_t votes = __ballot(some);
        __syncthreads();
        if (lane == 0) counts[wave] = __popcll(votes);
        __syncthreads();
        int at = before + __popcll(votes & ((uint64_t(1) << lane) - 1));
        for (int k = 0; k < 16; ++k) {
            if (k < wave) at += counts[k];
            before += counts[k];
        }
        if (i < n) place[i] = some ? at : -1;
        if (some) {
            const float beta = rows::sound(rows::scale_of(inv_temp, i)) ? rows::scale_of(inv_temp, i) : NAN;
            list[at] = i;
            out[at] = {beta * rows::kLog2e, stats[2 * (int64_t)i], stats[2 * (int64_t)i + 1] * rows::kLog2e,
                       beta * g / top * store_scale, beta * w / top * store_scale, ids && g != 0.0f ? ids[i] : -1};
        }
    }
    __syncthreads();  // the first row is there
    for (int i = before + t; i < padded_rows(before); i += 1024) out[i] = {out[0].c, out[0].m, out[0].l, 0.0f, 0.0f, -1};
    if (t == 0) *totals = {before, top / store_scale};
}

// ln p in base 2.  No probability is above 1: statistics of another product may have an M a rounding below the largest logit as it is
// formed here, which a large inverse temperature would make an infinity.  (A minimum that is NaN beside a NaN: one instruction.)
__device__ __forceinline__ float exponent_of(const Row &r, float z) { return __builtin_elementwise_minimum(fmaf(z - r.m, r.c, -r.l), 0.0f); }

// dz of a token.  At the row's own 1 - p is not a difference, and where p is above 2^-0.5 at M and the logit within 2^-0.25 of it, it
// is M's and taken as M (a second token as near would have made the sum 1.8, and p at M 2^-0.88): where the two differ by a rounding
// (statistics of another product, of more or fewer rows), 1 - p of a token that is almost certain would be that rounding over 1 - p off.
__device__ __forceinline__ float dlogit_of(const Row &r, float z, int token) {
    float y = (r.w - r.g) * __builtin_amdgcn_exp2f(exponent_of(r, z));
    if (token == r.id) {
        const float e = exponent_of(r, r.l < 0.5f && fabsf(z - r.m) * r.c < 0.25f ? r.m : z);
        y = r.g * -expm1f(e * (float)rows::kLn2) + r.w * __builtin_amdgcn_exp2f(e);
    }
    return y;
}

// dz of a piece's tokens (the first of them v0) for the listed rows, stored as [row][token] up to row n_end; in 16 bits the
// remainders `rest` rows further on.
template <int DT, typename S>
__global__ __launch_bounds__(S::THREADS, 2) void head_dlogits(Side w, Side x, int mt, int nt, int v0, const Row *meta, const Totals *totals, int rest, int n_end, char *d,
                                                              int64_t d_ld) {
    TT_TILE_LDS(S);
    using T = typename rows::Elem<DT>::T;
    f4 acc[S::FM][S::FN];
    int m0, n0;
    tile_of((int)blockIdx.x, (int)gridDim.x, mt, nt, m0, n0);
    m0 *= S::TM;
    n0 *= S::TN;
    if (n0 >= totals->rows) return;
    Product<DT, false, false, S>::run(w, x, m0, n0, 0, w.bytes / kStepBytes, lds, acc);
    Row r[S::FN];
    for_columns<S>(n0, [&](int n, int j) { r[j] = meta[n]; });
    bool special = m0 + S::TM > w.rows;  // the piece's end, or a row's token
#pragma unroll
    for (int j = 0; j < S::FN; ++j) special |= __any(r[j].id - v0 >= m0 && r[j].id - v0 < m0 + S::TM) != 0;
    const auto to = [&](int n) { return reinterpret_cast<T *>(d) + (int64_t)n * d_ld; };
    const auto exponent = [&](float z, int j) { return exponent_of(r[j], z); };
    // any of the workgroup's (by a word of the tile's memory, of which there is no more)
    int *flag = reinterpret_cast<int *>(lds);
    if (threadIdx.x == 0) *flag = 0;
    __syncthreads();
    if (special) *flag = 1;
    __syncthreads();
    special = *flag != 0;
    __syncthreads();
    const auto store = [&](auto values) {
        store_tile<DT, S, DT != TT_F32>(m0, (int)d_ld, n0, n_end, lds, lds + S::TM * kStepBytes, values, to, rest * d_ld);
    };
    if (special) {
        store([&](int, int j, int m, int i, float (&y)[4]) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                y[q] = m + q < w.rows ? dlogit_of(r[j], acc[i][j][q], v0 + m + q) : 0.0f;
            }
        });
    } else {
        store([&](int, int j, int, int i, float (&y)[4]) {
            const float f = r[j].w - r[j].g;
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = f * __builtin_amdgcn_exp2f(exponent(acc[i][j][q], j));
        });
    }
}

// Up to 16 rows: the logits by the same sums as head_parts_few has, so that what its statistics say of a token that is almost certain
// holds here, too (1 - p of 1e-4 would be off by a rounding of its logit over 1e-4, a few percent).  d: `again` rows of which the
// first x.rows are listed ones or pad the list, in 16 bits the remainders' as many; all of whole steps of tokens, zeros elsewhere.
template <int DT, bool WHOLE>
__global__ __launch_bounds__(kThinThreads, 4) void head_dlogits_few(Side w, Side x, int v0, const Row *meta, const Totals *totals, int again, char *d, int64_t d_ld) {
    __shared__ __attribute__((aligned(16))) char lds[kThinLds];
    __shared__ float sums[8][256];
    if (totals->rows == 0) return;
    using T = typename rows::Elem<DT>::T;
    const int n = (int)threadIdx.x >> 4;
    const bool there = n < x.rows;
    const Row r = meta[there ? n : 0];
    T *row = reinterpret_cast<T *>(d) + n * d_ld;
    product_few<DT, WHOLE>(w, x, lds, sums, [&](int m, int, float z) {
        if (!there || m >= w.rows) return;
        const float y = dlogit_of(r, z, v0 + m);
        const uint32_t bits = rows::encode<DT>(y);
        row[m] = (T)bits;
        if constexpr (DT != TT_F32) {
            const float stored = rows::decode<DT>(bits);
            row[again * d_ld + m] = (T)rows::encode<DT>(fabsf(stored) < INFINITY ? y - stored : 0.0f);
        }
    });
    const int end = (int)round_to(w.rows, step_elements(DT)), id = (int)(blockIdx.x * kThinThreads + threadIdx.x), all = (int)gridDim.x * kThinThreads;
    const int pieces = end * (int)sizeof(T) / 16, more = again - x.rows, tail = end - w.rows;
    for (int part = 0; part < (DT == TT_F32 ? 1 : 2); ++part) {
        T *from = reinterpret_cast<T *>(d) + part * again * d_ld;
        for (int64_t i = id; i < (int64_t)more * pieces; i += all) reinterpret_cast<u4 *>(from + (x.rows + i / pieces) * d_ld)[i % pieces] = u4{0, 0, 0, 0};
        for (int i = id; i < x.rows * tail; i += all) from[i / tail * d_ld + w.rows + i % tail] = 0;
    }
}

// dx of the listed rows over one piece of the vocabulary, split into parts of its tokens, added to what the pieces before
// gave: sums[split][row][h] in fp32.  twice, rest: the remainders are a second matrix.
template <int DT, typename S>
__global__ __launch_bounds__(S::THREADS, 2) void head_dhidden(Side w, Side d, int mt, int nt, int split_steps, const Totals *totals, float *sums, int64_t ld,
                                                    int64_t plane, int first, int twice, int64_t rest) {
    TT_TILE_LDS(S);
    f4 acc[S::FM][S::FN];
    const int split = (int)blockIdx.x / (mt * nt);
    int m0, n0;
    tile_of((int)blockIdx.x % (mt * nt), mt * nt, mt, nt, m0, n0);
    m0 *= S::TM;
    n0 *= S::TN;
    if (n0 >= totals->rows) return;
    const int steps = (w.rows + step_elements(DT) - 1) / step_elements(DT), from = split * split_steps;
    Product<DT, true, false, S>::run(w, d, m0, n0, from, min(split_steps, steps - from), lds, acc, twice, rest);
    for_columns<S>(n0, [&](int n, int j) {
        float *out = sums + split * plane + (int64_t)n * ld;
        for_rows<S>(m0, [&](int m, int i) {
            if (m >= ld) return;
            f4 *to = reinterpret_cast<f4 *>(out + m);
            *to = first ? acc[i][j] : *to + acc[i][j];
        });
    });
}

// The splits' sums, scaled, to the rows' places; zeros for rows without a weight.
template <int DT>
__global__ __launch_bounds__(256) void head_place(const float *sums, int64_t ld, int64_t plane, int splits, const int32_t *place, const Totals *totals,
                                                  int again, int h, void *dhidden, int64_t out_ld) {
    using T = typename rows::Elem<DT>::T;
    const int n = (int)blockIdx.x, c = (int)(blockIdx.y * 256 + threadIdx.x) * 4;
    if (c >= h) return;
    const int at = place[n];
    f4 y = {0, 0, 0, 0};
    if (at >= 0) {
        const auto add = [&](const float *from) {  // a loop for each: a condition inside would keep its loads from going out together
#pragma unroll 4
            for (int s = 0; s < splits; ++s) y += *reinterpret_cast<const f4 *>(from + s * plane);
        };
        add(sums + at * ld + c);
        if (again) add(sums + (at + again) * ld + c);
        y *= totals->scale;
    }
    const float z[4] = {y[0], y[1], y[2], y[3]};
    store4<DT>(static_cast<T *>(dhidden) + n * out_ld, c, h, z);
}

// A piece's rows of dW.
template <int DT, typename S>
__global__ __launch_bounds__(S::THREADS, 2) void head_dweight(Side x, Side d, int mt, int nt, const Totals *totals, int again, int n_tokens, int h, void *dweight, int64_t ld,
                                                              int twice, int64_t rest) {
    TT_TILE_LDS(S);
    using T = typename rows::Elem<DT>::T;
    f4 acc[S::FM][S::FN];
    int m0, n0;
    tile_of((int)blockIdx.x, (int)gridDim.x, mt, nt, m0, n0);
    m0 *= S::TM;
    n0 *= S::TN;
    const int n_rows = totals->rows == 0 ? 0 : again ? 2 * again : totals->rows, steps = (n_rows + step_elements(DT) - 1) / step_elements(DT);
    Product<DT, true, true, S>::run(x, d, m0, n0, 0, steps, lds, acc, twice, rest);
    const float scale = totals->scale;
    store_tile<DT, S>(m0, h, n0, n_tokens, lds, lds + S::TM * kStepBytes, [&](int, int j, int, int i, float (&y)[4]) {
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] = acc[i][j][q] * scale;
    }, [&](int n) { return static_cast<T *>(dweight) + (int64_t)n * ld; });
}

__global__ __launch_bounds__(256) void head_zero(int h, int e, char *out, int64_t ld) {
    for (int64_t c = threadIdx.x; c < (int64_t)h * e; c += 256) out[blockIdx.x * ld * e + c] = 0;
}

// ------------------------------------------------------------------------------------------------ workspaces
struct Layout {
    size_t total = 0;
    size_t take(size_t bytes) {
        const size_t at = total;
        total += round256(bytes);
        return at;
    }
};

struct ForwardLayout : Layout {
    size_t parts, token;
    ForwardLayout(int64_t n, int64_t v) {
        parts = take(most_parts(n, v) * sizeof(Part));
        token = take((size_t)n * 4);
    }
};

struct BackwardLayout : Layout {
    int64_t n_pad, d_rows, width, piece;  // d_rows: of dz with its remainders; width: elements of a hidden state in a copy
    int splits;
    size_t totals, place, list, meta, x, w, d, sums;
    BackwardLayout(int64_t n, int64_t v, int64_t h, int dtype) {
        const int64_t e = rows::element_bytes(dtype), all = round_to(v, kAlign);
        n_pad = padded_rows(n);
        d_rows = stored_rows(n, dtype);
        width = round_to(h, step_elements(dtype));
        const int64_t row = (d_rows + width) * e;  // of dz and of the weights' copy, for a token
        piece = std::min(all, std::max<int64_t>(kAlign, kPieceBytes / row / kAlign * kAlign));
        // pieces of one size, in whole rounds of the compute units where there are several
        const int64_t round = std::max<int64_t>(1, kCus / row_tiles(n, dtype)) * kTile, even = round_to(tiles_of(all, tiles_of(all, piece)), kAlign);
        if (piece < all) piece = std::min(piece, piece >= round ? std::min(round_to(even, round), piece / round * round) : even);
        const int64_t tiles = row_tiles(n, dtype) * tiles_of(width, dtype == TT_F32 ? 128 : kTile);
        splits = (int)std::min<int64_t>(std::max<int64_t>(1, kSplitTiles / tiles), std::max<int64_t>(1, all / (dtype == TT_F32 ? 128 : 512)));  // at least 4 or 8 steps each
        rows_of(n, e);
        d = take((size_t)(piece * d_rows * e));
        w = take((size_t)(piece * width * e));
        sums = take((size_t)(splits * n_pad * width * 4));
    }
    // What no number of rows up to n takes more than (fewer rows make longer pieces and more splits).
    static size_t most(int64_t n, int64_t v, int64_t h, int dtype) {
        BackwardLayout l;
        const int64_t e = rows::element_bytes(dtype);
        l.n_pad = padded_rows(n);
        l.width = round_to(h, step_elements(dtype));
        l.rows_of(n, e);
        const int64_t row = (stored_rows(n, dtype) + l.width) * e;
        l.take((size_t)std::min(round_to(v, kAlign) * row, std::max(kAlign * row, kPieceBytes)) + 256);
        l.take((size_t)(std::max(kSplitTiles / tiles_of(l.width, kTile), row_tiles(n, dtype)) * 384 * l.width * 4));  // n_pad is at most 384 a tile
        return l.total;
    }

  private:
    BackwardLayout() {}
    static int64_t stored_rows(int64_t n, int dtype) { return (dtype != TT_F32 && n > kBeside ? 2 : 1) * padded_rows(n); }
    static int64_t row_tiles(int64_t n, int dtype) { return tiles_of(n, dtype == TT_F32 ? 128 : 256); }
    void rows_of(int64_t n, int64_t e) {
        totals = take(sizeof(Totals));
        place = take((size_t)n * 4);
        list = take((size_t)n * 4);
        meta = take((size_t)n_pad * sizeof(Row));
        x = take((size_t)(n_pad * width * e));
    }
};

int status() { return hipGetLastError() == hipSuccess ? TT_OK : TT_ELAUNCH; }

Side matrix(const void *p, int64_t ld, int64_t n, int64_t width, int64_t e) { return {static_cast<const char *>(p), ld * e, (int)n, (int)(width * e)}; }

void copy_rows(const void *src, int64_t ld, int64_t n_rows, int64_t width, int64_t e, const int32_t *list, const Totals *totals, int again, char *out,
               int64_t out_width, hipStream_t stream) {
    const int64_t pieces = (totals ? padded_rows(n_rows) : n_rows) * out_width * e / 16;
    lay_out<<<(unsigned int)std::min<int64_t>((pieces + 255) / 256, 1 << 20), 256, 0, stream>>>(static_cast<const char *>(src), ld * e, (int)n_rows, (int)(width * e), list, totals,
                                                                  again, out, (int)(out_width * e));
}

template <int DT>
int forward(const HeadArgs &a, char *ws, hipStream_t stream) {
    const ForwardLayout lay(a.n_rows, a.v);
    const int64_t e = rows::element_bytes(DT);
    Part *parts = reinterpret_cast<Part *>(ws + lay.parts);
    float *token = reinterpret_cast<float *>(ws + lay.token);
    const int32_t *ids = a.logprob ? a.ids : nullptr;
    const Side w = matrix(a.weight, a.w_ld, a.v, a.h, e);
    int n_tiles = (int)tiles_of(a.v, kTile);
    if (a.n_rows <= kThinMost) {
        n_tiles = thin_groups(a.n_rows, a.v);
        const Side x = matrix(a.hidden, a.x_ld, a.n_rows, a.h, e);
        const auto run = [&](auto kernel) { kernel<<<n_tiles, kThinThreads, 0, stream>>>(w, x, a.inv_temp, ids, parts, token); };
        if (a.n_rows <= kFewMost && w.bytes % kFewBytes == 0) run(head_parts_few<DT, true>);
        else if (a.n_rows <= kFewMost) run(head_parts_few<DT, false>);
        else if (a.n_rows <= 32) run(head_parts_thin<DT, 2>);
        else run(head_parts_thin<DT, 4>);
    } else if (whole_steps(w) && whole_steps(matrix(a.hidden, a.x_ld, a.n_rows, a.h, e))) {
        for (int64_t n0 = 0; n0 < a.n_rows; n0 += kRowsPerLaunch) {
            const int64_t n = std::min<int64_t>(kRowsPerLaunch, a.n_rows - n0);
            const Side x = matrix(static_cast<const char *>(a.hidden) + n0 * a.x_ld * e, a.x_ld, n, a.h, e);
            with_shape<DT, kForward>(a.v, std::min<int64_t>(kRowsPerLaunch, a.n_rows), [&](auto shape) {
                typedef decltype(shape) S;
                const int nt = (int)tiles_of(n, S::TN);
                n_tiles = (int)tiles_of(a.v, S::TM);
                head_parts<DT, S><<<(unsigned int)(n_tiles * nt), S::THREADS, 0, stream>>>(w, x, n_tiles, nt, a.inv_temp ? a.inv_temp + n0 : nullptr,
                                                                                        ids ? ids + n0 : nullptr, parts + n0 * n_tiles, token + n0);
            });
        }
    } else {
        n_tiles = (int)tiles_of(a.v, Any::TM);
        const Side x = matrix(a.hidden, a.x_ld, a.n_rows, a.h, e);
        head_parts_any<DT><<<dim3(n_tiles, (unsigned int)tiles_of(a.n_rows, Any::TN)), Any::THREADS, 0, stream>>>(w, x, a.inv_temp, ids, parts, token);
    }
    head_join<<<(unsigned int)a.n_rows, 256, 0, stream>>>(parts, n_tiles, a.v, a.inv_temp, a.ids, token, a.logprob, a.lse, a.stats);
    return status();
}

// Whether the gradient's products need a copy of the weights' rows.
bool copies_weight(const HeadGradArgs &a) {
    const Side w = matrix(a.weight, a.w_ld, a.v, a.h, rows::element_bytes(a.dtype));
    return !whole_steps(w);
}

// Rows that the remainders lie behind as rows of their own, 0 where they do not.
template <int DT>
int beside(const HeadGradArgs &a) {
    return DT == TT_F32 || a.n_rows > kBeside ? 0 : a.n_rows > kBeside / 2 ? kBeside : kBeside / 2;
}

template <int DT>
void backward_piece(const HeadGradArgs &a, const BackwardLayout &lay, char *ws, int64_t v0, bool copy_w, hipStream_t stream) {
    const int64_t e = rows::element_bytes(DT), here = std::min<int64_t>(lay.piece, a.v - v0);
    const Totals *totals = reinterpret_cast<Totals *>(ws + lay.totals);
    const char *weight = static_cast<const char *>(a.weight) + v0 * a.w_ld * e;
    Side w = matrix(weight, a.w_ld, here, a.h, e);
    if (copy_w && (a.dhidden || a.n_rows > kFewMost)) {
        copy_rows(weight, a.w_ld, here, a.h, e, nullptr, nullptr, 0, ws + lay.w, lay.width, stream);
        w = matrix(ws + lay.w, lay.width, here, lay.width, e);
    }
    const int again = beside<DT>(a), twice = lay.d_rows > lay.n_pad;
    const int64_t rest = lay.n_pad * lay.piece * e;
    const Side x = matrix(ws + lay.x, lay.width, lay.n_pad, lay.width, e), d = matrix(ws + lay.d, lay.piece, lay.n_pad, lay.piece, e);
    const Row *meta = reinterpret_cast<const Row *>(ws + lay.meta);
    if (a.n_rows <= kFewMost) {
        const Side weights = matrix(weight, a.w_ld, here, a.h, e), few = matrix(ws + lay.x, lay.width, a.n_rows, lay.width, e);
        const auto run = [&](auto kernel) {
            kernel<<<thin_groups(a.n_rows, here), kThinThreads, 0, stream>>>(weights, few, (int)v0, meta, totals, kBeside / 2, ws + lay.d, lay.piece);
        };
        if (weights.bytes % kFewBytes == 0) run(head_dlogits_few<DT, true>);
        else run(head_dlogits_few<DT, false>);
    } else with_shape<DT, kGradLogits>(here, a.n_rows, [&](auto shape) {
        typedef decltype(shape) S;
        const int mt = (int)tiles_of(here, S::TM), nt = (int)tiles_of(a.n_rows, S::TN);
        head_dlogits<DT, S><<<mt * nt, S::THREADS, 0, stream>>>(w, x, mt, nt, (int)v0, meta, totals, again ? again : (int)lay.n_pad, again ? again : INT_MAX,
                                                               ws + lay.d, lay.piece);
    });
    if (a.dhidden)
        with_shape<DT, kGradHidden>(a.h, a.n_rows, [&](auto shape) {
            typedef decltype(shape) S;
            const int mt = (int)tiles_of(a.h, S::TM), nt = (int)tiles_of(a.n_rows, S::TN);
            const int steps = (int)tiles_of(here, step_elements(DT)), split = (int)tiles_of(steps, lay.splits);
            head_dhidden<DT, S><<<mt * nt * lay.splits, S::THREADS, 0, stream>>>(w, d, mt, nt, split, totals, reinterpret_cast<float *>(ws + lay.sums),
                                                                              lay.width, lay.n_pad * lay.width, v0 == 0, twice, rest);
        });
    if (a.dweight)
        with_shape<DT, kGradWeight>(a.h, a.n_rows, [&](auto shape) {
            typedef decltype(shape) S;
            const int mt = (int)tiles_of(a.h, S::TM), nt = (int)tiles_of(here, S::TN);
            head_dweight<DT, S><<<mt * nt, S::THREADS, 0, stream>>>(x, d, mt, nt, totals, again, (int)here, a.h,
                                                                    static_cast<char *>(a.dweight) + v0 * a.dw_ld * e, a.dw_ld, twice, rest);
        });
}

template <int DT>
int backward(const HeadGradArgs &a, char *ws, hipStream_t stream) {
    const bool copy_w = copies_weight(a);
    const BackwardLayout lay(a.n_rows, a.v, a.h, a.dtype);
    const int64_t e = rows::element_bytes(DT);
    Totals *totals = reinterpret_cast<Totals *>(ws + lay.totals);
    int32_t *place = reinterpret_cast<int32_t *>(ws + lay.place), *list = reinterpret_cast<int32_t *>(ws + lay.list);
    head_select<<<1, 1024, 0, stream>>>(a.n_rows, a.v, a.inv_temp, a.ids, a.stats, a.grad, a.grad_lse, DT == TT_F16 ? 0x1p14f : 1.0f, place, list,
                                        reinterpret_cast<Row *>(ws + lay.meta), totals);
    copy_rows(a.hidden, a.x_ld, a.n_rows, a.h, e, list, totals, beside<DT>(a), ws + lay.x, lay.width, stream);
    for (int64_t v0 = 0; v0 < a.v; v0 += lay.piece) backward_piece<DT>(a, lay, ws, v0, copy_w, stream);
    if (a.dhidden)
        head_place<DT><<<dim3(a.n_rows, (unsigned int)tiles_of(a.h, 1024)), 256, 0, stream>>>(reinterpret_cast<float *>(ws + lay.sums), lay.width,
                                                                                         lay.n_pad * lay.width, lay.splits, place, totals, beside<DT>(a), a.h,
                                                                                         a.dhidden, a.dx_ld);
    return status();
}

}  // namespace

size_t head_workspace_bytes(int32_t n_rows, int32_t v) { return ForwardLayout(n_rows, v).total; }

size_t head_backward_workspace_bytes(int32_t n_rows, int32_t v, int32_t h, int dtype) { return BackwardLayout::most(n_rows, v, h, dtype); }
size_t head_backward_workspace_used(int32_t n_rows, int32_t v, int32_t h, int dtype) { return BackwardLayout(n_rows, v, h, dtype).total; }

int launch_head_logprobs(const HeadArgs &a, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!workspace || workspace_bytes < head_workspace_bytes(a.n_rows, a.v)) return TT_EWORKSPACE;
    char *ws = static_cast<char *>(workspace);
    return a.dtype == TT_BF16 ? forward<TT_BF16>(a, ws, stream) : a.dtype == TT_F16 ? forward<TT_F16>(a, ws, stream) : forward<TT_F32>(a, ws, stream);
}

int launch_head_logprobs_backward(const HeadGradArgs &a, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (a.n_rows == 0) {  // dW of no rows
        if (!a.dweight) return TT_OK;
        head_zero<<<a.v, 256, 0, stream>>>(a.h, rows::element_bytes(a.dtype), static_cast<char *>(a.dweight), a.dw_ld);
        return status();
    }
    if (!workspace || workspace_bytes < head_backward_workspace_used(a.n_rows, a.v, a.h, a.dtype)) return TT_EWORKSPACE;
    char *ws = static_cast<char *>(workspace);
    return a.dtype == TT_BF16 ? backward<TT_BF16>(a, ws, stream) : a.dtype == TT_F16 ? backward<TT_F16>(a, ws, stream) : backward<TT_F32>(a, ws, stream);
}

}  // namespace tt
