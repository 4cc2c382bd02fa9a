// The output head without its logits: log probabilities of given tokens from hidden states x [n, h] and the head's
// weights W [v, h] (tt_head_logprobs), and their gradient (tt_head_logprobs_backward).
//
//   z = x W^T,  M = max z,  L = ln sum exp(beta (z - M)),  logprob = beta (z_t - M) - L
//   dz_j = beta (g ([j = t] - p_j) + q p_j),  dx = dz W,  dW = dz^T x
//
// Forward: one product by tiles (tiles.h), whose epilogue leaves each tile's largest logit and sum of exponentials for
// every row, and a second kernel that joins a row's parts.  Backward: the rows that carry a weight are gathered, with
// their transpose; then, for one piece of the vocabulary after another, the product again with an epilogue that makes dz of
// it, rounded to the operands' type (relative to the largest row weight, so that a small weight costs no digits), and two more
// products: dx += dz W (in fp32, over all pieces) and the piece's rows of dW, written once.  No atomics: results do not
// depend on scheduling.  fp32 operands are held as three bf16 parts and multiplied in six products (tiles.h).
#include <algorithm>

#include "tiles.h"

namespace tt {
namespace {

using namespace tiles;
using rows::round256;

constexpr int kTile = 128;      // rows of either side in a tile
constexpr int kAlign = 256;     // rows, tokens and pieces of the vocabulary in a workspace come in multiples of this
constexpr int kStepElements = kStepBytes / 2;
typedef Shape<kTile, kTile, 2, 2> Tile;

constexpr int64_t kSplitTiles = 768;  // workgroups that the sum over a piece's tokens is split into at most
constexpr size_t kPieceBytes = size_t(192) << 20;  // what the pieces of the vocabulary may take of the workspace

__host__ __device__ constexpr int parts_of(int dtype) { return dtype == TT_F32 ? kParts : 1; }
__host__ __device__ inline int64_t round_to(int64_t x, int64_t n) { return (x + n - 1) / n * n; }
// The type that the matrix cores are given.
template <int DT>
constexpr int kCore = DT == TT_F32 ? TT_BF16 : DT;

// A row that carries a weight, for the gradient's epilogue: p = 2^((z - m) c - l), dz = (w - g) p, and g (1 - p) + w p at
// its token; padding rows are zeros.
struct Row {
    float c, m, l, g, w;
    int32_t id;
};
struct Totals {
    int32_t rows;  // that carry a weight
    float scale;   // of the stored dz: the true one is scale times as large
};

// ------------------------------------------------------------------------------------------------ copies into parts
// A matrix's elements [r0, r0 + n_rows) x [0, cols) in the parts' layout: `out` [parts][out_rows][out_cols], rounded up with
// zeros, and its transpose `out_t` [parts][out_cols][out_rows], either of which may be null.  list: rows by their index
// in it, totals->rows of them (rounded up to a tile are written), or null.
template <int DT>
__global__ __launch_bounds__(256) void lay_out(const void *src, int64_t ld, int n_rows, int cols, const int32_t *list, const Totals *totals,
                                               uint16_t *out, int64_t out_ld, int64_t out_plane, uint16_t *out_t, int64_t t_ld, int64_t t_plane) {
    constexpr int P = parts_of(DT);
    __shared__ uint16_t block[P][64][66];
    using T = typename rows::Elem<DT>::T;
    const int r0 = (int)blockIdx.x * 64, c0 = (int)blockIdx.y * 64;
    const int count = totals ? totals->rows : n_rows;
    if (totals && r0 >= round_to(count, kTile)) return;
    const T *in = static_cast<const T *>(src);
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
        const int r = i * 4 + (int)threadIdx.x / 64, c = (int)threadIdx.x % 64;
        uint32_t part[kParts] = {0, 0, 0};
        if (r0 + r < count && c0 + c < cols) {
            const int64_t row = list ? list[r0 + r] : r0 + r;
            const T x = in[row * ld + c0 + c];
            if constexpr (DT == TT_F32) split(__uint_as_float(x), part);
            else part[0] = x;
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            block[p][r][c] = (uint16_t)part[p];
            if (out) out[p * out_plane + (int64_t)(r0 + r) * out_ld + c0 + c] = (uint16_t)part[p];
        }
    }
    if (!out_t) return;
    __syncthreads();
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
        const int c = i * 4 + (int)threadIdx.x / 64, r = (int)threadIdx.x % 64;
#pragma unroll
        for (int p = 0; p < P; ++p) out_t[p * t_plane + (int64_t)(c0 + c) * t_ld + r0 + r] = block[p][r][c];
    }
}

// ------------------------------------------------------------------------------------------------ forward
// Parts of the rows' distributions from the tokens [v0 + 128 tile, + 128), and the given tokens' logits.
template <int DT, int PASSES>
__global__ __launch_bounds__(Tile::THREADS) void head_parts(Side w, Side x, int64_t bytes, int v0, const float *inv_temp, const int32_t *ids,
                                                            Part *parts, int tile0, int n_tiles, float *token) {
    __shared__ __attribute__((aligned(16))) char lds[Tile::LDS];
    f4 acc[Tile::FM][Tile::FN];
    const int m0 = (int)blockIdx.x * kTile, n0 = (int)blockIdx.y * kTile;
    product<DT, Tile, PASSES>(w, x, m0, n0, 0, bytes, bytes, lds, acc);
    const int n_rows = x.rows, lane = (int)threadIdx.x & 63, wm = ((int)threadIdx.x >> 6) % Tile::WM;
    const int base = m0 + wm * Tile::FM * 16 + (lane >> 4) * 4;
    if (ids)
        for_blocks<Tile>(m0, n0, [&](int m, int n, int i, int j) {
            const int at = n < n_rows ? ids[n] - v0 - m : -1;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (at == q && m + q < w.rows) token[n] = acc[i][j][q];
        });
    const Part p = column_parts<Tile>(
        n0, lds, [&](int i, int j, int q) { return base + i * 16 + q < w.rows ? acc[i][j][q] : -INFINITY; },
        [&](int n) { return (n < n_rows ? rows::scale_of(inv_temp, n) : 1.0f) * rows::kLog2e; });
    const int n = n0 + (int)threadIdx.x;
    if ((int)threadIdx.x < kTile && n < n_rows) parts[(int64_t)n * n_tiles + tile0 + blockIdx.x] = p;
}

// A wave a row.
__global__ __launch_bounds__(256) void head_join(const Part *parts, int n_tiles, int n_rows, int v, const float *inv_temp, const int32_t *ids,
                                                 const float *token, float *logprob, float *lse, float *stats) {
    const int n = (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6);
    if (n >= n_rows) return;
    const float beta = rows::scale_of(inv_temp, n);
    Part r = join_row(parts + (int64_t)n * n_tiles, n_tiles, beta);
    if (((int)threadIdx.x & 63) != 0) return;
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
    for (int i = before + t; i < round_to(before, kAlign); i += 1024) out[i] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, -1};
    if (t == 0) *totals = {before, top / store_scale};
}

// dz of the piece's tokens [128 tile, + 128) for the listed rows, stored as [n][token] and [token][n].
template <int DT>
__global__ __launch_bounds__(Tile::THREADS) void head_dlogits(Side w, Side x, int64_t bytes, int v0, const Row *meta, const Totals *totals,
                                                              uint16_t *d, int64_t d_ld, int64_t d_plane, uint16_t *dt, int64_t dt_ld,
                                                              int64_t dt_plane) {
    constexpr int P = parts_of(DT);
    __shared__ __attribute__((aligned(16))) char lds[Tile::LDS];
    f4 acc[Tile::FM][Tile::FN];
    const int m0 = (int)blockIdx.x * kTile, n0 = (int)blockIdx.y * kTile;
    if (n0 >= totals->rows) return;
    product<kCore<DT>, Tile, P == 1 ? 1 : kPasses>(w, x, m0, n0, 0, bytes, bytes, lds, acc);
    for_blocks<Tile>(m0, n0, [&](int m, int n, int i, int j) {
        const Row r = meta[n];
        uint32_t part[4][kParts];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float y = fmaf(acc[i][j][q] - r.m, r.c, -r.l), p = __builtin_amdgcn_exp2f(y);
            float g = (r.w - r.g) * p;
            if (v0 + m + q == r.id) g = r.g * -expm1f(y * (float)rows::kLn2) + r.w * p;
            if (m + q >= w.rows) g = 0.0f;
            if constexpr (DT == TT_F32) split(g, part[q]);
            else part[q][0] = rows::encode<DT>(g);
        }
#pragma unroll
        for (int k = 0; k < P; ++k) {
            typedef unsigned int u2 __attribute__((ext_vector_type(2)));
            if (d) *reinterpret_cast<u2 *>(d + k * d_plane + (int64_t)n * d_ld + m) = u2{part[0][k] | part[1][k] << 16, part[2][k] | part[3][k] << 16};
            if (dt)
#pragma unroll
                for (int q = 0; q < 4; ++q) dt[k * dt_plane + (int64_t)(m + q) * dt_ld + n] = (uint16_t)part[q][k];
        }
    });
}

// dx of the listed rows over one piece of the vocabulary, split into parts of its tokens, added to what the pieces before
// gave: sums[split][n][h] in fp32.
template <int DT>
__global__ __launch_bounds__(Tile::THREADS) void head_dhidden(Side wt, Side d, int64_t bytes, int64_t split_bytes, const Totals *totals,
                                                              float *sums, int64_t ld, int64_t plane, int first) {
    __shared__ __attribute__((aligned(16))) char lds[Tile::LDS];
    f4 acc[Tile::FM][Tile::FN];
    const int m0 = (int)blockIdx.x * kTile, n0 = (int)blockIdx.y * kTile;
    if (n0 >= totals->rows) return;
    const int64_t k0 = (int64_t)blockIdx.z * split_bytes, k1 = k0 + split_bytes < bytes ? k0 + split_bytes : bytes;
    product<kCore<DT>, Tile, DT == TT_F32 ? kPasses : 1>(wt, d, m0, n0, k0, k1, bytes, lds, acc);
    float *out = sums + blockIdx.z * plane;
    for_blocks<Tile>(m0, n0, [&](int m, int n, int i, int j) {
        if (m >= ld) return;
        f4 *to = reinterpret_cast<f4 *>(out + (int64_t)n * ld + m);
        *to = first ? acc[i][j] : *to + acc[i][j];
    });
}

// The splits' sums, scaled, to the rows' places; zeros for rows without a weight.
template <int DT>
__global__ __launch_bounds__(256) void head_place(const float *sums, int64_t ld, int64_t plane, int splits, const int32_t *place, const Totals *totals,
                                                  int h, void *dhidden, int64_t out_ld) {
    using T = typename rows::Elem<DT>::T;
    const int n = (int)blockIdx.x, c = (int)(blockIdx.y * 256 + threadIdx.x);
    if (c >= h) return;
    const int at = place[n];
    float y = 0.0f;
    if (at >= 0) {
        for (int s = 0; s < splits; ++s) y += sums[s * plane + at * ld + c];
        y *= totals->scale;
    }
    static_cast<T *>(dhidden)[n * out_ld + c] = (T)rows::encode<DT>(y);
}

// A piece's rows of dW.
template <int DT>
__global__ __launch_bounds__(Tile::THREADS) void head_dweight(Side xt, Side dt, const Totals *totals, int h, void *dweight, int64_t ld) {
    __shared__ __attribute__((aligned(16))) char lds[Tile::LDS];
    f4 acc[Tile::FM][Tile::FN];
    const int m0 = (int)blockIdx.x * kTile, n0 = (int)blockIdx.y * kTile;
    const int64_t bytes = round_to(totals->rows, kStepElements) * 2;
    product<kCore<DT>, Tile, DT == TT_F32 ? kPasses : 1>(xt, dt, m0, n0, 0, bytes, bytes, lds, acc);
    const float scale = totals->scale;
    for_blocks<Tile>(m0, n0, [&](int m, int n, int i, int j) {
        if (n >= dt.rows) return;
        const float y[4] = {acc[i][j][0] * scale, acc[i][j][1] * scale, acc[i][j][2] * scale, acc[i][j][3] * scale};
        store4<DT>(static_cast<typename rows::Elem<DT>::T *>(dweight) + (int64_t)n * ld, m, h, y);
    });
}

__global__ __launch_bounds__(256) void head_zero(int h, int e, char *out, int64_t ld) {
    for (int64_t c = threadIdx.x; c < (int64_t)h * e; c += 256) out[blockIdx.x * ld * e + c] = 0;
}

unsigned int tiles_of(int64_t n) { return (unsigned int)((n + kTile - 1) / kTile); }

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
    int64_t piece;  // tokens of a piece (fp32: the weights' parts are made piece by piece)
    int64_t width;  // of a row of parts
    int n_tiles;
    size_t parts, token, x, w;
    ForwardLayout(int64_t n, int64_t v, int64_t h, int dtype) {
        n_tiles = (int)tiles_of(v);
        width = round_to(h, kStepElements);
        piece = v;
        parts = take((size_t)n * n_tiles * sizeof(Part));
        token = take((size_t)n * 4);
        x = w = 0;
        if (dtype == TT_F32) {
            const int64_t most = (int64_t)(kPieceBytes / (size_t)(kParts * width * 2));
            piece = std::min(round_to(v, kAlign), std::max<int64_t>(kAlign, most / kAlign * kAlign));
            x = take((size_t)(kParts * round_to(n, kAlign) * width * 2));
            w = take((size_t)(kParts * piece * width * 2));
        }
    }
};

struct BackwardLayout : Layout {
    int64_t n_pad, width, piece;
    int splits;
    size_t totals, place, list, meta, x, xt, w, wt, d, dt, sums;
    // most: what no number of rows up to n takes more than (fewer rows make longer pieces and more splits)
    BackwardLayout(int64_t n, int64_t v, int64_t h, int dtype, bool most = false) {
        const int64_t p = parts_of(dtype);
        n_pad = round_to(n, kAlign);
        width = round_to(h, kStepElements);
        const int64_t row = p * (2 * n_pad + (dtype == TT_F32 ? 2 : 1) * width) * 2, all = round_to(v, kAlign);
        const int64_t fit = most ? ((int64_t)kPieceBytes + row - 1) / row : (int64_t)kPieceBytes / row / kAlign * kAlign;
        piece = std::min(all, std::max<int64_t>(kAlign, fit));
        const int64_t tiles = (int64_t)tiles_of(n_pad) * tiles_of(width);
        splits = (int)std::min<int64_t>(std::max<int64_t>(1, most ? (kSplitTiles + tiles - 1) / tiles : kSplitTiles / tiles), std::max<int64_t>(1, all / 1024));
        totals = take(sizeof(Totals));
        place = take((size_t)n * 4);
        list = take((size_t)n * 4);
        meta = take((size_t)n_pad * sizeof(Row));
        x = take((size_t)(p * n_pad * width * 2));
        xt = take((size_t)(p * n_pad * width * 2));
        w = dtype == TT_F32 ? take((size_t)(p * piece * width * 2)) : 0;
        wt = take((size_t)(p * piece * width * 2));
        d = take((size_t)(p * piece * n_pad * 2));
        dt = take((size_t)(p * piece * n_pad * 2));
        sums = take((size_t)(splits * n_pad * width * 4));
    }
};

int status() { return hipGetLastError() == hipSuccess ? TT_OK : TT_ELAUNCH; }

template <int DT>
int forward(const HeadArgs &a, char *ws, hipStream_t stream) {
    const ForwardLayout lay(a.n_rows, a.v, a.h, a.dtype);
    const int64_t e = rows::element_bytes(DT);
    Part *parts = reinterpret_cast<Part *>(ws + lay.parts);
    float *token = reinterpret_cast<float *>(ws + lay.token);
    const int32_t *ids = a.logprob ? a.ids : nullptr;
    if constexpr (DT != TT_F32) {
        const Side w = {static_cast<const char *>(a.weight), a.w_ld * e, 0, a.v}, x = {static_cast<const char *>(a.hidden), a.x_ld * e, 0, a.n_rows};
        head_parts<DT, 1><<<dim3(tiles_of(a.v), tiles_of(a.n_rows)), Tile::THREADS, 0, stream>>>(w, x, a.h * e, 0, a.inv_temp, ids, parts, 0,
                                                                                              lay.n_tiles, token);
    } else {
        uint16_t *xp = reinterpret_cast<uint16_t *>(ws + lay.x), *wp = reinterpret_cast<uint16_t *>(ws + lay.w);
        const int64_t x_plane = round_to(a.n_rows, kAlign) * lay.width, w_plane = lay.piece * lay.width;
        const unsigned int wide = (unsigned int)(lay.width / 64);
        lay_out<DT><<<dim3((unsigned int)(round_to(a.n_rows, 64) / 64), wide), 256, 0, stream>>>(a.hidden, a.x_ld, a.n_rows, a.h, nullptr, nullptr, xp,
                                                                                             lay.width, x_plane, nullptr, 0, 0);
        for (int64_t v0 = 0; v0 < a.v; v0 += lay.piece) {
            const int here = (int)std::min<int64_t>(lay.piece, a.v - v0);
            lay_out<DT><<<dim3((unsigned int)(round_to(here, 64) / 64), wide), 256, 0, stream>>>(
                static_cast<const float *>(a.weight) + v0 * a.w_ld, a.w_ld, here, a.h, nullptr, nullptr, wp, lay.width, w_plane, nullptr, 0, 0);
            const Side w = {reinterpret_cast<const char *>(wp), lay.width * 2, w_plane * 2, here};
            const Side x = {reinterpret_cast<const char *>(xp), lay.width * 2, x_plane * 2, a.n_rows};
            head_parts<TT_BF16, kPasses><<<dim3(tiles_of(here), tiles_of(a.n_rows)), Tile::THREADS, 0, stream>>>(
                w, x, lay.width * 2, (int)v0, a.inv_temp, ids, parts, (int)(v0 / kTile), lay.n_tiles, token);
        }
    }
    head_join<<<(unsigned int)((a.n_rows + 3) / 4), 256, 0, stream>>>(parts, lay.n_tiles, a.n_rows, a.v, a.inv_temp, a.ids, token, a.logprob, a.lse,
                                                                   a.stats);
    return status();
}

template <int DT>
int backward(const HeadGradArgs &a, char *ws, hipStream_t stream) {
    const BackwardLayout lay(a.n_rows, a.v, a.h, a.dtype);
    const int64_t e = rows::element_bytes(DT);
    Totals *totals = reinterpret_cast<Totals *>(ws + lay.totals);
    int32_t *place = reinterpret_cast<int32_t *>(ws + lay.place), *list = reinterpret_cast<int32_t *>(ws + lay.list);
    Row *meta = reinterpret_cast<Row *>(ws + lay.meta);
    const auto part = [&](size_t at) { return reinterpret_cast<uint16_t *>(ws + at); };
    uint16_t *x = part(lay.x), *xt = part(lay.xt), *wp = part(lay.w), *wt = part(lay.wt), *d = part(lay.d), *dt = part(lay.dt);
    float *sums = reinterpret_cast<float *>(ws + lay.sums);
    const int64_t x_plane = lay.n_pad * lay.width, w_plane = lay.piece * lay.width, d_plane = lay.piece * lay.n_pad;
    const unsigned int wide = (unsigned int)(lay.width / 64);
    head_select<<<1, 1024, 0, stream>>>(a.n_rows, a.v, a.inv_temp, a.ids, a.stats, a.grad, a.grad_lse, DT == TT_F16 ? 0x1p14f : 1.0f, place, list, meta,
                                        totals);
    lay_out<DT><<<dim3((unsigned int)(lay.n_pad / 64), wide), 256, 0, stream>>>(a.hidden, a.x_ld, a.n_rows, a.h, list, totals, x, lay.width, x_plane,
                                                                             a.dweight ? xt : nullptr, lay.n_pad, x_plane);
    const Side xs = {reinterpret_cast<const char *>(x), lay.width * 2, x_plane * 2, (int)lay.n_pad};
    const Side xts = {reinterpret_cast<const char *>(xt), lay.n_pad * 2, x_plane * 2, (int)lay.width};
    for (int64_t v0 = 0; v0 < a.v; v0 += lay.piece) {
        const int here = (int)std::min<int64_t>(lay.piece, a.v - v0);
        const char *weight = static_cast<const char *>(a.weight) + v0 * a.w_ld * e;
        if (a.dhidden || DT == TT_F32)
            lay_out<DT><<<dim3((unsigned int)(round_to(here, 64) / 64), wide), 256, 0, stream>>>(
                weight, a.w_ld, here, a.h, nullptr, nullptr, DT == TT_F32 ? wp : nullptr, lay.width, w_plane, a.dhidden ? wt : nullptr, lay.piece, w_plane);
        const Side ws_ = DT == TT_F32 ? Side{reinterpret_cast<const char *>(wp), lay.width * 2, w_plane * 2, here} : Side{weight, a.w_ld * e, 0, here};
        head_dlogits<DT><<<dim3(tiles_of(here), tiles_of(a.n_rows)), Tile::THREADS, 0, stream>>>(
            ws_, xs, DT == TT_F32 ? lay.width * 2 : a.h * e, (int)v0, meta, totals, a.dhidden ? d : nullptr, lay.piece, d_plane, a.dweight ? dt : nullptr,
            lay.n_pad, d_plane);
        if (a.dhidden) {
            const int64_t bytes = round_to(here, kStepElements) * 2, split = round_to((bytes + lay.splits - 1) / lay.splits, kStepBytes);
            const Side wts = {reinterpret_cast<const char *>(wt), lay.piece * 2, w_plane * 2, (int)lay.width};
            const Side ds = {reinterpret_cast<const char *>(d), lay.piece * 2, d_plane * 2, (int)lay.n_pad};
            head_dhidden<DT><<<dim3(tiles_of(lay.width), tiles_of(a.n_rows), lay.splits), Tile::THREADS, 0, stream>>>(
                wts, ds, bytes, split, totals, sums, lay.width, x_plane, v0 == 0);
        }
        if (a.dweight) {
            const Side dts = {reinterpret_cast<const char *>(dt), lay.n_pad * 2, d_plane * 2, here};
            head_dweight<DT><<<dim3(tiles_of(a.h), tiles_of(here)), Tile::THREADS, 0, stream>>>(
                xts, dts, totals, a.h, static_cast<char *>(a.dweight) + v0 * a.dw_ld * e, a.dw_ld);
        }
    }
    if (a.dhidden)
        head_place<DT><<<dim3(a.n_rows, (unsigned int)((a.h + 255) / 256)), 256, 0, stream>>>(sums, lay.width, x_plane, lay.splits, place, totals, a.h,
                                                                                         a.dhidden, a.dx_ld);
    return status();
}

}  // namespace

size_t head_workspace_bytes(int32_t n_rows, int32_t v, int32_t h, int dtype) { return ForwardLayout(n_rows, v, h, dtype).total; }

size_t head_backward_workspace_bytes(int32_t n_rows, int32_t v, int32_t h, int dtype) { return BackwardLayout(n_rows, v, h, dtype, true).total; }
size_t head_backward_workspace_used(int32_t n_rows, int32_t v, int32_t h, int dtype) { return BackwardLayout(n_rows, v, h, dtype).total; }

int launch_head_logprobs(const HeadArgs &a, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!workspace || workspace_bytes < head_workspace_bytes(a.n_rows, a.v, a.h, a.dtype)) return TT_EWORKSPACE;
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
