// 8-bit integers: rows quantised with a scale each (tt_quantize_i8), and their matrix product with scales for each token
// and channel (tt_matmul_i8), which is an output head in 8 bits where the rows' log-sum-exp is wanted beside the logits.
//
//   scale_i = max_k |x_ik| / 127,  q_ik = rint(x_ik / scale_i)
//   y_ij = sx_i sw_j sum_k q_ik w_jk (+ bias_j)
#include "tiles.h"

namespace tt {
namespace {

using namespace tiles;
using rows::round256;

constexpr int kTile = 128;
typedef Shape<kTile, kTile, 2, 2> Tile;

// A workgroup a row, read twice (the second time from a cache).
template <int DT>
__global__ __launch_bounds__(256) void quantize_rows(int k, const void *x, int64_t ld, int8_t *q, int64_t q_ld, float *scale) {
    using T = typename rows::Elem<DT>::T;
    __shared__ float tops[4];
    __shared__ int bad[4];
    const int64_t n = blockIdx.x;
    const T *row = static_cast<const T *>(x) + n * ld;
    float top = 0.0f;
    bool odd = false;
    for (int i = (int)threadIdx.x; i < k; i += 256) {
        const float f = fabsf(rows::decode<DT>(row[i]));
        odd |= !(f < INFINITY);
        top = fmaxf(top, f);
    }
    top = rows::wave_max(top);
    const bool any = __ballot(odd) != 0;
    if (((int)threadIdx.x & 63) == 0) {
        tops[threadIdx.x >> 6] = top;
        bad[threadIdx.x >> 6] = any;
    }
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const bool none = bad[0] | bad[1] | bad[2] | bad[3];
    const float s = top / 127.0f;
    for (int i = (int)threadIdx.x; i < k; i += 256) {
        const float y = rows::decode<DT>(row[i]) / s;
        q[n * q_ld + i] = none || s == 0.0f ? 0 : (int8_t)rintf(fminf(fmaxf(y, -127.0f), 127.0f));
    }
    if (threadIdx.x == 0) scale[n] = none ? NAN : s;
}

template <int DT, bool LSE>
__global__ __launch_bounds__(Tile::THREADS) void product_i8(Side w, Side x, int k, const float *x_scale, const float *w_scale, const float *bias,
                                                            void *out, int64_t out_ld, const float *inv_temp, Part *parts, int n_tiles) {
    __shared__ __attribute__((aligned(16))) char lds[Tile::LDS];
    i4 acc[Tile::FM][Tile::FN];
    using T = typename rows::Elem<DT>::T;
    const int m0 = (int)blockIdx.x * kTile, n0 = (int)blockIdx.y * kTile;
    product<kI8, Tile, 1>(w, x, m0, n0, 0, k, k, lds, acc);
    const int n_rows = x.rows;
    float y[Tile::FM][Tile::FN][4];
    for_blocks<Tile>(m0, n0, [&](int m, int n, int i, int j) {
        const float sx = n < n_rows ? x_scale[n] : 0.0f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float f = -INFINITY;
            if (m + q < w.rows) {
                f = (float)acc[i][j][q] * sx * w_scale[m + q];
                if (bias) f += bias[m + q];
            }
            y[i][j][q] = f;
        }
        if (n < n_rows) store4<DT>(static_cast<T *>(out) + (int64_t)n * out_ld, m, w.rows, y[i][j]);
    });
    if constexpr (LSE) {
        const Part p = column_parts<Tile>(
            n0, lds, [&](int i, int j, int q) { return rows::decode<DT>(rows::encode<DT>(y[i][j][q])); },
            [&](int n) { return (n < n_rows ? rows::scale_of(inv_temp, n) : 1.0f) * rows::kLog2e; });
        const int n = n0 + (int)threadIdx.x;
        if ((int)threadIdx.x < kTile && n < n_rows) parts[(int64_t)n * n_tiles + blockIdx.x] = p;
    }
}

// A wave a row.
__global__ __launch_bounds__(256) void join_lse(const Part *parts, int n_tiles, int n_rows, const float *inv_temp, float *lse) {
    const int n = (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6);
    if (n >= n_rows) return;
    const float beta = rows::scale_of(inv_temp, n);
    const Part r = join_row(parts + (int64_t)n * n_tiles, n_tiles, beta);
    if (((int)threadIdx.x & 63) == 0) lse[n] = rows::sound(beta) && r.s == r.s ? fmaf(beta, r.m, r.s) : NAN;
}

template <int DT>
int multiply(const MatmulI8Args &a, Part *parts, hipStream_t stream) {
    const Side w = {reinterpret_cast<const char *>(a.w), a.w_ld, 0, a.n_cols}, x = {reinterpret_cast<const char *>(a.x), a.x_ld, 0, a.n_rows};
    const int n_tiles = (a.n_cols + kTile - 1) / kTile;
    const dim3 grid(n_tiles, (a.n_rows + kTile - 1) / kTile);
    if (a.lse) product_i8<DT, true><<<grid, Tile::THREADS, 0, stream>>>(w, x, a.k, a.x_scale, a.w_scale, a.bias, a.out, a.out_ld, a.inv_temp, parts, n_tiles);
    else product_i8<DT, false><<<grid, Tile::THREADS, 0, stream>>>(w, x, a.k, a.x_scale, a.w_scale, a.bias, a.out, a.out_ld, a.inv_temp, parts, n_tiles);
    if (a.lse) join_lse<<<(unsigned int)((a.n_rows + 3) / 4), 256, 0, stream>>>(parts, n_tiles, a.n_rows, a.inv_temp, a.lse);
    return hipGetLastError() == hipSuccess ? TT_OK : TT_ELAUNCH;
}

}  // namespace

int launch_quantize_i8(const QuantizeI8Args &a, hipStream_t stream) {
    const auto run = [&](auto kernel) { kernel<<<(unsigned int)a.n_rows, 256, 0, stream>>>(a.k, a.x, a.ld, a.q, a.q_ld, a.scale); };
    if (a.dtype == TT_BF16) run(quantize_rows<TT_BF16>);
    else if (a.dtype == TT_F16) run(quantize_rows<TT_F16>);
    else run(quantize_rows<TT_F32>);
    return hipGetLastError() == hipSuccess ? TT_OK : TT_ELAUNCH;
}

size_t matmul_i8_workspace_bytes(int32_t n_rows, int32_t n_cols, bool lse) {
    return lse ? round256((size_t)n_rows * ((n_cols + kTile - 1) / kTile) * sizeof(Part)) : 0;
}

int launch_matmul_i8(const MatmulI8Args &a, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const size_t need = matmul_i8_workspace_bytes(a.n_rows, a.n_cols, a.lse != nullptr);
    if (need && (!workspace || workspace_bytes < need)) return TT_EWORKSPACE;
    Part *parts = static_cast<Part *>(workspace);
    return a.out_dtype == TT_BF16 ? multiply<TT_BF16>(a, parts, stream)
           : a.out_dtype == TT_F16 ? multiply<TT_F16>(a, parts, stream)
                                   : multiply<TT_F32>(a, parts, stream);
}

}  // namespace tt
