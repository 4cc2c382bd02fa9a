// 8-bit integers: rows quantised with a scale each (tt_quantize_i8), and their matrix product with scales for each token
// and channel (tt_matmul_i8), which is an output head in 8 bits where the rows' log-sum-exp is wanted beside the logits.
//
//   scale_i = max_k |x_ik| / 127,  q_ik = rint(x_ik / scale_i)
//   y_ij = sx_i sw_j sum_k q_ik w_jk (+ bias_j)
#include <algorithm>

#include "tiles.h"

namespace tt {
namespace {

using namespace tiles;
using rows::round256;

typedef Shape<128, 128, 2, 2> Any;  // of the product of matrices that lie in any way
constexpr int kRowsPerLaunch = 1 << 14;
constexpr int64_t kGroupsPerLaunch = 1 << 20;  // of the quantisation: up to 1,024 threads each, of 2^32 that a launch can have

// fp32 quotients x / s rounded as a division rounds them, from r = 1 / s correctly rounded (Markstein 1990: a product and one
// correction by the exact remainder), where s is far from fp32's ends.  A tiny x leaves a remainder that is not exact, and a
// quotient that rounds to 0 all the same.
__device__ __forceinline__ float quotient(float x, float s, float r) {
    const float y = x * r;
    return fmaf(fmaf(-y, s, x), r, y);
}

// Rows quantised by WAVES waves each, 4 / WAVES rows to a workgroup (of 256 threads, WAVES = 16: 1,024): 16 bytes a
// lane and load.  NV > 0: the row stays in NV registers' worth of loads; 0: it is read again.  Bound by memory: 8,192 x 4,096
// bf16, 101 MB, 18.3 us (5.5 TB/s), fp32, 168 MB, 28.2 (6.0); 2,048 x 16,384 bf16, 101 MB, 18.4; 512 x 131,071 bf16, read twice, 67
// (3.0 TB/s of the 201 MB that one reading would be).
template <int DT, int WAVES, int NV>
__global__ __launch_bounds__(WAVES == 16 ? 1024 : 256) void quantize_rows(int n_rows, int k, const char *x, int64_t ld, int8_t *q, int64_t q_ld, float *scale) {
    constexpr int E = DT == TT_F32 ? 4 : 2, PER = 16 / E, ROWS = WAVES == 16 ? 1 : 4 / WAVES, LANES = WAVES * 64;
    const int lane = (int)threadIdx.x % LANES, wave = (int)threadIdx.x / 64;
    const int64_t n = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
    if (WAVES == 1 && n >= n_rows) return;
    const char *row = x + n * ld;
    const auto load = [&](int i) {
        const int at = i * PER;
        if (at + PER <= k) return (u4)*reinterpret_cast<const u4b *>(row + (int64_t)at * E);
        return at < k ? load_some(row + (int64_t)at * E, (k - at) * E) : u4{0, 0, 0, 0};
    };
    // the largest size, as bits: those of a NaN or an infinity are above all others
    uint32_t top = 0;
    const auto add = [&](u4 v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (DT == TT_F32) top = max(top, v[j] & 0x7FFFFFFFu);
            else top = max(top, max(v[j] & 0x7FFFu, v[j] >> 16 & 0x7FFFu));
        }
    };
    u4 held[NV ? NV : 1];
    const int vectors = (k + PER - 1) / PER;
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) held[i] = i * LANES + lane < vectors ? load(i * LANES + lane) : u4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NV; ++i) add(held[i]);
    } else {
        for (int i = lane; i < vectors; i += LANES) add(load(i));
    }
    top = rows::wave_max(top);
    if constexpr (WAVES > 1) {
        __shared__ uint32_t tops[16];
        if (((int)threadIdx.x & 63) == 0) tops[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = max(top, tops[w]);
    }
    const float most = rows::decode<DT>(top), s = most / 127.0f;
    const bool none = !(most < INFINITY) || s == 0.0f, plain = s > 0x1p-100f && s < 0x1p100f;
    const float r = 1.0f / s;
    int8_t *out = q + n * q_ld;
    const auto store = [&](int i, u4 v) {
        const int at = i * PER;
        uint32_t b[PER / 4];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            const float f = rows::value<DT>(w, j);
            const float y = plain ? quotient(f, s, r) : fminf(fmaxf(f / s, -127.0f), 127.0f);
            const uint32_t c = none ? 0 : (uint32_t)(int)rintf(y) & 0xFFu;
            b[j / 4] = j % 4 ? b[j / 4] | c << (j % 4 * 8) : c;
        }
        if (at + PER <= k) {
            typedef unsigned int u1b __attribute__((aligned(1)));
            typedef unsigned int u2b __attribute__((ext_vector_type(2), aligned(1)));
            if constexpr (PER == 8) *reinterpret_cast<u2b *>(out + at) = u2b{b[0], b[1]};
            else *reinterpret_cast<u1b *>(out + at) = b[0];
        } else {
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (at + j < k) out[at + j] = (int8_t)(b[j / 4] >> (j % 4 * 8));
        }
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES + lane < vectors) store(i * LANES + lane, held[i]);
    } else {
        for (int i = lane; i < vectors; i += LANES) store(i, load(i));
    }
    if (lane == 0) scale[n] = most < INFINITY ? s : NAN;
}

// Rows of up to 8 KB (16 bits: 4,096 elements) in one wave's registers, of up to 32 KB in four waves', longer ones by 16 waves,
// read twice.
template <int DT>
void quantize(const QuantizeI8Args &a, hipStream_t stream) {
    constexpr int per = DT == TT_F32 ? 4 : 8;
    const int vectors = (a.k + per - 1) / per;
    const auto run = [&](auto kernel, int rows, int threads) {
        const int64_t ld = a.ld * rows::element_bytes(DT), most = kGroupsPerLaunch * rows;
        for (int64_t n0 = 0; n0 < a.n_rows; n0 += most) {
            const int n = (int)std::min<int64_t>(most, a.n_rows - n0);
            kernel<<<(unsigned int)((n + rows - 1) / rows), threads, 0, stream>>>(n, a.k, static_cast<const char *>(a.x) + n0 * ld, ld, a.q + n0 * a.q_ld,
                                                                                 a.q_ld, a.scale + n0);
        }
    };
    if (vectors <= 64) run(quantize_rows<DT, 1, 1>, 4, 256);
    else if (vectors <= 128) run(quantize_rows<DT, 1, 2>, 4, 256);
    else if (vectors <= 256) run(quantize_rows<DT, 1, 4>, 4, 256);
    else if (vectors <= 512) run(quantize_rows<DT, 1, 8>, 4, 256);
    else if (vectors <= 1024) run(quantize_rows<DT, 4, 4>, 1, 256);
    else if (vectors <= 2048) run(quantize_rows<DT, 4, 8>, 1, 256);
    else run(quantize_rows<DT, 16, 0>, 1, 1024);
}

struct Scales {
    const float *x, *w, *bias, *inv_temp;
};

// A tile's scales and biases of its rows m in LDS: [rows] of either, ones and zeros past the end.
template <typename S>
__device__ __forceinline__ void stage_scales(const Scales &scales, int m0, int m_end, float *lds) {
    for (int t = (int)threadIdx.x; t < S::TM; t += S::THREADS) {
        const bool in = m0 + t < m_end;
        lds[t] = in ? scales.w[m0 + t] : 1.0f;
        lds[S::TM + t] = in && scales.bias ? scales.bias[m0 + t] : 0.0f;
    }
    __syncthreads();
}

// Four results of a column with scale sx, from the tile's row `at` on.
template <typename S>
__device__ __forceinline__ void scaled(const i4 &sum, float sx, const float *lds, int at, bool bias, float (&y)[4]) {
    const f4 sw = *reinterpret_cast<const f4 *>(lds + at);
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] = (float)sum[q] * sx * sw[q];
    if (!bias) return;
    const f4 b = *reinterpret_cast<const f4 *>(lds + S::TM + at);
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] += b[q];
}

// The parts of the rows' log-sum-exp from the results as they are written, left in acc as fp32 bits.
template <typename S>
__device__ __forceinline__ void leave_parts(const Side &x, int m0, int n0, const i4 (&acc)[S::FM][S::FN], const Scales &scales, Part *parts, int n_tiles, char *lds) {
    const int n_rows = x.rows;
    const Part p = column_parts<S, false>(
        n0, lds, [&](int i, int j, int q) { return __int_as_float(acc[i][j][q]); },
        [&](int n) { return (n < n_rows ? rows::scale_of(scales.inv_temp, n) : 1.0f) * rows::kLog2e; });
    const int n = n0 + (int)threadIdx.x;
    if ((int)threadIdx.x < S::TN && n < n_rows) parts[(int64_t)n * n_tiles + m0 / S::TM] = p;
}

template <int DT, bool LSE, typename S>
__global__ __launch_bounds__(S::THREADS, 2) void product_i8(Side w, Side x, int mt, int nt, Scales scales, void *out, int64_t out_ld, Part *parts) {
    TT_TILE_LDS(S);
    i4 acc[S::FM][S::FN];
    int m0, n0;
    tile_of((int)blockIdx.x, (int)gridDim.x, mt, nt, m0, n0);
    m0 *= S::TM;
    n0 *= S::TN;
    Product<kI8, false, false, S>::run(w, x, m0, n0, 0, w.bytes / kStepBytes, lds, acc);
    using T = typename rows::Elem<DT>::T;
    float *by_row = reinterpret_cast<float *>(lds + 2 * S::TM * kStepBytes);
    stage_scales<S>(scales, m0, w.rows, by_row);
    float sx[S::FN];
    for_columns<S>(n0, [&](int c, int j) { sx[j] = c < x.rows ? scales.x[c] : 0.0f; });
    store_tile<DT, S>(m0, w.rows, n0, x.rows, lds, lds + S::TM * kStepBytes, [&](int, int j, int row, int i, float (&y)[4]) {
        scaled<S>(acc[i][j], sx[j], by_row, row - m0, scales.bias != nullptr, y);
        if constexpr (LSE)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[i][j][q] = __float_as_int(row + q < w.rows ? rows::decode<DT>(rows::encode<DT>(y[q])) : -INFINITY);
    }, [&](int c) { return static_cast<T *>(out) + (int64_t)c * out_ld; });
    if constexpr (LSE) {
        __syncthreads();
        leave_parts<S>(x, m0, n0, acc, scales, parts, mt, lds);
    }
}

template <int DT, bool LSE>
__global__ __launch_bounds__(Any::THREADS) void product_i8_any(Side w, Side x, Scales scales, void *out, int64_t out_ld, Part *parts) {
    __shared__ __attribute__((aligned(16))) char lds[Any::LDS];
    i4 acc[Any::FM][Any::FN];
    const int m0 = (int)blockIdx.x * Any::TM, n0 = (int)blockIdx.y * Any::TN;
    product_any<kI8, Any>(w, x, m0, n0, lds, acc);
    using T = typename rows::Elem<DT>::T;
    __shared__ __attribute__((aligned(16))) float by_row[2 * Any::TM];
    stage_scales<Any>(scales, m0, w.rows, by_row);
    for_columns<Any>(n0, [&](int n, int j) {
        const float sx = n < x.rows ? scales.x[n] : 0.0f;
        for_rows<Any>(m0, [&](int m, int i) {
            float y[4];
            scaled<Any>(acc[i][j], sx, by_row, m - m0, scales.bias != nullptr, y);
            if constexpr (LSE)
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[i][j][q] = __float_as_int(m + q < w.rows ? rows::decode<DT>(rows::encode<DT>(y[q])) : -INFINITY);
            if (n < x.rows) store4<DT>(static_cast<T *>(out) + (int64_t)n * out_ld, m, w.rows, y);
        });
    });
    if constexpr (LSE) leave_parts<Any>(x, m0, n0, acc, scales, parts, gridDim.x, lds);
}

// Up to 16 rows.
template <int DT, bool LSE, bool WHOLE>
__global__ __launch_bounds__(kThinThreads, 4) void product_i8_few(Side w, Side x, Scales scales, void *out, int64_t out_ld, Part *parts) {
    __shared__ __attribute__((aligned(16))) char lds[kThinLds];
    __shared__ float sums[8][256];
    using T = typename rows::Elem<DT>::T;
    const int column = (int)threadIdx.x >> 4;
    const bool there = column < x.rows;
    const float c = LSE && there ? rows::scale_of(scales.inv_temp, column) * rows::kLog2e : 0.0f, sx = there ? scales.x[column] : 0.0f;
    T *row = static_cast<T *>(out) + column * out_ld;
    Part p = {-INFINITY, 0.0f};
    product_few<kI8, WHOLE>(w, x, lds, sums, [&](int m, int, int sum) {
        if (!there || m >= w.rows) return;
        float y = (float)sum * sx * scales.w[m];
        if (scales.bias) y += scales.bias[m];
        const uint32_t bits = rows::encode<DT>(y);
        row[m] = (T)bits;
        if constexpr (LSE) add_part<false>(p, rows::decode<DT>(bits), c);  // of the results as they are written
    });
    if constexpr (LSE) {
        p = join_quarter<false>(p, c);
        if (((int)threadIdx.x & 15) == 0 && there) parts[(int64_t)column * gridDim.x + blockIdx.x] = p;
    }
}

// Few rows.
template <int DT, bool LSE, int FN>
__global__ __launch_bounds__(kThinThreads, 4) void product_i8_thin(Side w, Side x, Scales scales, void *out, int64_t out_ld, Part *parts) {
    __shared__ __attribute__((aligned(16))) char lds[kThinLds];
    using T = typename rows::Elem<DT>::T;
    const int column = (int)threadIdx.x & 15;
    const auto scale = [&](int n) { return (n < x.rows ? rows::scale_of(scales.inv_temp, n) : 1.0f) * rows::kLog2e; };
    Part p[FN];
    float c[FN], sx[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        p[j] = {-INFINITY, 0.0f};
        c[j] = LSE ? scale(j * 16 + column) : 0.0f;
        sx[j] = j * 16 + column < x.rows ? scales.x[j * 16 + column] : 0.0f;
    }
    product_thin<kI8, FN>(w, x, lds, [&](int m, i4 (&acc)[FN]) {
        float sw[4], bias[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            sw[q] = scales.w[min(m + q, w.rows - 1)];
            bias[q] = scales.bias ? scales.bias[min(m + q, w.rows - 1)] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int n = j * 16 + column;
            float y[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                y[q] = (float)acc[j][q] * sx[j] * sw[q];
                if (scales.bias) y[q] += bias[q];
            }
            if (n < x.rows && m < w.rows) store4<DT>(static_cast<T *>(out) + (int64_t)n * out_ld, m, w.rows, y);
            if constexpr (LSE) {  // of the results as they are written
#pragma unroll
                for (int q = 0; q < 4; ++q) y[q] = m + q < w.rows ? rows::decode<DT>(rows::encode<DT>(y[q])) : -INFINITY;
                add_part<false>(p[j], y, c[j]);
            }
        }
    });
    if constexpr (LSE) {
        const Part r = join_lanes<FN, false>(p, x.rows, lds, scale);
        if ((int)threadIdx.x < x.rows) parts[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = r;
    }
}

// A workgroup a row.
__global__ __launch_bounds__(256) void join_lse(const Part *parts, int n_tiles, const float *inv_temp, float *lse) {
    const int n = (int)blockIdx.x;
    const float beta = rows::scale_of(inv_temp, n);
    const Part r = join_row(parts + (int64_t)n * n_tiles, n_tiles, beta);
    if (threadIdx.x == 0) lse[n] = rows::sound(beta) && r.s == r.s ? fmaf(beta, r.m, r.s) : NAN;
}

template <int DT, bool LSE>
int multiply(const MatmulI8Args &a, Part *parts, hipStream_t stream) {
    const Side w = {reinterpret_cast<const char *>(a.w), a.w_ld, a.n_cols, a.k}, x = {reinterpret_cast<const char *>(a.x), a.x_ld, a.n_rows, a.k};
    const int64_t e = rows::element_bytes(DT);
    int n_tiles = (a.n_cols + 255) / 256;
    if (a.n_rows <= kThinMost) {
        n_tiles = thin_groups(a.n_rows, a.n_cols);
        const Scales scales = {a.x_scale, a.w_scale, a.bias, a.inv_temp};
        const auto run = [&](auto kernel) { kernel<<<n_tiles, kThinThreads, 0, stream>>>(w, x, scales, a.out, a.out_ld, parts); };
        if (a.n_rows <= kFewMost && w.bytes % kFewBytes == 0) run(product_i8_few<DT, LSE, true>);
        else if (a.n_rows <= kFewMost) run(product_i8_few<DT, LSE, false>);
        else if (a.n_rows <= 32) run(product_i8_thin<DT, LSE, 2>);
        else run(product_i8_thin<DT, LSE, 4>);
    } else if (whole_steps(w) && whole_steps(x)) {
        for (int64_t n0 = 0; n0 < a.n_rows; n0 += kRowsPerLaunch) {
            const int n = (int)std::min<int64_t>(kRowsPerLaunch, a.n_rows - n0);
            const Side part = {x.p + n0 * x.ld, x.ld, n, x.bytes};
            const Scales scales = {a.x_scale + n0, a.w_scale, a.bias, a.inv_temp ? a.inv_temp + n0 : nullptr};
            with_shape<kI8, kForward>(a.n_cols, std::min<int64_t>(kRowsPerLaunch, a.n_rows), [&](auto shape) {
                typedef decltype(shape) S;
                const int nt = (n + S::TN - 1) / S::TN;
                n_tiles = (a.n_cols + S::TM - 1) / S::TM;
                product_i8<DT, LSE, S><<<(unsigned int)(n_tiles * nt), S::THREADS, 0, stream>>>(
                    w, part, n_tiles, nt, scales, static_cast<char *>(a.out) + n0 * a.out_ld * e, a.out_ld, parts + n0 * n_tiles);
            });
        }
    } else {
        n_tiles = (a.n_cols + Any::TM - 1) / Any::TM;
        product_i8_any<DT, LSE><<<dim3(n_tiles, (a.n_rows + Any::TN - 1) / Any::TN), Any::THREADS, 0, stream>>>(
            w, x, Scales{a.x_scale, a.w_scale, a.bias, a.inv_temp}, a.out, a.out_ld, parts);
    }
    if (LSE) join_lse<<<(unsigned int)a.n_rows, 256, 0, stream>>>(parts, n_tiles, a.inv_temp, a.lse);
    return hipGetLastError() == hipSuccess ? TT_OK : TT_ELAUNCH;
}

template <int DT>
int multiply(const MatmulI8Args &a, Part *parts, hipStream_t stream) {
    return a.lse ? multiply<DT, true>(a, parts, stream) : multiply<DT, false>(a, parts, stream);
}

}  // namespace

int launch_quantize_i8(const QuantizeI8Args &a, hipStream_t stream) {
    if (a.dtype == TT_BF16) quantize<TT_BF16>(a, stream);
    else if (a.dtype == TT_F16) quantize<TT_F16>(a, stream);
    else quantize<TT_F32>(a, stream);
    return hipGetLastError() == hipSuccess ? TT_OK : TT_ELAUNCH;
}

size_t matmul_i8_workspace_bytes(int32_t n_rows, int32_t n_cols, bool lse) {
    return lse ? round256(most_parts(n_rows, n_cols) * sizeof(Part)) : 0;
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
