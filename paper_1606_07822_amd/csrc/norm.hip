// Layer norm of rows, forward and backward.
//
//   mu = sum x / d,  r = 1 / sqrt(sum (x - mu)^2 / d + eps),  h = (x - mu) r,  y = h w + b
//   a = dy w,  dx = r (a - sum a / d - h sum(a h) / d),  dw = sum over rows of dy h,  db = sum over rows of dy
//
// Both passes read each row once into registers (the variance is taken from the centred values there, not from a
// difference of sums), so what bounds them is memory: 2 row transfers forward, 3 backward. A row is held by LPR
// lanes, each with NCH vectors of 16 bytes: 16 lanes for narrow rows, so that a wavefront's loads are full at 50 to
// 300 columns, a wavefront or a workgroup for wide ones: with few elements a lane there are enough wavefronts to keep
// memory busy (the forward pass of 16,384 rows of 4,096 bf16 columns takes 62 us with 256 lanes a row, 4.3 TB/s, and 170
// with 64; the backward pass of 65,536 rows of 300 floats 54 us, of which the rows 45, 5.5 TB/s). All sums are fp32, in a
// fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "w2v_ops.h"

namespace w2v {
namespace {

constexpr int kNormThreads = 256;

template <class T>
constexpr int kVec = 16 / sizeof(T);

// Sums of N values over the LPR lanes of a row, in every one of them. Rows of more than a wavefront go through LDS;
// `turn` alternates its two halves, so that one barrier a sum is enough.
template <int LPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int &turn) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = row_sum(v[k]);
    if constexpr (LPR > 16) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = rows_sum(v[k]);
    }
    if constexpr (LPR > kWave) {
        constexpr int kWaves = LPR / kWave;
        __shared__ float part[2][N][kWaves];
        const int wid = static_cast<int>(threadIdx.x) / kWave;
        if (lane_id() == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) part[turn][k][wid] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v[k] += part[turn][k][w];
        }
        turn ^= 1;
    }
}

// Weight or bias columns: in fp32, or in the rows' type (w_type tells).
template <class T, int N, bool WHOLE>
__device__ __forceinline__ void load_affine(const void *w, int32_t w_type, int col, int dim, float (&f)[N]) {
    if (w_type == W2V_F32)
        load_cols<float, N, WHOLE>(static_cast<const float *>(w), col, dim, f);
    else
        load_cols<T, N, WHOLE>(static_cast<const T *>(w), col, dim, f);
}

// WHOLE: dim is a multiple of a vector's elements. (Reading the elements of a last part of a vector one by one takes
// registers that rows without one had better keep for more wavefronts: 16,384 rows of 4,096 bf16 columns with 103
// registers a lane 81 us, with 62 62 us.)
template <class T, int LPR, int NCH, bool WHOLE>
__global__ __launch_bounds__(LPR > kNormThreads ? LPR : kNormThreads) void k_norm(NormArgs a) {
    constexpr int VEC = kVec<T>;
    const int lane = static_cast<int>(threadIdx.x) % LPR;
    const int groups = static_cast<int>(blockDim.x) / LPR;
    const float d = static_cast<float>(a.dim);
    int turn = 0;
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * groups + threadIdx.x / LPR; r < a.rows;
         r += static_cast<int64_t>(gridDim.x) * groups) {
        const T *x = static_cast<const T *>(a.x) + r * a.x_stride;
        float v[NCH][VEC], sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NCH; ++i) load_cols<T, VEC, WHOLE>(x, (i * LPR + lane) * VEC, a.dim, v[i]);
#pragma unroll
        for (int i = 0; i < NCH; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[0] += v[i][e];
        row_sums<LPR, 1>(sum, turn);
        const float mu = sum[0] / d;   // exact for a row of one value, which a product with 1 / d is not
        float sq[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NCH; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[i][e] = (i * LPR + lane) * VEC + e < a.dim ? v[i][e] - mu : 0.0f;
                sq[0] = fmaf(v[i][e], v[i][e], sq[0]);
            }
        row_sums<LPR, 1>(sq, turn);
        const float rs = 1.0f / sqrtf(sq[0] / d + a.eps);
        T *y = static_cast<T *>(a.out) + r * a.out_stride;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int col = (i * LPR + lane) * VEC;
            if (col >= a.dim) continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[i][e] *= rs;
            if (a.w) {
                float w[VEC];
                load_affine<T, VEC, WHOLE>(a.w, a.w_type, col, a.dim, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[i][e] *= w[e];
            }
            if (a.b) {
                float b[VEC];
                load_affine<T, VEC, WHOLE>(a.b, a.w_type, col, a.dim, b);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[i][e] += b[e];
            }
            store_cols<T, VEC, WHOLE>(y, col, a.dim, v[i]);
        }
        if (lane == 0 && a.mean) a.mean[r] = mu;
        if (lane == 0 && a.rstd) a.rstd[r] = rs;
    }
}

// The columns' sums of a workgroup's rows go to part[blockIdx.x][0..dim) (dw) and [dim..2 dim) (db). A row's elements are
// fetched while the row before it is worked on.
template <class T, int LPR, int NCH, bool WHOLE>
__global__ __launch_bounds__(LPR > kNormThreads ? LPR : kNormThreads) void k_norm_back(NormArgs a, float *part) {
    constexpr int VEC = kVec<T>;
    const int lane = static_cast<int>(threadIdx.x) % LPR;
    const int groups = static_cast<int>(blockDim.x) / LPR;
    const float inv_d = 1.0f / static_cast<float>(a.dim);
    int turn = 0;
    float dw[NCH][VEC], db[NCH][VEC];
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) dw[i][e] = db[i][e] = 0.0f;
    Pack<T, VEC> next_x[NCH], next_dy[NCH];
    float next_mu = 0.0f, next_rs = 0.0f;
    auto fetch = [&](int64_t r) {
        if (r >= a.rows) return;
        const T *x = static_cast<const T *>(a.x) + r * a.x_stride, *dy = static_cast<const T *>(a.dy) + r * a.dy_stride;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int col = (i * LPR + lane) * VEC;
            next_x[i] = raw_cols<T, VEC, WHOLE>(x, col, a.dim);
            next_dy[i] = raw_cols<T, VEC, WHOLE>(dy, col, a.dim);
        }
        next_mu = a.mean[r];
        next_rs = a.rstd[r];
    };
    const int64_t step = static_cast<int64_t>(gridDim.x) * groups;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * groups + threadIdx.x / LPR;
    constexpr bool kAhead = LPR <= 256;   // sixteen wavefronts a workgroup have registers for one row
    if (kAhead) fetch(first);
    for (int64_t r = first; r < a.rows; r += step) {
        if (!kAhead) fetch(r);
        float h[NCH][VEC], g[NCH][VEC], sum[2] = {0.0f, 0.0f};   // g: dy, then dy w
#pragma unroll
        for (int i = 0; i < NCH; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                h[i][e] = static_cast<float>(next_x[i].v[e]);
                g[i][e] = static_cast<float>(next_dy[i].v[e]);
            }
        const float mu = next_mu, rs = next_rs;
        if (kAhead) fetch(r + step);
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int col = (i * LPR + lane) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                h[i][e] = col + e < a.dim ? (h[i][e] - mu) * rs : 0.0f;
                dw[i][e] = fmaf(g[i][e], h[i][e], dw[i][e]);
                db[i][e] += g[i][e];
            }
            if (a.w && col < a.dim) {
                float w[VEC];
                load_affine<T, VEC, WHOLE>(a.w, a.w_type, col, a.dim, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) g[i][e] *= w[e];
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                sum[0] += g[i][e];
                sum[1] = fmaf(g[i][e], h[i][e], sum[1]);
            }
        }
        row_sums<LPR, 2>(sum, turn);
        const float c0 = sum[0] * inv_d, c1 = sum[1] * inv_d;
        T *dx = static_cast<T *>(a.out) + r * a.out_stride;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int col = (i * LPR + lane) * VEC;
            if (col >= a.dim) continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e) g[i][e] = rs * (g[i][e] - c0 - h[i][e] * c1);
            store_cols<T, VEC, WHOLE>(dx, col, a.dim, g[i]);
        }
    }
    if (!part) return;
    float *out = part + static_cast<int64_t>(blockIdx.x) * 2 * a.dim;
    if constexpr (LPR > kWave) {   // each column has one lane
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            store_cols<float, VEC>(out, (i * LPR + lane) * VEC, a.dim, dw[i]);
            store_cols<float, VEC>(out + a.dim, (i * LPR + lane) * VEC, a.dim, db[i]);
        }
    } else {
        constexpr int kCols = LPR * NCH * VEC, kWaves = kNormThreads / kWave;
        __shared__ float cols[kWaves][kCols];
        const int wid = static_cast<int>(threadIdx.x) / kWave;
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int i = 0; i < NCH; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float v = half ? db[i][e] : dw[i][e];
                    if constexpr (LPR == 16) v = rows_sum(v);
                    if (lane_id() < LPR) cols[wid][(i * LPR + lane) * VEC + e] = v;
                }
            __syncthreads();
            for (int c = threadIdx.x; c < a.dim; c += kNormThreads) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) v += cols[w][c];
                out[half * a.dim + c] = v;
            }
            __syncthreads();
        }
    }
}

// Column c of the n rows of part, summed: 64 columns a workgroup, the rows split over its wavefronts.
constexpr int kColThreads = 1024;
__global__ __launch_bounds__(kColThreads) void k_norm_columns(const float *__restrict__ part, int n, int dim,
                                                              float *__restrict__ dw, float *__restrict__ db) {
    constexpr int kWaves = kColThreads / kWave;
    __shared__ float sums[kWaves][kWave];
    const int lane = lane_id(), wid = static_cast<int>(threadIdx.x) / kWave;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kWave + lane, width = 2 * static_cast<int64_t>(dim);
    float v = 0.0f;
    if (c < width) {
        int k = wid;
        for (; k + 7 * kWaves < n; k += 8 * kWaves) {
            float t[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) t[u] = part[(k + u * kWaves) * width + c];
#pragma unroll
            for (int u = 0; u < 8; ++u) v += t[u];
        }
        for (; k < n; k += kWaves) v += part[k * width + c];
    }
    sums[wid][lane] = v;
    __syncthreads();
    if (wid == 0 && c < width) {
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += sums[w][lane];
        float *to = c < dim ? dw : db;
        if (to) to[c < dim ? c : c - dim] = v;
    }
}

// Calls f(LPR, NCH) with the smallest shape that holds a row of dim elements of T.
template <int A, int B, bool W = false>
struct Shape {
    static constexpr int lpr = A, nch = B;
    static constexpr bool whole = W;
    using Whole = Shape<A, B, true>;
};
template <class T, class F>
int with_shape(int32_t dim, F call) {
    const int chunks = static_cast<int>(ceil_div(dim, kVec<T>));
    auto f = [&](auto shape) { return dim % kVec<T> == 0 ? call(typename decltype(shape)::Whole{}) : call(shape); };
    // at most 20 elements a lane: with 32 the backward pass keeps a wavefront or two a SIMD
    if (chunks <= 16) return f(Shape<16, 1>{});
    if (chunks <= 32) return f(Shape<16, 2>{});
    if constexpr (sizeof(T) == 4) {
        if (chunks <= 48) return f(Shape<16, 3>{});
        if (chunks <= 80) return f(Shape<16, 5>{});
        if (chunks <= 128) return f(Shape<64, 2>{});
        if (chunks <= 256) return f(Shape<64, 4>{});
        if (chunks <= 512) return f(Shape<256, 2>{});
        if (chunks <= 1024) return f(Shape<256, 4>{});
        if (chunks <= 2048) return f(Shape<1024, 2>{});
        return f(Shape<1024, 4>{});
    } else {
        if (chunks <= 64) return f(Shape<64, 1>{});
        if (chunks <= 128) return f(Shape<64, 2>{});
        if (chunks <= 256) return f(Shape<256, 1>{});
        if (chunks <= 512) return f(Shape<256, 2>{});
        if (chunks <= 1024) return f(Shape<1024, 1>{});
        return f(Shape<1024, 2>{});
    }
}

// Workgroups of the backward pass, each with a row of partial sums.
constexpr int64_t kBackGroups = 512, kBackRows = 8;   // at most, and rows for each at least (1,024: 62 us, not 54)
int64_t back_groups(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(kBackGroups, rows / kBackRows)); }

}  // namespace

int run_layer_norm(const NormArgs &a, hipStream_t s) {
    if (a.rows == 0) return W2V_OK;
    return with_type(a.type, [&](auto zero) {
        using T = decltype(zero);
        return with_shape<T>(a.dim, [&](auto shape) {
            constexpr int threads = shape.lpr > kNormThreads ? shape.lpr : kNormThreads;
            const int64_t want = ceil_div(a.rows, threads / shape.lpr);
            const auto grid = static_cast<unsigned>(std::min<int64_t>(want, kMaxGroups * kNormThreads / threads));
            k_norm<T, shape.lpr, shape.nch, shape.whole><<<grid, threads, 0, s>>>(a);
            W2V_LAUNCH_CHECK("k_norm");
            return static_cast<int>(W2V_OK);
        });
    });
}

size_t norm_backward_bytes(int64_t rows, int32_t dim) {
    return static_cast<size_t>(back_groups(rows)) * 2 * static_cast<size_t>(dim) * sizeof(float);
}

int run_layer_norm_backward(const NormArgs &a, void *workspace, hipStream_t s) {
    const bool sums = a.dw || a.db;
    const int64_t groups = back_groups(a.rows);
    float *part = sums ? static_cast<float *>(workspace) : nullptr;
    if (a.rows > 0) {
        const int rc = with_type(a.type, [&](auto zero) {
            using T = decltype(zero);
            return with_shape<T>(a.dim, [&](auto shape) {
                constexpr int threads = shape.lpr > kNormThreads ? shape.lpr : kNormThreads;
                k_norm_back<T, shape.lpr, shape.nch, shape.whole><<<static_cast<unsigned>(groups), threads, 0, s>>>(a, part);
                W2V_LAUNCH_CHECK("k_norm_back");
                return static_cast<int>(W2V_OK);
            });
        });
        if (rc) return rc;
    }
    if (!sums) return W2V_OK;
    const auto grid = static_cast<unsigned>(ceil_div(2 * static_cast<int64_t>(a.dim), kWave));
    k_norm_columns<<<grid, kColThreads, 0, s>>>(part, a.rows > 0 ? static_cast<int>(groups) : 0, a.dim, a.dw, a.db);
    W2V_LAUNCH_CHECK("k_norm_columns");
    return W2V_OK;
}

}  // namespace w2v
