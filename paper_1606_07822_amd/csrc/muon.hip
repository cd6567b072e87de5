// Muon: momentum, and an update whose singular values five Newton-Schulz steps bring near one.
//
//   M = mu M + G,  U = G + mu M (Nesterov) or M,  X = U / (|U| + eps),  five times X = (a I + b A + c A A) X with A = X X',
//   W = W (1 - lr decay) - lr scale X
//
// A step is three products: A, of which half is made (it is symmetric), aI + bA + cAA with the sum and the unit matrix where
// the product's tiles end, and X; the last one's tiles become the result, or update the weights. A matrix taller than wide is
// multiplied from the other side, its long axis along k either way, and nothing is transposed: X is read along its rows by
// one product and down them by the other. Matrices of one shape and type go through the launches together.
//
// Numbers: a step multiplies errors by up to 3.9, so between the products everything has 22 bits in two fp16 parts (three
// products; 3.9e-6 of a 4,096 x 10,240 result in norm, fp32 products 6e-6) and sums are fp32. Norms are sums in 64 bits, so that
// squares neither overflow nor vanish.
//
// bf16 results take products of one part, 11 bits, a third of the work. Rounding X itself to 11 bits would not do: that is noise
// in all directions, and the steps multiply it by up to 3.4445 each where X has no singular value of note, 485 in all (0.1 of
// the result for an X of rank 1). So X is carried in two parts, and a step is
//
//   X = (a + d) X + Q X1,   Q + d = bA + cA1 A1,   A = X1 X1'
//
// where 1 marks first parts, Q is rounded to one and the diagonal d is what that leaves of Q's. Errors of Q and A now multiply
// X: they turn its singular vectors by a little and stay in its own rows' (columns') space, where p(s)/s is near one, so that
// no later step makes them grow; X's noise passes through Q X1 alone, and Q is next to nothing in the directions where it would
// grow. The last step, after which nothing grows, takes X1 for X. Error in norm: 1.1e-3 of the result for Gaussian matrices and
// 0.4 to 1.1e-3 for low ranks and decaying singular values, 3.6e-3 at the most that was found, where all of a matrix's roundings
// have one sign (all entries of one size, unit matrices); bf16's own rounding is 1.7e-3. The stack
// below takes 3.4 ms for the 2.9 of one part throughout, 5.6 with products of two; 4,096 x 10,240 3.2, 3.0 and 7.3.
//
// What bounds it: the matrix cores for large matrices (4,096 x 10,240: 7.3 ms, 1,200 TFLOP/s of 16-bit products); launches'
// starts and ends for stacks of middling ones (36 of 1,024 x 2,816 bf16: 3.4 ms, the products alone 1.5) and
// launches alone for small ones (100 x 400: 92 us, seventeen).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <tuple>
#include <type_traits>
#include <vector>

#include "w2v_ops.h"
#include "w2v_product.h"

namespace w2v {
namespace {

using E = _Float16;
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
// Everything that the steps hold is kept times 2^12 in fp16: entries of X are at most 1.21 in size, of A 1.45, of
// aI + bA + cAA 3.45 and of bA + cAA 2.81, and the second part's absolute error, 2^-25, is 2^-37 of one.
constexpr float kUp = 4096.0f, kDown = 1.0f / 4096.0f;
constexpr int kParts = 256;       // sums of squares of a matrix

// Where a matrix of a launch lies.
struct Entry {
    void *out;             // the parameter, or the orthogonalised matrix
    const void *grad;
    int64_t out_stride, grad_stride, moment;
    float decay, scale;
};
struct Batch {
    const Entry *table;    // null: `first`, and each next one `out_step` and `grad_step` bytes on
    Entry first;
    int64_t out_step, grad_step;
    int64_t rows, cols, count;
    float *m;              // null: no momentum
    float mu;
    int32_t nesterov, muon;
    float grad_scale;
    float lr;
    const float *lr_device;

    __device__ __forceinline__ Entry entry(int64_t z) const {
        if (table) return table[z];
        Entry e = first;
        e.out = static_cast<char *>(e.out) + z * out_step;
        e.grad = static_cast<const char *>(e.grad) + z * grad_step;
        return e;
    }
};

// ------------------------------------------------------------------ momentum and norms
// Two parts of 8 neighbouring elements in arrays of their own; second may be null.
__device__ __forceinline__ void store_apart8(E *first, E *second, int64_t at, int64_t valid, const float (&v)[8]) {
    Frag<E> part[2];
    to_parts8<E, 2>(valid, v, part);
    *reinterpret_cast<Frag<E> *>(first + at) = part[0];
    if (second) *reinterpret_cast<Frag<E> *>(second + at) = part[1];
}

// Both passes are bound by memory (momentum 5.6 TB/s). Block b of `blocks` of a matrix takes every `blocks`-th group of rows;
// its threads have a place in a row and go along it: f(row, column) for the first of each N columns up to `width`.
template <int N, class F>
__device__ __forceinline__ void each_chunk(int64_t rows, int64_t width, int64_t block, int64_t blocks, F f) {
    const int per = static_cast<int>(ceil_div(width, N)), wide = min(per, 256), tall = 256 / wide;
    const int tid = static_cast<int>(threadIdx.x), in = tid / wide, at = tid - in * wide;
    if (in >= tall) return;
    for (int64_t row = block * tall + in; row < rows; row += blocks * tall)
        for (int c = at; c < per; c += wide) f(row, c * N);
}

// Block b of matrix z: its share of the momentum and of U's sum of squares.
template <class T>
__global__ __launch_bounds__(256) void k_muon_momentum(const Batch b, double *part) {
    const int64_t z = blockIdx.x / kParts;
    const Entry e = b.entry(z);
    double sum = 0.0;
    each_chunk<8>(b.rows, b.cols, blockIdx.x % kParts, kParts, [&](int64_t row, int col) {
        const int64_t valid = b.cols - col;
        float g[8];
        load8<T>(static_cast<const T *>(e.grad) + row * e.grad_stride + col, valid, g);
        if (b.m) {
            float *at = b.m + e.moment + row * b.cols + col;
            float m[8];
            load8<float>(at, valid, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                g[i] *= b.grad_scale;
                m[i] = b.mu * m[i] + g[i];
                g[i] = b.nesterov ? g[i] + b.mu * m[i] : m[i];
            }
            store8<float>(at, valid, m);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += static_cast<double>(g[i]) * g[i];   // squares of fp32 leave its range
    });
    sum = wave_sum(sum);
    __shared__ double waves[4];
    if (lane_id() == 0) waves[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = waves[0] + waves[1] + waves[2] + waves[3];
}

// X's parts, in rows of `stride` elements with zeros behind the last column. P = 1: the second parts lie in an array of their
// own (null where the first step is the last).
template <class T, int P>
__global__ __launch_bounds__(256) void k_muon_start(const Batch b, const double *part, double eps, E *x, E *second, int64_t stride,
                                                    int64_t blocks) {
    const int64_t z = blockIdx.x / blocks;
    const Entry e = b.entry(z);
    double sum = wave_sum(part[z * kParts + threadIdx.x]);
    __shared__ double waves[4];
    if (lane_id() == 0) waves[threadIdx.x / kWave] = sum;
    __syncthreads();
    sum = waves[0] + waves[1] + waves[2] + waves[3];
    // one over the norm as a factor below one and a power of two: either may be out of fp32's range, X is not
    int power = 0;
    const float factor = static_cast<float>(frexp(kUp / (sqrt(sum) + eps), &power));
    each_chunk<8>(b.rows, stride, blockIdx.x % blocks, blocks, [&](int64_t row, int col) {
        const int64_t valid = b.cols - col;
        float g[8];
        load8<T>(static_cast<const T *>(e.grad) + row * e.grad_stride + col, valid, g);
        if (b.m) {
            float m[8];
            load8<float>(b.m + e.moment + row * b.cols + col, valid, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = b.nesterov ? g[i] * b.grad_scale + b.mu * m[i] : m[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = ldexpf(g[i] * factor, power);
        if constexpr (P == 1)
            store_apart8(x, second, (z * b.rows + row) * stride + col, valid, g);
        else
            store_parts8<E, P>(x + part_at<P>(z * b.rows + row, col, stride), valid, g);
    });
}

// ------------------------------------------------------------------ the products of a step
struct Spot {
    int64_t m0, n0, z;
};

// A symmetric r x r product of each matrix with itself: A = X X' (or X' X), or with `poly` aI + bA + cAA (P = 1: Q and d). Of it
// the tiles on and above the diagonal are made, and the others are their mirror images; of few tiles all are made
// (orthogonalize 100 x 400: a mirror image takes a second pass over LDS).
template <int P>
struct SquareJob {
    Side x;
    int64_t step;        // bytes from a matrix to the next
    int64_t r, k;
    int32_t g, poly, all;   // tiles along a side; all: none is a mirror image
    Tiling t;
    const E *old;        // A, where poly
    E *out;
    int64_t stride;
    float *diagonal;     // d, `stride` a matrix (P = 1, poly)

    template <class Q>
    __device__ __forceinline__ Spot at(int tile) const {
        const int each = all ? g * g : g * (g + 1) / 2, z = tile / each;
        int in = tile - z * each, tm = 0;
        if (all) return Spot{int64_t(in / g) * Q::BM, int64_t(in % g) * Q::BN, z};
        while (in >= g - tm) in -= g - tm++;
        return Spot{int64_t(tm) * Q::BM, int64_t(tm + in) * Q::BN, z};
    }
    template <class Q>
    __device__ __forceinline__ void multiply(const Spot &w, int from, int end, char *lds, f4 (&acc)[Q::FM][Q::FN]) const {
        Side s = x;
        s.p += w.z * step;
        Q::run(s, s, nullptr, nullptr, 0, w.m0, r, w.n0, r, k, int64_t(from) * Q::BK, std::min(k, int64_t(end) * Q::BK), lds, acc);
    }
    template <class Q>
    __device__ __forceinline__ void take(const Spot &w, int row, int col, char *region, Lanes lanes) const {
        E *to = out + w.z * r * stride * P;
        const E *a = old + w.z * r * stride * P;
        const bool mirror = !all && w.m0 != w.n0;
        Q::rows8(region, lanes, [&](int i, int j, float (&v)[8]) {
            const int64_t m = w.m0 + row + i, n = w.n0 + col + j;
            Frag<E> part[P] = {};
            if (m < r && n < stride) {
                finish(a + part_at<P>(m, n, stride), m, n, v);
                to_parts8<E, P>(r - n, v, part);
                store_parts8<E, P>(to + part_at<P>(m, n, stride), part);
                if constexpr (P == 1) {
                    if (poly)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (m == n + e) diagonal[w.z * stride + m] = (v[e] - static_cast<float>(part[0][e])) * kDown;
                }
            }
            if (mirror) Q::leave8(region, i, j, part);
        });
        if (!mirror) return;
        // the tile below the diagonal: row n has from column m on what column n had from row m on, zeros where there is none
        Q::mirror8(region, lanes, [&](int i, int j, const Frag<E> (&part)[P]) {
            const int64_t m = w.m0 + row + i, n = w.n0 + col + j;
            if (n < r && m < r) store_parts8<E, P>(to + part_at<P>(n, m, stride), part);
        });
    }
    // `from`: A's 8 elements from (row, col) on.
    __device__ __forceinline__ void finish(const E *from, int64_t row, int64_t col, float (&v)[8]) const {
        float a[8] = {};
        if (poly) {
#pragma unroll
            for (int p = P - 1; p >= 0; --p) {
                const Frag<E> o = *reinterpret_cast<const Frag<E> *>(from + p * 32);
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] += static_cast<float>(o[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] *= kDown;
            if (poly) v[e] = kC * v[e] + kB * a[e] + (P > 1 && row == col + e ? kA * kUp : 0.0f);
        }
    }
};

// X = (aI + bA + cAA) X, or X (aI + bA + cAA) where X is taller than wide; the last one goes into the result. P = 1:
// (a + d) X + Q X1, or X (a + d) + X1 Q.
template <class T, int P, bool LAST>
struct StepJob {
    Side a, b;
    int64_t a_step, b_step;   // bytes from a matrix to the next
    int64_t k;
    int32_t gm, gn;
    Tiling t;
    E *out;
    int64_t stride;
    Batch batch;
    // P = 1: X's first parts, and its second ones (LAST: none), which the new X's replace if `keep`
    const E *first;
    E *second;
    int32_t keep, wide;
    const float *diagonal;
    int64_t diagonal_stride;

    // The new X's 8 elements from (m, n) on, times 2^12, from the product's.
    __device__ __forceinline__ void finish(int64_t z, int64_t m, int64_t n, float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= kDown;
        if constexpr (P == 1) {
            const int64_t at = (z * batch.rows + m) * stride + n;
            const float *d = diagonal + z * diagonal_stride;
            const f4 low = wide ? f4{} + d[m] : *reinterpret_cast<const f4 *>(d + n),
                     high = wide ? low : *reinterpret_cast<const f4 *>(d + n + 4);
            const Frag<E> x1 = *reinterpret_cast<const Frag<E> *>(first + at);
            Frag<E> x2{};
            if constexpr (!LAST) x2 = *reinterpret_cast<const Frag<E> *>(second + at);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] += (kA + (e < 4 ? low[e & 3] : high[e & 3])) * (static_cast<float>(x1[e]) + static_cast<float>(x2[e]));
        }
    }

    template <class Q>
    __device__ __forceinline__ Spot at(int tile) const {
        const int z = tile / (gm * gn);
        int tm, tn;
        tile_at(tile - z * gm * gn, gm, gn, tm, tn);
        return Spot{int64_t(tm) * Q::BM, int64_t(tn) * Q::BN, z};
    }
    template <class Q>
    __device__ __forceinline__ void multiply(const Spot &w, int from, int end, char *lds, f4 (&acc)[Q::FM][Q::FN]) const {
        Side l = a, r = b;
        l.p += w.z * a_step;
        r.p += w.z * b_step;
        Q::run(l, r, nullptr, nullptr, 0, w.m0, batch.rows, w.n0, batch.cols, k, int64_t(from) * Q::BK, std::min(k, int64_t(end) * Q::BK), lds, acc);
    }
    template <class Q>
    __device__ __forceinline__ void take(const Spot &w, int row, int col, char *region, Lanes lanes) const {
        if constexpr (!LAST) {
            Q::rows8(region, lanes, [&](int i, int j, float (&v)[8]) {
                const int64_t m = w.m0 + row + i, n = w.n0 + col + j;
                if (m >= batch.rows || n >= stride) return;
                finish(w.z, m, n, v);
                if constexpr (P == 1)
                    store_apart8(out, keep ? second : nullptr, (w.z * batch.rows + m) * stride + n, batch.cols - n, v);
                else
                    store_parts8<E, P>(out + part_at<P>(w.z * batch.rows + m, n, stride), batch.cols - n, v);
            });
        } else {
            const Entry en = batch.entry(w.z);
            const float lr = batch.lr_device ? *batch.lr_device : batch.lr;
            const float keep = 1.0f - lr * en.decay, by = batch.muon ? -lr * en.scale * kDown : kDown;
            Q::rows8(region, lanes, [&](int i, int j, float (&v)[8]) {
                const int64_t m = w.m0 + row + i, n = w.n0 + col + j;
                if (m >= batch.rows || n >= batch.cols) return;
                finish(w.z, m, n, v);
                T *to = static_cast<T *>(en.out) + m * en.out_stride + n;
                float old[8] = {};
                if (batch.muon) load8<T>(to, batch.cols - n, old);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = batch.muon ? old[e] * keep + v[e] * by : v[e] * by;
                store8<T>(to, batch.cols - n, v);
            });
        }
    }
};

// SQUARE: tiles as wide as tall only.
template <int P, bool A, bool B, bool SQUARE>
struct Tiles;
template <bool A, bool B, bool SQUARE>
struct Tiles<1, A, B, SQUARE> {
    using Large = Tile<E, 1, 256, 256, 2, 4, 64, A, B>;
    using Small = Tile<E, 1, 128, 128, 2, 2, 64, A, B>;
    using Deep = Tile<E, 1, 128, 128, 2, 2, 64, A, B, false, false, 5>;
    using Tiny = Tile<E, 1, 64, 64, 2, 2, 64, A, B, false, false, 4>;
    using Middle = std::conditional_t<SQUARE, Deep, Tile<E, 1, 256, 128, 4, 2, 64, A, B, false, false, 3>>;
};
template <bool A, bool B, bool SQUARE>
struct Tiles<2, A, B, SQUARE> {
    using Large = Tile<E, 2, 256, 256, 2, 4, 32, A, B>;
    using Small = Tile<E, 2, 128, 128, 2, 2, 32, A, B>;
    using Deep = Tile<E, 2, 128, 128, 4, 2, 32, A, B, false, false, 5>;
    using Tiny = Tile<E, 2, 64, 64, 2, 2, 32, A, B, false, false, 4>;
    using Middle = std::conditional_t<SQUARE, Deep, Tile<E, 2, 256, 128, 4, 2, 32, A, B, false, false, 3>>;
};

// Whether a launch of `count` symmetric products of g x g tiles makes them all (up to a quarter of the CUs: with all of them
// 2,731 x 1,023 takes 396 us, by halves 348).
bool makes_all(int64_t g, int64_t count) { return count * g * g * 4 <= device_cu_count(); }
int64_t square_tiles(int64_t g, int64_t count) { return count * (makes_all(g, count) ? g * g : g * (g + 1) / 2); }

// Where the arrays of a launch of `count` matrices lie.
struct Arrays {
    double *part;
    E *x[2], *a, *b;
    E *second;           // one part: X's second parts, and d
    float *diagonal;
    float *sums;
    int64_t r, c, x_stride, a_stride;
    Cut gram, poly, step;
    size_t bytes;
};

template <int P>
Arrays arrays_of(int64_t rows, int64_t cols, int64_t count, void *workspace) {
    Arrays w{};
    w.r = std::min(rows, cols);
    w.c = std::max(rows, cols);
    w.x_stride = ceil_div(cols, 64) * 64;
    w.a_stride = ceil_div(w.r, 64) * 64;
    const auto square = [&](auto tile) { return square_tiles(ceil_div(w.r, decltype(tile)::type::BM), count); };
    w.gram = choose_cut<Tiles<P, true, true, true>>(w.c, 4 * P, square);
    w.poly = choose_cut<Tiles<P, true, true, true>>(w.r, 6 * P, square);
    w.step = choose_cut<Tiles<P, true, true, false>>(
        w.r, 2 * P, [&](auto tile) { return count * count_tiles<typename decltype(tile)::type>(rows, cols); });
    Carve k(workspace);
    w.part = k.take<double>(static_cast<size_t>(count * kParts));
    for (E *&x : w.x) x = k.take<E>(static_cast<size_t>(P * count * rows * w.x_stride));
    w.a = k.take<E>(static_cast<size_t>(P * count * w.r * w.a_stride));
    w.b = k.take<E>(static_cast<size_t>(P * count * w.r * w.a_stride));
    if (P == 1) {
        w.second = k.take<E>(static_cast<size_t>(count * rows * w.x_stride));
        w.diagonal = k.take<float>(static_cast<size_t>(count * w.a_stride));
    }
    w.sums = k.take<float>(std::max({w.gram.floats, w.poly.floats, w.step.floats}));
    w.bytes = k.used();
    return w;
}

template <class T, int P, bool WIDE>
int run_steps(const Batch &b, const Arrays &w, int32_t steps, hipStream_t s) {
    using Gram = Tiles<P, WIDE, WIDE, true>;
    using Poly = Tiles<P, true, true, true>;
    using Step = Tiles<P, true, !WIDE, false>;
    for (int32_t i = 0; i < steps; ++i) {
        const E *from = w.x[i % 2];
        const int64_t x_row = P * w.x_stride * 2, a_row = P * w.a_stride * 2;   // bytes
        const Side x{reinterpret_cast<const char *>(from), x_row};
        SquareJob<P> q{};
        q.x = x;
        q.step = b.rows * x_row;
        q.r = w.r;
        q.k = w.c;
        q.g = tiles_along(w.r, tile_m<Gram>(w.gram));
        q.all = makes_all(q.g, b.count);
        q.out = w.a;
        q.stride = w.a_stride;
        if (int rc = launch_cut<Gram>(w.gram, w.sums, q, s)) return rc;
        q.x = Side{reinterpret_cast<const char *>(w.a), a_row};
        q.step = w.r * a_row;
        q.k = w.r;
        q.g = tiles_along(w.r, tile_m<Poly>(w.poly));
        q.all = makes_all(q.g, b.count);
        q.poly = 1;
        q.old = w.a;
        q.out = w.b;
        q.diagonal = w.diagonal;
        if (int rc = launch_cut<Poly>(w.poly, w.sums, q, s)) return rc;
        const Side poly{reinterpret_cast<const char *>(w.b), a_row};
        auto step = [&](auto job) {
            job.a = WIDE ? poly : x;
            job.b = WIDE ? x : poly;
            job.a_step = WIDE ? w.r * a_row : b.rows * x_row;
            job.b_step = WIDE ? b.rows * x_row : w.r * a_row;
            job.k = w.r;
            job.gm = tiles_along(b.rows, tile_m<Step>(w.step));
            job.gn = tiles_along(b.cols, tile_n<Step>(w.step));
            job.out = w.x[1 - i % 2];
            job.stride = w.x_stride;
            job.batch = b;
            job.first = from;
            job.second = w.second;
            job.keep = i + 2 < steps;
            job.wide = WIDE;
            job.diagonal = w.diagonal;
            job.diagonal_stride = w.a_stride;
            return launch_cut<Step>(w.step, w.sums, job, s);
        };
        if (int rc = i + 1 < steps ? step(StepJob<T, P, false>{}) : step(StepJob<T, P, true>{})) return rc;
    }
    return W2V_OK;
}

// All matrices of one shape and type.
template <class T, class G, int P>
int run_batch(const Batch &b, const Arrays &w, double eps, int32_t steps, hipStream_t s) {
    if (std::max({w.gram.tiles, w.poly.tiles, w.step.tiles}) > kMaxTiles) return fail(W2V_E_RANGE, "a matrix is too large");
    k_muon_momentum<G><<<static_cast<unsigned>(b.count * kParts), 256, 0, s>>>(b, w.part);
    W2V_LAUNCH_CHECK("k_muon_momentum");
    // some four chunks of eight a thread, and no more than 4,096 workgroups a matrix
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(ceil_div(b.rows * (w.x_stride / 8), 1024), 4096));
    E *second = steps > 1 ? w.second : nullptr;
    k_muon_start<G, P><<<static_cast<unsigned>(b.count * blocks), 256, 0, s>>>(b, w.part, eps, w.x[0], second, w.x_stride, blocks);
    W2V_LAUNCH_CHECK("k_muon_start");
    return b.rows <= b.cols ? run_steps<T, P, true>(b, w, steps, s) : run_steps<T, P, false>(b, w, steps, s);
}

// bf16 results are made by products of one part, all others of two.
bool one_part(int32_t type) { return type == W2V_BF16; }

// Matrices that go through the steps together: launches of equal shares with X within 2^27 elements, and 4,096 matrices (a
// launch numbers its threads in 32 bits).
int64_t together(int64_t rows, int64_t cols, int64_t count) {
    const int64_t most = std::max<int64_t>(1, std::min(int64_t(4096), (int64_t(1) << 27) / (rows * ceil_div(cols, 64) * 64)));
    return ceil_div(count, ceil_div(count, most));
}

Arrays arrays_for(int64_t rows, int64_t cols, int64_t count, int32_t type, void *workspace) {
    return one_part(type) ? arrays_of<1>(rows, cols, count, workspace) : arrays_of<2>(rows, cols, count, workspace);
}

// The largest of the launches' needs: all but the last have `together` matrices.
size_t batch_workspace(int64_t rows, int64_t cols, int64_t count, int32_t type) {
    if (rows == 0 || cols == 0 || count == 0) return 0;
    const int64_t n = together(rows, cols, count), rest = count % n;
    const size_t most = arrays_for(rows, cols, n, type, nullptr).bytes;
    return rest == 0 ? most : std::max(most, arrays_for(rows, cols, rest, type, nullptr).bytes);
}

}  // namespace

size_t orthogonalize_bytes(int64_t batch, int64_t rows, int64_t cols, int32_t type) {
    return batch_workspace(rows, cols, batch, type);
}

int run_orthogonalize(const OrthArgs &a, void *workspace, size_t bytes, hipStream_t s) {
    if (a.batch == 0 || a.rows == 0 || a.cols == 0) return W2V_OK;
    const int64_t most = together(a.rows, a.cols, a.batch), size = type_bytes(a.type), rest = a.batch % most;
    const Arrays many = arrays_for(a.rows, a.cols, most, a.type, workspace);
    const Arrays last = rest == 0 ? many : arrays_for(a.rows, a.cols, rest, a.type, workspace);
    if (int rc = check_workspace(workspace, bytes, std::max(many.bytes, last.bytes))) return rc;
    for (int64_t z = 0; z < a.batch; z += most) {
        Batch b{};
        b.first.out = static_cast<char *>(a.out) + z * a.out_step * size;
        b.first.grad = static_cast<const char *>(a.g) + z * a.g_step * size;
        b.first.out_stride = a.out_stride;
        b.first.grad_stride = a.g_stride;
        b.out_step = a.out_step * size;
        b.grad_step = a.g_step * size;
        b.rows = a.rows;
        b.cols = a.cols;
        b.count = std::min(most, a.batch - z);
        const Arrays &w = b.count == most ? many : last;
        const int rc = with_type(a.type, [&](auto zero) {
            using T = decltype(zero);
            return run_batch<T, T, std::is_same<T, __bf16>::value ? 1 : 2>(b, w, a.eps, a.steps, s);
        });
        if (rc) return rc;
    }
    return W2V_OK;
}

// ------------------------------------------------------------------ Muon over many matrices
namespace {

bool same_kind(const w2v_muon_matrix &x, const w2v_muon_matrix &y) {
    return x.rows == y.rows && x.cols == y.cols && x.param_type == y.param_type && x.grad_type == y.grad_type;
}

// The matrices' order in the plan: kind after kind, each in the list's order.
std::vector<int32_t> plan_order(const w2v_muon_matrix *t, int32_t n) {
    std::vector<int32_t> order(n);
    for (int32_t i = 0; i < n; ++i) order[i] = i;
    std::stable_sort(order.begin(), order.end(), [&](int32_t i, int32_t j) {
        const auto key = [&](int32_t q) {
            return std::make_tuple(t[q].rows, t[q].cols, t[q].param_type, t[q].grad_type);
        };
        return key(i) < key(j);
    });
    return order;
}

}  // namespace

size_t muon_plan_bytes(int32_t n) { return static_cast<size_t>(n) * sizeof(Entry); }

size_t muon_bytes(const w2v_muon_matrix *t, int32_t n) {
    size_t most = 0;
    const std::vector<int32_t> order = plan_order(t, n);
    for (int32_t i = 0, j; i < n; i = j) {
        for (j = i; j < n && same_kind(t[order[i]], t[order[j]]);) ++j;
        const w2v_muon_matrix &x = t[order[i]];
        most = std::max(most, batch_workspace(x.rows, x.cols, j - i, x.param_type));
    }
    return most;
}

int run_muon_plan(const w2v_muon_matrix *t, int32_t n, void *plan, hipStream_t s) {
    std::vector<Entry> table;
    table.reserve(n);
    for (int32_t i : plan_order(t, n))
        table.push_back(Entry{t[i].param, t[i].grad, t[i].param_stride, t[i].grad_stride, t[i].moment_offset,
                              t[i].weight_decay, t[i].scale});
    if (n > 0) W2V_HIP(hipMemcpyAsync(plan, table.data(), table.size() * sizeof(Entry), hipMemcpyHostToDevice, s));
    W2V_HIP(hipStreamSynchronize(s));
    return W2V_OK;
}

int run_muon_step(const w2v_muon_matrix *t, int32_t n, const void *plan, float *m, const w2v_muon_params &p, void *workspace,
                  size_t bytes, hipStream_t s) {
    const std::vector<int32_t> order = plan_order(t, n);
    struct Launch {
        int32_t first, count;
        Arrays w;
    };
    std::vector<Launch> launches;
    size_t need = 0;
    for (int32_t i = 0, j; i < n; i = j) {
        for (j = i; j < n && same_kind(t[order[i]], t[order[j]]);) ++j;
        const w2v_muon_matrix &x = t[order[i]];
        if (x.rows == 0 || x.cols == 0) continue;
        const int32_t most = static_cast<int32_t>(together(x.rows, x.cols, j - i));
        for (int32_t z = i; z < j; z += most) {
            const int32_t count = std::min(most, j - z);
            launches.push_back(Launch{z, count, arrays_for(x.rows, x.cols, count, x.param_type, workspace)});
            need = std::max(need, launches.back().w.bytes);
        }
    }
    if (int rc = check_workspace(workspace, bytes, need)) return rc;
    for (const Launch &l : launches) {
        const w2v_muon_matrix &x = t[order[l.first]];
        Batch b{};
        b.table = static_cast<const Entry *>(plan) + l.first;
        b.rows = x.rows;
        b.cols = x.cols;
        b.count = l.count;
        b.m = m;
        b.mu = static_cast<float>(p.momentum);
        b.nesterov = p.nesterov;
        b.muon = 1;
        b.grad_scale = p.grad_scale;
        b.lr = static_cast<float>(p.lr);
        b.lr_device = p.lr_device;
        const int rc = with_type(x.param_type, [&](auto pz) {
            return with_type(x.grad_type, [&](auto gz) {
                using T = decltype(pz);
                return run_batch<T, decltype(gz), std::is_same<T, __bf16>::value ? 1 : 2>(b, l.w, p.eps, p.steps, s);
            });
        });
        if (rc) return rc;
    }
    return W2V_OK;
}

}  // namespace w2v
