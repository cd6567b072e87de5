// A gated feed-forward block of rows, forward and backward.
//
//   g = x Wg',  u = x Wu',  h = act(g) u,  y = h Wd'        act: g sigmoid(g), or g Phi(g) (the normal distribution's)
//   dh = dy Wd,  du = dh act(g),  dg = dh u act'(g),  dx = dg Wg + du Wu,  dWg = dg' x,  dWu = du' x,  dWd = dy' h
//
// Forward two products, backward three launches: dh, whose tiles become dg, du and h where they are made; dx, whose k goes
// through dg and Wg and on through du and Wu; the three weight gradients in one launch, their k the rows. Nothing is stored
// twice or transposed: a product reads an array along its rows or down them. 16-bit rows whose chunks are aligned are read
// where they are, all others copied once into aligned rows.
//
// Numbers: g, u and all sums are fp32. With 16-bit types h, dg and du are rounded to the type (R) between two products, as
// the matrix cores take them; that adds to a result's own rounding one of the same size, spread over its terms (bf16: 2.3e-3
// of the result in norm, where rounding the result alone leaves 1.7e-3). The forward pass of few rows keeps h in fp32. fp32 is
// multiplied as three bf16 parts of 8 bits, six products (2.4e-7 of the result; the library's fp32 product: 7e-7).
//
// What bounds it: the matrix cores for wide rows (16,384 rows of 4,096 bf16, hidden 10,240: 3.3 ms, 1,230 TFLOP/s; backward,
// 8,192 rows: 3.5 ms, 1,180); memory and the matrix cores in turn for narrow ones, whose tiles end after 10 steps (65,536 rows
// of 300, hidden 800: 0.70 ms forward, 1.67 backward); the weights' bytes for a single row (4,096 bf16, hidden 10,240: 57 us,
// 4.4 TB/s); launches for small ones (257 rows of 100: 32 us backward, five launches).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "w2v_ops.h"
#include "w2v_product.h"

namespace w2v {
namespace {

// ------------------------------------------------------------------ activations
// 1 / (1 + exp(-g)): exp's argument is rounded once (|g| 2^-24 of its value), the power and the reciprocal are the
// hardware's, 1 ulp each.
__device__ __forceinline__ float sigmoid(float g) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g));
}
// exp(-g^2 / 2) and the normal distribution's Phi(g). Of a negative g it is exp(-g^2 / 2) t p(t) with t = 1 / (1 - 0.35 g), of
// a positive one what that leaves of 1. p, of degree 8, is fitted to exp(z^2 / 2) Phi(-z) / t over 0 <= z <= 14.5 for the least
// relative error, 5e-8, so that the tail keeps its digits as far as fp32 goes, but for what the rounding of g^2 does to the
// power (g^2 2^-24 of it). 0.5 + 0.5 erf would cancel there: at -5 it is off by 4 %. Some 16 instructions beside the
// exponential; the library's erf has four times as many, and the backward pass of 4,099 rows of 1,023, hidden 2,731, spent 17 us
// on them.
__device__ __forceinline__ float normal_share(float g, float &density) {
    density = __builtin_amdgcn_exp2f(-0.72134752f * g * g);
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.35f * fabsf(g));
    constexpr float p[] = {0.139621302f, 0.139863521f, 0.119821295f, 0.105552472f, -0.0232122745f,
                           0.159319565f, -0.255838871f, 0.144030854f, -0.0291578695f};
    float sum = p[8];
#pragma unroll
    for (int i = 7; i >= 0; --i) sum = fmaf(sum, t, p[i]);
    const float tail = t * sum * density;
    return g < 0.0f ? tail : 1.0f - tail;
}

__device__ __forceinline__ float act_value(int act, float g) {
    float density;
    return g * (act == W2V_SILU ? sigmoid(g) : normal_share(g, density));
}

__device__ __forceinline__ void act_both(int act, float g, float &value, float &slope) {
    if (act == W2V_SILU) {
        const float p = sigmoid(g);
        value = g * p;
        slope = p + value * (1.0f - p);
    } else {
        float density;
        const float p = normal_share(g, density);
        value = g * p;
        slope = p + g * 0.39894228f * density;
    }
}

// ------------------------------------------------------------------ operands as parts
// An array as the matrix products read it: P 16-bit parts an element in rows of whole chunks, zeros behind the last column.
struct Source {
    const void *from;
    int64_t from_stride;   // elements
    void *to;
    int64_t rows, cols, to_stride;   // to_stride in elements, a multiple of 8 (of 32 with parts)
    int64_t first;         // number of its first chunk in the launch
};
struct Sources {
    Source s[7];
    int32_t count;
    int64_t chunks;
};

template <class T, class E, int P>
__global__ __launch_bounds__(256) void k_parts(const Sources all) {
    for (int64_t c = blockIdx.x * int64_t(256) + threadIdx.x; c < all.chunks; c += int64_t(gridDim.x) * 256) {
        int i = 0;
        while (i + 1 < all.count && c >= all.s[i + 1].first) ++i;
        const Source &s = all.s[i];
        const int64_t per = s.to_stride / 8, row = (c - s.first) / per, chunk = (c - s.first) % per;
        float v[8];
        const int64_t left = s.cols - chunk * 8;
        load8<T>(static_cast<const T *>(s.from) + row * s.from_stride + chunk * 8, left, v);
        store_parts8<E, P>(static_cast<E *>(s.to) + part_at<P>(row, chunk * 8, s.to_stride), left, v);
    }
}

// ------------------------------------------------------------------ jobs
struct Place {
    int64_t m0, n0;
    int32_t which;
};

// Up to three products of one kind and k, or two whose results are added.
struct Product {
    Side a, b;
    int64_t m, n;
    int32_t gm, gn, first;   // tiles, and the number of the first one
    void *out;
    int64_t out_stride;
};
template <class T>
struct ProductJob {
    Product p[3];
    int32_t count;
    const char *a2, *b2;           // what p[0]'s k goes on with, or null
    int64_t k;
    Tiling t;

    template <class Q>
    __device__ __forceinline__ Place at(int tile) const {
        Place w;
        w.which = count > 2 && tile >= p[2].first ? 2 : count > 1 && tile >= p[1].first ? 1 : 0;
        int tm, tn;
        tile_at(tile - p[w.which].first, p[w.which].gm, p[w.which].gn, tm, tn);
        w.m0 = int64_t(tm) * Q::BM;
        w.n0 = int64_t(tn) * Q::BN;
        return w;
    }
    template <class Q>
    __device__ __forceinline__ void multiply(const Place &w, int step, int end, char *lds, f4 (&acc)[Q::FM][Q::FN]) const {
        const Product &x = p[w.which];
        const int64_t all = Q::TWO ? ceil_div(k, Q::BK) * Q::BK + k : k;
        Q::run(x.a, x.b, a2, b2, 0, w.m0, x.m, w.n0, x.n, k, int64_t(step) * Q::BK, std::min(all, int64_t(end) * Q::BK), lds, acc);
    }
    template <class Q>
    __device__ __forceinline__ void take(const Place &w, int row, int col, char *region, Lanes lanes) const {
        const Product &x = p[w.which];
        Q::rows8(region, lanes, [&](int r, int c, const float (&v)[8]) {
            const int64_t m = w.m0 + row + r, n = w.n0 + col + c;
            if (m < x.m) store8<T>(static_cast<T *>(x.out) + m * x.out_stride + n, x.n - n, v);
        });
    }
};

// g and u of 16 columns each side by side in a tile; h's parts, and g and u themselves where they are wanted.
template <class T, class E, int P>
struct UpJob {
    Side x, w;
    int64_t other;   // from Wg to Wu, bytes
    int64_t m, n, k;
    int32_t gm, gn;
    int32_t act;
    Tiling t;
    E *h;
    int64_t h_stride;
    T *gate, *up;
    int64_t gate_stride, up_stride;

    template <class Q>
    __device__ __forceinline__ Place at(int tile) const {
        int tm, tn;
        tile_at(tile, gm, gn, tm, tn);
        return Place{int64_t(tm) * Q::BM, int64_t(tn) * (Q::BN / 2), 0};
    }
    template <class Q>
    __device__ __forceinline__ void multiply(const Place &w0, int step, int end, char *lds, f4 (&acc)[Q::FM][Q::FN]) const {
        Q::run(x, w, nullptr, nullptr, other, w0.m0, m, w0.n0, n, k, int64_t(step) * Q::BK, std::min(k, int64_t(end) * Q::BK), lds, acc);
    }
    template <class Q>
    __device__ __forceinline__ void take(const Place &w0, int row, int col, char *region, Lanes lanes) const {
        Q::pairs8(region, lanes, [&](int i, int j, const float (&g)[8], const float (&u)[8]) {
            const int64_t r = w0.m0 + row + i, c = w0.n0 + col / 2 + j, valid = n - c;
            if (r >= m || c >= h_stride) return;
            if (gate) store8<T>(gate + r * gate_stride + c, valid, g);
            if (up) store8<T>(up + r * up_stride + c, valid, u);
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = act_value(act, g[e]) * u[e];
            store_parts8<E, P>(h + part_at<P>(r, c, h_stride), valid, v);
        });
    }
};

// dh, from which the parts of dg, du and h are made where it lies in registers.
template <class T, class E, int P>
struct BackJob {
    Side dy, w;
    int64_t m, n, k;
    int32_t gm, gn;
    int32_t act;
    Tiling t;
    E *dg, *du, *h;
    int64_t h_stride;
    const T *gate, *up;
    int64_t gate_stride, up_stride;

    template <class Q>
    __device__ __forceinline__ Place at(int tile) const {
        int tm, tn;
        tile_at(tile, gm, gn, tm, tn);
        return Place{int64_t(tm) * Q::BM, int64_t(tn) * Q::BN, 0};
    }
    template <class Q>
    __device__ __forceinline__ void multiply(const Place &w0, int step, int end, char *lds, f4 (&acc)[Q::FM][Q::FN]) const {
        Q::run(dy, w, nullptr, nullptr, 0, w0.m0, m, w0.n0, n, k, int64_t(step) * Q::BK, std::min(k, int64_t(end) * Q::BK), lds, acc);
    }
    template <class Q>
    __device__ __forceinline__ void take(const Place &w0, int row, int col, char *region, Lanes lanes) const {
        Q::rows8(region, lanes, [&](int i, int j, const float (&dh)[8]) {
            const int64_t r = w0.m0 + row + i, c = w0.n0 + col + j, valid = n - c;
            if (r >= m || c >= h_stride) return;
            float g[8], u[8], vg[8], vu[8], vh[8];
            load8<T>(gate + r * gate_stride + c, valid, g);
            load8<T>(up + r * up_stride + c, valid, u);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float value, slope;
                act_both(act, g[e], value, slope);
                vh[e] = value * u[e];
                vu[e] = dh[e] * value;
                vg[e] = dh[e] * u[e] * slope;
            }
            const int64_t at = part_at<P>(r, c, h_stride);
            store_parts8<E, P>(dg + at, valid, vg);
            store_parts8<E, P>(du + at, valid, vu);
            store_parts8<E, P>(h + at, valid, vh);
        });
    }
};

// ------------------------------------------------------------------ tiles and how a product is cut into them
template <class E, bool A, bool B, bool PAIR, bool TWO>
struct Tiles1 {
    using Large = Tile<E, 1, 256, 256, PAIR ? 4 : 2, PAIR ? 2 : 4, 64, A, B, PAIR, TWO>;
    using Small = Tile<E, 1, 128, 128, 2, 2, 64, A, B, PAIR, TWO>;
    using Deep = Tile<E, 1, 128, 128, 2, 2, 64, A, B, PAIR, TWO, 5>;
    using Tiny = Tile<E, 1, 64, 64, 2, 2, 64, A, B, PAIR, TWO, 4>;
    using Middle = Tile<E, 1, 256, 128, 4, 2, 64, A, B, PAIR, TWO, 3>;
};
template <class E, bool A, bool B, bool PAIR, bool TWO>
struct Tiles3 {
    using Large = Tile<E, 3, 256, 128, 4, 2, 32, A, B, PAIR, TWO>;
    using Small = Tile<E, 3, 128, 64, 2, 2, 32, A, B, PAIR, TWO>;
    using Deep = Tile<E, 3, 128, 128, 4, 2, 32, A, B, PAIR, TWO, 3>;
    using Tiny = Tile<E, 3, 64, 64, 2, 2, 32, A, B, PAIR, TWO, 3>;
    using Middle = Deep;
};
template <class T>
struct Kind {   // 16-bit rows are multiplied as they are
    using E = T;
    static constexpr int P = 1;
    template <bool A, bool B, bool PAIR = false, bool TWO = false>
    using Tiles = Tiles1<E, A, B, PAIR, TWO>;
};
template <>
struct Kind<float> {   // fp32 rows as three parts of 8 bits, 24 in all
    using E = __bf16;
    static constexpr int P = 3;
    template <bool A, bool B, bool PAIR = false, bool TWO = false>
    using Tiles = Tiles3<E, A, B, PAIR, TWO>;
};

// ------------------------------------------------------------------ operands
// 16-bit rows of whole, aligned chunks are read where they are.
bool in_place(int32_t type, const Rows &r, int64_t rows, int64_t cols) {
    return type != W2V_F32 && cols % 8 == 0 && reinterpret_cast<uintptr_t>(r.p) % 16 == 0 &&
           (rows <= 1 || (r.stride % 8 == 0 && r.stride < (1 << 23)));
}

// Two arrays of the same sizes that a product reads with one stride.
bool in_place(int32_t type, const Rows &r, const Rows &q, int64_t rows, int64_t cols) {
    return in_place(type, r, rows, cols) && in_place(type, q, rows, cols) && (rows <= 1 || r.stride == q.stride);
}

struct Packing {
    Sources all{};
    int32_t type;
    int parts;
    Carve *carve;

    Side operand(const Rows &r, int64_t rows, int64_t cols) {
        return in_place(type, r, rows, cols) ? as_is(r, rows, cols) : packed(r, rows, cols);
    }
    void operands(const Rows &r, const Rows &q, int64_t rows, int64_t cols, Side &a, Side &b) {
        const bool both = in_place(type, r, q, rows, cols);
        a = both ? as_is(r, rows, cols) : packed(r, rows, cols);
        b = both ? as_is(q, rows, cols) : packed(q, rows, cols);
    }
    static Side as_is(const Rows &r, int64_t rows, int64_t cols) {
        return Side{static_cast<const char *>(r.p), (rows <= 1 ? cols : r.stride) * 2};
    }
    Side packed(const Rows &r, int64_t rows, int64_t cols) {
        const int64_t unit = parts > 1 ? 32 : 8, stride = ceil_div(cols, unit) * unit;
        char *to = carve->take<char>(static_cast<size_t>(parts * rows * stride * 2));
        all.s[all.count++] = Source{r.p, r.stride, to, rows, cols, stride, all.chunks};
        all.chunks += rows * (stride / 8);
        return Side{to, parts * stride * 2};
    }
};

template <class T>
int launch_parts(const Packing &p, hipStream_t s) {
    if (p.all.chunks == 0) return W2V_OK;
    const auto grid = static_cast<unsigned>(std::min<int64_t>(ceil_div(p.all.chunks, 256), kMaxGroups));
    k_parts<T, typename Kind<T>::E, Kind<T>::P><<<grid, 256, 0, s>>>(p.all);
    W2V_LAUNCH_CHECK("k_parts");
    return W2V_OK;
}

// ------------------------------------------------------------------ few rows
// Where there are few rows every weight is read for them, and the weights' bytes are the time. A workgroup takes 16 columns
// of the result, its wavefronts take turns along k, 128 bytes of each of the 16 weight rows at a time straight from memory
// into the matrix cores' registers (rows need no alignment but their elements'); the wavefronts' sums are joined in LDS in
// their order. fp32 is multiplied in fp32. h stays fp32; 16-bit weights meet it as two parts, or in fp32 in rows where one h is
// past the type's range (its two parts would be opposite infinities): the sums are made again for these, and the others keep
// theirs.
constexpr int kFewWaves = 8;   // wavefronts a workgroup

// The least number that a 16-bit type rounds to an infinity.
template <class T>
constexpr float kPast = std::is_same<T, __bf16>::value ? 0x1.ffp127f : 65520.0f;

// fp32 rows go this way up to 64 (64 rows, 4,096 x 10,240: 0.28 ms, in tiles, whose parts are 1.5 times as many bytes, 0.43),
// 16-bit ones where the products are small (weights from memory: 1 row, 4,096 x 10,240: 57 us, in tiles 61; 16 rows, 1,024 x
// 2,816: 16 and 20; weights in cache: 48 and 51; 15 and 19; 16 rows, 4,096 x 10,240: 63 and 50) or tiles would need copies of the
// weights. What they read of x again and again grows with the rows.
template <class T>
bool few_rows(const FfnArgs &a, bool copies) {
    return a.rows <= 64 && (sizeof(T) == 4 || a.rows == 1 || (copies && a.rows <= 16) ||
                            a.rows * a.dim * a.hidden <= int64_t(1) << 26);
}

struct FewArgs {
    const void *x, *w, *w2;              // n rows of X, cols rows of T (gate's and up's, or w alone)
    int64_t x_stride, w_stride, w2_stride;
    int32_t n, cols, k, act;
    void *out, *gate, *up;               // float (PAIR) or T, and T
    int64_t out_stride, gate_stride, up_stride;
};

// Products of 16 weight rows' chunks (V elements of each lane's row) with 16 rows' of x.
template <bool FP32, class T, class X, int V>
__device__ __forceinline__ f4 few_product(const Pack<T, V> &w, const Pack<X, V> &x, f4 acc) {
    if constexpr (FP32) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(static_cast<float>(w.v[e]), static_cast<float>(x.v[e]), acc, 0, 0, 0);
    } else {
        Frag<T> a, hi, lo;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            a[e] = w.v[e];
            hi[e] = static_cast<T>(x.v[e]);
            if constexpr (sizeof(X) == 4) lo[e] = static_cast<T>(x.v[e] - static_cast<float>(hi[e]));
        }
        if constexpr (sizeof(X) == 4) acc = mfma32(a, lo, acc);
        acc = mfma32(a, hi, acc);
    }
    return acc;
}

template <class T, class X, int NT, bool PAIR>
__global__ __launch_bounds__(kFewWaves * kWave) void k_few(const FewArgs a) {
    constexpr int V = 16 / sizeof(T), kGroup = 8 * V, kArrays = PAIR ? 2 : 1;
    constexpr bool kParts = sizeof(T) == 2 && sizeof(X) == 4;
    const int lane = lane_id(), wave = static_cast<int>(threadIdx.x) / kWave, c0 = static_cast<int>(blockIdx.x) * 16;
    const int64_t row = min(c0 + lane % 16, a.cols - 1);
    const T *w[kArrays];
    w[0] = static_cast<const T *>(a.w) + row * a.w_stride;
    if constexpr (PAIR) w[1] = static_cast<const T *>(a.w2) + row * a.w2_stride;
    const X *x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) x[t] = static_cast<const X *>(a.x) + min(t * 16 + lane % 16, a.n - 1) * a.x_stride;
    f4 acc[NT][kArrays] = {};
    float most[NT] = {};   // the largest |x| that the lane has met
    const int full = a.k / kGroup, lead = lane / 16 * V;
    // a lane's chunks of a group: number lane / 16 and 4 further on
    auto group = [&](int g, auto whole, auto fp32) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int at = g * kGroup + c * 4 * V + lead;
            const int valid = decltype(whole)::value ? V : a.k - at;
            Pack<T, V> pw[kArrays];
#pragma unroll
            for (int i = 0; i < kArrays; ++i)
                pw[i] = decltype(whole)::value ? *reinterpret_cast<const Pack<T, V> *>(w[i] + at) : raw_cols<T, V>(w[i] + at, 0, valid);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const Pack<X, V> px = decltype(whole)::value ? *reinterpret_cast<const Pack<X, V> *>(x[t] + at)
                                                             : raw_cols<X, V>(x[t] + at, 0, valid);
#pragma unroll
                for (int i = 0; i < kArrays; ++i) acc[t][i] = few_product<decltype(fp32)::value>(pw[i], px, acc[t][i]);
                if constexpr (kParts)
#pragma unroll
                    for (int e = 0; e < V; ++e) most[t] = fmaxf(most[t], fabsf(px.v[e]));
            }
        }
    };
    auto groups = [&](auto fp32) {
        for (int g = wave; g < full; g += kFewWaves) group(g, std::true_type{}, fp32);
        if (a.k % kGroup != 0 && full % kFewWaves == wave) group(full, std::false_type{}, fp32);
    };
    groups(std::bool_constant<sizeof(T) == 4>{});
    if constexpr (kParts) {
        uint64_t past[NT], any = 0;
#pragma unroll
        for (int t = 0; t < NT; ++t) any |= past[t] = __ballot(!(most[t] < kPast<T>));
        if (any) {   // once more in fp32; rows without such a number keep their sums
            f4 parts[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                parts[t] = acc[t][0];
                acc[t][0] = f4{};
            }
            groups(std::true_type{});
#pragma unroll
            for (int t = 0; t < NT; ++t)   // four lanes have one row
                if (!((past[t] | past[t] >> 16 | past[t] >> 32 | past[t] >> 48) >> lane % 16 & 1)) acc[t][0] = parts[t];
        }
    }
    __shared__ f4 part[kFewWaves][NT][kArrays][kWave];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < kArrays; ++i) part[wave][t][i][lane] = acc[t][i];
    __syncthreads();
    if (wave >= NT) return;
    f4 v[kArrays] = {};
#pragma unroll
    for (int q = 0; q < kFewWaves; ++q)
#pragma unroll
        for (int i = 0; i < kArrays; ++i) v[i] += part[q][wave][i][lane];
    // the lane has four columns of one row
    const int64_t r = wave * 16 + lane % 16;
    const int c = c0 + lane / 16 * 4;
    if (r >= a.n) return;
    auto store = [&](auto *to, int64_t stride, const f4 &f) {
        const float e[4] = {f[0], f[1], f[2], f[3]};
        store_cols<std::remove_pointer_t<decltype(to)>, 4>(to + r * stride, c, a.cols, e);
    };
    if constexpr (PAIR) {
        if (a.gate) store(static_cast<T *>(a.gate), a.gate_stride, v[0]);
        if (a.up) store(static_cast<T *>(a.up), a.up_stride, v[1]);
        f4 h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = act_value(a.act, v[0][e]) * v[1][e];
        store(static_cast<float *>(a.out), a.out_stride, h);
    } else {
        store(static_cast<T *>(a.out), a.out_stride, v[0]);
    }
}

template <class T, class X, bool PAIR>
int launch_few(const FewArgs &a, hipStream_t s) {
    const auto grid = static_cast<unsigned>(ceil_div(a.cols, 16));
    const int threads = kFewWaves * kWave;
    if (a.n <= 16)
        k_few<T, X, 1, PAIR><<<grid, threads, 0, s>>>(a);
    else if (a.n <= 32)
        k_few<T, X, 2, PAIR><<<grid, threads, 0, s>>>(a);
    else
        k_few<T, X, 4, PAIR><<<grid, threads, 0, s>>>(a);
    W2V_LAUNCH_CHECK("k_few");
    return W2V_OK;
}

template <class T>
int forward_few(const FfnArgs &a, Carve &c, bool launch, hipStream_t s) {
    const int64_t hs = ceil_div(a.hidden, 64) * 64;
    float *h = c.take<float>(static_cast<size_t>(a.rows * hs));
    if (!launch) return W2V_OK;
    if (int rc = check_workspace(c.base, c.cap, c.used())) return rc;
    FewArgs u{};
    u.x = a.x.p;
    u.w = a.w_gate.p;
    u.w2 = a.w_up.p;
    u.x_stride = a.x.stride;
    u.w_stride = a.w_gate.stride;
    u.w2_stride = a.w_up.stride;
    u.n = static_cast<int32_t>(a.rows);
    u.cols = a.hidden;
    u.k = a.dim;
    u.act = a.act;
    u.out = h;
    u.out_stride = hs;
    u.gate = const_cast<void *>(a.gate.p);
    u.up = const_cast<void *>(a.up.p);
    u.gate_stride = a.gate.stride;
    u.up_stride = a.up.stride;
    if (int rc = launch_few<T, T, true>(u, s)) return rc;
    FewArgs d{};
    d.x = h;
    d.w = a.w_down.p;
    d.x_stride = hs;
    d.w_stride = a.w_down.stride;
    d.n = u.n;
    d.cols = a.dim;
    d.k = a.hidden;
    d.out = const_cast<void *>(a.y.p);
    d.out_stride = a.y.stride;
    return launch_few<T, float, false>(d, s);
}

// One plan of a pass: where its arrays lie, without a workspace only how many bytes they are.
template <class T>
int forward(const FfnArgs &a, Carve &c, bool launch, hipStream_t s) {
    const bool copies = !in_place(a.type, a.w_gate, a.w_up, a.hidden, a.dim) || !in_place(a.type, a.w_down, a.dim, a.hidden);
    if (launch ? few_rows<T>(a, copies) : few_rows<T>(a, false) && few_rows<T>(a, true)) return forward_few<T>(a, c, launch, s);
    using K = Kind<T>;
    using E = typename K::E;
    using Up = typename K::template Tiles<true, true, true>;
    using Down = typename K::template Tiles<true, true>;
    const int64_t n = a.rows, d = a.dim, f = a.hidden, hs = ceil_div(f, 64) * 64;
    Packing pack{{}, a.type, K::P, &c};
    const Side x = pack.operand(a.x, n, d);
    Side wg, wu;
    pack.operands(a.w_gate, a.w_up, f, d, wg, wu);
    const Side wd = pack.operand(a.w_down, d, f);
    E *h = c.take<E>(static_cast<size_t>(K::P * n * hs));
    // bytes that an element of a product's result stands for: g or u, and half of h's parts; y
    const Cut up = choose_cut_of<Up>(n, 2 * f, d, sizeof(T) + K::P),
              down = choose_cut_of<Down>(n, d, f, sizeof(T));
    float *part = c.take<float>(std::max(up.floats, down.floats));
    if (!launch) {   // arrays that need no copies may go the other way
        Carve other;
        if (few_rows<T>(a, true)) forward_few<T>(a, other, false, s);
        c.off = std::max(c.off, other.off);
        return W2V_OK;
    }
    if (int rc = check_workspace(c.base, c.cap, c.used())) return rc;
    if (up.tiles > kMaxTiles || down.tiles > kMaxTiles) return fail(W2V_E_RANGE, "too many rows for one call");
    if (int rc = launch_parts<T>(pack, s)) return rc;
    UpJob<T, E, K::P> u{};
    u.x = x;
    u.w = wg;
    u.other = wu.p - wg.p;
    u.m = n;
    u.n = f;
    u.gm = tiles_along(n, tile_m<Up>(up));
    u.gn = tiles_along(2 * f, tile_n<Up>(up));
    u.k = d;
    u.act = a.act;
    u.h = h;
    u.h_stride = hs;
    u.gate = static_cast<T *>(const_cast<void *>(a.gate.p));
    u.up = static_cast<T *>(const_cast<void *>(a.up.p));
    u.gate_stride = a.gate.stride;
    u.up_stride = a.up.stride;
    if (int rc = launch_cut<Up>(up, part, u, s)) return rc;
    ProductJob<T> y{};
    y.p[0] = Product{Side{reinterpret_cast<char *>(h), K::P * hs * 2}, wd, n, d, tiles_along(n, tile_m<Down>(down)),
                     tiles_along(d, tile_n<Down>(down)), 0, const_cast<void *>(a.y.p), a.y.stride};
    y.count = 1;
    y.k = f;
    return launch_cut<Down>(down, part, y, s);
}

template <class T>
int backward(const FfnArgs &a, Carve &c, bool launch, hipStream_t s) {
    using K = Kind<T>;
    using E = typename K::E;
    using Hidden = typename K::template Tiles<true, false>;
    using Input = typename K::template Tiles<true, false, false, true>;
    using Weights = typename K::template Tiles<false, false>;
    const int64_t n = a.rows, d = a.dim, f = a.hidden, hs = ceil_div(f, 64) * 64;
    Packing pack{{}, a.type, K::P, &c};
    const Side dy = pack.operand(a.dy, n, d), wd = pack.operand(a.w_down, d, f);
    const Side x = pack.operand(a.x, n, d);
    Side wg, wu;
    pack.operands(a.w_gate, a.w_up, f, d, wg, wu);
    E *h[3];
    Side hid[3];
    for (int i = 0; i < 3; ++i) {
        h[i] = c.take<E>(static_cast<size_t>(K::P * n * hs));
        hid[i] = Side{reinterpret_cast<char *>(h[i]), K::P * hs * 2};
    }
    const Cut back = choose_cut_of<Hidden>(n, f, d, 2 * sizeof(T) + 6 * K::P),
              in = choose_cut_of<Input>(n, d, f, sizeof(T), true);
    const auto cut_weights = [&](int inputs, int outputs) {
        return choose_cut<Weights>(n, sizeof(T), [&](auto tile) {
            using Q = typename decltype(tile)::type;
            return inputs * count_tiles<Q>(f, d) + outputs * count_tiles<Q>(d, f);
        });
    };
    Cut weights = cut_weights(2, 1);
    float *part = c.take<float>(std::max({back.floats, in.floats, weights.floats}));
    if (!launch) return W2V_OK;
    if (int rc = check_workspace(c.base, c.cap, c.used())) return rc;
    if (back.tiles > kMaxTiles || in.tiles > kMaxTiles || weights.tiles > kMaxTiles)
        return fail(W2V_E_RANGE, "too many rows for one call");
    if (!a.dw_gate.p || !a.dw_up.p || !a.dw_down.p) {   // fewer gradients: whole tiles where their pieces have no room
        const size_t room = std::max({back.floats, in.floats, weights.floats});
        weights = cut_weights((a.dw_gate.p ? 1 : 0) + (a.dw_up.p ? 1 : 0), a.dw_down.p ? 1 : 0);
        if (weights.floats > room) weights.whole = weights.tiles;
    }
    if (int rc = launch_parts<T>(pack, s)) return rc;
    BackJob<T, E, K::P> b{};
    b.dy = dy;
    b.w = wd;
    b.m = n;
    b.n = f;
    b.gm = tiles_along(n, tile_m<Hidden>(back));
    b.gn = tiles_along(f, tile_n<Hidden>(back));
    b.k = d;
    b.act = a.act;
    b.dg = h[0];
    b.du = h[1];
    b.h = h[2];
    b.h_stride = hs;
    b.gate = static_cast<const T *>(a.gate.p);
    b.up = static_cast<const T *>(a.up.p);
    b.gate_stride = a.gate.stride;
    b.up_stride = a.up.stride;
    if (int rc = launch_cut<Hidden>(back, part, b, s)) return rc;
    ProductJob<T> j{};
    const Rows outs[3] = {a.dw_gate, a.dw_up, a.dw_down};
    int32_t first = 0;
    for (int i = 0; i < 3; ++i) {
        if (!outs[i].p) continue;
        const int64_t m = i < 2 ? f : d, cols = i < 2 ? d : f;
        const int32_t gm = tiles_along(m, tile_m<Weights>(weights)), gn = tiles_along(cols, tile_n<Weights>(weights));
        j.p[j.count++] = Product{i < 2 ? hid[i] : dy, i < 2 ? x : hid[2], m, cols, gm, gn, first, const_cast<void *>(outs[i].p),
                                 outs[i].stride};
        first += gm * gn;
    }
    j.k = n;
    if (j.count > 0)
        if (int rc = launch_cut<Weights>(weights, part, j, s)) return rc;
    // dx last: it may lie where dy or x did
    if (!a.dx.p) return W2V_OK;
    ProductJob<T> i{};
    i.p[0] = Product{hid[0], wg, n, d, tiles_along(n, tile_m<Input>(in)), tiles_along(d, tile_n<Input>(in)), 0,
                     const_cast<void *>(a.dx.p), a.dx.stride};
    i.a2 = hid[1].p;
    i.b2 = wu.p;
    i.count = 1;
    i.k = f;
    return launch_cut<Input>(in, part, i, s);
}

// Gradients of no rows: zeros, by a kernel (a captured graph takes no memset).
template <class T>
__global__ __launch_bounds__(256) void k_zero_rows(T *p, int64_t rows, int64_t cols, int64_t stride) {
    for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < rows * cols; i += int64_t(gridDim.x) * 256)
        p[i / cols * stride + i % cols] = static_cast<T>(0.0f);
}

}  // namespace

size_t ffn_bytes(int64_t rows, int32_t dim, int32_t hidden, int32_t type, bool backward_pass) {
    if (rows == 0) return 0;
    // the sizes are those of arrays none of which can be read in place
    FfnArgs a{};
    a.rows = rows;
    a.dim = dim;
    a.hidden = hidden;
    a.type = type;
    Rows odd{reinterpret_cast<const void *>(uintptr_t(2)), 1};
    a.x = a.w_gate = a.w_up = a.w_down = a.dy = odd;
    Carve c;
    with_type(type, [&](auto zero) {
        using T = decltype(zero);
        return backward_pass ? backward<T>(a, c, false, nullptr) : forward<T>(a, c, false, nullptr);
    });
    return c.used();
}

int run_ffn(const FfnArgs &a, void *workspace, size_t bytes, hipStream_t s) {
    if (a.rows == 0) return W2V_OK;
    Carve c(workspace, bytes);
    return with_type(a.type, [&](auto zero) { return forward<decltype(zero)>(a, c, true, s); });
}

int run_ffn_backward(const FfnArgs &a, void *workspace, size_t bytes, hipStream_t s) {
    Carve c(workspace, bytes);
    if (a.rows > 0) return with_type(a.type, [&](auto zero) { return backward<decltype(zero)>(a, c, true, s); });
    const Rows outs[3] = {a.dw_gate, a.dw_up, a.dw_down};
    for (int i = 0; i < 3; ++i) {
        if (!outs[i].p) continue;
        const int64_t rows = i < 2 ? a.hidden : a.dim, cols = i < 2 ? a.dim : a.hidden;
        const auto grid = static_cast<unsigned>(std::min<int64_t>(ceil_div(rows * cols, 256), kMaxGroups));
        const int rc = with_type(a.type, [&](auto zero) {
            using T = decltype(zero);
            k_zero_rows<T><<<grid, 256, 0, s>>>(static_cast<T *>(const_cast<void *>(outs[i].p)), rows, cols, outs[i].stride);
            W2V_LAUNCH_CHECK("k_zero_rows");
            return static_cast<int>(W2V_OK);
        });
        if (rc) return rc;
    }
    return W2V_OK;
}

}  // namespace w2v
