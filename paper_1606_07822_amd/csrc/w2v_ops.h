// Declarations and device helpers shared by the operators of a mini-batch step (layer norm, the hierarchical
// softmax as a loss, AdamW) and the training path that calls them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "w2v_internal.h"

namespace w2v {

// ------------------------------------------------------------------ element types
// bf16 and fp16 are converted to fp32 exactly on loading; a result is rounded once, to nearest (ties to even), when it is
// stored.
inline bool type_ok(int32_t t) { return t == W2V_F32 || t == W2V_BF16 || t == W2V_F16; }
inline int64_t type_bytes(int32_t t) { return t == W2V_F32 ? 4 : 2; }

// N neighbouring elements that need no more than an element's alignment: gfx950's vector loads and stores take any
// element-aligned address, so odd strides and views keep the wide accesses.
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    T v[N];
};

template <class T, int N>
__device__ __forceinline__ void load_pack(const T *p, float (&f)[N]) {
    const Pack<T, N> u = *reinterpret_cast<const Pack<T, N> *>(p);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = static_cast<float>(u.v[e]);
}

template <class T, int N>
__device__ __forceinline__ void store_pack(T *p, const float (&f)[N]) {
    Pack<T, N> u;
#pragma unroll
    for (int e = 0; e < N; ++e) u.v[e] = static_cast<T>(f[e]);
    *reinterpret_cast<Pack<T, N> *>(p) = u;
}

// The same for the columns from `col` of a row of dim elements; columns past it read as zeros and are not written. WHOLE:
// dim and col are multiples of N.
template <class T, int N, bool WHOLE = false>
__device__ __forceinline__ Pack<T, N> raw_cols(const T *row, int col, int dim) {
    Pack<T, N> u{};
    if (WHOLE ? col < dim : col + N <= dim) {
        u = *reinterpret_cast<const Pack<T, N> *>(row + col);
    } else if (!WHOLE) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (col + e < dim) u.v[e] = row[col + e];
    }
    return u;
}

template <class T, int N, bool WHOLE = false>
__device__ __forceinline__ void load_cols(const T *row, int col, int dim, float (&f)[N]) {
    const Pack<T, N> u = raw_cols<T, N, WHOLE>(row, col, dim);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = static_cast<float>(u.v[e]);
}

template <class T, int N, bool WHOLE = false>
__device__ __forceinline__ void store_cols(T *row, int col, int dim, const float (&f)[N]) {
    if (WHOLE ? col < dim : col + N <= dim) {
        store_pack<T, N>(row + col, f);
    } else if (!WHOLE) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (col + e < dim) row[col + e] = static_cast<T>(f[e]);
    }
}

// Sum over the four rows of 16 lanes, lane by lane: every lane gets the sum of the lanes at its place in a row.
__device__ __forceinline__ float rows_sum(float v) {
    float a = v, b = v;
    swap16(a, b);
    v = a + b;
    a = v;
    b = v;
    swap32(a, b);
    return a + b;
}

// Whether a workspace of `have` bytes is there where `need` are wanted.
int check_workspace(const void *ws, size_t have, size_t need);   // ops_api.hip

// Calls f with a value of the element type that t names.
template <class F>
int with_type(int32_t t, F f) {
    switch (t) {
        case W2V_F32: return f(float{});
        case W2V_BF16: return f(static_cast<__bf16>(0.0f));
        default: return f(static_cast<_Float16>(0.0f));
    }
}

// ------------------------------------------------------------------ layer norm (norm.hip)
constexpr int32_t kNormMaxDim = 16384;
struct NormArgs {
    const void *x, *dy;            // rows of dim elements of `type`
    int64_t rows;
    int32_t dim, type, w_type;
    int64_t x_stride, dy_stride, out_stride;   // elements
    const void *w, *b;             // dim elements of w_type, or null
    float eps;
    void *out;                     // y, or dx
    float *mean, *rstd;            // float[rows]; written by the forward pass (null: not), read by the backward pass
    float *dw, *db;                // float[dim] each, or null
};
int run_layer_norm(const NormArgs &a, hipStream_t s);
size_t norm_backward_bytes(int64_t rows, int32_t dim);
int run_layer_norm_backward(const NormArgs &a, void *workspace, hipStream_t s);

// ------------------------------------------------------------------ hierarchical softmax as a loss (hs_loss.hip)
struct HsLossArgs {
    int32_t V, dim, stride, longest;   // longest: code length that no word of the tree passes
    const float *syn1;
    const uint8_t *codelen;
    const uint64_t *code;
    const int32_t *point_off, *points;
    const void *x;                     // rows of dim elements of `type`
    int32_t type;
    int64_t rows, x_stride;
    const int32_t *targets;
    const float *weights;              // null: ones
    float *loss;                       // float[rows], or null
    void *dx;                          // rows of `type`, or null
    int64_t dx_stride;
    float *dsyn1;                      // V-1 rows, or null
    int64_t dsyn1_stride;
    bool dsyn1_whole;                  // zeros may go into the rows' padding
};
size_t hs_loss_bytes(int64_t rows, int32_t dim, int32_t longest);
int run_hs_loss(const HsLossArgs &a, void *workspace, hipStream_t s);

// out[w] = sum of the rows x_i with words[i] = w, in the rows' order (rows of out without one: zeros; a word outside
// [0, V): none; the padding of out's rows may be written with zeros).
size_t word_sums_bytes(int64_t rows, int32_t dim);
int run_word_sums(const int32_t *words, const float *x, int64_t rows, int32_t dim, int64_t x_stride, int32_t V, float *out,
                  int64_t out_stride, void *workspace, hipStream_t s);

// ------------------------------------------------------------------ AdamW (adamw.hip)
constexpr int kMomentBlock = 256;   // elements that share a scale, moments in 8 bits

int run_adamw_plan(const w2v_adamw_tensor *t, int32_t n, void *plan, hipStream_t s);
size_t adamw_plan_bytes(const w2v_adamw_tensor *t, int32_t n);
int64_t adamw_chunks(const w2v_adamw_tensor *t, int32_t n);
int run_adamw_step(void *plan, int64_t n_chunks, int32_t bits, void *m, void *v, float *m_scale, float *v_scale,
                   const w2v_adamw_params &p, hipStream_t s);
int run_adamw_moments(const void *m, const void *v, const float *m_scale, const float *v_scale, int64_t n, float *m_out,
                      float *v_out, hipStream_t s);

// ------------------------------------------------------------------ gated feed-forward block (ffn.hip)
struct Rows {
    const void *p;
    int64_t stride;   // elements
};
struct FfnArgs {
    int64_t rows;
    int32_t dim, hidden, type, act;
    Rows x, w_gate, w_up, w_down;          // rows x dim, hidden x dim twice, dim x hidden
    Rows gate, up;                         // rows x hidden: written by the forward pass (null: not), read by the backward pass
    Rows y;                                // rows x dim
    Rows dy, dx, dw_gate, dw_up, dw_down;  // a gradient may be null: not wanted
};
constexpr int32_t kFfnMaxDim = 1 << 20;
size_t ffn_bytes(int64_t rows, int32_t dim, int32_t hidden, int32_t type, bool backward);
int run_ffn(const FfnArgs &a, void *workspace, size_t bytes, hipStream_t s);
int run_ffn_backward(const FfnArgs &a, void *workspace, size_t bytes, hipStream_t s);

// ------------------------------------------------------------------ orthogonalised updates (muon.hip)
struct OrthArgs {
    const void *g;
    void *out;
    int32_t type, steps;
    int64_t batch, rows, cols;
    int64_t g_stride, out_stride, g_step, out_step;   // elements from a row, and from a matrix, to the next
    double eps;
};
constexpr int32_t kMuonMaxSide = 1 << 20;
size_t orthogonalize_bytes(int64_t batch, int64_t rows, int64_t cols, int32_t type);
int run_orthogonalize(const OrthArgs &a, void *workspace, size_t bytes, hipStream_t s);
size_t muon_plan_bytes(int32_t n);
size_t muon_bytes(const w2v_muon_matrix *t, int32_t n);
int run_muon_plan(const w2v_muon_matrix *t, int32_t n, void *plan, hipStream_t s);
int run_muon_step(const w2v_muon_matrix *t, int32_t n, const void *plan, float *m, const w2v_muon_params &p, void *workspace,
                  size_t bytes, hipStream_t s);

// ------------------------------------------------------------------ training in mini-batches (batch.hip)
int check_training_args(const w2v_model *m, const w2v_params *p);   // api.hip
int64_t batch_moments(const w2v_model *m, const w2v_batch_params *b);
size_t batch_bytes(const w2v_model *m, int64_t n_tokens, const w2v_params *p, const w2v_batch_params *b, bool train);
int run_batches(const w2v_model *m, const int32_t *tokens, int64_t n_tokens, const w2v_params *p, const w2v_batch_params *b,
                bool train, int64_t *stats, int64_t *steps_host, double *sum_ll_host, int64_t *n_terms_host,
                void *workspace, hipStream_t s);

}  // namespace w2v
