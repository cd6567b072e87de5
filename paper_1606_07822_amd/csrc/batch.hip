// CBOW in mini-batches: the hidden vector of a centre is the mean of its window words' vectors, normalised if the
// caller has a gain and a bias for it; the loss is the hierarchical softmax of the centre word. All gradients of a
// batch of consecutive kept centres are taken against the model at its start, and AdamW updates both tables.
//
// Per batch: k_batch_rows (means and targets), layer norm, the loss with its gradients, layer norm's backward pass,
// k_batch_words (each kept position's share of the gradient of its word), the positions' sums by word, AdamW. A
// position takes part in the windows of at most 2 W neighbours, so its gradient is gathered from their rows, without
// atomics; every sum has a fixed order, and a call's results are the same bits each time.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "w2v_ops.h"
#include "w2v_scan.h"

namespace w2v {
namespace {

constexpr int kBatchThreads = 256;
constexpr int kBatchWaves = kBatchThreads / kWave;

struct BatchArgs {
    const float *syn0;
    int32_t V, dim, stride, window;
    const int32_t *kept_vid;
    const uint32_t *kept_meta;
    const int32_t *doc_kept;
    const int64_t *kept_off;   // exclusive prefix of doc_kept
    int32_t n_docs, doc_len;
    int64_t kept;              // kept centres of the call
    int64_t lo;                // first centre of the batch
    int32_t n;                 // its centres
    int64_t first_raw, epoch_base, blk0;
    const float *alpha_tab;
    float *lr;                 // out: the batch's learning rate, that of its first centre
    float *hidden;             // [n][row]
    int32_t row;               // floats between the batch's rows
    int32_t *targets;          // [n]: the centre word, -1 where it has no window
    const uint8_t *codelen;
    int32_t *lengths;          // [n]: nodes on that word's path
    const float *dhidden;
    float *dword;              // [n + 2 window][row]: gradient of the word at each kept position around the batch
    int32_t *words;            // [n + 2 window], -1 where no centre of the batch has the position in its window
};

// Document and place of kept centre g.
__device__ __forceinline__ int32_t place_of(const BatchArgs &a, int64_t g, int32_t *j) {
    const int32_t d = wave_partition_point(0, a.n_docs, [&](int32_t m) { return a.kept_off[m] <= g; }) - 1;
    *j = static_cast<int32_t>(g - a.kept_off[d]);
    return d;
}

// The sum of the table's rows index / divisor of the lanes that `in` marks, in the lanes' order.
// Two rows at a time are on their way, whatever the row's width (NE elements a lane, 64 columns apart).
template <int NE>
__device__ __forceinline__ void sum_rows(const float *table, int64_t row_floats, int32_t dim, uint64_t in, int32_t index,
                                         float divisor, float (&sum)[NE]) {
    const int lane = lane_id(), bytes = dim * 4;
#pragma unroll
    for (int i = 0; i < NE; ++i) sum[i] = 0.0f;
    while (in) {
        float x[2][NE], d[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {   // an empty range for a row past the last
            const bool on = in != 0;
            const int l = on ? __builtin_ctzll(in) : 0;
            in &= in - 1;
            const float of = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, divisor), l));
            d[u] = on ? of : 1.0f;
            const int64_t r = __builtin_amdgcn_readlane(index, l);
            buf_load_row<NE>(x[u], __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(table) + r * row_floats, 0,
                                                                    on ? bytes : 0, kRawBufferWord3), lane);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < NE; ++i) sum[i] += x[u][i] / d[u];
    }
}

template <int NE>
__global__ __launch_bounds__(kBatchThreads) void k_batch_rows(BatchArgs a) {
    const int lane = lane_id();
    const int32_t i = static_cast<int32_t>(blockIdx.x) * kBatchWaves + static_cast<int32_t>(threadIdx.x) / kWave;
    if (i >= a.n) return;
    int32_t j = 0;
    const int32_t d = place_of(a, a.lo + i, &j);
    const int64_t base = static_cast<int64_t>(d) * a.doc_len;
    const int32_t nk = a.doc_kept[d];
    const uint32_t meta = a.kept_meta[base + j];
    const int32_t eff = static_cast<int32_t>(meta >> 16);
    const int32_t from = max(0, j - eff), P = min(nk - 1, j + eff) - from;
    if (i == 0 && lane == 0) {
        const int64_t g = a.epoch_base + a.first_raw + base + static_cast<int64_t>(meta & 0xFFFFu);
        *a.lr = a.alpha_tab[g / 10000 - a.blk0];
    }
    if (lane == 0) {
        const int32_t v = P > 0 ? a.kept_vid[base + j] : -1;
        a.targets[i] = v;
        a.lengths[i] = v >= 0 ? a.codelen[v] : 0;
    }
    const int32_t at = from + lane + (from + lane >= j ? 1 : 0);   // lane q: the q-th window word
    const int32_t mine = lane < P ? a.kept_vid[base + at] : 0;
    float h[NE];
    sum_rows<NE>(a.syn0, a.stride, a.dim, (1ull << P) - 1, mine, 1.0f, h);
#pragma unroll
    for (int e = 0; e < NE; ++e) h[e] = P > 0 ? h[e] / static_cast<float>(P) : 0.0f;
    buf_store_row<NE>(h, row_rsrc(a.hidden, i, a.row, a.dim * 4), lane);
}

template <int NE>
__global__ __launch_bounds__(kBatchThreads) void k_batch_words(BatchArgs a) {
    const int lane = lane_id();
    const int32_t k = static_cast<int32_t>(blockIdx.x) * kBatchWaves + static_cast<int32_t>(threadIdx.x) / kWave;
    if (k >= a.n + 2 * a.window) return;
    const int64_t g = a.lo - a.window + k;
    if (g < 0 || g >= a.kept) {
        if (lane == 0) a.words[k] = -1;
        return;
    }
    int32_t j = 0;
    const int32_t d = place_of(a, g, &j);
    const int64_t base = static_cast<int64_t>(d) * a.doc_len;
    const int32_t nk = a.doc_kept[d];
    // lane l: the centre at place j - window + l, if it is in the batch and has this position in its window
    const int32_t c = j - a.window + lane;
    const int64_t of = g - a.window + lane - a.lo;   // its row of the batch
    float share = 0.0f;
    if (lane <= 2 * a.window && c >= 0 && c < nk && c != j && of >= 0 && of < a.n) {
        const int32_t eff = static_cast<int32_t>(a.kept_meta[base + c] >> 16);
        if (abs(c - j) <= eff) share = static_cast<float>(min(nk - 1, c + eff) - max(0, c - eff));
    }
    const uint64_t in = __ballot(share > 0.0f);
    if (lane == 0) a.words[k] = in ? a.kept_vid[base + j] : -1;
    if (!in) return;
    float e[NE];   // a centre's mean has a part of 1 / its window words in each of them
    sum_rows<NE>(a.dhidden, a.row, a.dim, in, static_cast<int32_t>(of), share, e);
    buf_store_row<NE>(e, row_rsrc(a.dword, k, a.row, a.dim * 4), lane);
}

struct Totals {
    double loss;
    int64_t terms, nodes;
};

// A batch's loss, terms and path nodes, summed by up to kTotalGroups workgroups (one alone fetches 65,536 rows' numbers in
// 54 us), whose sums k_batch_totals adds to the call's. In a fixed order. A centre without a window gets an rstd of
// 0 for the norm's backward pass, so that its normalised row is zeros there: with norm_eps 0 the forward pass leaves an
// infinite one and a row of NaN, which the zeros of the row's gradient would not take out of the gain's sums.
constexpr int kTotalThreads = 1024;
constexpr int kTotalGroups = 64;   // a wavefront adds them up
__global__ __launch_bounds__(kTotalThreads) void k_batch_parts(const float *__restrict__ loss,
                                                               const int32_t *__restrict__ targets,
                                                               const int32_t *__restrict__ lengths, int32_t n,
                                                               float *__restrict__ rstd, Totals *parts) {
    constexpr int kWaves = kTotalThreads / kWave;
    __shared__ double s_loss[kWaves];
    __shared__ int64_t s_terms[kWaves], s_nodes[kWaves];
    double sum = 0.0;
    int64_t terms = 0, nodes = 0;
    const int32_t step = static_cast<int32_t>(gridDim.x) * kTotalThreads;
    for (int32_t i = static_cast<int32_t>(blockIdx.x) * kTotalThreads + static_cast<int32_t>(threadIdx.x); i < n; i += step) {
        if (targets[i] < 0) {
            if (rstd) rstd[i] = 0.0f;
            continue;
        }
        sum += static_cast<double>(loss[i]);
        ++terms;
        nodes += lengths[i];
    }
    sum = wave_sum(sum);
    terms = wave_sum(terms);
    nodes = wave_sum(nodes);
    const int wid = static_cast<int>(threadIdx.x) / kWave;
    if (lane_id() == 0) {
        s_loss[wid] = sum;
        s_terms[wid] = terms;
        s_nodes[wid] = nodes;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; ++w) {
            sum += s_loss[w];
            terms += s_terms[w];
            nodes += s_nodes[w];
        }
        parts[blockIdx.x] = Totals{sum, terms, nodes};
    }
}

__global__ __launch_bounds__(kWave) void k_batch_totals(const Totals *parts, int n, Totals *to) {
    const int lane = lane_id();
    const Totals mine = lane < n ? parts[lane] : Totals{0.0, 0, 0};
    const double sum = wave_sum(mine.loss);
    const int64_t terms = wave_sum(mine.terms), nodes = wave_sum(mine.nodes);
    if (lane == 0) {
        to->loss += sum;
        to->terms += terms;
        to->nodes += nodes;
    }
}

__global__ __launch_bounds__(kScanThreads) void k_batch_scan(const int32_t *__restrict__ in, int64_t n,
                                                             int64_t *__restrict__ out, Totals *totals) {
    block_exclusive_scan(in, n, out);
    if (threadIdx.x == 0) *totals = Totals{0.0, 0, 0};
}

__global__ void k_batch_stats(const int64_t *sampled, const Totals *t, int64_t *stats) {
    if (threadIdx.x < 4) stats[threadIdx.x] = sampled[threadIdx.x];
    if (threadIdx.x == 4) stats[4] = t->nodes;
}

// Calls f with the elements that a lane holds of a row of dim floats.
template <class F>
void with_columns(int32_t dim, F f) {
    const int64_t ne = ceil_div(dim, kWave);
    if (ne <= 1) f(std::integral_constant<int, 1>{});
    else if (ne <= 2) f(std::integral_constant<int, 2>{});
    else if (ne <= 4) f(std::integral_constant<int, 4>{});
    else if (ne <= 5) f(std::integral_constant<int, 5>{});
    else if (ne <= 8) f(std::integral_constant<int, 8>{});
    else f(std::integral_constant<int, 16>{});
}

struct Buffers {
    SampleBufs sample;
    float *alpha_tab, *lr, *hidden, *normed, *dnormed, *loss, *mean, *rstd, *dgain, *dsyn0, *dsyn1, *dword;
    int64_t *kept_off;
    Totals *totals, *parts;
    int32_t *targets, *lengths, *words;
    char *loss_ws, *norm_ws, *sum_ws, *plan;
    int32_t row;
};

int64_t blocks_of(int64_t n) { return ceil_div(n, kMomentBlock) * kMomentBlock; }

// syn0, syn1 and, with a layer norm, its gain and bias.
int fill_tensors(const w2v_model *m, const w2v_batch_params *b, const Buffers &w, w2v_adamw_tensor (&t)[4]) {
    const int64_t d = m->dim;
    int64_t at = 0;
    auto add = [&](int k, float *p, float *g, int64_t rows, int64_t p_stride, int64_t g_stride, float decay) {
        t[k] = w2v_adamw_tensor{p, g, rows, d, p_stride, g_stride, at, W2V_F32, W2V_F32, decay, 0};
        at += blocks_of(rows * d);
    };
    add(0, m->syn0, w.dsyn0, m->V, m->row_stride, w.row, b->weight_decay);
    add(1, m->syn1, w.dsyn1, m->V - 1, m->row_stride, w.row, b->weight_decay);
    if (!b->gain) return 2;
    add(2, b->gain, w.dgain, 1, d, d, 0.0f);
    add(3, b->bias, w.dgain ? w.dgain + d : nullptr, 1, d, d, 0.0f);
    return 4;
}

Buffers carve(Carve &c, const w2v_model *m, int64_t n_tokens, const w2v_params *p, const w2v_batch_params *b, bool train) {
    Buffers w{};
    w.sample = sample_bufs_carve(c, m->V, n_tokens, p->doc_len);
    w.row = static_cast<int32_t>(ceil_div(m->dim, 4) * 4);
    const int64_t n_docs = std::max<int64_t>(1, ceil_div(n_tokens, p->doc_len));
    const auto rows = static_cast<size_t>(p->sync_batch), wide = rows * static_cast<size_t>(w.row);
    w.alpha_tab = c.take<float>(static_cast<size_t>(std::max<int64_t>(1, n_tokens) / 10000 + 3));
    w.kept_off = c.take<int64_t>(static_cast<size_t>(n_docs));
    w.totals = c.take<Totals>(1);
    w.parts = c.take<Totals>(kTotalGroups);
    w.lr = c.take<float>(1);
    w.targets = c.take<int32_t>(rows);
    w.lengths = c.take<int32_t>(rows);
    w.loss = c.take<float>(rows);
    w.hidden = c.take<float>(wide);
    w.normed = w.hidden;
    if (b->gain) {
        w.normed = c.take<float>(wide);
        w.mean = c.take<float>(rows);
        w.rstd = c.take<float>(rows);
    }
    if (!train) return w;
    const size_t around = rows + 2 * static_cast<size_t>(p->window);
    w.dnormed = c.take<float>(wide);   // layer norm's backward pass turns it into the hidden vectors' gradient
    w.words = c.take<int32_t>(around);
    w.dword = c.take<float>(around * static_cast<size_t>(w.row));
    w.dsyn0 = c.take<float>(static_cast<size_t>(m->V) * w.row);
    w.dsyn1 = c.take<float>(static_cast<size_t>(m->V) * w.row);
    w.loss_ws = c.take<char>(hs_loss_bytes(p->sync_batch, m->dim, b->max_code_len));
    w.sum_ws = c.take<char>(word_sums_bytes(static_cast<int64_t>(around), m->dim));
    if (b->gain) {
        w.dgain = c.take<float>(2 * static_cast<size_t>(m->dim));
        w.norm_ws = c.take<char>(norm_backward_bytes(p->sync_batch, m->dim));
    }
    w2v_adamw_tensor t[4];
    const int n = fill_tensors(m, b, w, t);
    w.plan = c.take<char>(adamw_plan_bytes(t, n));
    return w;
}

}  // namespace

int64_t batch_moments(const w2v_model *m, const w2v_batch_params *b) {
    const int64_t d = m->dim;
    return blocks_of(m->V * d) + blocks_of((m->V - 1) * d) + (b->gain ? 2 * blocks_of(d) : 0);
}

size_t batch_bytes(const w2v_model *m, int64_t n_tokens, const w2v_params *p, const w2v_batch_params *b, bool train) {
    Carve c;
    carve(c, m, n_tokens, p, b, train);
    return c.used();
}

int run_batches(const w2v_model *m, const int32_t *tokens, int64_t n_tokens, const w2v_params *p, const w2v_batch_params *b,
                bool train, int64_t *stats, int64_t *steps_host, double *sum_ll_host, int64_t *n_terms_host,
                void *workspace, hipStream_t s) {
    Carve c(workspace);
    const Buffers w = carve(c, m, n_tokens, p, b, train);
    if (int rc = launch_sampling(tokens, n_tokens, m->V, m->vocab_counts, m->train_words, p, w.sample, nullptr, s)) return rc;
    const int64_t n_docs = n_tokens > 0 ? ceil_div(n_tokens, p->doc_len) : 0, span = std::max<int64_t>(1, n_tokens);
    const int64_t epoch_base = static_cast<int64_t>(p->epoch) * p->corpus_tokens;
    const int64_t blk0 = (epoch_base + p->first_raw_index) / 10000;
    const int64_t blk1 = (epoch_base + p->first_raw_index + span - 1) / 10000;
    if (int rc = launch_alpha_table(p, blk0, blk1 - blk0 + 1, w.alpha_tab, s)) return rc;
    k_batch_scan<<<1, kScanThreads, 0, s>>>(w.sample.doc_kept, n_docs, w.kept_off, w.totals);
    W2V_LAUNCH_CHECK("k_batch_scan");
    int64_t sampled[4];
    W2V_HIP(hipMemcpyAsync(sampled, w.sample.totals, sizeof(sampled), hipMemcpyDeviceToHost, s));
    W2V_HIP(hipStreamSynchronize(s));
    int64_t chunks = 0;
    if (train) {
        w2v_adamw_tensor t[4];
        const int n = fill_tensors(m, b, w, t);
        if (int rc = run_adamw_plan(t, n, w.plan, s)) return rc;
        chunks = adamw_chunks(t, n);
    }
    BatchArgs a{};
    a.syn0 = m->syn0;
    a.V = m->V;
    a.dim = m->dim;
    a.stride = m->row_stride;
    a.window = p->window;
    a.kept_vid = w.sample.kept_vid;
    a.kept_meta = w.sample.kept_meta;
    a.doc_kept = w.sample.doc_kept;
    a.kept_off = w.kept_off;
    a.n_docs = static_cast<int32_t>(n_docs);
    a.doc_len = p->doc_len;
    a.kept = sampled[2];
    a.first_raw = p->first_raw_index;
    a.epoch_base = epoch_base;
    a.blk0 = blk0;
    a.alpha_tab = w.alpha_tab;
    a.lr = w.lr;
    a.hidden = w.hidden;
    a.row = w.row;
    a.targets = w.targets;
    a.codelen = m->codelen;
    a.lengths = w.lengths;
    a.dhidden = w.dnormed;
    a.dword = w.dword;
    a.words = w.words;
    int64_t step = b->step0;
    for (a.lo = 0; a.lo < a.kept; a.lo += p->sync_batch) {
        a.n = static_cast<int32_t>(std::min<int64_t>(p->sync_batch, a.kept - a.lo));
        with_columns(m->dim, [&](auto ne) {
            k_batch_rows<decltype(ne)::value>
                <<<static_cast<unsigned>(ceil_div(a.n, kBatchWaves)), kBatchThreads, 0, s>>>(a);
        });
        W2V_LAUNCH_CHECK("k_batch_rows");
        NormArgs f{};
        if (b->gain) {
            f.x = w.hidden;
            f.rows = a.n;
            f.dim = m->dim;
            f.type = f.w_type = W2V_F32;
            f.x_stride = f.dy_stride = f.out_stride = w.row;
            f.w = b->gain;
            f.b = b->bias;
            f.eps = b->norm_eps;
            f.out = w.normed;
            f.mean = w.mean;
            f.rstd = w.rstd;
            if (int rc = run_layer_norm(f, s)) return rc;
        }
        HsLossArgs h{};
        h.V = m->V;
        h.dim = m->dim;
        h.stride = m->row_stride;
        h.longest = b->max_code_len;
        h.syn1 = m->syn1;
        h.codelen = m->codelen;
        h.code = m->code;
        h.point_off = m->point_off;
        h.points = m->points;
        h.x = w.normed;
        h.type = W2V_F32;
        h.rows = a.n;
        h.x_stride = w.row;
        h.targets = w.targets;
        h.loss = w.loss;
        if (train) {
            h.dx = w.dnormed;
            h.dx_stride = w.row;
            h.dsyn1 = w.dsyn1;
            h.dsyn1_stride = w.row;
            h.dsyn1_whole = true;
        }
        if (int rc = run_hs_loss(h, w.loss_ws, s)) return rc;
        const auto groups = static_cast<int>(std::min<int64_t>(kTotalGroups, ceil_div(a.n, kTotalThreads)));
        k_batch_parts<<<static_cast<unsigned>(groups), kTotalThreads, 0, s>>>(w.loss, w.targets, w.lengths, a.n,
                                                                                  w.rstd, w.parts);
        W2V_LAUNCH_CHECK("k_batch_parts");
        k_batch_totals<<<1, kWave, 0, s>>>(w.parts, groups, w.totals);
        W2V_LAUNCH_CHECK("k_batch_totals");
        if (!train) continue;
        if (b->gain) {
            f.dy = w.dnormed;
            f.out = w.dnormed;
            f.dw = w.dgain;
            f.db = w.dgain + m->dim;
            if (int rc = run_layer_norm_backward(f, w.norm_ws, s)) return rc;
        }
        const int64_t around = a.n + 2 * static_cast<int64_t>(p->window);
        with_columns(m->dim, [&](auto ne) {
            k_batch_words<decltype(ne)::value>
                <<<static_cast<unsigned>(ceil_div(around, kBatchWaves)), kBatchThreads, 0, s>>>(a);
        });
        W2V_LAUNCH_CHECK("k_batch_words");
        if (int rc = run_word_sums(w.words, w.dword, around, m->dim, w.row, m->V, w.dsyn0, w.row, w.sum_ws, s)) return rc;
        w2v_adamw_params o{};
        o.beta1 = b->beta1;
        o.beta2 = b->beta2;
        o.eps = b->eps;
        o.step = ++step;
        o.lr_device = w.lr;
        o.grad_scale = 1.0f / static_cast<float>(a.n);
        o.seed = b->seed;
        if (int rc = run_adamw_step(w.plan, chunks, b->bits, b->m, b->v, b->m_scale, b->v_scale, o, s)) return rc;
        *steps_host = step - b->step0;   // kept up to date: a later error leaves the steps that were launched
    }
    if (stats) {
        k_batch_stats<<<1, kWave, 0, s>>>(w.sample.totals, w.totals, stats);
        W2V_LAUNCH_CHECK("k_batch_stats");
    }
    Totals t{};
    W2V_HIP(hipMemcpyAsync(&t, w.totals, sizeof(t), hipMemcpyDeviceToHost, s));
    W2V_HIP(hipStreamSynchronize(s));
    if (sum_ll_host) *sum_ll_host = -t.loss;
    if (n_terms_host) *n_terms_host = t.terms;
    return W2V_OK;
}

}  // namespace w2v
