// The hierarchical softmax as a loss with gradients, for a batch of hidden vectors x_i with target words v_i:
//
//   z_j = x . syn1[n_j] along v's path, s_j = 1 - 2 t_j,  loss = sum_j log(1 + exp(-s_j z_j))
//   g_j = -w s_j sigmoid(-s_j z_j),  dx = sum_j g_j syn1[n_j],  dsyn1[n] = sum over the rows through n of g x
//
// The walk (k_hs_walk) is a wavefront per row: four inner nodes at a time, the next four on their way, dot products
// reduced together. It reads a path's rows once for z and dx, and leaves the row's coefficients g_j.
//
// dsyn1 is a sum over rows without atomics, in a fixed order. Rows are sorted by their word's code, left-aligned, so
// that the rows through an inner node are neighbours: node (row, j) continues its neighbour's where their codes share
// j bits. A wavefront holds kRows sorted rows' x in registers, 64 columns a lane each, and goes down the levels: a
// level's nodes are runs of rows, summed and written out where a run ends. Runs that reach over a block's border are
// written as partial sums, which k_hs_join adds up in order, 64 blocks at a time. The same sum with one level, every row
// for its own word's row of the table, is the gradient of a table's looked-up rows (run_word_sums).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "w2v_ops.h"

namespace w2v {
namespace {

constexpr int kSlab = 65536;      // rows sorted and summed together; a longer batch takes several, each adding to dsyn1
constexpr int kSortBlock = 2048;  // rows ranked against each other
constexpr int kRows = 64;         // sorted rows of a wavefront's sum
constexpr int kFan = 64;          // blocks that one wavefront joins
constexpr int kXcds = 8;

// What a row's target stands for: a word's path, or (codelen null, longest 1) one row of the table, the word's own.
struct Tree {
    int32_t V, longest;
    const uint8_t *codelen;
    const uint64_t *code;
    const int32_t *point_off, *points;
};

// Inner nodes on a target's path: none for a row without a target, nor for a word that is not in the tree (its loss is
// a NaN, see k_hs_walk).
__device__ __forceinline__ int path_len(const Tree &t, int32_t v) {
    if (v < 0 || v >= t.V) return 0;
    const int len = t.codelen ? t.codelen[v] : 1;
    return len <= t.longest ? len : 0;
}

// The code with its first turn in the top bit; rows without a path come last.
__device__ __forceinline__ uint64_t sort_key(const Tree &t, int32_t v) {
    const int len = path_len(t, v);
    if (len == 0) return ~0ull;
    return t.codelen ? __brevll(t.code[v]) & (~0ull << (64 - len)) : static_cast<uint64_t>(v);
}

// Levels that two neighbouring sorted rows share an inner node at.
__device__ __forceinline__ int shared_levels(const Tree &t, int32_t va, int la, uint64_t ka, int32_t vb, int lb,
                                             uint64_t kb) {
    if (la == 0 || lb == 0) return 0;
    if (va == vb) return la;
    return t.codelen ? min(min(la, lb), static_cast<int>(__clzll(static_cast<long long>(ka ^ kb))) + 1) : 0;
}

__device__ __forceinline__ int node_at(const Tree &t, int32_t v, int level) {   // of a path that long
    return t.codelen ? t.points[t.point_off[v] + level] : v;
}

// ------------------------------------------------------------------ order
// Each key's place among the kSortBlock keys of its block, by counting the smaller ones (equal keys keep their order):
// a workgroup places 64 rows, its wavefronts count in a sixteenth of the block each. Two instructions a comparison.
constexpr int kRankThreads = 1024;
constexpr int kRankWaves = kRankThreads / kWave;
__global__ __launch_bounds__(kRankThreads) void k_hs_rank(Tree t, const int32_t *__restrict__ targets, int32_t n,
                                                          uint64_t *__restrict__ key_out, int32_t *__restrict__ row_out) {
    __shared__ uint64_t keys[kSortBlock];
    __shared__ int32_t counts[kRankWaves][kWave];
    constexpr int kPerBlock = kSortBlock / kWave;
    const int32_t lo = static_cast<int32_t>(blockIdx.x) / kPerBlock * kSortBlock;
    const int own = static_cast<int>(blockIdx.x) % kPerBlock;   // this workgroup's 64 rows of the block
    const int len = min(kSortBlock, n - lo);
    if (own * kWave >= len) return;
    for (int i = threadIdx.x; i < kSortBlock; i += kRankThreads) keys[i] = i < len ? sort_key(t, targets[lo + i]) : ~0ull;
    __syncthreads();
    const int lane = lane_id(), wid = static_cast<int>(threadIdx.x) / kWave;
    const uint64_t mine = keys[own * kWave + lane];
    int32_t c = 0;
    for (int seg = wid; seg * kWave < len; seg += kRankWaves) {
        const uint64_t *k = keys + seg * kWave;
        const int most = min(kWave, len - seg * kWave);
        if (seg < own) {
            for (int j = 0; j < most; ++j) c += k[j] <= mine ? 1 : 0;
        } else if (seg > own) {
            for (int j = 0; j < most; ++j) c += k[j] < mine ? 1 : 0;
        } else {
            for (int j = 0; j < most; ++j) c += k[j] < mine || (k[j] == mine && j < lane) ? 1 : 0;
        }
    }
    counts[wid][lane] = c;
    __syncthreads();
    if (wid == 0 && own * kWave + lane < len) {
        int32_t at = lo;
#pragma unroll
        for (int w = 0; w < kRankWaves; ++w) at += counts[w][lane];
        key_out[at] = mine;
        row_out[at] = lo + own * kWave + lane;
    }
}

// Each key's place among all: its place in its own sorted block and, in every other, the keys before it (equal ones
// count where their block comes first), found by bisection in LDS, four blocks at once.
constexpr int kMergeThreads = 256;
constexpr int kMergeBlocks = 4;
__global__ __launch_bounds__(kMergeThreads) void k_hs_merge(const uint64_t *__restrict__ key_in,
                                                            const int32_t *__restrict__ row_in, int32_t n,
                                                            uint64_t *__restrict__ key_out, int32_t *__restrict__ row_out) {
    __shared__ uint64_t keys[kMergeBlocks][kSortBlock];
    const int32_t i = static_cast<int32_t>(blockIdx.x) * kMergeThreads + static_cast<int32_t>(threadIdx.x);
    const int own = i / kSortBlock, blocks = static_cast<int>(ceil_div(n, kSortBlock));
    const uint64_t mine = i < n ? key_in[i] : 0;
    int32_t at = i % kSortBlock;
    for (int b0 = 0; b0 < blocks; b0 += kMergeBlocks) {
        __syncthreads();
        for (int j = threadIdx.x; j < kMergeBlocks * kSortBlock; j += kMergeThreads) {
            const int32_t k = b0 * kSortBlock + j;
            (&keys[0][0])[j] = k < n ? key_in[k] : ~0ull;   // past the end: after every key
        }
        __syncthreads();
        int32_t lo[kMergeBlocks], len[kMergeBlocks];
#pragma unroll
        for (int u = 0; u < kMergeBlocks; ++u) {
            lo[u] = 0;
            len[u] = max(0, min(kSortBlock, n - (b0 + u) * kSortBlock));
        }
        for (int step = kSortBlock; step > 0; step >>= 1) {
#pragma unroll
            for (int u = 0; u < kMergeBlocks; ++u) {
                const int32_t p = lo[u] + step;
                if (p > len[u]) continue;
                const uint64_t k = keys[u][p - 1];
                if (k < mine || (k == mine && b0 + u < own)) lo[u] = p;
            }
        }
#pragma unroll
        for (int u = 0; u < kMergeBlocks; ++u)
            if (b0 + u != own) at += lo[u];
    }
    if (i < n) {
        key_out[at] = mine;
        row_out[at] = row_in[i];
    }
}

// ------------------------------------------------------------------ the walk
struct WalkArgs {
    Tree t;
    const float *syn1;
    int32_t stride, dim;
    const void *x;
    int64_t x_stride;
    const int32_t *targets;
    const float *weights;   // null: ones
    const int32_t *order;   // sorted place -> row; null: the rows' own order
    int32_t n;
    float *loss;            // null: not written
    void *dx;               // null: not written
    int64_t dx_stride;
    float *coef;            // [block of kRows][level][row of the block]; null: not written
};

constexpr int kWalkThreads = 256;

template <class T, int NE, bool GRADS>
__global__ __launch_bounds__(kWalkThreads) void k_hs_walk(WalkArgs a) {
    const int lane = lane_id();
    // neighbouring sorted rows share most of their path: each XCD, with an L2 of its own, takes one stretch of them
    const int per = static_cast<int>(gridDim.x) / kXcds;
    const int group = static_cast<int>(blockIdx.x) < per * kXcds
                          ? static_cast<int>(blockIdx.x) % kXcds * per + static_cast<int>(blockIdx.x) / kXcds
                          : static_cast<int>(blockIdx.x);
    const int pos = group * (kWalkThreads / kWave) + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    if (pos >= a.n) return;
    const int row = a.order ? a.order[pos] : pos;
    const int32_t v = a.targets[row];
    const int len = path_len(a.t, v);
    const int pt = lane < len ? a.t.points[a.t.point_off[v] + lane] : 0;
    const uint64_t code = len > 0 ? a.t.code[v] : 0;
    const float weight = GRADS && a.weights ? a.weights[row] : 1.0f;
    const T *xr = static_cast<const T *>(a.x) + row * a.x_stride;
    float x[NE], dx[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const int col = lane + i * kWave;
        x[i] = len > 0 && col < a.dim ? static_cast<float>(xr[col]) : 0.0f;
        dx[i] = 0.0f;
    }
    float y[4][NE];
    auto load = [&](int j) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {   // zeros past the path's end
            const bool in = j + u < len;
            const int node = __builtin_amdgcn_readlane(pt, min(j + u, kWave - 1));
            buf_load_row<NE>(y[u], row_rsrc(const_cast<float *>(a.syn1), in ? node : 0, a.stride, in ? a.dim * 4 : 0), lane);
        }
    };
    load(0);
    // log(1 + e) of a path's nodes as the logarithm of their product, at most 2^64
    float wrong = 0.0f, prod = 1.0f, g_all = 0.0f;
    for (int j = 0; j < len; j += 4) {
        float now[4][NE];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < NE; ++i) now[u][i] = y[u][i];
        load(j + 4);
        const float z = reduce4(dot_partial<NE>(x, now[0]), dot_partial<NE>(x, now[1]), dot_partial<NE>(x, now[2]),
                                dot_partial<NE>(x, now[3]));   // lanes 16u..16u+15: node j + u
        const int level = j + (lane >> 4);
        const bool in = level < len;
        const float sz = (code >> min(level, 63)) & 1ull ? -z : z;
        const float e = in ? __expf(-fabsf(z)) : 0.0f;
        prod *= 1.0f + e;
        wrong += in && sz < 0.0f ? -sz : 0.0f;
        if constexpr (GRADS) {
            const float f = (sz < 0.0f ? 1.0f : e) / (1.0f + e);   // sigmoid(-s z)
            const float g = in ? (((code >> min(level, 63)) & 1ull) ? f : -f) * weight : 0.0f;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float gu = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, g), 16 * u));
#pragma unroll
                for (int i = 0; i < NE; ++i) dx[i] = fmaf(gu, now[u][i], dx[i]);
                if (lane == j + u) g_all = gu;
            }
        }
    }
    if (a.loss) {
        // a row of lanes holds every fourth node's sums
        const float p0 = __shfl(prod, 0, kWave), p1 = __shfl(prod, 16, kWave), p2 = __shfl(prod, 32, kWave),
                    p3 = __shfl(prod, 48, kWave);
        const float s = rows_sum(wrong) + logf((p0 * p1) * (p2 * p3));
        const bool missing = v >= 0 && len == 0;   // a target that the tree does not hold
        if (lane == 0) a.loss[row] = missing ? __builtin_nanf("") : s;
    }
    if constexpr (GRADS) {
        if (a.dx) {
            T *out = static_cast<T *>(a.dx) + row * a.dx_stride;
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                const int col = lane + i * kWave;
                if (col < a.dim) out[col] = static_cast<T>(dx[i]);
            }
        }
        if (a.coef && lane < a.t.longest) {
            float *c = a.coef + static_cast<int64_t>(pos / kRows) * a.t.longest * kRows;
            c[lane * kRows + pos % kRows] = g_all;
        }
    }
}

// ------------------------------------------------------------------ the inner nodes' sums
// Of a block of sorted rows: the levels that its first row shares with the row before it, and the fewest that two of
// its neighbouring rows share.
struct Borders {
    int32_t *left, *inner;
};

struct NodeArgs {
    Tree t;
    const uint64_t *keys;
    const int32_t *order, *targets;
    int32_t n, dim;
    const void *x;
    int64_t x_stride;
    const float *coef;  // null: ones
    float *part;        // [block][2][level][dim]: sums of runs that come in from the left, and of those that go on right
    Borders borders;
    float *dsyn1;
    int64_t out_stride;
    int32_t add;        // dsyn1 holds an earlier slab's sums
};

__device__ __forceinline__ void put(float *to, float v, bool add) { *to = add ? *to + v : v; }

template <class T, bool COEF>
__global__ __launch_bounds__(kWave) void k_hs_nodes(NodeArgs a) {
    const int lane = lane_id();
    const int blk = static_cast<int>(blockIdx.x), longest = a.t.longest;
    const int col = static_cast<int>(blockIdx.y) * kWave + lane;
    const int p0 = blk * kRows, rows = min(kRows, a.n - p0);
    // lane q: row q of the block
    const int pos = p0 + lane;
    const bool on = lane < rows;
    const int row = on ? a.order[pos] : 0;
    const int32_t v = on ? a.targets[row] : -1;
    const int len = path_len(a.t, v);
    auto neighbour = [&](int at) {   // levels that the row at place `at` shares with the one before it
        const int32_t va = a.targets[a.order[at - 1]], vb = a.targets[a.order[at]];
        return shared_levels(a.t, va, path_len(a.t, va), a.keys[at - 1], vb, path_len(a.t, vb), a.keys[at]);
    };
    const int before = on && pos > 0 ? neighbour(pos) : 0;
    const int after = on && pos + 1 < a.n ? neighbour(pos + 1) : 0;
    const int left = __builtin_amdgcn_readlane(before, 0);
    const int right = __builtin_amdgcn_readlane(after, kWave - 1);
    int deepest = len, inner = on && lane > 0 ? before : kWave;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        deepest = max(deepest, __shfl_xor(deepest, m, kWave));
        inner = min(inner, __shfl_xor(inner, m, kWave));
    }
    deepest = __builtin_amdgcn_readfirstlane(deepest);
    if (blockIdx.y == 0 && lane == 0) {
        a.borders.left[blk] = left;
        a.borders.inner[blk] = inner;
    }
    float x[kRows];
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
        x[q] = 0.0f;
        const int r = __builtin_amdgcn_readlane(row, q);
        if (q < rows && col < a.dim) x[q] = static_cast<float>((static_cast<const T *>(a.x) + r * a.x_stride)[col]);
    }
    const float *coef = COEF ? a.coef + static_cast<int64_t>(blk) * longest * kRows : nullptr;
    for (int j = 0; j < deepest; ++j) {
        const uint64_t active = __ballot(len > j);
        const uint64_t ends = __ballot(len > j && (after <= j || lane == kWave - 1));
        const int node = len > j ? node_at(a.t, v, j) : 0;
        const float *c = COEF ? coef + j * kRows : nullptr;
        float acc = 0.0f;
#pragma unroll
        for (int q = 0; q < kRows; ++q) {
            if ((active >> q) & 1ull) {
                acc = COEF ? fmaf(c[q], x[q], acc) : acc + x[q];
                if ((ends >> q) & 1ull) {
                    const bool from_left = left > j && (ends & ((1ull << q) - 1)) == 0;
                    const bool to_right = q == kRows - 1 && right > j;
                    if (col < a.dim) {
                        if (from_left || to_right) {
                            const int64_t slot = (static_cast<int64_t>(blk) * 2 + (from_left ? 0 : 1)) * longest + j;
                            a.part[slot * a.dim + col] = acc;
                        } else {
                            put(a.dsyn1 + __builtin_amdgcn_readlane(node, q) * a.out_stride + col, acc, a.add);
                        }
                    }
                    acc = 0.0f;
                }
            }
        }
    }
}

struct JoinArgs {
    Tree t;
    const int32_t *order, *targets;
    int32_t n, dim;
    const float *in;    // [block][2][level][dim]
    Borders borders;
    int32_t blocks, rows;   // rows of a block
    float *out;         // the same of kFan blocks together
    Borders out_borders;
    float *dsyn1;
    int64_t out_stride;
    int32_t add;
};

// Partial sums of kFan neighbouring blocks at one level, in order: a run's first part lies on a block's right, the
// others on the left of the blocks that follow.
__global__ __launch_bounds__(kWave) void k_hs_join(JoinArgs a) {
    const int lane = lane_id(), level = static_cast<int>(blockIdx.z), longest = a.t.longest;
    const int first = static_cast<int>(blockIdx.x) * kFan, blk = first + lane;
    const int col = static_cast<int>(blockIdx.y) * kWave + lane;
    const bool on = blk < a.blocks;
    const int left = on ? a.borders.left[blk] : 0, inner = on ? a.borders.inner[blk] : kWave;
    const int right = on && blk + 1 < a.blocks ? a.borders.left[blk + 1] : 0;
    if (blockIdx.y == 0 && level == 0) {
        int least = on ? min(inner, lane > 0 ? left : kWave) : kWave;
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) least = min(least, __shfl_xor(least, m, kWave));
        if (lane == 0) {
            a.out_borders.left[blockIdx.x] = left;
            a.out_borders.inner[blockIdx.x] = least;
        }
    }
    const uint64_t has_left = __ballot(left > level);
    const uint64_t through = __ballot(left > level && inner > level && right > level);
    const uint64_t has_right = __ballot(right > level) & ~through;
    if (!(has_left | has_right)) return;
    // the node that comes in from a block's left lies on its first row's path
    int node = 0;
    if (left > level) {
        node = node_at(a.t, a.targets[a.order[static_cast<int64_t>(blk) * a.rows]], level);
    }
    const int bytes = a.dim * 4;
    const int64_t block_rows = static_cast<int64_t>(2) * longest;
    float *in = const_cast<float *>(a.in);
    bool outside = has_left & 1ull;   // the run at hand began before these blocks
    float acc = 0.0f;
    constexpr int kAhead = 16;
    for (int b0 = 0; b0 < kFan && first + b0 < a.blocks; b0 += kAhead) {
        float l[kAhead], r[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {   // an empty range where there is none: no branch around the loads
            const int b = b0 + u;
            const int64_t at = (first + b) * block_rows + level;
            const bool hl = (has_left >> b) & 1ull, hr = (has_right >> b) & 1ull;
            l[u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(
                row_rsrc(in, hl ? at : 0, a.dim, hl ? bytes : 0), col * 4, 0, 0));
            r[u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(
                row_rsrc(in, hr ? at + longest : 0, a.dim, hr ? bytes : 0), col * 4, 0, 0));
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int b = b0 + u;
            if ((has_left >> b) & 1ull) {
                acc += l[u];
                if (!((through >> b) & 1ull)) {
                    if (col < a.dim) {
                        if (outside)
                            a.out[(static_cast<int64_t>(blockIdx.x) * 2 * longest + level) * a.dim + col] = acc;
                        else
                            put(a.dsyn1 + __builtin_amdgcn_readlane(node, b) * a.out_stride + col, acc, a.add);
                    }
                    outside = false;
                    acc = 0.0f;
                }
            }
            if ((has_right >> b) & 1ull) {
                acc = r[u];
                outside = false;
            }
        }
    }
    // a run that goes on past the last block
    if (((has_right | through) >> (kFan - 1)) & 1ull) {
        if (col < a.dim)
            a.out[((static_cast<int64_t>(blockIdx.x) * 2 + (outside ? 0 : 1)) * longest + level) * a.dim + col] = acc;
    }
}

// The first dim columns of the rows set to zero: four at a time where dim is a multiple of 4.
__global__ __launch_bounds__(256) void k_hs_zero(float *p, int64_t rows, int32_t dim, int64_t stride) {
    const int per = dim % 4 == 0 ? 4 : 1, width = dim / per;
    const int64_t step = static_cast<int64_t>(gridDim.x) * blockDim.x;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < rows * width; i += step) {
        const int64_t r = i / width;
        float *to = p + r * stride + (i - r * width) * per;
        if (per == 4) {
            const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            store_pack<float, 4>(to, zero);
        } else {
            *to = 0.0f;
        }
    }
}

struct Buffers {
    uint64_t *key0, *key1;
    int32_t *row0, *row1;
    float *coef, *part[2];
    Borders borders[3];
};

int64_t blocks_of(int64_t n) { return ceil_div(n, kRows); }

Buffers carve(Carve &c, int64_t rows, int32_t dim, int32_t longest) {
    const auto n = static_cast<size_t>(std::min<int64_t>(std::max<int64_t>(rows, 1), kSlab));
    const auto blocks = static_cast<size_t>(blocks_of(static_cast<int64_t>(n)));
    const size_t fans = (blocks + kFan - 1) / kFan, level = static_cast<size_t>(2) * longest * dim;
    Buffers b;
    b.key0 = c.take<uint64_t>(n);
    b.key1 = c.take<uint64_t>(n);
    b.row0 = c.take<int32_t>(n);
    b.row1 = c.take<int32_t>(n);
    b.coef = c.take<float>(blocks * longest * kRows);
    b.part[0] = c.take<float>(blocks * level);
    b.part[1] = c.take<float>(fans * level);
    const size_t counts[3] = {blocks, fans, 1};
    for (int k = 0; k < 3; ++k) {
        b.borders[k].left = c.take<int32_t>(counts[k]);
        b.borders[k].inner = c.take<int32_t>(counts[k]);
    }
    return b;
}

template <class T, int NE>
void launch_walk(const WalkArgs &w, bool grads, unsigned grid, hipStream_t s) {
    if (grads)
        k_hs_walk<T, NE, true><<<grid, kWalkThreads, 0, s>>>(w);
    else
        k_hs_walk<T, NE, false><<<grid, kWalkThreads, 0, s>>>(w);
}

int zero_rows(float *p, int64_t rows, int32_t dim, int64_t stride, hipStream_t s) {
    const auto grid = static_cast<unsigned>(std::min<int64_t>(ceil_div(rows * dim, 1024), 64LL * device_cu_count()));
    k_hs_zero<<<grid, 256, 0, s>>>(p, rows, dim, stride);
    W2V_LAUNCH_CHECK("k_hs_zero");
    return W2V_OK;
}

// Sorts n <= kSlab rows by their targets' keys.
int sort_rows(const Tree &t, const int32_t *targets, int32_t n, const Buffers &b, const int32_t **order,
              const uint64_t **keys, hipStream_t s) {
    const auto rank_grid = static_cast<unsigned>(ceil_div(n, kSortBlock) * (kSortBlock / kWave));
    k_hs_rank<<<rank_grid, kRankThreads, 0, s>>>(t, targets, n, b.key0, b.row0);
    W2V_LAUNCH_CHECK("k_hs_rank");
    *order = b.row0;
    *keys = b.key0;
    if (n > kSortBlock) {
        k_hs_merge<<<static_cast<unsigned>(ceil_div(n, kMergeThreads)), kMergeThreads, 0, s>>>(b.key0, b.row0, n, b.key1,
                                                                                             b.row1);
        W2V_LAUNCH_CHECK("k_hs_merge");
        *order = b.row1;
        *keys = b.key1;
    }
    return W2V_OK;
}

// The sorted rows' sums, into rows of `out` that hold zeros or an earlier slab's sums.
int sum_rows(const NodeArgs &m, int32_t type, const Buffers &b, hipStream_t s) {
    const auto blocks = static_cast<int32_t>(blocks_of(m.n));
    const auto tiles = static_cast<unsigned>(ceil_div(m.dim, kWave));
    (void)with_type(type, [&](auto zero) {
        using T = decltype(zero);
        const dim3 grid(static_cast<unsigned>(blocks), tiles);
        if (m.coef)
            k_hs_nodes<T, true><<<grid, kWave, 0, s>>>(m);
        else
            k_hs_nodes<T, false><<<grid, kWave, 0, s>>>(m);
        return 0;
    });
    W2V_LAUNCH_CHECK("k_hs_nodes");
    // 1,024 blocks at most: two joins
    int32_t left = blocks, rows = kRows;
    for (int k = 0; k < 2 && left > 1; ++k) {
        const auto fans = static_cast<int32_t>(ceil_div(left, kFan));
        JoinArgs j{m.t, m.order, m.targets, m.n, m.dim, b.part[k], b.borders[k], left, rows, b.part[1], b.borders[k + 1],
                   m.dsyn1, m.out_stride, m.add};
        k_hs_join<<<dim3(static_cast<unsigned>(fans), tiles, static_cast<unsigned>(m.t.longest)), kWave, 0, s>>>(j);
        W2V_LAUNCH_CHECK("k_hs_join");
        left = fans;
        rows *= kFan;
    }
    return W2V_OK;
}

}  // namespace

size_t hs_loss_bytes(int64_t rows, int32_t dim, int32_t longest) {
    Carve c;
    carve(c, rows, dim, longest);
    return c.used();
}

int run_hs_loss(const HsLossArgs &a, void *workspace, hipStream_t s) {
    const Tree t{a.V, a.longest, a.codelen, a.code, a.point_off, a.points};
    const bool grads = a.dx || a.dsyn1;
    Buffers b{};
    if (a.dsyn1) {
        Carve c(workspace);
        b = carve(c, a.rows, a.dim, a.longest);
        if (int rc = zero_rows(a.dsyn1, a.V - 1, a.dim, a.dsyn1_stride, s)) return rc;
    }
    for (int64_t lo = 0; lo < a.rows; lo += kSlab) {
        const auto n = static_cast<int32_t>(std::min<int64_t>(kSlab, a.rows - lo));
        const int32_t *targets = a.targets + lo;
        const char *x = static_cast<const char *>(a.x) + lo * a.x_stride * type_bytes(a.type);
        const int32_t *order = nullptr;
        const uint64_t *keys = nullptr;
        if (a.dsyn1)
            if (int rc = sort_rows(t, targets, n, b, &order, &keys, s)) return rc;
        WalkArgs w{};
        w.t = t;
        w.syn1 = a.syn1;
        w.stride = a.stride;
        w.dim = a.dim;
        w.x = x;
        w.x_stride = a.x_stride;
        w.targets = targets;
        w.weights = a.weights ? a.weights + lo : nullptr;
        w.order = order;
        w.n = n;
        w.loss = a.loss ? a.loss + lo : nullptr;
        w.dx = a.dx ? static_cast<char *>(a.dx) + lo * a.dx_stride * type_bytes(a.type) : nullptr;
        w.dx_stride = a.dx_stride;
        w.coef = a.dsyn1 ? b.coef : nullptr;
        const auto grid = static_cast<unsigned>(ceil_div(n, kWalkThreads / kWave));
        const int ne = static_cast<int>(ceil_div(a.dim, kWave));
        (void)with_type(a.type, [&](auto zero) {
            using T = decltype(zero);
            if (ne <= 1) launch_walk<T, 1>(w, grads, grid, s);
            else if (ne <= 2) launch_walk<T, 2>(w, grads, grid, s);
            else if (ne <= 4) launch_walk<T, 4>(w, grads, grid, s);
            else if (ne <= 5) launch_walk<T, 5>(w, grads, grid, s);
            else if (ne <= 8) launch_walk<T, 8>(w, grads, grid, s);
            else launch_walk<T, 16>(w, grads, grid, s);
            return 0;
        });
        W2V_LAUNCH_CHECK("k_hs_walk");
        if (!a.dsyn1) continue;
        const NodeArgs m{t, keys, order, targets, n, a.dim, x, a.x_stride, b.coef, b.part[0], b.borders[0],
                         a.dsyn1, a.dsyn1_stride, lo > 0 ? 1 : 0};
        if (int rc = sum_rows(m, a.type, b, s)) return rc;
    }
    return W2V_OK;
}

size_t word_sums_bytes(int64_t rows, int32_t dim) {
    Carve c;
    carve(c, rows, dim, 1);
    return c.used();
}

int run_word_sums(const int32_t *words, const float *x, int64_t rows, int32_t dim, int64_t x_stride, int32_t V, float *out,
                  int64_t out_stride, void *workspace, hipStream_t s) {
    const Tree t{V, 1, nullptr, nullptr, nullptr, nullptr};
    Carve c(workspace);
    const Buffers b = carve(c, rows, dim, 1);
    if (int rc = zero_rows(out, V, dim, out_stride, s)) return rc;
    for (int64_t lo = 0; lo < rows; lo += kSlab) {
        const auto n = static_cast<int32_t>(std::min<int64_t>(kSlab, rows - lo));
        const int32_t *order = nullptr;
        const uint64_t *keys = nullptr;
        if (int rc = sort_rows(t, words + lo, n, b, &order, &keys, s)) return rc;
        const NodeArgs m{t, keys, order, words + lo, n, dim, x + lo * x_stride, x_stride, nullptr, b.part[0],
                         b.borders[0], out, out_stride, lo > 0 ? 1 : 0};
        if (int rc = sum_rows(m, W2V_F32, b, s)) return rc;
    }
    return W2V_OK;
}

}  // namespace w2v
