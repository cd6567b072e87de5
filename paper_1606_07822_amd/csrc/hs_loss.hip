// The hierarchical softmax as a loss with gradients, for a batch of hidden vectors x_i with target words v_i:
//
//   z_j = x . syn1[n_j] along v's path, s_j = 1 - 2 t_j,  loss = sum_j log(1 + exp(-s_j z_j))
//   g_j = -w s_j sigmoid(-s_j z_j),  dx = sum_j g_j syn1[n_j],  dsyn1[n] = sum over the rows through n of g x
//
// The walk (k_hs_walk) is a wavefront per row, in large batches per four rows: four inner nodes at a time, the next four
// on their way, dot products reduced together. It reads a path's rows once for z and dx, and leaves the row's
// coefficients g_j.
//
// dsyn1 is a sum over rows without atomics, in a fixed order. Rows are sorted by their word's code, left-aligned, so
// that the rows through an inner node are neighbours: node (row, j) continues its neighbour's where their codes share
// j bits. A wavefront holds up to 32 sorted rows' x in registers, up to five columns a lane, and goes down the levels: a
// level's nodes are runs of rows, summed and written out where a run ends. Runs that reach over a block's border are
// written as partial sums, which k_hs_join adds up in order. The same sum with one level, every row for its own word's
// row of the table, is the gradient of a table's looked-up rows (run_word_sums).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "w2v_ops.h"

namespace w2v {
namespace {

constexpr int kSlab = 33 * 2048;  // rows sorted and summed together; a longer batch takes several, each adding to dsyn1
constexpr int kSortBlock = 2048;  // rows ranked against each other
constexpr int kRows = 32;         // sorted rows of a wavefront's sum
// Fewer of them in batches of at most kFewBlocks times as many, which have few wavefronts otherwise (257 rows of 100: 21.7
// us in all, not 23.6; 2,048: 27.5, not 29.5; 4,096: 36.1, not 37.5; but 8,192: 45.9, not 42.4).
constexpr int kFewRows = 16;
constexpr int kFewBlocks = 256;
constexpr int kFan = 16;          // blocks whose sums one wavefront joins
// Rows up to which a workgroup ranks 64 of them, not 256, which reads each key four times as often (1,024 rows of 100:
// 24 us in all, not 27; 16,384: 59, not 65; 32,768 of 200: 118, not 120; but 65,536: 180, not 170).
constexpr int kRankNarrow = 32768;
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

// ------------------------------------------------------------------ zeros
// Rows set to zero by workgroups of kFillThreads threads, a group each. Sorting leaves memory idle, so its launches have
// such workgroups behind their own (65,536 rows, 1M rows of 300 floats: 458 -> 443 us in all; in the walk as well, which
// needs memory itself, 456).
constexpr int kFillThreads = 1024;
constexpr int kFillFloats = kFillThreads * 4 * 8;   // of a group, whole rows
constexpr int kFillRows = kFillThreads / kWave * 4;   // of a group, rows without their padding
struct Fill {
    float *p;
    int64_t rows, stride;
    int32_t dim, whole;   // whole: with their padding, as one array
    int64_t first;        // group of this launch's first filling workgroup
};

__device__ __forceinline__ void fill_group(const Fill &f, int64_t group) {
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (f.whole) {
        const int64_t n = f.rows * f.stride, lo = group * kFillFloats, at = lo + threadIdx.x * 4;
        if (lo + kFillFloats <= n) {
#pragma unroll
            for (int u = 0; u < kFillFloats / kFillThreads; u += 4) store_pack<float, 4>(f.p + at + u * kFillThreads, zero);
        } else {
            for (int64_t i = lo + threadIdx.x; i < n; i += kFillThreads) f.p[i] = 0.0f;
        }
        return;
    }
    const int64_t end = min(f.rows, (group + 1) * kFillRows);
    for (int64_t r = group * kFillRows + threadIdx.x / kWave; r < end; r += kFillThreads / kWave)
        for (int c = lane_id() * 4; c < f.dim; c += kWave * 4) store_cols<float, 4>(f.p + r * f.stride, c, f.dim, zero);
}

__global__ __launch_bounds__(kFillThreads) void k_hs_zero(Fill f) { fill_group(f, f.first + blockIdx.x); }

// ------------------------------------------------------------------ order
// A row of the batch, its target and what is needed of that word's path.
struct Item {
    int32_t row, word, off, len;
    uint64_t code;
};

__device__ __forceinline__ Item item_of(const Tree &t, int32_t row, int32_t word) {
    const int len = path_len(t, word);
    Item i{row, word, 0, len, 0};
    if (len > 0 && t.codelen) {
        i.off = t.point_off[word];
        i.code = t.code[word];
    }
    return i;
}

__device__ __forceinline__ int node_of(const Tree &t, const Item &i, int level) {   // of a path that long
    return t.codelen ? t.points[i.off + level] : i.word;
}

// Levels that two neighbouring sorted rows share an inner node at.
__device__ __forceinline__ int shared_levels(const Tree &t, const Item &a, const Item &b) {
    if (a.len == 0 || b.len == 0) return 0;
    if (a.word == b.word) return a.len;
    return t.codelen ? min(min(a.len, b.len), static_cast<int>(__ffsll(static_cast<long long>(a.code ^ b.code)))) : 0;
}

// What the rows are sorted by: the code with its first turn in the top bit, and after all of them the rows without a
// path, whose key is all ones. A code's 64th turn is left out: it leads to one of two words and to no inner node, so rows
// that agree in 63 turns share every node of theirs in any order, and no code is all ones. 32 bits do where no code is
// longer than 31, and cost half as much to compare.
template <class K>
__device__ __forceinline__ K sort_key(const Tree &t, int32_t v) {
    const int len = path_len(t, v);
    if (len == 0) return static_cast<K>(~0ull);
    if (!t.codelen) return static_cast<K>(v);
    return static_cast<K>((__brevll(t.code[v]) & (~0ull << (64 - min(len, 63)))) >> (64 - 8 * sizeof(K)));
}

// Each key's place among the kSortBlock keys of its block, by counting the smaller ones (equal keys keep their order).
// A workgroup places R rows; its wavefronts share the pairs of 64 of them and 64 keys of the block, two instructions a
// comparison: keys that come first count where they are equal, too, later ones where they are smaller, and only a
// pair of the same 64 compares the places as well.
constexpr int kRankThreads = 1024;
constexpr int kRankWaves = kRankThreads / kWave;
template <class K, int R>
__global__ __launch_bounds__(kRankThreads) void k_hs_rank(Tree t, const int32_t *__restrict__ targets, int32_t n,
                                                          K *__restrict__ key_out, int32_t *__restrict__ row_out,
                                                          Item *__restrict__ item_out, int32_t ranking, Fill fill) {
    if (static_cast<int32_t>(blockIdx.x) >= ranking) {
        fill_group(fill, fill.first + blockIdx.x - ranking);
        return;
    }
    __shared__ __align__(16) K keys[kSortBlock];
    __shared__ int32_t counts[kRankWaves][R];
    constexpr int kGroups = kSortBlock / R, kSets = R / kWave;
    const int32_t lo = static_cast<int32_t>(blockIdx.x) / kGroups * kSortBlock;
    const int own = static_cast<int>(blockIdx.x) % kGroups * R;   // this workgroup's rows of the block
    const int len = min(kSortBlock, n - lo);
    if (own >= len) return;
    const int i = static_cast<int>(threadIdx.x);
    Item item{};
    if (item_out && i < R && own + i < len) item = item_of(t, lo + own + i, targets[lo + own + i]);
    for (int i = threadIdx.x; i < kSortBlock; i += kRankThreads) keys[i] = i < len ? sort_key<K>(t, targets[lo + i]) : static_cast<K>(~0ull);
    __syncthreads();
    const int lane = lane_id(), wid = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    int32_t c[kSets];
#pragma unroll
    for (int r = 0; r < kSets; ++r) c[r] = 0;
    for (int seg = wid; seg * kWave < len; seg += kRankWaves) {   // keys past the end are the largest: they count for none
        const K *k = keys + seg * kWave;
#pragma unroll
        for (int r = 0; r < kSets; ++r) {
            const int mine_seg = own / kWave + r;
            const K mine = keys[mine_seg * kWave + lane];
            if (seg < mine_seg) {
#pragma unroll 16
                for (int j = 0; j < kWave; ++j) c[r] += k[j] <= mine ? 1 : 0;
            } else if (seg > mine_seg) {
#pragma unroll 16
                for (int j = 0; j < kWave; ++j) c[r] += k[j] < mine ? 1 : 0;
            } else {
#pragma unroll 16
                for (int j = 0; j < kWave; ++j) c[r] += k[j] < mine || (k[j] == mine && j < lane) ? 1 : 0;
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kSets; ++r) counts[wid][r * kWave + lane] = c[r];
    __syncthreads();
    if (i < R && own + i < len) {
        int32_t at = lo;
#pragma unroll
        for (int w = 0; w < kRankWaves; ++w) at += counts[w][i];
        if (item_out) {
            item_out[at] = item;
        } else {
            key_out[at] = keys[own + i];
            row_out[at] = lo + own + i;
        }
    }
}

// Each key's place among all: its place in its own sorted block and, in every other, the keys before it (equal ones
// count where their block comes first), found by bisection in LDS. A workgroup places 256 keys; each of its four parts
// takes two of the eight blocks that are in LDS at a time (a bisection is a chain of LDS reads, so several run at once),
// and the next eight are on their way meanwhile.
constexpr int kMergeKeys = 256;
constexpr int kMergeParts = 4;
constexpr int kMergeThreads = kMergeKeys * kMergeParts;
constexpr int kMergePer = 2;
constexpr int kMergeBlocks = kMergeParts * kMergePer;
template <class K>
__global__ __launch_bounds__(kMergeThreads) void k_hs_merge(Tree t, const int32_t *__restrict__ targets,
                                                            const K *__restrict__ key_in,
                                                            const int32_t *__restrict__ row_in, int32_t n,
                                                            Item *__restrict__ item_out, int32_t merging, Fill fill) {
    if (static_cast<int32_t>(blockIdx.x) >= merging) {
        fill_group(fill, fill.first + blockIdx.x - merging);
        return;
    }
    __shared__ K keys[kMergeBlocks * kSortBlock];
    __shared__ int32_t counts[kMergeParts][kMergeKeys];
    const int slot = static_cast<int>(threadIdx.x) % kMergeKeys, part = static_cast<int>(threadIdx.x) / kMergeKeys;
    const int32_t i = static_cast<int32_t>(blockIdx.x) * kMergeKeys + slot;
    const int own = i / kSortBlock, blocks = static_cast<int>(ceil_div(n, kSortBlock));
    const K mine = i < n ? key_in[i] : 0;
    const int32_t row = part == 0 && i < n ? row_in[i] : 0;
    constexpr int kLoads = kMergeBlocks * kSortBlock / kMergeThreads;
    K next[kLoads];
    auto load = [&](int b0) {
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int32_t k = b0 * kSortBlock + u * kMergeThreads + static_cast<int32_t>(threadIdx.x);
            next[u] = k < n ? key_in[k] : static_cast<K>(~0ull);   // past the end: after every key
        }
    };
    load(0);
    Item item{};   // fetched while the places are counted
    if (part == 0 && i < n) item = item_of(t, row, targets[row]);
    int32_t at = 0;
    for (int b0 = 0; b0 < blocks; b0 += kMergeBlocks) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kLoads; ++u) keys[u * kMergeThreads + static_cast<int>(threadIdx.x)] = next[u];
        __syncthreads();
        if (b0 + kMergeBlocks < blocks) load(b0 + kMergeBlocks);
        const int mine0 = part * kMergePer;
        int32_t lo[kMergePer], len[kMergePer];
#pragma unroll
        for (int u = 0; u < kMergePer; ++u) {
            lo[u] = 0;
            len[u] = max(0, min(kSortBlock, n - (b0 + mine0 + u) * kSortBlock));
        }
#pragma unroll
        for (int step = kSortBlock; step > 0; step >>= 1) {
            K k[kMergePer];
#pragma unroll
            for (int u = 0; u < kMergePer; ++u)
                k[u] = keys[(mine0 + u) * kSortBlock + min(lo[u] + step, kSortBlock) - 1];
#pragma unroll
            for (int u = 0; u < kMergePer; ++u) {
                const bool before = b0 + mine0 + u < own ? k[u] <= mine : k[u] < mine;
                if (lo[u] + step <= len[u] && before) lo[u] += step;
            }
        }
#pragma unroll
        for (int u = 0; u < kMergePer; ++u)
            if (b0 + mine0 + u != own) at += lo[u];
    }
    counts[part][slot] = at;
    __syncthreads();
    if (part == 0 && i < n) {
        at = i % kSortBlock;
#pragma unroll
        for (int k = 0; k < kMergeParts; ++k) at += counts[k][slot];
        item_out[at] = item;
    }
}

// A lane's C columns of a row of `bytes` bytes, 64 apart from `col` on: zeros past the row, and no store there.
template <int C, class T>
__device__ __forceinline__ void load_columns(const T *row, int col, int bytes, float (&v)[C]) {
    const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(row), 0, bytes, kRawBufferWord3);
    const int at = col * static_cast<int>(sizeof(T));
#pragma unroll
    for (int e = 0; e < C; ++e) {
        if constexpr (sizeof(T) == 4)
            v[e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, at + e * kWave * 4, 0, 0));
        else
            v[e] = static_cast<float>(__builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b16(rs, at + e * kWave * 2, 0, 0)));
    }
}

template <int C, class T>
__device__ __forceinline__ void store_columns(T *row, int col, int bytes, const float (&v)[C]) {
    const auto rs = __builtin_amdgcn_make_buffer_rsrc(row, 0, bytes, kRawBufferWord3);
    const int at = col * static_cast<int>(sizeof(T));
#pragma unroll
    for (int e = 0; e < C; ++e) {
        if constexpr (sizeof(T) == 4)
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v[e]), rs, at + e * kWave * 4, 0, 0);
        else
            __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, static_cast<T>(v[e])), rs, at + e * kWave * 2,
                                                  0, 0);
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
    const Item *items;      // the rows sorted; null: in their own order
    int32_t n;
    float *loss;            // null: not written
    void *dx;               // null: not written
    int64_t dx_stride;
    float *coef;            // [block of block_rows][level][row of the block]; null: not written
    int32_t block_rows;
};

constexpr int kWalkThreads = 64;   // a wavefront a workgroup: 65,536 rows of 200, 184 -> 181 us in all against four

// (1 + a) (1 + b) - 1, in two roundings that are relative to it: the products of a path are held less one, as a node
// with e below 2^-24 would not enter 1 + e, nor the digits of a small e.
__device__ __forceinline__ float product_less_one(float a, float b) { return fmaf(a, b, a + b); }

// What a node adds for s z (sz) at the lane: e = exp(-|z|) into the product of 1 + e (prod: less one; at most 2^64), whose
// logarithm is the path's sum of log(1 + e), and the rest of the loss; the value is sigmoid(-s z).
__device__ __forceinline__ float node_terms(float sz, bool in, float &prod, float &wrong) {
    const float e = in ? __expf(-fabsf(sz)) : 0.0f;
    prod = product_less_one(prod, e);
    wrong += in && sz < 0.0f ? -sz : 0.0f;
    return (sz < 0.0f ? 1.0f : e) * __builtin_amdgcn_rcpf(1.0f + e);
}

__device__ __forceinline__ float lane_value(float v, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// log(1 + q), q >= 0, to a few units in the last place: u = 1 + q is rounded, and log(u) / (u - 1) changes so little with u
// that a factor q in its place takes the rounding out (Kahan; q itself where u is 1).
__device__ __forceinline__ float log_one_more(float q) {
    const float u = 1.0f + q, d = u - 1.0f;
    return d == 0.0f ? q : logf(u) * (q * __builtin_amdgcn_rcpf(d));
}

// product_less_one over the four rows of 16 lanes, lane by lane.
__device__ __forceinline__ float rows_product_less_one(float v) {
    float a = v, b = v;
    swap16(a, b);
    v = product_less_one(a, b);
    a = v;
    b = v;
    swap32(a, b);
    return product_less_one(a, b);
}

// A wavefront's stretch of the sorted rows: neighbouring ones share most of their path, so each XCD, with an L2 of its
// own, takes one stretch of workgroups.
__device__ __forceinline__ int walk_wave() {
    const int per = static_cast<int>(gridDim.x) / kXcds, b = static_cast<int>(blockIdx.x);
    const int group = b < per * kXcds ? b % kXcds * per + b / kXcds : b;
    return group * (kWalkThreads / kWave) + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
}

// R rows a wavefront, 1 or 4 (sorted ones). The levels that all four share are walked once for the four: a node's row
// is loaded once, its four products are reduced together, and row r's terms are worked out in the r-th sixteen lanes.
// Then each row's own levels follow, four at a time. The next four nodes are on their way meanwhile.
template <class T, int NE, bool GRADS, int R>
__global__ __launch_bounds__(kWalkThreads) void k_hs_walk(WalkArgs a) {
    const int lane = lane_id(), quarter = lane >> 4;
    const int pos0 = walk_wave() * R;
    if (pos0 >= a.n) return;
    const int pos = pos0 + (R == 4 ? quarter : 0);   // the row that a lane loads for
    Item item{0, -1, 0, 0, 0};
    if (pos < a.n) item = a.items ? a.items[pos] : item_of(a.t, pos, a.targets[pos]);
    const uint64_t code = item.code;
    const float weight = GRADS && a.weights && pos < a.n ? a.weights[item.row] : 1.0f;
    int len[R], row[R], pt[R];
    float x[R][NE], dx[R][NE];
    const int x_bytes = a.dim * static_cast<int>(sizeof(T));
#pragma unroll
    for (int r = 0; r < R; ++r) {
        len[r] = __builtin_amdgcn_readlane(item.len, 16 * r);
        row[r] = __builtin_amdgcn_readlane(item.row, 16 * r);
        const int off = __builtin_amdgcn_readlane(item.off, 16 * r);
        pt[r] = lane < len[r] ? a.t.points[off + lane] : 0;
        load_columns<NE>(static_cast<const T *>(a.x) + row[r] * a.x_stride, lane, len[r] > 0 ? x_bytes : 0, x[r]);
#pragma unroll
        for (int i = 0; i < NE; ++i) dx[r][i] = 0.0f;
    }
    int shared = 0;
    if constexpr (R == 4) {
        auto item_at = [&](int l) {
            return Item{0, __builtin_amdgcn_readlane(item.word, l), 0, __builtin_amdgcn_readlane(item.len, l),
                        static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(code >> 32), l)))
                                << 32 | static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(code), l))};
        };
        shared = shared_levels(a.t, item_at(0), item_at(48));
    }
    float y[4][NE], now[4][NE];
    const int bytes = a.dim * 4;
    auto load = [&](int r, int j, int end) {   // zeros past the end
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const bool in = j + u < end;
            const int node = __builtin_amdgcn_readlane(pt[r], min(j + u, kWave - 1));
            load_columns<NE>(a.syn1 + static_cast<int64_t>(in ? node : 0) * a.stride, lane, in ? bytes : 0, y[u]);
        }
    };
    auto take = [&] {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < NE; ++i) now[u][i] = y[u][i];
    };
    float wrong = 0.0f, prod = 0.0f;   // a lane's (prod less one): of its row's shared levels, later of all its row's
    float g_all[R];                    // lane j: a row's coefficient at level j
#pragma unroll
    for (int r = 0; r < R; ++r) g_all[r] = 0.0f;
    if constexpr (R == 4) {
        load(0, 0, shared > 0 ? shared : len[0]);
        for (int j = 0; j < shared; j += 4) {
            take();
            if (j + 4 < shared)
                load(0, j + 4, shared);
            else
                load(0, shared, len[0]);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (j + u >= shared) break;
                const float z = reduce4(dot_partial<NE>(x[0], now[u]), dot_partial<NE>(x[R / 4], now[u]),
                                        dot_partial<NE>(x[R / 2], now[u]), dot_partial<NE>(x[R - 1], now[u]));
                const bool turn = (code >> (j + u)) & 1ull;
                const float f = node_terms(turn ? -z : z, true, prod, wrong);
                if constexpr (GRADS) {
                    const float g = (turn ? f : -f) * weight;
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const float gr = lane_value(g, 16 * r);
#pragma unroll
                        for (int i = 0; i < NE; ++i) dx[r][i] = fmaf(gr, now[u][i], dx[r][i]);
                        if (lane == j + u) g_all[r] = gr;
                    }
                }
            }
        }
    } else {
        load(0, 0, len[0]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint64_t turns = static_cast<uint64_t>(static_cast<uint32_t>(
                                   __builtin_amdgcn_readlane(static_cast<int>(code >> 32), 16 * r))) << 32 |
                               static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(code), 16 * r));
        const float w = lane_value(weight, 16 * r);
        float row_wrong = 0.0f, row_prod = 0.0f;
        if (r + 1 < R && len[r] <= shared) load(r + 1 < R ? r + 1 : r, shared, len[r + 1 < R ? r + 1 : r]);
        for (int j = shared; j < len[r]; j += 4) {
            take();
            if (j + 4 < len[r])
                load(r, j + 4, len[r]);
            else if (r + 1 < R)
                load(r + 1 < R ? r + 1 : r, shared, len[r + 1 < R ? r + 1 : r]);
            const float z = reduce4(dot_partial<NE>(x[r], now[0]), dot_partial<NE>(x[r], now[1]),
                                    dot_partial<NE>(x[r], now[2]), dot_partial<NE>(x[r], now[3]));   // lanes 16u..: node j + u
            const int level = j + quarter;
            const bool in = level < len[r], turn = (turns >> min(level, 63)) & 1ull;
            const float f = node_terms(turn ? -z : z, in, row_prod, row_wrong);
            if constexpr (GRADS) {
                const float g = in ? (turn ? f : -f) * w : 0.0f;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float gu = lane_value(g, 16 * u);
#pragma unroll
                    for (int i = 0; i < NE; ++i) dx[r][i] = fmaf(gu, now[u][i], dx[r][i]);
                    if (lane == j + u) g_all[r] = gu;
                }
            }
        }
        row_wrong = rows_sum(row_wrong);
        row_prod = rows_product_less_one(row_prod);
        if (R == 1 || quarter == r) {
            wrong += row_wrong;
            prod = product_less_one(prod, row_prod);
        }
    }
    if (a.loss && (lane & 15) == 0 && quarter < R && pos < a.n) {
        const bool missing = item.word >= 0 && item.len == 0;   // a target that the tree does not hold
        a.loss[item.row] = missing ? __builtin_nanf("") : wrong + log_one_more(prod);
    }
    if constexpr (GRADS) {
        if (a.dx) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (pos0 + r < a.n) store_columns<NE>(static_cast<T *>(a.dx) + row[r] * a.dx_stride, lane, x_bytes, dx[r]);
        }
        if (a.coef && lane < a.t.longest) {
            float *c = a.coef + (static_cast<int64_t>(pos0 / a.block_rows) * a.t.longest + lane) * a.block_rows +
                       pos0 % a.block_rows;
            store_pack<float, R>(c, g_all);   // a block's rows are a multiple of four
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
    const Item *items;
    int32_t n, dim;
    const void *x;
    int64_t x_stride;
    const float *coef;  // null: ones
    float *part;        // [level][block][2][dim]: sums of runs that come in from the left, and of those that go on right
    int32_t *part_node; // [level][block]: the node of a run that comes in from the left
    Borders borders;
    float *dsyn1;
    int64_t out_stride;
    int32_t add;        // dsyn1 holds an earlier slab's sums
    int32_t tiles;      // wavefronts for a row's columns
};

// Stores a sum, or adds it to what an earlier slab left.
template <int C>
__device__ __forceinline__ void put_columns(float *row, int col, int bytes, const float (&v)[C], bool add) {
    if (add) {
        float sum[C];
        load_columns<C>(row, col, bytes, sum);
#pragma unroll
        for (int e = 0; e < C; ++e) sum[e] += v[e];
        store_columns<C>(row, col, bytes, sum);
    } else {
        store_columns<C>(row, col, bytes, v);
    }
}

// A wavefront holds RB sorted rows, C columns a lane, and takes every so many of the levels; a workgroup has wavefronts
// for all columns of the rows and, where there are few rows, for several parts of the levels. What bounds it is
// the instructions around a row's multiply-adds, so a wavefront takes as many columns as its registers hold. What a
// level's rows need (coefficient, node, where a run that ends with the row goes) is worked out by the row's lane and
// read from there; the coefficients and nodes of all levels are fetched into LDS first, as a load waits for the stores
// that went before it. Eight rows inside one run take a multiply-add a column each; elsewhere a row also takes a branch
// for whether it has the level and whether its run ends.
template <int RB>   // of a workgroup: 256 registers a lane, or 128
constexpr int kNodeWaves = RB == kFewRows ? 16 : 8;
template <class T, bool COEF, int RB, int C>
__global__ __launch_bounds__(kNodeWaves<RB> *kWave) void k_hs_nodes(NodeArgs a) {
    extern __shared__ int32_t level_node[];   // [longest][RB], then the coefficients alike
    const int lane = lane_id(), wid = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    const int waves = static_cast<int>(blockDim.x) / kWave, level_step = waves / a.tiles;
    const int blk = static_cast<int>(blockIdx.x), longest = a.t.longest;
    const int col = wid % a.tiles * C * kWave + lane;
    const int p0 = blk * RB, rows = min(RB, a.n - p0);
    // lane q: row q of the block and the rows beside it
    const int pos = p0 + lane;
    const bool on = lane < rows;
    Item item{0, -1, 0, 0, 0}, last = item, next = item;
    if (on) {
        item = a.items[pos];
        if (pos > 0) last = a.items[pos - 1];
        if (pos + 1 < a.n) next = a.items[pos + 1];
    }
    const int len = item.len, before = shared_levels(a.t, last, item), after = shared_levels(a.t, item, next);
    float x[RB][C];
#pragma unroll
    for (int q = 0; q < RB; ++q) {
        const int64_t r = __builtin_amdgcn_readlane(item.row, q);
        load_columns<C>(static_cast<const T *>(a.x) + r * a.x_stride, col, q < rows ? a.dim * static_cast<int>(sizeof(T)) : 0,
                        x[q]);
    }
    const int left = __builtin_amdgcn_readlane(before, 0);
    const int right = __builtin_amdgcn_readlane(after, RB - 1);
    int deepest = len, inner = on && lane > 0 ? before : kWave;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        deepest = max(deepest, __shfl_xor(deepest, m, kWave));
        inner = min(inner, __shfl_xor(inner, m, kWave));
    }
    deepest = __builtin_amdgcn_readfirstlane(deepest);
    if (threadIdx.x == 0) {
        a.borders.left[blk] = left;
        a.borders.inner[blk] = inner;
    }
    const int cells = longest * RB;
    float *level_coef = reinterpret_cast<float *>(level_node + cells);
    if (lane < RB) {
        for (int j = wid; j < deepest; j += waves) level_node[j * RB + lane] = j < len ? node_of(a.t, item, j) : 0;
    }
    if constexpr (COEF) {
        const float *coef = a.coef + static_cast<int64_t>(blk) * cells;
        for (int i = threadIdx.x; i < deepest * RB; i += blockDim.x) level_coef[i] = coef[i];
    }
    __syncthreads();
    const int bytes = a.dim * 4;
    const uint64_t lower = (1ull << lane) - 1;
    for (int j = wid / a.tiles; j < deepest; j += level_step) {
        const int node = level_node[j * RB + lane % RB];
        const float coefs = COEF ? level_coef[j * RB + lane % RB] : 1.0f;
        const uint64_t active = __ballot(len > j);
        const uint64_t ends = __ballot(len > j && (after <= j || lane == RB - 1));
        // where the run that ends with this lane's row goes
        const bool from_left = left > j && (ends & lower) == 0;
        const bool to_right = lane == RB - 1 && right > j;
        const int64_t slot = (static_cast<int64_t>(j) * gridDim.x + blk) * 2 + (from_left ? 0 : 1);
        const uint64_t to = reinterpret_cast<uint64_t>(from_left || to_right ? a.part + slot * a.dim
                                                                             : a.dsyn1 + node * a.out_stride);
        const int to_lo = static_cast<int>(to), to_hi = static_cast<int>(to >> 32);
        const uint64_t direct = a.add ? ~__ballot(from_left || to_right) : 0;   // rows whose sum is added to dsyn1
        if (left > j && lane == 0) a.part_node[static_cast<int64_t>(j) * gridDim.x + blk] = node;
        float acc[C];
#pragma unroll
        for (int e = 0; e < C; ++e) acc[e] = 0.0f;
        auto add_row = [&](int q) {
            const float c = COEF ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, coefs), q)) : 1.0f;
#pragma unroll
            for (int e = 0; e < C; ++e) acc[e] = COEF ? fmaf(c, x[q][e], acc[e]) : acc[e] + x[q][e];
        };
        auto end_run = [&](int q) {
            const auto lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(to_lo, q));
            const auto hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(to_hi, q));
            put_columns<C>(reinterpret_cast<float *>(static_cast<uint64_t>(hi) << 32 | lo), col, bytes, acc, (direct >> q) & 1ull);
#pragma unroll
            for (int e = 0; e < C; ++e) acc[e] = 0.0f;
        };
#pragma unroll
        for (int q0 = 0; q0 < RB; q0 += 8) {
            const uint32_t act = static_cast<uint32_t>(active >> q0) & 255u, end = static_cast<uint32_t>(ends >> q0) & 255u;
            if (act == 255u && (end & 127u) == 0) {
#pragma unroll
                for (int q = q0; q < q0 + 8; ++q) add_row(q);
                if (end) end_run(q0 + 7);
            } else if (act) {
#pragma unroll
                for (int q = q0; q < q0 + 8; ++q)
                    if ((act >> (q - q0)) & 1u) {
                        add_row(q);
                        if ((end >> (q - q0)) & 1u) end_run(q);
                    }
            }
        }
    }
}

struct JoinArgs {
    int32_t dim;
    const float *in;        // [level][block][2][dim]
    const int32_t *in_node; // [level][block]
    Borders borders;
    int32_t blocks;
    float *out;             // the same of a workgroup's blocks together
    int32_t *out_node;
    Borders out_borders;
    float *dsyn1;
    int64_t out_stride;
    int32_t add;
};

// The partial sums of one level added up in the blocks' order, 64 columns of up to kJoinWaves kFan blocks a workgroup: a
// run's first part lies on a block's right, the others on the left of the blocks that follow. Each wavefront fetches the
// parts of kFan blocks at once (another XCD wrote them: a fetch takes a microsecond, whatever it is of) and adds up the
// runs among them; the first one then puts together what leaves one wavefront's blocks for the next one's.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(kJoinWaves *kWave) void k_hs_join(JoinArgs a) {
    __shared__ float s_in[kJoinWaves][kWave], s_out[kJoinWaves][kWave];
    __shared__ int32_t s_flags[kJoinWaves], s_node[kJoinWaves], s_least[kJoinWaves];
    const int lane = lane_id(), wid = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    const int level = static_cast<int>(blockIdx.z), super = static_cast<int>(blockIdx.x);
    const int col = static_cast<int>(blockIdx.y) * kWave + lane, bytes = a.dim * 4;
    const int first = (super * kJoinWaves + wid) * kFan, blk = first + lane;
    const bool on = lane < kFan && blk < a.blocks;
    const int left = on ? a.borders.left[blk] : 0, inner = on ? a.borders.inner[blk] : kWave;
    const int right = on && blk + 1 < a.blocks ? a.borders.left[blk + 1] : 0;
    int least = on ? min(inner, lane > 0 || wid > 0 ? left : kWave) : kWave;
    if (blockIdx.y == 0 && level == 0) {
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) least = min(least, __shfl_xor(least, m, kWave));
    }
    const auto has_left = static_cast<uint32_t>(__ballot(left > level));
    const auto through = static_cast<uint32_t>(__ballot(left > level && inner > level && right > level));
    const auto has_right = static_cast<uint32_t>(__ballot(right > level)) & ~through;
    float acc[1] = {0.0f};
    bool outside = has_left & 1u;   // the run at hand began before these blocks
    int first_node = 0;
    if (has_left | has_right) {
        const int node = left > level ? a.in_node[static_cast<int64_t>(level) * a.blocks + blk] : 0;
        const auto rs = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<float *>(a.in + (static_cast<int64_t>(level) * a.blocks + first) * 2 * a.dim), 0,
            min(kFan, a.blocks - first) * 2 * bytes, kRawBufferWord3);
        float l[kFan], r[kFan];
#pragma unroll
        for (int b = 0; b < kFan; ++b) {   // out of range where there is none: no branch around the loads
            const int at = col * 4 + b * 2 * bytes;
            l[b] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, (has_left >> b) & 1u ? at : -4, 0, 0));
            r[b] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, (has_right >> b) & 1u ? at + bytes : -4, 0, 0));
        }
        first_node = __builtin_amdgcn_readlane(node, 0);
#pragma unroll
        for (int b = 0; b < kFan; ++b) {
            if ((has_left >> b) & 1u) {
                acc[0] += l[b];
                if (!((through >> b) & 1u)) {
                    if (outside)
                        s_in[wid][lane] = acc[0];
                    else
                        put_columns<1>(a.dsyn1 + __builtin_amdgcn_readlane(node, b) * a.out_stride, col, bytes, acc, a.add);
                    outside = false;
                    acc[0] = 0.0f;
                }
            }
            if ((has_right >> b) & 1u) {
                acc[0] = r[b];
                outside = false;
            }
        }
    }
    const bool leaves = ((has_right | through) >> (kFan - 1)) & 1u;
    if (leaves) (outside ? s_in : s_out)[wid][lane] = acc[0];
    if (lane == 0) {
        s_flags[wid] = (has_left & 1u ? 1 : 0) | (leaves ? (outside ? 2 : 4) : 0);   // a run comes in, goes through, leaves
        s_node[wid] = first_node;
        s_least[wid] = least;
    }
    __syncthreads();
    if (wid > 0) return;
    float *out = a.out + (static_cast<int64_t>(level) * gridDim.x + super) * 2 * a.dim;
    const int waves = static_cast<int>(blockDim.x) / kWave;
    outside = has_left & 1u;
    acc[0] = 0.0f;
    int flags = 0;
    for (int w = 0; w < waves; ++w) {
        flags = __builtin_amdgcn_readfirstlane(s_flags[w]);
        if (flags & 1) {
            acc[0] += s_in[w][lane];
            if (!(flags & 2)) {
                if (outside)
                    put_columns<1>(out, col, bytes, acc, false);
                else
                    put_columns<1>(a.dsyn1 + __builtin_amdgcn_readfirstlane(s_node[w]) * a.out_stride, col, bytes, acc, a.add);
                outside = false;
                acc[0] = 0.0f;
            }
        }
        if (flags & 4) {
            acc[0] = s_out[w][lane];
            outside = false;
        }
    }
    if (flags & 6) put_columns<1>(out + (outside ? 0 : a.dim), col, bytes, acc, false);
    if (blockIdx.y == 0 && lane == 0) {
        if (has_left & 1u) a.out_node[static_cast<int64_t>(level) * gridDim.x + super] = first_node;
        if (level == 0) {
            for (int w = 0; w < waves; ++w) least = min(least, s_least[w]);
            a.out_borders.left[super] = left;
            a.out_borders.inner[super] = least;
        }
    }
}

struct Buffers {
    void *keys;
    int32_t *row;
    Item *items;
    float *coef, *part[2];
    int32_t *node[2];
    Borders borders[3];
};

// Rows of a wavefront's sum: few, so that there are more wavefronts, in a small batch.
int block_rows(int64_t n) { return n <= kFewRows * kFewBlocks ? kFewRows : kRows; }

Buffers carve(Carve &c, int64_t rows, int32_t dim, int32_t longest) {
    const auto n = static_cast<size_t>(std::min<int64_t>(std::max<int64_t>(rows, 1), kSlab));
    // a last slab of few rows has blocks of kFewRows, at most kFewBlocks of them
    const auto blocks = std::max<size_t>((n + kRows - 1) / kRows, std::min<size_t>((n + kFewRows - 1) / kFewRows, kFewBlocks));
    const size_t fans = (blocks + kFan * kJoinWaves - 1) / (kFan * kJoinWaves), level = static_cast<size_t>(2) * longest * dim;
    Buffers b;
    b.keys = c.take<uint64_t>(n);
    b.row = c.take<int32_t>(n);
    b.items = c.take<Item>(n);
    b.coef = c.take<float>(blocks * longest * kRows);
    b.part[0] = c.take<float>(blocks * level);
    b.part[1] = c.take<float>(fans * level);
    b.node[0] = c.take<int32_t>(blocks * longest);
    b.node[1] = c.take<int32_t>(fans * longest);
    const size_t counts[3] = {blocks, fans, 1};
    for (int k = 0; k < 3; ++k) {
        b.borders[k].left = c.take<int32_t>(counts[k]);
        b.borders[k].inner = c.take<int32_t>(counts[k]);
    }
    return b;
}

// Four rows a wavefront from here on: fewer take longer one after the other than the loads they share save (in all,
// four and one: 8,192 rows of 200 62 and 56 us; 16,384 83 and 83, of 100 59 and 57; 32,768 of 200 120 and 124; 65,536 170
// and 186).
constexpr int kWalkFour = 20480;

template <class T, int NE>
void launch_walk(const WalkArgs &w, bool grads, hipStream_t s) {
    constexpr int kWaves = kWalkThreads / kWave;
    const auto grid = static_cast<unsigned>(ceil_div(w.n, kWaves));
    if constexpr (NE <= 8) {   // registers for four rows
        if (grads && w.items && w.n >= kWalkFour) {
            k_hs_walk<T, NE, true, 4><<<static_cast<unsigned>(ceil_div(w.n, 4 * kWaves)), kWalkThreads, 0, s>>>(w);
            return;
        }
    }
    if (grads)
        k_hs_walk<T, NE, true, 1><<<grid, kWalkThreads, 0, s>>>(w);
    else
        k_hs_walk<T, NE, false, 1><<<grid, kWalkThreads, 0, s>>>(w);
}

// The groups of a filling, none for rows that hold an earlier slab's sums. whole: the rows' padding may be written too.
// Rows that end inside a 128-byte line cost memory a read for the rest of it (1M rows of 300 floats, 320 apart: 329 us,
// 204 with the padding), so padding of less than kShortPadding floats is then written with them (callers may rely on it).
constexpr int64_t kShortPadding = 32;
struct Zeros {
    Fill fill{};
    int64_t groups = 0;
    Zeros() = default;
    Zeros(float *p, int64_t rows, int32_t dim, int64_t stride, bool whole) {
        fill = Fill{p, rows, stride, dim, whole && stride - dim < kShortPadding ? 1 : 0, 0};
        groups = fill.whole ? ceil_div(rows * stride, kFillFloats) : ceil_div(rows, kFillRows);
    }
    // The next of them, at most `most`.
    unsigned take(int64_t most, Fill *part) {
        *part = fill;
        const int64_t n = std::min(groups, most);
        fill.first += n;
        groups -= n;
        return static_cast<unsigned>(n);
    }
};
constexpr int64_t kFillLaunch = int64_t(1) << 20;   // groups of one launch

int zero_rows(Zeros z, hipStream_t s) {
    while (z.groups > 0) {
        Fill part;
        const unsigned n = z.take(kFillLaunch, &part);
        k_hs_zero<<<n, kFillThreads, 0, s>>>(part);
        W2V_LAUNCH_CHECK("k_hs_zero");
    }
    return W2V_OK;
}

// Sorts n <= kSlab rows by their targets' keys, and sets z's rows to zero.
template <class K>
int sort_rows(const Tree &t, const int32_t *targets, int32_t n, Zeros z, const Buffers &b, hipStream_t s) {
    static_assert(kFillThreads == kRankThreads && kFillThreads == kMergeThreads);
    const bool one = n <= kSortBlock;   // the ranks are the order
    Item *now = one ? b.items : nullptr;
    K *keys = static_cast<K *>(b.keys);
    Fill part;
    unsigned filling = z.take(std::min(kFillLaunch, one ? z.groups : z.groups / 2), &part);
    const auto ranking = static_cast<unsigned>(ceil_div(n, kSortBlock) * (kSortBlock / (n <= kRankNarrow ? 64 : 256)));
    if (n <= kRankNarrow)
        k_hs_rank<K, 64><<<ranking + filling, kRankThreads, 0, s>>>(t, targets, n, keys, b.row, now,
                                                                  static_cast<int32_t>(ranking), part);
    else
        k_hs_rank<K, 256><<<ranking + filling, kRankThreads, 0, s>>>(t, targets, n, keys, b.row, now,
                                                                   static_cast<int32_t>(ranking), part);
    W2V_LAUNCH_CHECK("k_hs_rank");
    if (one) return zero_rows(z, s);
    filling = z.take(kFillLaunch, &part);
    const auto merging = static_cast<unsigned>(ceil_div(n, kMergeKeys));
    k_hs_merge<K><<<merging + filling, kMergeThreads, 0, s>>>(t, targets, keys, b.row, n, b.items,
                                                             static_cast<int32_t>(merging), part);
    W2V_LAUNCH_CHECK("k_hs_merge");
    return zero_rows(z, s);
}

int sort_rows(const Tree &t, const int32_t *targets, int32_t n, const Zeros &z, const Buffers &b, hipStream_t s) {
    return t.longest <= 31 ? sort_rows<uint32_t>(t, targets, n, z, b, s) : sort_rows<uint64_t>(t, targets, n, z, b, s);
}

template <int R, int C>
struct SumShape {
    static constexpr int rows = R, cols = C;
};

// The sorted rows' sums, into rows of `out` that hold zeros or an earlier slab's sums.
int sum_rows(NodeArgs m, int32_t type, const Buffers &b, hipStream_t s) {
    const int rb = block_rows(m.n), columns = static_cast<int>(ceil_div(m.dim, kWave));
    const auto blocks = static_cast<int32_t>(ceil_div(m.n, rb));
    const int per = columns <= 5 ? columns : 4;   // columns of a lane
    m.tiles = static_cast<int32_t>(ceil_div(columns, per));
    // The levels are shared out, to more than four parts while that gives a SIMD no more than two wavefronts (rows of
    // 200, 4,096 of them: 54 us in all with four parts, 48 with eight; 16,384: 82, 85), to up to four while it gives ten
    // (65,536: 184 us with one part, 173 with four). Batches of few rows: 257 of 100, 22 us with eight parts, 21 with 16.
    const int64_t waves = static_cast<int64_t>(blocks) * m.tiles, cus = device_cu_count();
    int parts = std::min(m.t.longest, (rb == kRows ? kNodeWaves<kRows> : kNodeWaves<kFewRows>) / m.tiles);
    while (parts > 1 && waves * parts > (parts > 4 ? 8 : 40) * cus) parts /= 2;
    const auto threads = static_cast<unsigned>(m.tiles * parts * kWave);
    const size_t lds = static_cast<size_t>(m.t.longest) * rb * (m.coef ? 8 : 4);
    (void)with_type(type, [&](auto zero) {
        using T = decltype(zero);
        auto launch = [&](auto shape) {
            constexpr int RB = decltype(shape)::rows, C = decltype(shape)::cols;
            if (m.coef)
                k_hs_nodes<T, true, RB, C><<<static_cast<unsigned>(blocks), threads, lds, s>>>(m);
            else if constexpr (sizeof(T) == 4)
                k_hs_nodes<T, false, RB, C><<<static_cast<unsigned>(blocks), threads, lds, s>>>(m);
        };
        auto with_rows = [&](auto cols) {
            constexpr int C = decltype(cols)::value;
            rb == kRows ? launch(SumShape<kRows, C>{}) : launch(SumShape<kFewRows, C>{});
        };
        switch (per) {
            case 1: with_rows(std::integral_constant<int, 1>{}); break;
            case 2: with_rows(std::integral_constant<int, 2>{}); break;
            case 3: with_rows(std::integral_constant<int, 3>{}); break;
            case 4: with_rows(std::integral_constant<int, 4>{}); break;
            default: with_rows(std::integral_constant<int, 5>{}); break;
        }
        return 0;
    });
    W2V_LAUNCH_CHECK("k_hs_nodes");
    const auto tiles = static_cast<unsigned>(ceil_div(m.dim, kWave));
    static_assert(kSlab / kRows <= kFan * kJoinWaves * kFan * kJoinWaves, "two joins are enough");
    int32_t left = blocks;
    for (int k = 0; k < 2 && left > 1; ++k) {
        const auto supers = static_cast<int32_t>(ceil_div(left, kFan * kJoinWaves));
        const auto waves = std::min<int64_t>(kJoinWaves, ceil_div(left, kFan));
        JoinArgs j{m.dim, b.part[k], b.node[k], b.borders[k], left, b.part[1], b.node[1], b.borders[k + 1],
                   m.dsyn1, m.out_stride, m.add};
        k_hs_join<<<dim3(static_cast<unsigned>(supers), tiles, static_cast<unsigned>(m.t.longest)),
                    static_cast<unsigned>(waves * kWave), 0, s>>>(j);
        W2V_LAUNCH_CHECK("k_hs_join");
        left = supers;
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
    Zeros zeros;
    if (a.dsyn1) {
        Carve c(workspace);
        b = carve(c, a.rows, a.dim, a.longest);
        zeros = Zeros(a.dsyn1, a.V - 1, a.dim, a.dsyn1_stride, a.dsyn1_whole);
        if (a.rows == 0) return zero_rows(zeros, s);
    }
    for (int64_t lo = 0; lo < a.rows; lo += kSlab) {
        const auto n = static_cast<int32_t>(std::min<int64_t>(kSlab, a.rows - lo));
        const int32_t *targets = a.targets + lo;
        const char *x = static_cast<const char *>(a.x) + lo * a.x_stride * type_bytes(a.type);
        if (a.dsyn1)
            if (int rc = sort_rows(t, targets, n, lo == 0 ? zeros : Zeros(), b, s)) return rc;
        WalkArgs w{};
        w.t = t;
        w.syn1 = a.syn1;
        w.stride = a.stride;
        w.dim = a.dim;
        w.x = x;
        w.x_stride = a.x_stride;
        w.targets = targets;
        w.weights = a.weights ? a.weights + lo : nullptr;
        w.items = a.dsyn1 ? b.items : nullptr;
        w.n = n;
        w.loss = a.loss ? a.loss + lo : nullptr;
        w.dx = a.dx ? static_cast<char *>(a.dx) + lo * a.dx_stride * type_bytes(a.type) : nullptr;
        w.dx_stride = a.dx_stride;
        w.coef = a.dsyn1 ? b.coef : nullptr;
        w.block_rows = block_rows(n);
        const int ne = static_cast<int>(ceil_div(a.dim, kWave));
        (void)with_type(a.type, [&](auto zero) {
            using T = decltype(zero);
            if (ne <= 1) launch_walk<T, 1>(w, grads, s);
            else if (ne <= 2) launch_walk<T, 2>(w, grads, s);
            else if (ne <= 4) launch_walk<T, 4>(w, grads, s);
            else if (ne <= 5) launch_walk<T, 5>(w, grads, s);
            else if (ne <= 8) launch_walk<T, 8>(w, grads, s);
            else launch_walk<T, 16>(w, grads, s);
            return 0;
        });
        W2V_LAUNCH_CHECK("k_hs_walk");
        if (!a.dsyn1) continue;
        const NodeArgs m{t, b.items, n, a.dim, x, a.x_stride, b.coef, b.part[0], b.node[0], b.borders[0],
                         a.dsyn1, a.dsyn1_stride, lo > 0 ? 1 : 0, 1};
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
    const Zeros zeros(out, V, dim, out_stride, true);
    if (rows == 0) return zero_rows(zeros, s);
    for (int64_t lo = 0; lo < rows; lo += kSlab) {
        const auto n = static_cast<int32_t>(std::min<int64_t>(kSlab, rows - lo));
        if (int rc = sort_rows(t, words + lo, n, lo == 0 ? zeros : Zeros(), b, s)) return rc;
        const NodeArgs m{t, b.items, n, dim, x + lo * x_stride, x_stride, nullptr, b.part[0],
                         b.node[0], b.borders[0], out, out_stride, lo > 0 ? 1 : 0, 1};
        if (int rc = sum_rows(m, W2V_F32, b, s)) return rc;
    }
    return W2V_OK;
}

}  // namespace w2v
