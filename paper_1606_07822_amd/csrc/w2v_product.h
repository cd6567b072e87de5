// Tiles of a matrix product C[m][n] = sum_k A(m, k) B(n, k) on the matrix cores, for the kernels that put their own
// last step (an activation, a gradient, a weight's update) on a tile while it is in registers.
//
// An operand is 16-bit elements in rows of whole 16-byte chunks, with k along the rows (ALONG) or down them: the second
// kind is read from LDS by a transposing load, so that no array is needed in two layouts. An element is one number, or P
// whose sum is the value (parts of 8 bits in bf16, of 11 in fp16): products p, q with p + q < P are taken, smallest
// first, which leaves out what lies below the last part. The sums are fp32. A row holds the first parts of 32 elements,
// then their second parts, and so on, so that a step's 64 bytes of each part lie in common 128-byte lines (rows of one part
// after the other's took 40 % longer with 128 x 64 tiles of three parts: half of every line came for nothing).
//
// A workgroup of WM x WN wavefronts makes BM x BN of C. Each step, BK of k, goes from global memory straight into one
// of two LDS buffers while the matrix cores work on the other; a wavefront waits for its own loads and a barrier makes
// them everybody's, once a step. Chunks change places within 256 bytes by their row, so that the 16 lanes of a phase
// read all 64 banks. Measured on 8,192^3 with results in bf16, TFLOP/s: 256 x 256 tiles of one part 1,280 (the library's
// product 1,370), two fp16 parts 477 (three products: 1,430), 256 x 128 of three bf16 parts 218 (six: 1,310; the library's
// product in fp32: 153); 128 x 128 tiles 1,130 and 420, 128 x 64 of three parts 168. Large tiles read LDS least and are
// bound by the matrix cores; of short products and few tiles a launch's start and end are the larger part (some 10 us of 37
// with 16 steps), which two small tiles a CU do not hide either: they stay in step with each other.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "w2v_ops.h"

namespace w2v {

template <class E>
using Frag = E __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f4 mfma32(Frag<__bf16> a, Frag<__bf16> b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f4 mfma32(Frag<_Float16> a, Frag<_Float16> b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// The lane, as a number that the compiler does not know anything of: what a loop's body computes from it stays in there, and
// out of the registers that the body's products need.
__device__ __forceinline__ int lane_here() {
    int lane = lane_id();
    asm volatile("" : "+v"(lane));
    return lane;
}

// 64 lanes' 16 bytes each from global memory into LDS, lane after lane from `lds` (the same in all lanes) on. In assembly,
// because the compiler lets a transposing read of LDS wait for every such load before it, also of the other buffer; the
// kernels wait for them themselves. M0 holds nothing else here: no other instruction of these kernels reads it.
__device__ __forceinline__ void load_to_lds(uint32_t lds, const char *base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds(uint32_t lds, const char *from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory");
}

namespace {
__device__ __attribute__((aligned(16))) const char kZeroChunk[16] = {};   // what a step reads past the end of k
}

// A wavefront's writes of LDS before it, for its other lanes' reads behind it (and the other way round).
__device__ __forceinline__ void lds_order() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// The first `valid` of 8 neighbouring elements (any number: none below 1, all from 8 on).
template <class T>
__device__ __forceinline__ void store8(T *to, int64_t valid, const float (&v)[8]) {
    store_cols<T, 8>(to, 0, static_cast<int>(std::min<int64_t>(valid, 8)), v);
}
template <class T>
__device__ __forceinline__ void load8(const T *from, int64_t valid, float (&v)[8]) {
    load_cols<T, 8>(from, 0, static_cast<int>(std::min<int64_t>(valid, 8)), v);
}

// The threads that share a region: number `at` of `step`.
struct Lanes {
    int at, step;
};

struct Side {
    const char *p;
    int64_t row;   // bytes from a row to the next
};

// Where element (row, col) of an array of P parts has its first one; the others follow 32 elements apart. stride: elements
// of a row, a multiple of 32 where there are several parts.
template <int P>
__device__ __forceinline__ int64_t part_at(int64_t row, int64_t col, int64_t stride) {
    return P == 1 ? row * stride + col : row * stride * P + col / 32 * (32 * P) + col % 32;
}

// The values of 1, 2 or 3 parts. The last part takes what is left, to nearest.
template <class E, int P>
__device__ __forceinline__ void to_parts(float v, E (&part)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        // values within half a step of fp32's largest would round to an infinity in bf16
        const float near = P == 3 && p == 0 && fabsf(v) < __builtin_inff() ? fminf(fmaxf(v, -0x1.fep127f), 0x1.fep127f) : v;
        part[p] = static_cast<E>(near);
        v -= static_cast<float>(part[p]);
    }
}

// Parts of 8 neighbouring elements of an array (the first a multiple of 8), zeros from number `valid` on.
template <class E, int P>
__device__ __forceinline__ void to_parts8(int64_t valid, const float (&v)[8], Frag<E> (&part)[P]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        E one[P];
        to_parts<E, P>(e < valid ? v[e] : 0.0f, one);
#pragma unroll
        for (int p = 0; p < P; ++p) part[p][e] = one[p];
    }
}
template <class E, int P>
__device__ __forceinline__ void store_parts8(E *to, const Frag<E> (&part)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) *reinterpret_cast<Frag<E> *>(to + p * 32) = part[p];
}
template <class E, int P>
__device__ __forceinline__ void store_parts8(E *to, int64_t valid, const float (&v)[8]) {
    Frag<E> part[P];
    to_parts8<E, P>(valid, v, part);
    store_parts8<E, P>(to, part);
}

// PAIR: B's rows come in groups of 16 from two arrays in turn. TWO: k runs through a second pair of operands after the
// first.
template <class E_, int P_, int BM_, int BN_, int WM_, int WN_, int BK_, bool ALONG_A, bool ALONG_B, bool PAIR_ = false,
          bool TWO_ = false, int STAGES_ = 2>
struct Tile {
    using E = E_;
    static constexpr int P = P_, BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_;
    static constexpr bool PAIR = PAIR_, TWO = TWO_, kAlong = ALONG_A || ALONG_B;
    static constexpr int STAGES = STAGES_;
    static constexpr int kWaves = WM * WN, kThreads = kWaves * kWave;
    static constexpr int kA = P * BM * BK * 2, kB = P * BN * BK * 2, kStage = kA + kB, kLds = STAGES * kStage;
    static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;   // fragments of 16 x 16 a wavefront
    static constexpr int kPerCu = 160 * 1024 / kLds, kPerSimd = std::max(1, std::min(2, kPerCu) * kWaves / 4);
    static_assert(FN % 2 == 0 && kPerCu >= 1, "pairs of fragments, one CU's LDS");

    // The part of a stage that holds one operand: rows of k (ALONG) or rows at one k.
    template <bool ALONG, int R>
    struct Half {
        static constexpr int kRow = (ALONG ? BK : R) * 2, kRows = ALONG ? R : BK;
        static constexpr int kChunks = kRow / 16;
        static constexpr int kPlane = kRow * kRows, kLoads = kPlane / (kWave * 16) / kWaves;
        static constexpr int kRowsPerLoad = kWave / kChunks;
        static_assert(kLoads >= 1 && kRowsPerLoad >= 1, "every wavefront loads");

        // ALONG: the 16 lanes that LDS serves at a time read one chunk of rows 0..3 and 12..15 of 16 and the next chunk of
        // the others, or the other way round: all places of 256 bytes differ. Down: 32 lanes read two chunks of the rows 0..3
        // and 8..11 of a group of 16: pairs of chunks change places.
        static __device__ __forceinline__ int place(int row, int chunk) {
            if constexpr (ALONG && kChunks == 4) return chunk ^ (0x78 >> (row / 4 % 4 * 2) & 3);   // 0, 2, 3, 1
            if constexpr (ALONG) return chunk ^ (row / (256 / kRow)) % kChunks;
            if constexpr (kRow == 128) return chunk ^ ((row >> 1 & 1) | (row >> 2 & 2)) << 1;
            return chunk ^ ((row & 3) | (row >> 1 & 4)) << 1;
        }

        const char *p;
        int64_t step, corner;          // corner: bytes from an operand's start to the tile's first row or column
        uint32_t off[kLoads];
        int32_t left;                  // of k, from the step that is loaded next on

        // A chunk's first part in a row that starts with 32 elements'.
        static __device__ __forceinline__ uint32_t at_chunk(int chunk) {
            return static_cast<uint32_t>(P == 1 ? chunk * 16 : chunk / 4 * (64 * P) + chunk % 4 * 16);
        }

        // valid: rows (ALONG) or columns from the tile's first one on that the operand has; what lies past them is read
        // from the last one and dropped with its results.
        __device__ __forceinline__ void start(const Side &s, int64_t first, int64_t valid, int64_t k0, int64_t k1, int wave, int lane) {
            corner = ALONG ? first * s.row : first * (2 * P);
            p = s.p + corner + k0 * (ALONG ? 2 * P : s.row);
            step = ALONG ? kRow * P : BK * s.row;
            left = static_cast<int32_t>(k1 - k0);
            const int last = static_cast<int>(std::min<int64_t>(valid, R)) - 1;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int row = (wave * kLoads + i) * kRowsPerLoad + lane / kChunks;
                const int chunk = place(row, lane % kChunks);
                if constexpr (ALONG)
                    off[i] = static_cast<uint32_t>(min(row, last)) * static_cast<uint32_t>(s.row) + at_chunk(chunk);
                else
                    off[i] = static_cast<uint32_t>(row) * static_cast<uint32_t>(s.row) + at_chunk(min(chunk, last / 8));
            }
        }

        __device__ __forceinline__ void turn(const char *second, int64_t k) {
            p = second + corner;
            left = static_cast<int32_t>(k);
        }

        // other: bytes to a second operand that every second group of 16 rows comes from.
        __device__ __forceinline__ void load(uint32_t lds, int wave, int lane, int64_t other = 0) {
            if (left >= BK) {
                each_load(lds, wave, other, [&](uint32_t at, const char *from, int i, int) { load_to_lds(at, from, off[i]); });
            } else {
                each_load(lds, wave, other, [&](uint32_t at, const char *from, int i, int first) {
                    const int row = first + lane / kChunks;
                    const int k = ALONG ? place(row, lane % kChunks) * 8 : row;
                    load_to_lds(at, k < left ? from + off[i] : kZeroChunk);
                });
            }
            p += step;
            left -= BK;
        }
        template <class F>
        __device__ __forceinline__ void each_load(uint32_t lds, int wave, int64_t other, F f) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
#pragma unroll
                for (int q = 0; q < P; ++q) {
                    const int first = (wave * kLoads + i) * kRowsPerLoad;
                    f(lds + static_cast<uint32_t>(q * kPlane + first * kRow),
                      p + q * 64 + (PAIR && first / 16 % 2 ? other : 0), i, first);
                }
        }

        // The fragment of 16 rows (ALONG) or columns from `first` on, at the 32 k from 32 ks on: lane l holds number
        // l % 16 of them, at the 8 k from 8 (l / 16) on.
        static __device__ __forceinline__ Frag<E> frag(const char *lds, int q, int first, int ks, int lane) {
            if constexpr (ALONG) {
                const int row = first + lane % 16;
                return *reinterpret_cast<const Frag<E> *>(lds + q * kPlane + row * kRow + place(lane % 16, ks * 4 + lane / 16) * 16);
            } else {
                // lanes 4 r .. 4 r + 3 of 16 give the address of row r of 4, lane c of them gets column c of the four rows
                using S4 = short __attribute__((ext_vector_type(4)));
                const int row = ks * 32 + lane / 16 * 8 + lane % 16 / 4;
                const char *a = lds + q * kPlane + row * kRow + place(row & 15, first / 8 + lane % 4 / 2) * 16 + lane % 2 * 8;
                union {
                    S4 h[2];
                    Frag<E> f;
                } u;
                u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4 *)(a));
                u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4 *)(a + 4 * kRow));
                return u.f;
            }
        }
    };
    using HalfA = Half<ALONG_A, BM>;
    using HalfB = Half<ALONG_B, BN>;
    static constexpr int kStepLoads = P * (HalfA::kLoads + HalfB::kLoads);

    // The product over k0 <= k < k1 (k0 a multiple of BK) of the tile from (m0, n0) on of an m x n one. Element e of
    // acc[i][j] is C at row m0 + 16 (wm FM + i) + lane % 16, column n0 + 16 (wn FN + j) + 4 (lane / 16) + e. PAIR: the second
    // array lies `other` bytes behind b; n and n0 count one array's rows. TWO: both pairs of operands have k elements of k,
    // the second's count from k rounded up to BK on; they share the first's strides.
    static __device__ __forceinline__ void run(const Side &a, const Side &b, const char *a2, const char *b2, int64_t other,
                                               int64_t m0, int64_t m, int64_t n0, int64_t n, int64_t k, int64_t k0,
                                               int64_t k1, char *lds, f4 (&acc)[FM][FN]) {
        const int lane = lane_here(), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
        const int wm = wave / WN, wn = wave % WN;
        HalfA ha;
        HalfB hb;
        int turn_at = -1;   // the step with which the second operands begin
        const int64_t whole = (k + BK - 1) / BK * BK;
        if (TWO && k0 >= whole) {
            ha.start(Side{a2, a.row}, m0, m - m0, k0 - whole, k1 - whole, wave, lane);
            hb.start(Side{b2, b.row}, n0, n - n0, k0 - whole, k1 - whole, wave, lane);
        } else {
            if (TWO && k1 > whole) turn_at = static_cast<int>((whole - k0) / BK);
            ha.start(a, m0, m - m0, k0, std::min(k1, k), wave, lane);
            hb.start(b, n0, n - n0, k0, std::min(k1, k), wave, lane);
        }
        if constexpr (PAIR) {   // row r of the tile is row 16 (r / 32) + r % 16 of an array
            const int last = static_cast<int>(std::min<int64_t>(n - n0, BN / 2)) - 1;
#pragma unroll
            for (int i = 0; i < HalfB::kLoads; ++i) {
                const int row = (wave * HalfB::kLoads + i) * HalfB::kRowsPerLoad + lane / HalfB::kChunks;
                hb.off[i] = static_cast<uint32_t>(min(row / 32 * 16 + row % 16, last)) * static_cast<uint32_t>(b.row) +
                            HalfB::at_chunk(HalfB::place(row, lane % HalfB::kChunks));
            }
        }
        const auto base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds));
        const int steps = static_cast<int>((k1 - k0 + BK - 1) / BK);
        int next = 0;       // the step that is loaded next on, and its place
        uint32_t to = base;
        auto load = [&] {
            if (TWO && next == turn_at) {
                ha.turn(a2, k1 - whole);
                hb.turn(b2, k1 - whole);
            }
            ha.load(to, wave, lane);
            hb.load(to + kA, wave, lane, other);
            ++next;
            to = to + kStage == base + kLds ? base : to + kStage;
        };
        f4 low[P == 3 ? FM : 1][P == 3 ? FN : 1] = {};
        for (int s = 0; s < STAGES - 1 && s < steps; ++s) load();
        int stage = 0;
        for (int s = 0; s < steps; ++s) {
            // this wavefront's loads of the step have landed (of STAGES - 2 further steps they may be on their way) and its
            // reads of the step before are done; then everybody's
            if (STAGES > 2 && s + STAGES - 1 <= steps)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * kStepLoads) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (next < steps) load();
            const char *la = lds + stage, *lb = la + kA;
            stage = stage + kStage == kLds ? 0 : stage + kStage;
#pragma unroll
            for (int ks = 0; ks < BK / 32; ++ks) {
                Frag<E> fb[P][FN];
#pragma unroll
                for (int q = 0; q < P; ++q)
#pragma unroll
                    for (int j = 0; j < FN; ++j) fb[q][j] = HalfB::frag(lb, q, (wn * FN + j) * 16, ks, lane);
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    Frag<E> fa[P];
#pragma unroll
                    for (int p = 0; p < P; ++p) fa[p] = HalfA::frag(la, p, (wm * FM + i) * 16, ks, lane);
#pragma unroll
                    for (int p = P - 1; p >= 0; --p)
#pragma unroll
                        for (int q = P - 1 - p; q >= 0; --q)
#pragma unroll
                            for (int j = 0; j < FN; ++j) {
                                // three parts: what lies below the first parts' product is summed apart, so that the large
                                // sum is rounded once for each 32 k and not six times
                                f4 &to = P == 3 && p + q > 0 ? low[P == 3 ? i : 0][P == 3 ? j : 0] : acc[i][j];
                                to = mfma32(fb[q][j], fa[p], to);
                            }
                }
            }
            // reads of LDS two rows of fragments ahead of the products that need them
            constexpr int kReadA = P * (ALONG_A ? 1 : 2), kReadB = P * FN * (ALONG_B ? 1 : 2), kGroups = FM * (BK / 32);
            constexpr int kFirst = kReadB + 2 * kReadA, kRest = (BK / 32) * (kReadB + FM * kReadA) - kFirst;
            constexpr int kEach = kGroups > 2 ? (kRest + kGroups - 3) / (kGroups - 2) : 1;
            __builtin_amdgcn_sched_group_barrier(0x100, kFirst, 0);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                __builtin_amdgcn_sched_group_barrier(0x008, FN * P * (P + 1) / 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, kEach, 0);
            }
        }
        if constexpr (P == 3) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] += low[i][j];
        }
    }

    // ---- what becomes of acc: it goes through LDS, a wavefront's rows (in kPhases parts) in a region of its own, so that
    // the code behind it is a loop over whole 128-byte lines, not acc's fragments written out one by one.
    static constexpr int kCols = FN * 16, kPhases = FM * FN * 1024 * kWaves <= kLds ? 1 : 2, kRows = FM * 16 / kPhases;
    static constexpr int kRegion = kRows * kCols * 4;
    static_assert(kRegion * kWaves <= kLds && (kCols == 32 || kCols % 64 == 0), "regions fit");

    // Four columns of a row; their place changes with the row, so that 16 rows' same columns fill all banks.
    static __device__ __forceinline__ f4 &cell(char *region, int row, int chunk) {
        const int to = kCols == 32 ? chunk ^ (row >> 1 & 7) : (chunk & ~15) + ((chunk & 15) ^ (row & 15) ^ (chunk >> 4) * 4);
        return *reinterpret_cast<f4 *>(region + row * (kCols * 4) + to * 16);
    }
    template <int phase>
    static __device__ __forceinline__ void fill(const f4 (&acc)[FM][FN], char *region) {
        const int lane = lane_here();
#pragma unroll
        for (int i = 0; i < FM; ++i)
            if (i / (FM / kPhases) == phase)
#pragma unroll
                for (int j = 0; j < FN; ++j) cell(region, i % (FM / kPhases) * 16 + lane % 16, j * 4 + lane / 16) = acc[i][j];
    }
    static __device__ __forceinline__ void get8(char *region, int row, int chunk, float (&v)[8]) {
        const f4 x = cell(region, row, chunk), y = cell(region, row, chunk + 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = x[e];
            v[4 + e] = y[e];
        }
    }
    // f(row, column, values of 8 columns) for a region.
    template <class F>
    static __device__ __forceinline__ void rows8(char *region, Lanes lanes, F f) {
        constexpr int kPer = kCols / 8;
#pragma unroll 2
        for (int c = lanes.at; c < kRows * kPer; c += lanes.step) {
            float v[8];
            get8(region, c / kPer, c % kPer * 2, v);
            f(c / kPer, c % kPer * 8, v);
        }
    }
    // PAIR: f(row, column of an array, the first's 8 columns, the second's).
    template <class F>
    static __device__ __forceinline__ void pairs8(char *region, Lanes lanes, F f) {
        constexpr int kPer = kCols / 16;
#pragma unroll 2
        for (int c = lanes.at; c < kRows * kPer; c += lanes.step) {
            const int row = c / kPer, col = c % kPer * 8, chunk = col / 16 * 8 + col % 16 / 4;
            float v[8], w[8];
            get8(region, row, chunk, v);
            get8(region, row, chunk + 4, w);
            f(row, col, v, w);
        }
    }
    // Where a region's row keeps the 32 bytes with a part's 16 columns from `col` on, once its values have become parts: in the
    // row's own place, pairs of chunks turned as a transposing read of 4 rows wants them.
    static __device__ __forceinline__ char *pair(char *region, int row, int p, int col) {
        constexpr int kPairs = kCols / 8;
        const int at = (p * (kCols / 16) + col / 16) ^ (((row & 3) | (row >> 1 & 4)) & (kPairs - 1));
        return region + row * (kCols * 4) + at * 32;
    }
    // rows8's f may leave 8 columns' parts there (all of a row's lanes have read it by then) ...
    static __device__ __forceinline__ void leave8(char *region, int row, int col, const Frag<E> (&part)[P]) {
#pragma unroll
        for (int p = 0; p < P; ++p) *reinterpret_cast<Frag<E> *>(pair(region, row, p, col) + col % 16 * 2) = part[p];
    }
    // ... for f(row, column, parts of 8 rows).
    template <class F>
    static __device__ __forceinline__ void mirror8(char *region, Lanes lanes, F f) {
        static_assert(P <= 2 && kRows % 32 == 0, "a row's parts take its own place");
        using S4 = short __attribute__((ext_vector_type(4)));
        if (lanes.step > kWave)
            __syncthreads();
        else
            lds_order();
        const int lane = lanes.at % kWave;
#pragma unroll 1
        for (int u = lanes.at / kWave; u < kRows / 32 * (kCols / 16); u += lanes.step / kWave) {
            const int row = u % (kRows / 32) * 32 + lane / 16 * 8, col = u / (kRows / 32) * 16;
            Frag<E> part[P];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                union {
                    S4 h[2];
                    Frag<E> f;
                } v;
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    v.h[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4 *)(
                        pair(region, row + i * 4 + lane % 16 / 4, p, col) + lane % 4 * 8));
                part[p] = v.f;
            }
            f(row, col + lane % 16, part);
        }
    }
};

// The workgroups of an XCD (every eighth) take neighbouring numbers, so that its L2 holds what they share.
__device__ __forceinline__ int by_xcd(int id, int count) {
    const int each = count / 8, more = count % 8, x = id % 8;
    return x * each + min(x, more) + id / 8;
}

// Tile number id of a gm x gn grid, column by column in bands of four rows.
__device__ __forceinline__ void tile_at(int id, int gm, int gn, int &tm, int &tn) {
    constexpr int kBand = 4;
    const int band = id / (kBand * gn), rows = min(gm - band * kBand, kBand), in = id - band * (kBand * gn);
    tm = band * kBand + in % rows;
    tn = in / rows;
}

// ------------------------------------------------------------------ kernels over a job's tiles
// How a launch's tiles are taken. `whole` workgroups make a tile each; the steps along k of the `tiles - whole` others are
// shared out to `parts` workgroups: each tile's in the same number of pieces, the same piece of all tiles side by side (they
// read the same k at a time), or all tiles' steps, one tile's after the other's, evenly, so that a workgroup has pieces of
// one or two tiles. Sums of pieces wait in memory and are joined in k's order by k_join: results do not depend on what ends
// first.
template <class T>
struct Which {
    using type = T;
};
enum { kLarge, kSmall, kDeep, kTiny, kMiddle };
struct Cut {
    int32_t kind, parts;
    int64_t tiles, whole, steps;   // steps: of one tile
    bool evenly;                   // parts of all shared tiles' steps, not the same pieces of each
    size_t floats;                 // of the pieces' sums
};
struct Tiling {
    int32_t tiles, whole, steps, parts;
    int32_t each, more;            // steps of a part; the first `more` parts have one more (evenly), or pieces of a tile: -more
    float *part;

    // Part j's first tile, and its steps from that tile's first one on.
    __device__ __forceinline__ void part_of(int j, int &tile, int &step, int &end) const {
        if (more < 0) {
            const int shared = tiles - whole, piece = j / shared;
            tile = whole + j - piece * shared;
            step = piece * each;
            end = min(step + each, steps);
        } else {
            const int in = begin(j) / steps;
            tile = whole + in;
            step = begin(j) - in * steps;
            end = begin(j + 1) - in * steps;
        }
    }
    __device__ __forceinline__ int begin(int j) const { return j * each + min(j, more); }
    // Of the shared tiles' number `shared` (evenly): the part that has a step.
    __device__ __forceinline__ int owner(int step) const {
        const int with = more * (each + 1);
        return step < with ? step / (each + 1) : more + (step - with) / each;
    }
};
inline Tiling tiling_of(const Cut &c, float *part) {
    const int64_t rest = c.tiles - c.whole, shared = rest * c.steps;
    Tiling t{static_cast<int32_t>(c.tiles), static_cast<int32_t>(c.whole), static_cast<int32_t>(c.steps), c.parts, 0, 0, part};
    if (rest > 0 && c.evenly) {
        t.each = static_cast<int32_t>(shared / c.parts);
        t.more = static_cast<int32_t>(shared % c.parts);
    } else if (rest > 0) {
        const int64_t pieces = c.parts / rest;
        t.each = static_cast<int32_t>(ceil_div(c.steps, pieces));
        t.more = static_cast<int32_t>(-pieces);
    }
    return t;
}

// A job says which tiles it has, multiplies one and puts its elements where they belong:
//   Tiling t
//   Place at<T>(tile)                                 where the tile lies
//   multiply<T>(place, step, end, lds, acc)           its product over some of k's steps
//   take<T>(place, row, column, region, lanes)        what a region holds, from that row and column of the tile on
template <class T, class J>
__device__ __forceinline__ void take_region(const J &job, const decltype(job.template at<T>(0)) &place, int wave, int phase,
                                            char *region, Lanes lanes) {
    const int row = wave / T::WN * T::FM * 16 + phase * T::kRows, col = wave % T::WN * T::kCols;
    job.template take<T>(place, row, col, region, lanes);
}

template <class T, class J>
__global__ __launch_bounds__(T::kThreads, T::kPerSimd) void k_tiles(const J job) {
    __shared__ __attribute__((aligned(1024))) char lds[T::kLds];
    const Tiling &t = job.t;
    const int wave = static_cast<int>(threadIdx.x) / kWave;
    char *region = lds + wave * T::kRegion;
    const int id = static_cast<int>(blockIdx.x);
    int j = 0, tile, step = 0, end = t.steps;
    if (id < t.whole) {
        tile = by_xcd(id, t.whole);
    } else {
        j = by_xcd(id - t.whole, t.parts);
        t.part_of(j, tile, step, end);
    }
#pragma unroll 1
    for (int piece = 0; step < end; ++piece) {   // steps from `step` to `end` of this tile, and on to the next one's
        const auto place = job.template at<T>(tile);
        const int last = min(end, t.steps);
        f4 acc[T::FM][T::FN] = {};
        if (piece > 0) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // everybody has left the regions
        job.template multiply<T>(place, step, last, lds, acc);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // everybody's reads of the last step
        // one copy of what follows for both phases: half the code, in the same time
#pragma unroll 1
        for (int phase = 0; phase < T::kPhases; ++phase) {
            lds_order();
            if (phase == 0)
                T::template fill<0>(acc, region);
            else
                T::template fill<T::kPhases - 1>(acc, region);
            lds_order();
            if (step == 0 && last == t.steps) {
                take_region<T>(job, place, wave, phase, region, Lanes{lane_here(), kWave});
                continue;
            }
            float *to = t.part + (((static_cast<int64_t>(j) * 2 + piece) * T::kWaves + wave) * T::kPhases + phase) * (T::kRegion / 4);
            for (int c = lane_here(); c < T::kRegion / 16; c += kWave)
                reinterpret_cast<f4 *>(to)[c] = T::cell(region, c / (T::kCols / 4), c % (T::kCols / 4));
        }
        ++tile;
        end -= t.steps;
        step = 0;
    }
}

constexpr int kJoinThreads = 256;   // of a region

template <class T, class J>
__global__ __launch_bounds__(kJoinThreads) void k_join(const J job) {
    __shared__ __attribute__((aligned(1024))) char region[T::kRegion];
    const Tiling &t = job.t;
    constexpr int size = T::kRegion / 16, per = T::kWaves * T::kPhases;
    const int shared = static_cast<int>(blockIdx.x) / per, at = static_cast<int>(blockIdx.x) % per;
    const int step = shared * t.steps, rest = t.tiles - t.whole;
    const int first = t.more < 0 ? 0 : t.owner(step), last = t.more < 0 ? (t.steps - 1) / t.each : t.owner(step + t.steps - 1);
    if (t.more >= 0 && first == last) return;   // one workgroup had it whole
    const f4 *part = reinterpret_cast<const f4 *>(t.part) + at * size + threadIdx.x;
    constexpr int kMine = T::kRegion / 16 / kJoinThreads;
    f4 v[kMine] = {};
    constexpr int kAhead = kMine == 1 ? 8 : 4;
#pragma unroll kAhead
    for (int j = first; j <= last; ++j) {
        // evenly: the piece is its workgroup's second where that began with the tile before
        const int slot = t.more < 0 ? (j * rest + shared) * 2 : j * 2 + (j == first && t.begin(j) / t.steps != shared);
        const f4 *from = part + static_cast<int64_t>(slot) * per * size;
#pragma unroll
        for (int i = 0; i < kMine; ++i) v[i] += from[i * kJoinThreads];
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int c = i * kJoinThreads + static_cast<int>(threadIdx.x);
        T::cell(region, c / (T::kCols / 4), c % (T::kCols / 4)) = v[i];
    }
    __syncthreads();
    take_region<T>(job, job.template at<T>(t.whole + shared), at / T::kPhases, at % T::kPhases, region,
                   Lanes{static_cast<int>(threadIdx.x), kJoinThreads});
}

// A launch numbers its threads in 32 bits.
constexpr int64_t kMaxTiles = int64_t(1) << 22;

template <class T, class J>
int launch_tiles(const J &job, hipStream_t s) {
    const int rest = job.t.tiles - job.t.whole;
    k_tiles<T, J><<<static_cast<unsigned>(job.t.whole + (rest > 0 ? job.t.parts : 0)), T::kThreads, 0, s>>>(job);
    W2V_LAUNCH_CHECK("k_tiles");
    if (rest > 0) {
        k_join<T, J><<<static_cast<unsigned>(rest * T::kWaves * T::kPhases), kJoinThreads, 0, s>>>(job);
        W2V_LAUNCH_CHECK("k_join");
    }
    return W2V_OK;
}

// Microseconds of a step (all of a tile's products over BK of k), measured: by whether k runs along a row of either operand,
// by parts, and by kind, where a CU has one tile at a time, and where there are more. Large tiles do 1.4 to 1.5 PFLOP/s; small
// ones read LDS more often.
constexpr double kStepUs[2][3][5][2] = {{{{1.50, 1.56}, {0.67, 0.44}, {0.65, 0.59}, {0.28, 0.19}, {0.90, 0.93}},
                                         {{2.07, 2.12}, {0.71, 0.56}, {0.67, 0.67}, {0.32, 0.21}, {1.15, 1.15}},
                                         {{2.16, 2.20}, {0.73, 0.56}, {1.20, 1.22}, {0.45, 0.32}, {}}},
                                        {{{1.46, 1.57}, {0.65, 0.43}, {0.64, 0.59}, {0.30, 0.20}, {0.87, 0.97}},
                                         {{2.10, 2.10}, {0.73, 0.59}, {0.66, 0.68}, {0.31, 0.22}, {1.12, 1.16}},
                                         {{2.20, 2.20}, {0.80, 0.68}, {1.17, 1.22}, {0.43, 0.36}, {}}}};

// The cut with the least time by this model: the CUs take tiles in turns of their steps and two more until the first product,
// 1 us and what an element of the result moves behind them (`bytes` of it; a CU's share of memory is 20 KB a us). Sums of
// pieces go through memory twice, and joining them is another launch, 0.2 us a piece of a tile. count(tile): the tiles of all products of a launch that
// have k in common. S: the tiles, Large, Small, Tiny, and Deep, which are small ones with more steps on their way where a CU
// has but one.
template <class S, class F>
Cut choose_cut(int64_t k, double bytes, F count, bool two = false) {
    Cut best{};
    double least = 1e300;
    const int64_t cus = device_cu_count();
    auto weigh = [&](int32_t kind, auto tile) {
        using T = typename decltype(tile)::type;
        const int64_t tiles = count(tile), steps = ceil_div(k, T::BK) * (two ? 2 : 1), area = T::BM * T::BN;
        const double *step_us = kStepUs[T::kAlong][T::P - 1][kind], out_us = 1.0 + area * (0.03 + 0.05 * bytes) * 1e-3;
        auto offer = [&](int64_t whole, int64_t parts, bool evenly) {
            const int64_t rest = tiles - whole, turns = ceil_div(whole, cus) + (rest > 0 ? ceil_div(parts, cus) : 0);
            const double step = step_us[turns > 1];
            double us = static_cast<double>(ceil_div(whole, cus)) * ((steps + 2) * step + out_us);
            size_t floats = 0;
            if (rest > 0) {
                // sharing steps out evenly has the workgroups read different k at a time: 15 % more
                const double piece = evenly ? 1.15 * (rest * steps) / parts + 2 : static_cast<double>(ceil_div(steps, parts / rest));
                us += ceil_div(parts, cus) * ((piece + 2) * step + (evenly ? 2 : 1) * (1.0 + area * 0.23e-3)) + 6.0 +
                      0.2 * parts / rest + 4.0 * parts * area / 4e6 + rest * area * bytes / 4e6;
                floats = static_cast<size_t>(2 * parts * area);
            }
            if (us >= least * 0.999) return;
            least = us;
            best = Cut{kind, static_cast<int32_t>(parts), tiles, whole, steps, evenly, floats};
        };
        offer(tiles, 1, false);
        // the last turn's tiles, or with the turn before it
        const int64_t left = tiles % cus;
        for (int64_t rest : {left, left + cus}) {
            if (rest == 0 || rest > tiles || rest * steps >= INT32_MAX) continue;
            for (int64_t n = 2; n <= 64 && n * 2 <= steps && n * rest <= 2 * cus; ++n) offer(tiles - rest, n * rest, false);
            if (rest * steps >= 4 * cus) offer(tiles - rest, rest > cus ? 2 * cus : cus, true);
        }
    };
    weigh(kLarge, Which<typename S::Large>{});
    weigh(kSmall, Which<typename S::Small>{});
    weigh(kDeep, Which<typename S::Deep>{});
    weigh(kTiny, Which<typename S::Tiny>{});
    if constexpr (!std::is_same<typename S::Middle, typename S::Deep>::value) weigh(kMiddle, Which<typename S::Middle>{});
    return best;
}

// The tiles of an m x n product.
template <class T>
int64_t count_tiles(int64_t m, int64_t n) {
    return ceil_div(m, T::BM) * ceil_div(n, T::BN);
}
template <class S>
Cut choose_cut_of(int64_t m, int64_t n, int64_t k, double bytes, bool two = false) {
    return choose_cut<S>(k, bytes, [&](auto tile) { return count_tiles<typename decltype(tile)::type>(m, n); }, two);
}

inline int32_t tiles_along(int64_t size, int64_t tile) { return static_cast<int32_t>(ceil_div(size, tile)); }

// A cut's tile sizes.
template <class S>
int64_t tile_m(const Cut &c) {
    constexpr int size[] = {S::Large::BM, S::Small::BM, S::Deep::BM, S::Tiny::BM, S::Middle::BM};
    return size[c.kind];
}
template <class S>
int64_t tile_n(const Cut &c) {
    constexpr int size[] = {S::Large::BN, S::Small::BN, S::Deep::BN, S::Tiny::BN, S::Middle::BN};
    return size[c.kind];
}

template <class S, class J>
int launch_cut(const Cut &c, float *part, J &job, hipStream_t s) {
    job.t = tiling_of(c, part);
    switch (c.kind) {
        case kLarge: return launch_tiles<typename S::Large, J>(job, s);
        case kSmall: return launch_tiles<typename S::Small, J>(job, s);
        case kDeep: return launch_tiles<typename S::Deep, J>(job, s);
        case kMiddle: return launch_tiles<typename S::Middle, J>(job, s);
        default: return launch_tiles<typename S::Tiny, J>(job, s);
    }
}

}  // namespace w2v
