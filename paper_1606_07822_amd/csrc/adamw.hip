// AdamW over many tensors in one launch.
//
//   g = grad * grad_scale;  m = b1 m + (1-b1) g;  v = b2 v + (1-b2) g^2
//   p = p (1 - lr wd) - (lr / (1-b1^t)) m / (sqrt(v) / sqrt(1-b2^t) + eps)
//
// Memory bounds it (28 bytes an element with fp32 parameters, gradients and moments): every array is read and written
// once, 16 bytes a lane and access. The tensors are cut into chunks of kChunk elements; a table in device memory, laid
// out once, says for each chunk which tensor it belongs to, so a launch covers tensors of any number and size.
//
// Moments in 8 bits, in blocks of 256 elements of a tensor with a scale each: m as e4m3 times the scale (the largest
// |m| of the block is 448), rounded to nearest; v as its root r, an unsigned float of 4 exponent and 4 fraction bits
// (c < 16: c 2^-18; else (1 + (c & 15) / 16) 2^((c >> 4) - 15)) times the scale (the largest r is 31/16). With
// b2 = 0.999 a step changes r by less than half a code's width for most gradients, so rounding to nearest would hold r
// where it is; r is rounded up or down at random in proportion instead, by 16 bits of a hash of (seed, step, element),
// and a positive r never becomes 0 (m / eps would follow). Moments, their scales and the root are computed in fp32,
// each operation rounded by itself (no contraction), so that the codes are a function of the inputs alone.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "w2v_ops.h"

namespace w2v {
namespace {

constexpr int kAdamThreads = 256;
constexpr int kPer = 4;                                // neighbouring elements of a lane; a wavefront's are one block of 256
constexpr int kSteps = 4;
constexpr int kChunk = kAdamThreads * kPer * kSteps;   // elements of a workgroup
static_assert(kPer * kWave == kMomentBlock, "a wavefront reduces a block's scale");

struct Scalars {
    float b1, c1, b2, c2, size, root, eps, grad_scale;
    double lr;
    uint32_t key;
};

struct Entry {
    void *p;
    const void *g;
    int64_t n, cols, p_stride, g_stride, offset;
    float decay;
    int32_t p_type, g_type, flat;   // flat: both arrays packed
};

struct Place {
    int32_t tensor, chunk;
};

// The plan's memory: this header, the entries, the chunks' places.
struct Header {
    uint64_t mark;   // kMark in a plan that was built: a step on other memory does nothing
    int64_t n_chunks;
    const Entry *entries;
    const Place *places;
    Scalars scalars;   // of the last step whose learning rate or step count lay in device memory
};
constexpr size_t kHeaderBytes = 256;
constexpr uint64_t kMark = 0x6e616c7077616461ull;
static_assert(sizeof(Header) <= kHeaderBytes);

__host__ __device__ inline uint32_t mix32(uint32_t h) {   // MurmurHash3's finaliser
    h = (h ^ (h >> 16)) * 0x85EBCA6Bu;
    h = (h ^ (h >> 13)) * 0xC2B2AE35u;
    return h ^ (h >> 16);
}

__host__ __device__ inline Scalars make_scalars(const w2v_adamw_params &p, double lr, int64_t step) {
    const double t = static_cast<double>(step);
    Scalars s;
    s.b1 = static_cast<float>(p.beta1);
    s.c1 = static_cast<float>(1.0 - p.beta1);
    s.b2 = static_cast<float>(p.beta2);
    s.c2 = static_cast<float>(1.0 - p.beta2);
    s.size = static_cast<float>(lr / (1.0 - pow(p.beta1, t)));
    s.root = static_cast<float>(1.0 / sqrt(1.0 - pow(p.beta2, t)));
    s.eps = static_cast<float>(p.eps);
    s.grad_scale = p.grad_scale;
    s.lr = lr;
    s.key = mix32(p.seed ^ (static_cast<uint32_t>(step) * 0x9E3779B9u));
    return s;
}

__global__ void k_adamw_scalars(Header *h, w2v_adamw_params p) {
    if (h->mark == kMark) h->scalars = make_scalars(p, p.lr_device ? static_cast<double>(*p.lr_device) : p.lr,
                              p.step_device ? *p.step_device : p.step);
}

// Largest of the wavefront's values, in every lane: of non-negative floats' bit patterns, so a NaN stays.
__device__ __forceinline__ float wave_max_bits(float v) {
    uint32_t b = __builtin_bit_cast(uint32_t, v);
    auto take = [&](uint32_t o) { b = max(b, o); };
    take(__builtin_amdgcn_update_dpp(0, b, 0xB1, 0xF, 0xF, true));
    take(__builtin_amdgcn_update_dpp(0, b, 0x4E, 0xF, 0xF, true));
    take(__builtin_amdgcn_update_dpp(0, b, 0x141, 0xF, 0xF, true));
    take(__builtin_amdgcn_update_dpp(0, b, 0x140, 0xF, 0xF, true));
    auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    b = max(static_cast<uint32_t>(r[0]), static_cast<uint32_t>(r[1]));
    r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __builtin_bit_cast(float, max(static_cast<uint32_t>(r[0]), static_cast<uint32_t>(r[1])));
}

// Four codes in a word, the first in the low byte.
__device__ __forceinline__ void decode_m(uint32_t c, float scale, float (&m)[kPer]) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c), false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c), true);
    m[0] = lo[0] * scale;
    m[1] = lo[1] * scale;
    m[2] = hi[0] * scale;
    m[3] = hi[1] * scale;
}

__device__ __forceinline__ uint32_t encode_m(const float (&m)[kPer], float inverse) {
#pragma clang fp contract(off)
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(m[0] * inverse, m[1] * inverse, 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(m[2] * inverse, m[3] * inverse, c, true);
    return static_cast<uint32_t>(c);
}

// The root's codes are the exponent and fraction bits of an fp32 number 2^-112 as large, subnormal ones among them:
// either way is a product with a power of two and a shift, and rounding one up or down is an addition below the code.
__device__ __forceinline__ float decode_r(uint32_t c) { return __builtin_bit_cast(float, c << 19) * 0x1p112f; }

// r / scale as a code, rounded by the 16 random bits h.
__device__ __forceinline__ uint32_t encode_r(float r, float inverse, uint32_t h) {
#pragma clang fp contract(off)
    const float t = (r * inverse) * 0x1p-112f;
    const uint32_t c = min((__builtin_bit_cast(uint32_t, t) + (h * 8 + 4)) >> 19, 255u);
    return r > 0.0f ? max(c, 1u) : c;
}

// One element: new moments (m, v) and v's root.
__device__ __forceinline__ void update_moments(float g, float &m, float &v, float &r, const Scalars &s) {
#pragma clang fp contract(off)
    g *= s.grad_scale;
    m = m * s.b1 + g * s.c1;
    v = v * s.b2 + (g * g) * s.c2;
    r = sqrtf(v);
}

// The new parameter. The quotient's reciprocal is the hardware's, off by one unit in the last place.
__device__ __forceinline__ float updated(float p, float m, float r, float keep, const Scalars &s) {
    return fmaf(p, keep, -(m * s.size) * __builtin_amdgcn_rcpf(fmaf(r, s.root, s.eps)));
}

// The tensors' addresses come from the plan, where the compiler can't tell global memory from the rest.
template <class T>
using Global = __attribute__((address_space(1))) T;

// N neighbouring elements as words, at any element-aligned address. Each is used once: non-temporal, which leaves the
// caches to what is read again (600 M fp32 parameters: 3.83 -> 3.20 ms, 4.4 -> 5.3 TB/s).
template <class T, int N>
struct Words {
    static constexpr int count = N * sizeof(T) / 4;
    typedef uint32_t type __attribute__((ext_vector_type(count), aligned(sizeof(T))));
};

template <class T, int N>
__device__ __forceinline__ void load_global(const T *p, float (&f)[N]) {
    using W = typename Words<T, N>::type;
    const W w = __builtin_nontemporal_load((const Global<W> *)(p));
    const auto u = __builtin_bit_cast(Pack<T, N>, w);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = static_cast<float>(u.v[e]);
}

template <class T, int N>
__device__ __forceinline__ void store_global(T *p, const float (&f)[N]) {
    using W = typename Words<T, N>::type;
    Pack<T, N> u;
#pragma unroll
    for (int e = 0; e < N; ++e) u.v[e] = static_cast<T>(f[e]);
    __builtin_nontemporal_store(__builtin_bit_cast(W, u), (Global<W> *)(p));
}

// A chunk's elements, four neighbouring ones of a lane at a time. kPacked: every element lies in the tensor and both
// arrays are packed; kRows: every element lies in the tensor, whose rows have gaps and a multiple of four columns, so
// that any four lie in one row; kAny: all else, where four that lie in one row are still one access. (A table of rows of
// 300 floats, 320 apart, as kAny: 600 M parameters in 3.84 ms, with a branch around every load.)
enum Layout { kPacked, kRows, kAny };
template <class TP, class TG, int BITS, Layout LAYOUT>
__device__ __forceinline__ void chunk_update(const Entry &t, int64_t first, void *mv, void *vv, float *m_scale,
                                             float *v_scale, const Scalars &s) {
    TP *pp = static_cast<TP *>(t.p);
    const TG *gp = static_cast<const TG *>(t.g);
    const float keep = static_cast<float>(1.0 - s.lr * static_cast<double>(t.decay));
    constexpr bool FULL = LAYOUT != kAny;   // no element past the tensor's end
    const int64_t row0 = LAYOUT == kPacked || t.flat ? 0 : first / t.cols;
    const int64_t rem0 = LAYOUT == kPacked || t.flat ? first : first - row0 * t.cols;
    float p[kSteps][kPer], g[kSteps][kPer], m[kSteps][kPer], v[kSteps][kPer];
    uint32_t mc[kSteps], vc[kSteps];
    int64_t po[kSteps], go[kSteps];
    int in_row[kSteps];   // elements of the four that lie in the first one's row
    uint32_t col[kSteps];
    auto rows_on = [&](int i, int k) -> uint32_t {   // rows between the four's first element and its i-th
        if (i < in_row[k]) return 0;
        return t.cols >= kPer ? 1 : (col[k] + static_cast<uint32_t>(i)) / static_cast<uint32_t>(t.cols);
    };
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        const int local = (k * kAdamThreads + static_cast<int>(threadIdx.x)) * kPer;
        const int64_t e = first + local, at = t.offset + e;
        if constexpr (FULL) {
            po[k] = go[k] = e;
            if constexpr (LAYOUT == kRows) {
                const uint32_t c = static_cast<uint32_t>(t.cols), at_row = static_cast<uint32_t>(rem0) + local;
                const uint32_t q = at_row / c, at_col = at_row - q * c;
                po[k] = (row0 + q) * t.p_stride + at_col;
                go[k] = (row0 + q) * t.g_stride + at_col;
            }
            load_global<TP, kPer>(pp + po[k], p[k]);
            load_global<TG, kPer>(gp + go[k], g[k]);
        } else {
            in_row[k] = 0;
            po[k] = go[k] = col[k] = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) p[k][i] = g[k][i] = 0.0f;
            if (e < t.n) {
                if (t.flat) {
                    po[k] = go[k] = e;
                    in_row[k] = static_cast<int>(min<int64_t>(kPer, t.n - e));
                } else {   // rem0 + local < cols + kChunk, below 2^32
                    const uint32_t c = static_cast<uint32_t>(t.cols), at_row = static_cast<uint32_t>(rem0) + local;
                    const uint32_t q = at_row / c;
                    col[k] = at_row - q * c;
                    po[k] = (row0 + q) * t.p_stride + col[k];
                    go[k] = (row0 + q) * t.g_stride + col[k];
                    in_row[k] = static_cast<int>(min<uint32_t>(kPer, c - col[k]));
                }
                if (in_row[k] == kPer) {
                    load_global<TP, kPer>(pp + po[k], p[k]);
                    load_global<TG, kPer>(gp + go[k], g[k]);
                } else {
#pragma unroll
                    for (int i = 0; i < kPer; ++i)
                        if (e + i < t.n) {
                            const uint32_t d = rows_on(i, k);
                            p[k][i] = static_cast<float>(((const Global<TP> *)pp)[po[k] + i + d * (t.p_stride - t.cols)]);
                            g[k][i] = static_cast<float>(((const Global<TG> *)gp)[go[k] + i + d * (t.g_stride - t.cols)]);
                        }
                }
            }
        }
        if constexpr (BITS == 32) {
            if (FULL || e < t.n) {   // the moments' places go on to the end of a block
                load_global<float, kPer>(static_cast<const float *>(mv) + at, m[k]);
                load_global<float, kPer>(static_cast<const float *>(vv) + at, v[k]);
            }
        } else {
            mc[k] = vc[k] = 0;
            if (FULL || e < t.n) {
                mc[k] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(mv) + at));
                vc[k] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(vv) + at));
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        const int64_t wave_e = first + (k * kAdamThreads + (static_cast<int>(threadIdx.x) & ~(kWave - 1))) * kPer;
        if (!FULL && wave_e >= t.n) continue;   // the same for the whole wavefront
        const int64_t e = wave_e + lane_id() * kPer, at = t.offset + e;
        const int64_t block = (t.offset + wave_e) / kMomentBlock;
        float r[kPer];
        if constexpr (BITS == 8) {
            decode_m(mc[k], m_scale[block], m[k]);
            const float vs = v_scale[block];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const float x = decode_r((vc[k] >> (8 * i)) & 255u) * vs;
                v[k][i] = x * x;
            }
        }
        float m_max = 0.0f, r_max = 0.0f;
        auto larger = [](float a, float b) {   // of non-negative floats, a NaN above all
            return __builtin_bit_cast(float, max(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)));
        };
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (!FULL && e + i >= t.n) continue;
            update_moments(g[k][i], m[k][i], v[k][i], r[i], s);
            p[k][i] = updated(p[k][i], m[k][i], r[i], keep, s);
            m_max = larger(m_max, fabsf(m[k][i]));
            r_max = larger(r_max, r[i]);
        }
        if constexpr (BITS == 32) {
            if (FULL || e < t.n) {
                store_global<float, kPer>(static_cast<float *>(mv) + at, m[k]);
                store_global<float, kPer>(static_cast<float *>(vv) + at, v[k]);
            }
        } else {
            float ms = wave_max_bits(m_max) * (1.0f / 448.0f), rs = wave_max_bits(r_max) * (16.0f / 31.0f);
            if (ms < 0x1p-126f) ms = 0.0f;   // its inverse would overflow: the block's m is zero
            const float mi = ms > 0.0f ? 1.0f / ms : 0.0f, ri = rs > 0.0f ? 1.0f / rs : 0.0f;
            const uint32_t old_m = mc[k], old_v = vc[k];
            uint32_t new_m = 0, new_v = 0;
            if (!FULL) {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (e + i >= t.n) m[k][i] = r[i] = 0.0f;
            }
            new_m = encode_m(m[k], mi);
#pragma unroll
            for (int i = 0; i < kPer; i += 2) {
                const uint32_t h = mix32(static_cast<uint32_t>(static_cast<uint64_t>(at + i) >> 1) ^ s.key);
                new_v |= encode_r(r[i], ri, h & 0xFFFFu) << (8 * i);
                new_v |= encode_r(r[i + 1], ri, h >> 16) << (8 * (i + 1));
            }
            if (!FULL && e + kPer > t.n) {   // codes past the tensor stay as they are
                const int live = static_cast<int>(max<int64_t>(0, t.n - e));
                const uint32_t mask = live == 0 ? 0u : 0xFFFFFFFFu >> (8 * (kPer - live));
                new_m = (new_m & mask) | (old_m & ~mask);
                new_v = (new_v & mask) | (old_v & ~mask);
            }
            if (FULL || e < t.n) {
                __builtin_nontemporal_store(new_m, reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(mv) + at));
                __builtin_nontemporal_store(new_v, reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(vv) + at));
            }
            if (lane_id() == 0) {
                m_scale[block] = ms;
                v_scale[block] = rs;
            }
        }
        if constexpr (FULL) {
            store_global<TP, kPer>(pp + po[k], p[k]);
        } else if (in_row[k] == kPer) {
            store_global<TP, kPer>(pp + po[k], p[k]);
        } else if (in_row[k] > 0) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (e + i < t.n) {
                    const uint32_t d = rows_on(i, k);
                    ((Global<TP> *)pp)[po[k] + i + d * (t.p_stride - t.cols)] = static_cast<TP>(p[k][i]);
                }
        }
    }
}

template <int BITS>
__global__ __launch_bounds__(kAdamThreads) void k_adamw(const Header *__restrict__ h, int64_t n_chunks, void *mv, void *vv,
                                                        float *m_scale, float *v_scale, Scalars given, int32_t device_scalars) {
    if (h->mark != kMark) return;
    const int64_t n = min(n_chunks, h->n_chunks);
    const Scalars s = device_scalars ? h->scalars : given;
    for (int64_t b = blockIdx.x; b < n; b += gridDim.x) {
        const Place at = h->places[b];
        const Entry t = h->entries[at.tensor];
        const int64_t first = static_cast<int64_t>(at.chunk) * kChunk;
        const bool full = first + kChunk <= t.n;
        auto with = [&](auto p0, auto g0) {
            using TP = decltype(p0);
            using TG = decltype(g0);
            if (full && t.flat)
                chunk_update<TP, TG, BITS, kPacked>(t, first, mv, vv, m_scale, v_scale, s);
            else if (full && t.cols % kPer == 0)
                chunk_update<TP, TG, BITS, kRows>(t, first, mv, vv, m_scale, v_scale, s);
            else
                chunk_update<TP, TG, BITS, kAny>(t, first, mv, vv, m_scale, v_scale, s);
        };
        auto with_grad = [&](auto p0) {
            if (t.g_type == W2V_F32)
                with(p0, float{});
            else if (t.g_type == W2V_BF16)
                with(p0, static_cast<__bf16>(0.0f));
            else
                with(p0, static_cast<_Float16>(0.0f));
        };
        if (t.p_type == W2V_F32)
            with_grad(float{});
        else if (t.p_type == W2V_BF16)
            with_grad(static_cast<__bf16>(0.0f));
        else
            with_grad(static_cast<_Float16>(0.0f));
    }
}

// The values that 8-bit moments stand for.
__global__ __launch_bounds__(kAdamThreads) void k_moments(const uint32_t *__restrict__ mc, const uint32_t *__restrict__ vc,
                                                          const float *__restrict__ m_scale,
                                                          const float *__restrict__ v_scale, int64_t blocks,
                                                          float *__restrict__ m_out, float *__restrict__ v_out) {
    const int64_t step = static_cast<int64_t>(gridDim.x) * (kAdamThreads / kWave);
    for (int64_t b = static_cast<int64_t>(blockIdx.x) * (kAdamThreads / kWave) + threadIdx.x / kWave; b < blocks; b += step) {
        const int64_t w = b * kWave + lane_id();
        float m[kPer], v[kPer];
        decode_m(mc[w], m_scale[b], m);
        const uint32_t c = vc[w];
        const float vs = v_scale[b];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const float x = decode_r((c >> (8 * i)) & 255u) * vs;
            v[i] = x * x;
        }
        store_global<float, kPer>(m_out + w * kPer, m);
        store_global<float, kPer>(v_out + w * kPer, v);
    }
}

}  // namespace

int64_t adamw_chunks(const w2v_adamw_tensor *t, int32_t n) {
    int64_t c = 0;
    for (int32_t i = 0; i < n; ++i) c += ceil_div(t[i].rows * t[i].cols, kChunk);
    return c;
}

size_t adamw_plan_bytes(const w2v_adamw_tensor *t, int32_t n) {
    Carve c;
    c.take<char>(kHeaderBytes);
    c.take<Entry>(static_cast<size_t>(n));
    c.take<Place>(static_cast<size_t>(adamw_chunks(t, n)));
    return c.used();
}

int run_adamw_plan(const w2v_adamw_tensor *t, int32_t n, void *plan, hipStream_t s) {
    Carve c(plan);
    const int64_t chunks = adamw_chunks(t, n);
    void *at = c.take<char>(kHeaderBytes);
    Entry *entries = c.take<Entry>(static_cast<size_t>(n));
    Place *places = c.take<Place>(static_cast<size_t>(chunks));
    Header h{};
    h.mark = kMark;
    h.n_chunks = chunks;
    h.entries = entries;
    h.places = places;
    std::vector<Entry> e(static_cast<size_t>(n));
    std::vector<Place> p;
    p.reserve(static_cast<size_t>(chunks));
    for (int32_t i = 0; i < n; ++i) {
        const w2v_adamw_tensor &x = t[i];
        const int64_t count = x.rows * x.cols;
        const bool flat = x.rows <= 1 || (x.param_stride == x.cols && x.grad_stride == x.cols);
        e[static_cast<size_t>(i)] = Entry{x.param, x.grad, count, x.cols, x.param_stride, x.grad_stride, x.moment_offset,
                                          x.weight_decay, x.param_type, x.grad_type, flat ? 1 : 0};
        for (int64_t k = 0; k < ceil_div(count, kChunk); ++k) p.push_back(Place{i, static_cast<int32_t>(k)});
    }
    W2V_HIP(hipMemcpyAsync(at, &h, sizeof(h), hipMemcpyHostToDevice, s));
    W2V_HIP(hipMemcpyAsync(entries, e.data(), e.size() * sizeof(Entry), hipMemcpyHostToDevice, s));
    if (!p.empty()) W2V_HIP(hipMemcpyAsync(places, p.data(), p.size() * sizeof(Place), hipMemcpyHostToDevice, s));
    W2V_HIP(hipStreamSynchronize(s));   // the host copies end here
    return W2V_OK;
}

int run_adamw_step(void *plan, int64_t n_chunks, int32_t bits, void *m, void *v, float *m_scale, float *v_scale,
                   const w2v_adamw_params &p, hipStream_t s) {
    if (n_chunks == 0) return W2V_OK;
    Header *h = static_cast<Header *>(plan);
    const int32_t device_scalars = p.lr_device || p.step_device ? 1 : 0;
    Scalars given{};
    if (device_scalars) {
        k_adamw_scalars<<<1, 1, 0, s>>>(h, p);
        W2V_LAUNCH_CHECK("k_adamw_scalars");
    } else {
        given = make_scalars(p, p.lr, p.step);
    }
    const auto grid = static_cast<unsigned>(std::min<int64_t>(n_chunks, kMaxGroups));
    if (bits == 32)
        k_adamw<32><<<grid, kAdamThreads, 0, s>>>(h, n_chunks, m, v, m_scale, v_scale, given, device_scalars);
    else
        k_adamw<8><<<grid, kAdamThreads, 0, s>>>(h, n_chunks, m, v, m_scale, v_scale, given, device_scalars);
    W2V_LAUNCH_CHECK("k_adamw");
    return W2V_OK;
}

int run_adamw_moments(const void *m, const void *v, const float *m_scale, const float *v_scale, int64_t n, float *m_out,
                      float *v_out, hipStream_t s) {
    const int64_t blocks = n / kMomentBlock;
    if (blocks == 0) return W2V_OK;
    const auto grid = static_cast<unsigned>(std::min<int64_t>(ceil_div(blocks, kAdamThreads / kWave), kMaxGroups));
    k_moments<<<grid, kAdamThreads, 0, s>>>(static_cast<const uint32_t *>(m), static_cast<const uint32_t *>(v), m_scale,
                                           v_scale, blocks, m_out, v_out);
    W2V_LAUNCH_CHECK("k_moments");
    return W2V_OK;
}

}  // namespace w2v
