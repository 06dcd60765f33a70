// What ends a training step: the norm of all gradients, and AdamW over a list of tensors (formulas in include/moe.h).
//
//   grad_norm_partial_kernel  sums of squares, in 64 bits, of runs of 16 KiB
//   grad_norm_finish_kernel   the norm and the factor that clips it
//   adamw_kernel              the step, a piece of 512 (fp32 states) or 2048 elements (8-bit) to a workgroup
//
// A launch takes a list of tensors, described in its arguments; every tensor is cut into pieces, and a workgroup finds its
// tensor from the first pieces.  All are bound by memory, read and written once and streamed past the caches.
//
// Measured: norm of 1.11G bf16 gradients 322 us (6.9 TB/s).  AdamW of 1.11G weights with fp32 masters and states and bf16
// gradients, 28 bytes each: 4.91 ms (6.3 TB/s; with as many waves as there is room for, in workgroups of four, 5.67, and through
// the caches 5.9).  1.41G bf16 weights with 8-bit states, 10.1 bytes each: 2.40 ms (5.9 TB/s; two pieces to a workgroup 2.6; four
// elements to a lane, rounding in plain operations 3.9).  60 fp32 tensors of 400 thousand elements in all 6 us.
#include <string.h>

#include <type_traits>

#include "wave_sum.h"

namespace moe {

namespace {

constexpr int kBlock = 32;         // elements that share a scale
constexpr int64_t kLaunchPieces = (1 << 24) - 1;   // of up to 256 threads: a grid has less than 2^32 of them

// -------------------------------------------------------------------------------------------------------------
// lists

// A gradient's bytes are cut into runs; the tensors of a launch have at most 192 pointers, lengths and first runs in 4 KiB.
constexpr int kGradTensors = 192;
constexpr int kRunBytes = 256 * 16 * 4;   // four 16-byte loads of every thread

struct GradList {
    const void* grad[kGradTensors];
    uint64_t n[kGradTensors];        // elements; bit 63: bf16
    int32_t first[kGradTensors];     // first run
    int32_t count, runs;
};

__device__ __forceinline__ int find_tensor(const GradList& l, int run) {
    int lo = 0, hi = l.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= run) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ float load_value(const void* p, bool bf16, int64_t i) {
    return bf16 ? bf16_to_f32(static_cast<const bf16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

// -------------------------------------------------------------------------------------------------------------
// norm

constexpr int kNormGroups = 1024;   // workgroups, and partial sums, of a launch at most

// Sum over the workgroup's four waves, in its first wave.
__device__ __forceinline__ double group_sum(double v, double* red) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// Sum of the squares of 16 bytes of values.  In 64 bits: a square of an fp32 number neither overflows nor vanishes, and the
// additions stay far below the rate at which memory delivers.
template <bool BF16>
__device__ __forceinline__ double square_sum(const u32x4& r) {
    double a = 0., b = 0.;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (BF16) {
            const double lo = __uint_as_float(r[j] << 16), hi = __uint_as_float(r[j] & 0xffff0000u);
            a = fma(lo, lo, a);
            b = fma(hi, hi, b);
        } else {
            const double x = __uint_as_float(r[j]);
            if (j & 1) b = fma(x, x, b);
            else a = fma(x, x, a);
        }
    }
    return a + b;
}

template <bool BF16>
__device__ __forceinline__ double run_square_sum(const void* grad, uint64_t n, uint64_t run) {
    constexpr int kVec = BF16 ? 8 : 4;                     // elements of a load
    constexpr int kElements = kRunBytes / (BF16 ? 2 : 4);
    const uint64_t at = run * kElements;
    if (at + kElements <= n) {
        const u32x4* p = reinterpret_cast<const u32x4*>(grad) + at / kVec + threadIdx.x;
        u32x4 r[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) r[u] = __builtin_nontemporal_load(p + u * 256);
        double acc = 0.;
#pragma unroll
        for (int u = 0; u < 4; ++u) acc += square_sum<BF16>(r[u]);
        return acc;
    }
    double acc = 0.;
    for (uint64_t j = at + threadIdx.x; j < n; j += 256) {
        const double g = load_value(grad, BF16, (int64_t)j);
        acc = fma(g, g, acc);
    }
    return acc;
}

// Workgroup g takes the runs [g runs / G, (g + 1) runs / G): the order of the sums depends on the sizes alone.
__global__ __launch_bounds__(256) void grad_norm_partial_kernel(GradList l, double* __restrict__ partial) {
    __shared__ double red[4];
    const int from = (int)((int64_t)l.runs * blockIdx.x / gridDim.x), to = (int)((int64_t)l.runs * (blockIdx.x + 1) / gridDim.x);
    double acc = 0.;
    int i = find_tensor(l, from);
    for (int run = from; run < to; ++run) {
        while (i + 1 < l.count && l.first[i + 1] <= run) ++i;
        const uint64_t n = l.n[i];
        acc += n >> 63 ? run_square_sum<true>(l.grad[i], n & ~(1ull << 63), run - l.first[i])
                       : run_square_sum<false>(l.grad[i], n, run - l.first[i]);
    }
    acc = group_sum(acc, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = acc;
}

__global__ __launch_bounds__(256) void grad_norm_finish_kernel(const double* __restrict__ partial, int parts, float max_norm,
                                                               float multiplier, float* __restrict__ out) {
    __shared__ double red[4];
    double acc = 0.;
    for (int i = threadIdx.x; i < parts; i += 256) acc += partial[i];
    acc = group_sum(acc, red);
    if (threadIdx.x == 0) {
        const float norm = (float)(fabs((double)multiplier) * sqrt(acc));
        float scale = multiplier;
        if (max_norm > 0.f) scale *= fminf(1.f, max_norm / (norm + 1e-6f));
        out[0] = norm;
        out[1] = norm < INFINITY ? scale : NAN;
    }
}

// -------------------------------------------------------------------------------------------------------------
// AdamW

// A tensor in a launch's arguments, which are limited to 4 KiB: six words of 64 bits and up to three more where its types need
// them, so that a launch takes 70 tensors in fp32, 60 in bf16 with masters, 46 of those with 8-bit states.
//   n | kind << 34 | place in the caller's list << 37;  1 - lr wd, lr / (1 - beta1^t);  grad;  what is stepped (param or
//   master);  m;  v;  [scales of m; of v];  [param, where there is a master]
constexpr int kAdamTensors = 70, kAdamWords = 420, kWordsMost = 9;

struct AdamList {
    // pointers, so that they are known to point to device memory; as many as the longest tensor has are read of each
    void* word[kAdamWords + kWordsMost - 6];
    struct {
        int32_t first, at;                        // first piece, first word
    } tensor[kAdamTensors];
    int32_t count;
};

// How a launch is shaped, by its tensors' states.  With fp32 states fewer waves are better, once enough is in flight: the launch
// asks for a share of the LDS, which it does not use, so that a compute unit holds six or eight workgroups of two waves.  TB/s
// with 5, 6, 7, 8 and 10 of them, and with as many as there is room for (400M weights; of type / gradient's): fp32 / fp32 6.08,
// 6.09, 6.10, 6.12, 6.07, 5.88; fp32 / bf16 6.19, 6.20, 6.36, 6.37, 6.41, 6.15; masters / fp32 6.25, 6.25, 6.18, 6.17, 6.13, 6.02;
// masters / bf16 6.26, 6.24, 6.23, 6.21, 6.13, 5.76; bf16 / fp32 5.93, 5.96, 6.33, 6.36, 6.31, 6.00; bf16 / bf16 5.66, 5.67, 6.26,
// 6.22, 6.21, 5.94.  Four waves to a workgroup lose 6 %.  The arithmetic of 8-bit states needs all waves.
template <bool MXFP8>
struct Shape {
    static constexpr int V = MXFP8 ? 8 : 4;               // elements of a lane
    static constexpr int kThreads = MXFP8 ? 256 : 128;
    static constexpr int kPiece = V * kThreads;           // elements of a workgroup; a multiple of the 8-bit states' blocks
    // bytes of LDS to a workgroup, where most elements have masters and where not
    static int lds(bool masters) { return MXFP8 ? 0 : masters ? 27000 : 20000; }
};

struct AdamTensor {
    const void* grad;
    void* stepped;
    void* m;
    void* v;
    void* copy;                // the bf16 weights beside a master
    uint8_t* m_scale;
    uint8_t* v_scale;
    int64_t n;
    float decay, step_size;
    int index;
};

struct AdamStep {
    float beta1, one_minus_beta1, beta2, one_minus_beta2, eps, rsqrt_bc2;
    uint32_t seed;
    const float* grad_scale;
};

// a mixing function published by C. Wellons, "Prospecting for Hash Functions" (2018)
__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x7feb352du;
    x ^= x >> 15;
    x *= 0x846ca68bu;
    return x ^ (x >> 16);
}

__device__ __forceinline__ uint32_t random_bits(uint32_t seed, int tensor, int64_t j) {
    const uint32_t key = mix(seed + 0x9e3779b9u * (uint32_t)(tensor + 1) + 0x85ebca6bu * (uint32_t)(j >> 32));
    return mix((uint32_t)j ^ key);
}

// value of an E8M0 scale, and the scale byte of a block whose largest magnitude has these bits: the smallest power of two
// that leaves at most 448 = 1.75 * 2^8, so the exponent goes up where the mantissa is above 1.75
__device__ __forceinline__ float scale_value(uint32_t byte) {
    const uint32_t bits = byte == 255 ? 0x7fc00000u : byte == 0 ? 0x00400000u : byte << 23;
    return __uint_as_float(bits);
}
__device__ __forceinline__ uint32_t scale_of(uint32_t top) {
    if (top >= 0x7f800000u) return 255;
    return (uint32_t)max((int)((top + 0x1fffffu) >> 23) - 8, 1);
}

// V consecutive values of a lane as they lie in memory: words of 32 bits.  `left` of them exist; in a whole piece of a
// tensor all do, and the access is as wide as it can be.
template <int V, typename T>
struct Packed {
    static constexpr int kWords = V * sizeof(T) / 4, kPer = 4 / sizeof(T), kBits = 8 * sizeof(T);
    typedef __attribute__((ext_vector_type(kWords < 4 ? kWords : 4))) uint32_t access_t;
    static constexpr int kAccess = sizeof(access_t) / 4;
    uint32_t w[kWords];

    __device__ __forceinline__ void load(const void* base, int64_t j) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(static_cast<const T*>(base) + j);
#pragma unroll
        for (int q = 0; q < kWords; q += kAccess) {
            const access_t r = __builtin_nontemporal_load(reinterpret_cast<const access_t*>(p + q));
#pragma unroll
            for (int u = 0; u < kAccess; ++u) w[q + u] = r[u];
        }
    }
    __device__ __forceinline__ void load_some(const void* base, int64_t j, int left) {
        const T* p = static_cast<const T*>(base) + j;
#pragma unroll
        for (int q = 0; q < kWords; ++q) w[q] = 0;
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (u < left) w[u / kPer] |= (uint32_t)p[u] << (kBits * (u % kPer));
    }
    __device__ __forceinline__ void store(void* base, int64_t j) const {
        uint32_t* p = reinterpret_cast<uint32_t*>(static_cast<T*>(base) + j);
#pragma unroll
        for (int q = 0; q < kWords; q += kAccess) {
            access_t r;
#pragma unroll
            for (int u = 0; u < kAccess; ++u) r[u] = w[q + u];
            __builtin_nontemporal_store(r, reinterpret_cast<access_t*>(p + q));
        }
    }
    __device__ __forceinline__ void store_some(void* base, int64_t j, int left) const {
        T* p = static_cast<T*>(base) + j;
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (u < left) p[u] = (T)(w[u / kPer] >> (kBits * (u % kPer)));
    }
    // values of fp32 or bf16 words
    __device__ __forceinline__ void values(float (&x)[V]) const {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            if (sizeof(T) == 4) x[u] = __uint_as_float(w[u]);
            else x[u] = __uint_as_float(u & 1 ? w[u / 2] & 0xffff0000u : w[u / 2] << 16);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[V]) {
#pragma unroll
        for (int u = 0; u < V; ++u) w[u] = __float_as_uint(x[u]);
    }
};

enum { kParamF32, kParamMaster, kParamBf16 };

// The largest of the four neighbouring lanes that hold a block of 32 elements.
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));          // quad_perm 1, 0, 3, 2
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));       // quad_perm 2, 3, 0, 1
}

// E4M3 codes and scale of a lane's eight values.  The conversion instruction adds the upper 20 bits of its random number
// below the last bit that is kept, in the denormal range too, and truncates: the rounding the interface defines, with 16
// random bits in the middle of their step.  UPPER: which half of a value's 32 bits is its random number; those of the
// second moment, which also stays above zero where it is (2^-9 is the smallest code).
template <bool UPPER>
__device__ __forceinline__ void quantize(const float (&x)[8], const uint32_t (&bits)[8], uint32_t (&codes)[2], uint32_t& scale) {
    uint32_t top = 0;   // as bits, which order NaN above all; the second moment has no sign but a NaN's
#pragma unroll
    for (int u = 0; u < 8; ++u) top = max(top, UPPER ? __float_as_uint(x[u]) : __float_as_uint(x[u]) & 0x7fffffffu);
    scale = scale_of(block_max(top));
    const float inverse = __uint_as_float((254 - (int)scale) << 23);
    float y[8];
    uint32_t r[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        y[u] = x[u] * inverse;
        if (UPPER) y[u] = fmaxf(y[u], x[u] > 0.f ? 0x1p-9f : 0.f);
        r[u] = (UPPER ? bits[u] & 0xffff0000u : bits[u] << 16) | 0x8000u;
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        int c = 0;
        c = __builtin_amdgcn_cvt_sr_fp8_f32(y[4 * q], r[4 * q], c, 0);
        c = __builtin_amdgcn_cvt_sr_fp8_f32(y[4 * q + 1], r[4 * q + 1], c, 1);
        c = __builtin_amdgcn_cvt_sr_fp8_f32(y[4 * q + 2], r[4 * q + 2], c, 2);
        c = __builtin_amdgcn_cvt_sr_fp8_f32(y[4 * q + 3], r[4 * q + 3], c, 3);
        codes[q] = scale == 255 ? 0x7f7f7f7fu : (uint32_t)c;
    }
}

__device__ __forceinline__ void dequantize(const uint32_t (&codes)[2], float scale, float (&x)[8]) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        x[4 * q] = __builtin_amdgcn_cvt_f32_fp8((int)codes[q], 0) * scale;
        x[4 * q + 1] = __builtin_amdgcn_cvt_f32_fp8((int)codes[q], 1) * scale;
        x[4 * q + 2] = __builtin_amdgcn_cvt_f32_fp8((int)codes[q], 2) * scale;
        x[4 * q + 3] = __builtin_amdgcn_cvt_f32_fp8((int)codes[q], 3) * scale;
    }
}

// What a lane reads of its V elements: four with fp32 states, so that every access of a wave is one run of memory; eight
// with 8-bit ones, where the work on a block is shared by fewer lanes.
template <int PARAM, bool GRAD_BF16, bool MXFP8>
struct AdamInput {
    static constexpr int V = Shape<MXFP8>::V;
    typedef typename std::conditional<GRAD_BF16, bf16_t, uint32_t>::type grad_t;
    typedef typename std::conditional<PARAM == kParamBf16, bf16_t, uint32_t>::type param_t;   // what is stepped
    typedef typename std::conditional<MXFP8, uint8_t, uint32_t>::type state_t;
    Packed<V, grad_t> g;
    Packed<V, param_t> p;
    Packed<V, state_t> m, v;
    uint32_t m_scale, v_scale;

    __device__ __forceinline__ void load(const AdamTensor& t, int64_t j, bool whole, int left) {
        if (whole) {
            g.load(t.grad, j);
            p.load(t.stepped, j);
            m.load(t.m, j);
            v.load(t.v, j);
        } else {
            g.load_some(t.grad, j, left);
            p.load_some(t.stepped, j, left);
            m.load_some(t.m, j, left);
            v.load_some(t.v, j, left);
        }
        if constexpr (MXFP8) {
            const int64_t block = min(j, t.n - 1) / kBlock;
            m_scale = t.m_scale[block];
            v_scale = t.v_scale[block];
        }
    }
};

// One piece of a tensor.
template <int PARAM, bool GRAD_BF16, bool MXFP8>
__device__ __forceinline__ void adamw_piece(const AdamTensor& t, const AdamStep& h, float scale, int64_t piece) {
#pragma clang fp contract(off)
    typedef AdamInput<PARAM, GRAD_BF16, MXFP8> Input;
    constexpr int V = Input::V;
    const int64_t base = piece * Shape<MXFP8>::kPiece, j = base + V * threadIdx.x;
    const bool whole = base + Shape<MXFP8>::kPiece <= t.n;
    const int left = (int)min((int64_t)V, t.n - j);   // none or negative: this lane has nothing
    Input cur;
    cur.load(t, j, whole, left);
    if (scale != scale) return;   // here, where what is read is on its way
    float p[V], g[V], m[V], v[V];
    cur.g.values(g);
    cur.p.values(p);
    if constexpr (MXFP8) {
        dequantize(cur.m.w, scale_value(cur.m_scale), m);
        dequantize(cur.v.w, scale_value(cur.v_scale), v);
    } else {
        cur.m.values(m);
        cur.v.values(v);
    }
    uint32_t bits[V];
    if (MXFP8 || PARAM == kParamBf16) {
#pragma unroll
        for (int u = 0; u < V; ++u) bits[u] = random_bits(h.seed, t.index, j + u);
    }
#pragma unroll
    for (int u = 0; u < V; ++u) {
        g[u] *= scale;
        m[u] = m[u] * h.beta1 + g[u] * h.one_minus_beta1;
        v[u] = v[u] * h.beta2 + (g[u] * g[u]) * h.one_minus_beta2;
        if constexpr (MXFP8) {
            // the instructions' own square root and reciprocal, each within a unit of fp32: some 45 instructions an element
            // are nearly as long as its 10 to 16 bytes take
            const float denom = fmaf(__builtin_amdgcn_sqrtf(v[u]), h.rsqrt_bc2, h.eps);
            p[u] = fmaf(-t.step_size * m[u], __builtin_amdgcn_rcpf(denom), p[u] * t.decay);
        } else {
            const float denom = sqrtf(v[u]) * h.rsqrt_bc2 + h.eps;
            p[u] = p[u] * t.decay - (m[u] / denom) * t.step_size;
        }
    }
    // new weights and states as they go to memory
    Packed<V, uint32_t> p32;
    Packed<V, bf16_t> p16;
    Packed<V, typename Input::state_t> pm, pv;
    if (PARAM != kParamBf16) p32.set(p);
    if constexpr (PARAM == kParamMaster) {
#pragma unroll
        for (int q = 0; q < V / 2; ++q) p16.w[q] = pack2_bf16(p[2 * q], p[2 * q + 1]);
    }
    if constexpr (PARAM == kParamBf16) {
#pragma unroll
        for (int q = 0; q < V / 2; ++q) {
            uint32_t x[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                // 16 random bits below the last kept one; infinities stay what they are, a NaN might carry over
                const float x32 = p[2 * q + u];
                x[u] = x32 != x32 ? 0x7fc00000u : __float_as_uint(x32) + ((bits[2 * q + u] * 0x9e3779b1u) >> 16);
            }
            p16.w[q] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302);   // the upper halves
        }
    }
    uint32_t sm, sv;
    if constexpr (MXFP8) {
        if (!whole) {
#pragma unroll
            for (int u = 0; u < V; ++u) {
                m[u] = u < left ? m[u] : 0.f;   // what lies past the end has no part in the scale
                v[u] = u < left ? v[u] : 0.f;
            }
        }
        quantize<false>(m, bits, pm.w, sm);
        quantize<true>(v, bits, pv.w, sv);
    } else {
        pm.set(m);
        pv.set(v);
    }
    if (whole) {
        if (PARAM != kParamBf16) p32.store(t.stepped, j);
        if (PARAM != kParamF32) p16.store(PARAM == kParamMaster ? t.copy : t.stepped, j);
        pm.store(t.m, j);
        pv.store(t.v, j);
    } else {
        if (PARAM != kParamBf16) p32.store_some(t.stepped, j, left);
        if (PARAM != kParamF32) p16.store_some(PARAM == kParamMaster ? t.copy : t.stepped, j, left);
        pm.store_some(t.m, j, left);
        pv.store_some(t.v, j, left);
    }
    if constexpr (MXFP8) {
        if (threadIdx.x % 4 == 0 && left > 0) {
            t.m_scale[j / kBlock] = (uint8_t)sm;
            t.v_scale[j / kBlock] = (uint8_t)sv;
        }
    }
}

template <bool MXFP8>
__global__ __launch_bounds__(Shape<MXFP8>::kThreads) void adamw_kernel(AdamList l, AdamStep h) {
    const float scale = h.grad_scale ? *h.grad_scale : 1.f;
    int lo = 0, hi = l.count, first = 0, at = 0;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        const auto m = l.tensor[mid];
        if (m.first <= (int)blockIdx.x) {
            lo = mid;
            first = m.first;
            at = m.at;
        } else {
            hi = mid;
        }
    }
    const int64_t piece = (int)blockIdx.x - first;
    void* w[kWordsMost];
#pragma unroll
    for (int k = 0; k < kWordsMost; ++k) w[k] = l.word[at + k];
    const uint64_t size = reinterpret_cast<uint64_t>(w[0]), rates = reinterpret_cast<uint64_t>(w[1]);
    const AdamTensor t = {w[2], w[3], w[4], w[5], MXFP8 ? w[8] : w[6], static_cast<uint8_t*>(w[6]), static_cast<uint8_t*>(w[7]),
                          (int64_t)(size & ((1ull << 34) - 1)), __uint_as_float((uint32_t)rates),
                          __uint_as_float((uint32_t)(rates >> 32)), (int)(size >> 37)};
    switch ((int)(size >> 34) & 7) {
        case 0: return adamw_piece<kParamF32, false, MXFP8>(t, h, scale, piece);
        case 1: return adamw_piece<kParamF32, true, MXFP8>(t, h, scale, piece);
        case 2: return adamw_piece<kParamMaster, false, MXFP8>(t, h, scale, piece);
        case 3: return adamw_piece<kParamMaster, true, MXFP8>(t, h, scale, piece);
        case 4: return adamw_piece<kParamBf16, false, MXFP8>(t, h, scale, piece);
        default: return adamw_piece<kParamBf16, true, MXFP8>(t, h, scale, piece);
    }
}

// place of a tensor's types in the switch above
inline int kind_of(const moe_adamw_tensor_t& t) {
    const int param = t.param_dt == MOE_F32 ? kParamF32 : t.master ? kParamMaster : kParamBf16;
    return 2 * param + (t.grad_dt == MOE_BF16 ? 1 : 0);
}

// The tensors of one kind of states, in as few launches as hold them.
template <bool MXFP8>
void launch_adamw_states(const moe_adamw_tensor_t* tensors, int count, double lr, double bc1, const AdamStep& h, hipStream_t s) {
    AdamList l;
    int64_t pieces = 0, all = 0, mastered = 0;
    int words = 0;
    l.count = 0;
    auto flush = [&] {
        if (pieces)
            hipLaunchKernelGGL(adamw_kernel<MXFP8>, dim3((unsigned)pieces), dim3(Shape<MXFP8>::kThreads),
                               Shape<MXFP8>::lds(2 * mastered > all), s, l, h);
        l.count = words = 0;
        pieces = all = mastered = 0;
    };
    auto put = [&](const void* p) { l.word[words++] = const_cast<void*>(p); };
    auto put_bits = [&](uint64_t b) { l.word[words++] = reinterpret_cast<void*>(b); };
    auto bits = [](float f) {
        uint32_t u;
        memcpy(&u, &f, sizeof u);
        return (uint64_t)u;
    };
    for (int i = 0; i < count; ++i) {
        const moe_adamw_tensor_t& t = tensors[i];
        if (t.n == 0 || (t.state == MOE_STATE_MXFP8) != MXFP8) continue;
        const int64_t more = (t.n + Shape<MXFP8>::kPiece - 1) / Shape<MXFP8>::kPiece;
        if (l.count == kAdamTensors || words + 6 + (t.master ? 1 : 0) + (MXFP8 ? 2 : 0) > kAdamWords || pieces + more > kLaunchPieces)
            flush();
        const AdamRates rates = adam_rates(t, lr, bc1);
        l.tensor[l.count].first = (int32_t)pieces;
        l.tensor[l.count++].at = words;
        put_bits((uint64_t)t.n | (uint64_t)kind_of(t) << 34 | (uint64_t)i << 37);
        put_bits(bits(rates.decay) | bits(rates.step_size) << 32);
        put(t.grad);
        put(t.master ? t.master : t.param);
        put(t.exp_avg);
        put(t.exp_avg_sq);
        if (MXFP8) {
            put(t.exp_avg_scale);
            put(t.exp_avg_sq_scale);
        }
        if (t.master) put(t.param);
        pieces += more;
        all += t.n;
        if (t.master) mastered += t.n;
    }
    flush();
}

}  // namespace

size_t grad_norm_workspace_bytes(int count) {
    const size_t launches = ((size_t)count + kGradTensors - 1) / kGradTensors;
    return (launches > 0 ? launches : 1) * kNormGroups * sizeof(double);
}

void launch_grad_norm(const moe_grad_tensor_t* tensors, int count, float max_norm, float multiplier, float* out, void* ws,
                      hipStream_t s) {
    double* partial = static_cast<double*>(ws);
    int parts = 0;
    GradList l;
    int64_t runs = 0;
    l.count = 0;
    auto flush = [&] {
        if (l.count == 0) return;
        l.runs = (int32_t)runs;
        const int groups = (int)(runs < kNormGroups ? runs : kNormGroups);
        hipLaunchKernelGGL(grad_norm_partial_kernel, dim3(groups), dim3(256), 0, s, l, partial + parts);
        parts += groups;
        l.count = 0;
        runs = 0;
    };
    for (int i = 0; i < count; ++i) {
        const bool bf16 = tensors[i].dt == MOE_BF16;
        const int64_t more = (tensors[i].n * (bf16 ? 2 : 4) + kRunBytes - 1) / kRunBytes;
        if (more == 0) continue;
        if (l.count == kGradTensors) flush();   // 192 tensors of 2^33 elements at most: under 2^29 runs
        l.grad[l.count] = tensors[i].grad;
        l.n[l.count] = (uint64_t)tensors[i].n | (bf16 ? 1ull << 63 : 0);
        l.first[l.count++] = (int32_t)runs;
        runs += more;
    }
    flush();
    hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(256), 0, s, partial, parts, max_norm, multiplier, out);
}

void launch_adamw(const moe_adamw_tensor_t* tensors, int count, double lr, double beta1, double beta2, double eps,
                  int64_t step, uint32_t seed, const float* grad_scale, hipStream_t s) {
    const double bc1 = 1. - pow(beta1, (double)step), bc2 = 1. - pow(beta2, (double)step);
    const AdamStep h = {(float)beta1, (float)(1. - beta1), (float)beta2, (float)(1. - beta2), (float)eps,
                        (float)(1. / sqrt(bc2)), seed, grad_scale};
    launch_adamw_states<false>(tensors, count, lr, bc1, h, s);
    launch_adamw_states<true>(tensors, count, lr, bc1, h, s);
}

}  // namespace moe
