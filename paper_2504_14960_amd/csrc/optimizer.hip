// What ends a training step: the norm of all gradients, and AdamW over a list of tensors (formulas in include/moe.h).
//
// A launch takes up to kListTensors tensors, described in its arguments; every tensor is cut into chunks of kChunk
// elements, and a workgroup finds its tensor from the first chunks.  Both are bound by memory.
#include "common.h"

namespace moe {

namespace {

constexpr int kListTensors = 48;   // 80 bytes each: a launch's arguments are limited to 4 KiB
constexpr int kChunk = 2048;       // elements of a workgroup; a multiple of the 8-bit states' blocks
constexpr int kBlock = 32;         // elements that share a scale
constexpr int64_t kLaunchChunks = (1 << 24) - 1;   // 256 threads each: a grid has less than 2^32 threads

// -------------------------------------------------------------------------------------------------------------
// lists

struct GradList {
    const void* grad[kListTensors];
    int64_t n[kListTensors];
    int32_t first[kListTensors];   // first chunk
    uint8_t bf16[kListTensors];
    int32_t count, chunks;
};

template <typename List>
__device__ __forceinline__ int find_tensor(const List& l, int chunk) {
    int lo = 0, hi = l.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= chunk) lo = mid;
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

__device__ __forceinline__ double group_sum(double v, double* red) {
    red[threadIdx.x] = v;
    __syncthreads();
    for (int d = 128; d > 0; d >>= 1) {
        if (threadIdx.x < d) red[threadIdx.x] += red[threadIdx.x + d];
        __syncthreads();
    }
    return red[0];
}

__global__ __launch_bounds__(256) void grad_norm_partial_kernel(GradList l, double* __restrict__ partial) {
    __shared__ double red[256];
    double acc = 0.;
    for (int chunk = blockIdx.x; chunk < l.chunks; chunk += gridDim.x) {
        const int i = find_tensor(l, chunk);
        const int64_t at = (int64_t)(chunk - l.first[i]) * kChunk;
        for (int64_t j = at + threadIdx.x; j < min(at + kChunk, l.n[i]); j += 256) {
            const double g = load_value(l.grad[i], l.bf16[i], j);
            acc += g * g;
        }
    }
    acc = group_sum(acc, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = acc;
}

__global__ __launch_bounds__(256) void grad_norm_finish_kernel(const double* __restrict__ partial, int parts, float max_norm,
                                                               float multiplier, float* __restrict__ out) {
    __shared__ double red[256];
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

struct AdamTensor {
    void* param;
    float* master;
    const void* grad;
    void* m;
    void* v;
    uint8_t* m_scale;
    uint8_t* v_scale;
    int64_t n;
    float decay, step_size;   // 1 - lr wd, lr / (1 - beta1^t)
    int32_t index;            // place in the caller's list
    uint8_t param_bf16, grad_bf16, mxfp8;
};

struct AdamList {
    AdamTensor t[kListTensors];
    int32_t first[kListTensors];
    int32_t count;
};

struct AdamStep {
    float beta1, one_minus_beta1, beta2, one_minus_beta2, eps, rsqrt_bc2;
    uint32_t seed;
    const float* grad_scale;
};

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

__device__ __forceinline__ float from_e4m3(uint32_t code) { return __builtin_amdgcn_cvt_f32_fp8((int)code, 0); }

// magnitude of an E4M3 code, |x| <= 448, rounded up with the probability of the part cut off: 16 random bits in the middle
// of their step are added below the last kept bit
__device__ __forceinline__ uint32_t to_e4m3(float magnitude, uint32_t random16) {
    const uint32_t r = (random16 << 4) | 8u;
    if (magnitude >= 0x1p-6f) return ((__float_as_uint(magnitude) + r) >> 20) - (120u << 3);
    return ((uint32_t)(magnitude * 0x1p29f) + r) >> 20;   // steps of 2^-9
}

__global__ __launch_bounds__(256) void adamw_kernel(AdamList l, AdamStep h) {
#pragma clang fp contract(off)
    const float scale = h.grad_scale ? *h.grad_scale : 1.f;
    if (scale != scale) return;
    const int i = find_tensor(l, blockIdx.x);
    const AdamTensor& t = l.t[i];
    const int64_t at = (int64_t)((int)blockIdx.x - l.first[i]) * kChunk;
    for (int64_t j = at + threadIdx.x; j - (int)threadIdx.x < min(at + kChunk, t.n); j += 256) {
        const bool ok = j < t.n;
        const int64_t k = ok ? j : t.n - 1;
        const int64_t block = k / kBlock;
        const float g = load_value(t.grad, t.grad_bf16, k) * scale;
        float p = t.master ? t.master[k] : load_value(t.param, t.param_bf16, k);
        float m, v;
        if (t.mxfp8) {
            m = from_e4m3(static_cast<uint8_t*>(t.m)[k]) * scale_value(t.m_scale[block]);
            v = from_e4m3(static_cast<uint8_t*>(t.v)[k]) * scale_value(t.v_scale[block]);
        } else {
            m = static_cast<float*>(t.m)[k];
            v = static_cast<float*>(t.v)[k];
        }
        m = m * h.beta1 + g * h.one_minus_beta1;
        v = v * h.beta2 + (g * g) * h.one_minus_beta2;
        const float denom = sqrtf(v) * h.rsqrt_bc2 + h.eps;
        p = p * t.decay - (m / denom) * t.step_size;
        const uint32_t bits = random_bits(h.seed, t.index, k);
        if (t.mxfp8) {
            // the largest magnitudes of the block: 32 lanes, as bits, which order NaN above all
            uint32_t top_m = ok ? __float_as_uint(m) & 0x7fffffffu : 0u, top_v = ok ? __float_as_uint(v) & 0x7fffffffu : 0u;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) {
                top_m = max(top_m, (uint32_t)__shfl_xor((int)top_m, off, 32));
                top_v = max(top_v, (uint32_t)__shfl_xor((int)top_v, off, 32));
            }
            const uint32_t sm = scale_of(top_m), sv = scale_of(top_v);
            uint32_t cm = 0x7f, cv = 0x7f;
            if (sm != 255) {
                const float y = m * __uint_as_float((254 - sm) << 23);
                cm = to_e4m3(fabsf(y), bits & 0xffffu) | (__float_as_uint(y) >> 24 & 0x80u);
            }
            if (sv != 255) {
                cv = to_e4m3(v * __uint_as_float((254 - sv) << 23), bits >> 16);
                if (cv == 0 && v > 0.f) cv = 1;
            }
            if (ok) {
                static_cast<uint8_t*>(t.m)[k] = (uint8_t)cm;
                static_cast<uint8_t*>(t.v)[k] = (uint8_t)cv;
                if (k % kBlock == 0) {
                    t.m_scale[block] = (uint8_t)sm;
                    t.v_scale[block] = (uint8_t)sv;
                }
            }
        } else if (ok) {
            static_cast<float*>(t.m)[k] = m;
            static_cast<float*>(t.v)[k] = v;
        }
        if (!ok) continue;
        if (!t.param_bf16) {
            static_cast<float*>(t.param)[k] = p;
        } else if (t.master) {
            t.master[k] = p;
            static_cast<bf16_t*>(t.param)[k] = f32_to_bf16(p);
        } else {
            const uint32_t u = __float_as_uint(p);
            const bool finite = (u & 0x7f800000u) != 0x7f800000u;
            static_cast<bf16_t*>(t.param)[k] = finite ? (bf16_t)((u + ((bits * 0x9e3779b1u) >> 16)) >> 16) : f32_to_bf16(p);
        }
    }
}

inline int64_t chunks_of(int64_t n) { return (n + kChunk - 1) / kChunk; }

}  // namespace

size_t grad_norm_workspace_bytes(int count) {
    // a launch takes one tensor at least; more than one launch for fewer than kListTensors only where chunks run out
    return (size_t)(count > 0 ? count : 1) * kNormGroups * sizeof(double);
}

void launch_grad_norm(const moe_grad_tensor_t* tensors, int count, float max_norm, float multiplier, float* out, void* ws,
                      hipStream_t s) {
    double* partial = static_cast<double*>(ws);
    int parts = 0;
    GradList l;
    int64_t chunks = 0;
    l.count = 0;
    auto flush = [&] {
        if (l.count == 0) return;
        l.chunks = (int32_t)chunks;
        const int groups = (int)(chunks < kNormGroups ? chunks : kNormGroups);
        hipLaunchKernelGGL(grad_norm_partial_kernel, dim3(groups), dim3(256), 0, s, l, partial + parts);
        parts += groups;
        l.count = 0;
        chunks = 0;
    };
    for (int i = 0; i < count; ++i) {
        const int64_t more = chunks_of(tensors[i].n);
        if (more == 0) continue;
        if (l.count == kListTensors || chunks + more > kLaunchChunks) flush();
        l.grad[l.count] = tensors[i].grad;
        l.n[l.count] = tensors[i].n;
        l.bf16[l.count] = tensors[i].dt == MOE_BF16;
        l.first[l.count++] = (int32_t)chunks;
        chunks += more;
    }
    flush();
    hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(256), 0, s, partial, parts, max_norm, multiplier, out);
}

void launch_adamw(const moe_adamw_tensor_t* tensors, int count, double lr, double beta1, double beta2, double eps,
                  int64_t step, uint32_t seed, const float* grad_scale, hipStream_t s) {
    const double bc1 = 1. - pow(beta1, (double)step), bc2 = 1. - pow(beta2, (double)step);
    const AdamStep h = {(float)beta1, (float)(1. - beta1), (float)beta2, (float)(1. - beta2), (float)eps,
                        (float)(1. / sqrt(bc2)), seed, grad_scale};
    AdamList l;
    int64_t chunks = 0;
    l.count = 0;
    auto flush = [&] {
        if (l.count) hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)chunks), dim3(256), 0, s, l, h);
        l.count = 0;
        chunks = 0;
    };
    for (int i = 0; i < count; ++i) {
        const moe_adamw_tensor_t& t = tensors[i];
        const int64_t more = chunks_of(t.n);
        if (more == 0) continue;
        if (l.count == kListTensors || chunks + more > kLaunchChunks) flush();
        const double lr_i = lr * t.lr_scale;
        l.first[l.count] = (int32_t)chunks;
        l.t[l.count++] = {t.param, t.master, t.grad, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale, t.n,
                          (float)(1. - lr_i * t.weight_decay), (float)(lr_i / bc1), i, t.param_dt == MOE_BF16,
                          t.grad_dt == MOE_BF16, t.state == MOE_STATE_MXFP8};
        chunks += more;
    }
    flush();
}

}  // namespace moe
