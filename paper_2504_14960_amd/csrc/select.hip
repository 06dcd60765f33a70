// Routing by scores: experts and gates of every token from its logits, where what decides is not the logit but its score
// (softmax or sigmoid) plus a balancing bias, within the best groups of experts; the gradient of the gates; and the step of the
// bias.
//
// Scores decide what is selected, so they are rounded to fp32 once, from 64 bits: two programs that follow the definition then
// select the same experts.
#include "common.h"
#include "wave_sum.h"

namespace moe {

namespace {

struct SelectArgs {
    const float* logits;
    const float* bias;   // [E] or null
    int32_t* idx;
    float* gate;
    float scale;
    int T, E, K, sigmoid, groups, topk_groups, group_best, renorm;
};

constexpr double kNever = -__builtin_huge_val();   // the key of an expert that is not selected whatever else there is

// What an expert is ranked by, as one number: its score and bias, and in the bits behind fp32's its index, so that of equal ones
// the lower index is the larger number.
__device__ __forceinline__ double select_key(float choice, int e) {
    if (!(choice > -INFINITY)) return kNever;                // NaN and -inf
    choice = fminf(choice, __FLT_MAX__) + 0.f;               // -0 to +0
    uint64_t b = __builtin_bit_cast(uint64_t, (double)choice);
    b |= (uint64_t)(choice < 0.f ? e : 255 - e);
    return __builtin_bit_cast(double, b);
}
__device__ __forceinline__ int key_expert(double key) {
    const uint64_t b = __builtin_bit_cast(uint64_t, key);
    return (int)(b >> 63 ? b & 255u : 255u - (b & 255u));
}
__device__ __forceinline__ float key_choice(double key) {
    return (float)__builtin_bit_cast(double, __builtin_bit_cast(uint64_t, key) & ~0x1fffffffull);
}
// the larger key (neither is a NaN, which fmax would look for)
__device__ __forceinline__ double max_key(double a, double b) {
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// f over the 64 lanes of a wave, in all of them
template <typename T, typename F>
__device__ __forceinline__ T wave_fold(T v, F&& f) {
    v = f(v, dpp<0x121>(v));   // row_ror 1, 2, 4, 8
    v = f(v, dpp<0x122>(v));
    v = f(v, dpp<0x124>(v));
    v = f(v, dpp<0x128>(v));
    v = with_swapped<false>(v, f);
    return with_swapped<true>(v, f);
}
__device__ __forceinline__ double wave_max_key(double v) {
    return wave_fold(v, [](double a, double b) { return max_key(a, b); });
}
__device__ __forceinline__ float wave_max(float v) {
    return wave_fold(v, [](float a, float b) { return fmaxf(a, b); });
}

__device__ __forceinline__ double sigmoid64(float x) { return 1. / (1. + exp(-(double)x)); }
// exp(x - m) for x <= m; of equal infinities 1
__device__ __forceinline__ double shifted_exp64(float x, float m) { return x == m ? 1. : exp((double)x - (double)m); }

constexpr int kSelectWaves = 4;

// One token to a wave, any K, any groups.  Lane l holds experts l + 64 j.
template <int VPL>
__global__ __launch_bounds__(64 * kSelectWaves) void select_wave_kernel(SelectArgs p) {
    __shared__ double keys[kSelectWaves][64 * VPL];
    __shared__ double best[kSelectWaves][64 * VPL];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = blockIdx.x * kSelectWaves + wave;
    if (t >= p.T) return;
    const float* const row = p.logits + (size_t)t * p.E;
    float x[VPL], m = -INFINITY;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        const int e = lane + 64 * j;
        x[j] = e < p.E ? row[e] : -INFINITY;
        if (!(x[j] > -INFINITY)) x[j] = -INFINITY;
        m = fmaxf(m, x[j]);
    }
    double z = 0.;
    if (!p.sigmoid) {
        m = wave_max(m);
#pragma unroll
        for (int j = 0; j < VPL; ++j) z += x[j] > -INFINITY ? shifted_exp64(x[j], m) : 0.;
        z = wave_sum(z);
    }
    auto score = [&](float l) { return p.sigmoid ? sigmoid64(l) : shifted_exp64(l, m) / z; };
    double key[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        const int e = lane + 64 * j;
        key[j] = kNever;
        if (x[j] > -INFINITY) key[j] = select_key((float)score(x[j]) + (p.bias ? p.bias[e] : 0.f), e);
    }
    if (p.groups > 1) {
        // a lane takes a group: the sum of its best keys, then its rank among the groups
        const int size = p.E / p.groups;
#pragma unroll
        for (int j = 0; j < VPL; ++j) keys[wave][lane + 64 * j] = key[j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        double mine[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int g = lane + 64 * j;
            mine[j] = kNever;
            if (g < p.groups) {
                double first = kNever, second = kNever;
                for (int i = 0; i < size; ++i) {
                    const double k = keys[wave][g * size + i];
                    second = k > first ? first : max_key(second, k);
                    first = max_key(first, k);
                }
                if (first > kNever) {
                    float sum = key_choice(first);
                    if (p.group_best > 1 && second > kNever) sum += key_choice(second);
                    mine[j] = select_key(sum, g);
                }
                best[wave][g] = mine[j];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        int rank[VPL] = {};
        for (int g = 0; g < p.groups; ++g) {
            const double other = best[wave][g];
#pragma unroll
            for (int j = 0; j < VPL; ++j) rank[j] += other > mine[j];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            if (lane + 64 * j < p.groups && rank[j] >= p.topk_groups) best[wave][lane + 64 * j] = kNever;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int e = lane + 64 * j;
            if (e < p.E && !(best[wave][e / size] > kNever)) key[j] = kNever;
        }
    }
    int my_e = -1;
    for (int k = 0; k < p.K; ++k) {
        double top = key[0];
#pragma unroll
        for (int j = 1; j < VPL; ++j) top = max_key(top, key[j]);
        top = wave_max_key(top);
        if (!(top > kNever)) break;                          // the same in every lane
        const int e = key_expert(top);
        if (lane == k) my_e = e;
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            if (e == lane + 64 * j) key[j] = kNever;
    }
    // slot k in lane k
    double g = my_e >= 0 ? score(row[my_e]) : 0.;
    if (p.renorm) {
        const double sum = wave_sum(g);
        g = sum > 0. ? g / sum : 0.;
    }
    if (lane < p.K) {
        p.idx[(size_t)t * p.K + lane] = my_e;
        p.gate[(size_t)t * p.K + lane] = (float)(g * (double)p.scale);
    }
}

// ---- the gradient ----
struct SelectBackwardArgs {
    const float* logits;
    const int32_t* idx;
    const float* dgate;
    const float* addend;   // [T, E] or null
    float* dlogits;
    float scale;
    int T, E, K, sigmoid, renorm;
};

// f over L consecutive lanes (a power of two), in all of them
template <typename F>
__device__ __forceinline__ float lanes_fold(float v, int L, F&& f) {
    for (int d = 1; d < L; d <<= 1) v = f(v, __shfl_xor(v, d, 64));
    return v;
}

// L = 1 .. 64 lanes to a token, four experts to a lane: 4 sub .. 4 sub + 3 (VEC: E is a multiple of 4), else sub + L j.  Lane sub
// works out the slots sub, sub + L, ..: as E <= 4 L there are at most four.
template <bool VEC>
__global__ __launch_bounds__(256) void select_dlogits_kernel(SelectBackwardArgs p, int L) {
    const int sub = threadIdx.x & (L - 1);
    const int t = (int)(((size_t)blockIdx.x * 256 + threadIdx.x) / L);
    const bool valid = t < p.T;                              // the same for the lanes of a token
    const size_t at = (size_t)(valid ? t : 0);
    const float* const row = p.logits + at * p.E;
    auto add = [](float a, float b) { return a + b; };
    auto expert = [&](int j) { return VEC ? 4 * sub + j : sub + L * j; };
    // probabilities (softmax), 0 of experts that are not open
    float pe[4] = {}, m = -INFINITY, rz = 0.f;
    if (!p.sigmoid) {
        float x[4];
        if (VEC) {
            f32x4 v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (4 * sub < p.E) v = *reinterpret_cast<const f32x4*>(row + 4 * sub);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = v[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = expert(j) < p.E ? row[expert(j)] : -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) m = fmaxf(m, x[j]);      // of NaN and a number the number
        m = lanes_fold(m, L, [](float a, float b) { return fmaxf(a, b); });
        float z = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (x[j] > -INFINITY) pe[j] = x[j] == m ? 1.f : expf(x[j] - m);
            z += pe[j];
        }
        z = lanes_fold(z, L, add);
        rz = z > 0.f ? 1.f / z : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) pe[j] *= rz;
    }
    // this lane's slots: expert, score, 1 - score (sigmoid), gradient of the gate
    int e[4];
    float s[4], rest[4], d[4], sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int k = sub + L * j;
        e[j] = -1;
        s[j] = rest[j] = d[j] = 0.f;
        if (k < p.K) {
            const int i = p.idx[at * p.K + k];
            if ((unsigned)i < (unsigned)p.E) {
                const float l = row[i];
                if (l > -INFINITY) {
                    e[j] = i;
                    d[j] = p.dgate[at * p.K + k] * p.scale;
                    if (p.sigmoid) {
                        const float q = expf(-fabsf(l)), r = 1.f / (1.f + q);
                        s[j] = l >= 0.f ? r : q * r;
                        rest[j] = l >= 0.f ? q * r : r;
                    } else {
                        s[j] = (l == m ? 1.f : expf(l - m)) * rz;
                    }
                }
            }
        }
        sum += s[j];
    }
    float c[4], total = 0.f;                                 // gradient of the logarithm of the score (sigmoid: divided by `rest`)
    if (p.renorm) {
        sum = lanes_fold(sum, L, add);
        float mean = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s[j] = sum > 0.f ? s[j] / sum : 0.f;
            mean += e[j] >= 0 ? d[j] * s[j] : 0.f;
        }
        mean = lanes_fold(mean, L, add);
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = e[j] >= 0 ? (d[j] - mean) * s[j] : 0.f;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = e[j] >= 0 ? d[j] * s[j] : 0.f;
    }
    if (p.sigmoid) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] *= rest[j];
    } else {
        total = lanes_fold(c[0] + c[1] + c[2] + c[3], L, add);
    }
    float out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = -pe[j] * total;
    // slots in ascending order; an expert named twice adds up
    const int lane = threadIdx.x & 63, first = lane & ~(L - 1);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        for (int k = 0; k < L && k + L * j < p.K; ++k) {
            const int ek = __shfl(e[j], first + k, 64);
            const float ck = __shfl(c[j], first + k, 64);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (ek == expert(i)) out[i] += ck;
        }
    if (!valid) return;
    if (VEC) {
        if (4 * sub >= p.E) return;
        f32x4 v = {out[0], out[1], out[2], out[3]};
        if (p.addend) v += *reinterpret_cast<const f32x4*>(p.addend + at * p.E + 4 * sub);
        *reinterpret_cast<f32x4*>(p.dlogits + at * p.E + 4 * sub) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (expert(j) < p.E) p.dlogits[at * p.E + expert(j)] = out[j] + (p.addend ? p.addend[at * p.E + expert(j)] : 0.f);
    }
}

// ---- the step of the bias ----
constexpr int kBiasRows = 64;   // rows of counts that a workgroup adds up

// part[b][e] = sum of a workgroup's rows
__global__ __launch_bounds__(256) void bias_sum_kernel(const int32_t* __restrict__ counts, int n_rows, int E,
                                                       int64_t* __restrict__ part) {
    const int r0 = blockIdx.x * kBiasRows, r1 = min(n_rows, r0 + kBiasRows);
    int64_t n = 0;
    if ((int)threadIdx.x < E)
        for (int r = r0; r < r1; ++r) n += counts[(size_t)r * E + threadIdx.x];
    if ((int)threadIdx.x < E) part[(size_t)blockIdx.x * E + threadIdx.x] = n;
}

// bias[e] += rate * sign(sum_j n_j - E n_e), n the sums of `rows` rows
template <typename N>
__global__ __launch_bounds__(256) void bias_step_kernel(const N* __restrict__ rows, int n_rows, int E, float rate,
                                                        float* __restrict__ bias) {
    __shared__ int64_t part[4];
    const int e = threadIdx.x;
    int64_t n = 0;
    if (e < E)
        for (int r = 0; r < n_rows; ++r) n += rows[(size_t)r * E + e];
    const int64_t sum = wave_sum(n);
    if ((e & 63) == 0) part[e >> 6] = sum;
    __syncthreads();
    const int64_t off = part[0] + part[1] + part[2] + part[3] - (int64_t)E * n;
    if (e < E && off != 0) bias[e] += off > 0 ? rate : -rate;
}

}  // namespace

void launch_select(const float* logits, const float* bias, int T, int E, int K, moe_score_t score, int groups, int topk_groups,
                   int group_best, int renorm, float scale, int32_t* idx, float* gate, hipStream_t s) {
    const SelectArgs p = {logits, bias, idx, gate, scale, T, E, K, score == MOE_SCORE_SIGMOID, groups, topk_groups, group_best, renorm};
    const dim3 grid((T + kSelectWaves - 1) / kSelectWaves), block(64 * kSelectWaves);
    if (E <= 64) hipLaunchKernelGGL(select_wave_kernel<1>, grid, block, 0, s, p);
    else if (E <= 128) hipLaunchKernelGGL(select_wave_kernel<2>, grid, block, 0, s, p);
    else hipLaunchKernelGGL(select_wave_kernel<4>, grid, block, 0, s, p);
}

void launch_select_dlogits(const float* logits, const int32_t* idx, const float* dgate, const float* addend, int T, int E, int K,
                           moe_score_t score, int renorm, float scale, float* dlogits, hipStream_t s) {
    const SelectBackwardArgs p = {logits, idx, dgate, addend, dlogits, scale, T, E, K, score == MOE_SCORE_SIGMOID, renorm};
    int L = 1;
    while (4 * L < E) L <<= 1;
    const dim3 grid((unsigned)(((size_t)T * L + 255) / 256));
    if (E % 4 == 0) hipLaunchKernelGGL(select_dlogits_kernel<true>, grid, dim3(256), 0, s, p, L);
    else hipLaunchKernelGGL(select_dlogits_kernel<false>, grid, dim3(256), 0, s, p, L);
}

size_t bias_update_workspace_bytes(int n_rows, int E) {
    return n_rows <= kBiasRows ? 0 : (size_t)((n_rows + kBiasRows - 1) / kBiasRows) * E * sizeof(int64_t);
}

void launch_bias_update(const int32_t* counts, int n_rows, int E, float rate, float* bias, void* ws, hipStream_t s) {
    if (n_rows <= kBiasRows) {
        hipLaunchKernelGGL(bias_step_kernel<int32_t>, dim3(1), dim3(256), 0, s, counts, n_rows, E, rate, bias);
        return;
    }
    const int parts = (n_rows + kBiasRows - 1) / kBiasRows;
    int64_t* part = static_cast<int64_t*>(ws);
    hipLaunchKernelGGL(bias_sum_kernel, dim3(parts), dim3(256), 0, s, counts, n_rows, E, part);
    hipLaunchKernelGGL(bias_step_kernel<int64_t>, dim3(1), dim3(256), 0, s, part, parts, E, rate, bias);
}

}  // namespace moe
