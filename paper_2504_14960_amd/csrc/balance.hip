// Balance loss and z loss of a router, per-expert counts, and their gradient in the logits (formulas in include/moe.h).
//
//   balance_partial_kernel   a chunk of one sequence's tokens: sums of probabilities, counts, squares of the
//                            log-sum-exps and valid tokens of the chunk
//   balance_sequence_kernel  the chunks of one sequence added up in order
//   balance_total_kernel     the two losses from all sequences
//   balance_backward_kernel  the gradient, token by token
//
// All are bound by memory: the forward reads the logits once, the backward reads and writes them once.
#include "common.h"

namespace moe {

namespace {

// Tokens of a chunk: a function of T only, so that the order of the sums is reproducible.
__host__ __device__ inline int chunk_tokens(int T) { return T > 65536 ? 256 : 64; }

inline int chunk_count(int T, int n_seq, bool packed) {
    const int c = chunk_tokens(T);
    return packed ? T / c + n_seq : (T + c - 1) / c + (T == 0);
}

__device__ __forceinline__ int clamp_token(int t, int T) { return min(max(t, 0), T); }

// Chunks are numbered across the sequences without a table: sequence s starts at chunk offsets[s] / c + s, which leaves it
// ceil(length / c) of them or one more (floor((a + n) / c) + 1 - floor(a / c) >= ceil(n / c)).
__device__ __forceinline__ int first_chunk(const int32_t* offsets, int s, int T) {
    return clamp_token(offsets[s], T) / chunk_tokens(T) + s;
}

struct Chunk {
    int seq, t0, t1;
};

__device__ __forceinline__ Chunk find_chunk(int b, const int32_t* offsets, int n_seq, int T) {
    const int c = chunk_tokens(T);
    if (offsets == nullptr) return {0, b * c, min(T, (b + 1) * c)};
    int lo = 0, hi = n_seq;   // the last sequence that starts at chunk b or before it
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first_chunk(offsets, mid, T) <= b) lo = mid;
        else hi = mid;
    }
    const int begin = clamp_token(offsets[lo], T), end = clamp_token(offsets[lo + 1], T);
    const long long t0 = begin + (long long)(b - first_chunk(offsets, lo, T)) * c;
    const int from = (int)(t0 < end ? t0 : end);
    return {lo, max(from, 0), min(end, max(from, 0) + c)};
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// p[j] = softmax of the token's logits for expert lane + 64 j; returns the log-sum-exp.  NaN stays NaN; a token of -inf
// only has p = 0 and a log-sum-exp that counts as 0.
__device__ __forceinline__ float token_softmax(const float* logits, int E, int lane, float (&p)[4]) {
    float m = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        p[j] = lane + 64 * j < E ? logits[lane + 64 * j] : -INFINITY;
        nan |= p[j] != p[j];
        m = fmaxf(m, p[j]);
    }
    m = wave_max(m);
    if (m == -INFINITY && !__any(nan)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = 0.f;
        return 0.f;
    }
    float z = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        p[j] = lane + 64 * j < E ? expf(p[j] - m) : 0.f;
        z += p[j];
    }
    z = wave_sum(z);
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] /= z;
    return m + logf(z);
}

// Workspace: what every chunk leaves, then what every sequence leaves.
struct Partials {
    float* prob;      // [chunks, E]
    int32_t* count;   // [chunks, E]
    float* z;         // [chunks]
    int32_t* tokens;  // [chunks]
    double* seq_loss; // [n_seq]
    double* seq_z;    // [n_seq]
};

inline size_t carve(void* ws, int chunks, int E, int n_seq, Partials* out) {
    uint8_t* base = static_cast<uint8_t*>(ws);
    size_t o = 0;
    auto take = [&](size_t bytes) { uint8_t* p = base + o; o = up256(o + bytes); return p; };
    Partials p;
    p.prob = reinterpret_cast<float*>(take((size_t)chunks * E * 4));
    p.count = reinterpret_cast<int32_t*>(take((size_t)chunks * E * 4));
    p.z = reinterpret_cast<float*>(take((size_t)chunks * 4));
    p.tokens = reinterpret_cast<int32_t*>(take((size_t)chunks * 4));
    p.seq_loss = reinterpret_cast<double*>(take((size_t)n_seq * 8));
    p.seq_z = reinterpret_cast<double*>(take((size_t)n_seq * 8));
    if (out) *out = p;
    return o;
}

__global__ __launch_bounds__(256) void balance_partial_kernel(const float* __restrict__ logits, const int32_t* __restrict__ idx,
                                                              const uint8_t* __restrict__ mask,
                                                              const int32_t* __restrict__ offsets, int T, int E, int K,
                                                              int n_seq, Partials out) {
    __shared__ int32_t hist[kMaxExperts];
    __shared__ float sums[4][kMaxExperts];
    __shared__ float zs[4];
    __shared__ int32_t ns[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.x;
    const Chunk c = find_chunk(b, offsets, n_seq, T);
    hist[threadIdx.x] = 0;
    __syncthreads();
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, z = 0.f;
    int n = 0;
    for (int t = c.t0 + wave; t < c.t1; t += 4) {
        if (mask && mask[t] == 0) continue;
        ++n;
        float p[4];
        const float lse = token_softmax(logits + (size_t)t * E, E, lane, p);
        z += lse * lse;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += p[j];
        if (lane < K) {
            const int e = idx[(size_t)t * K + lane];
            if ((unsigned)e < (unsigned)E) atomicAdd(&hist[e], 1);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[wave][lane + 64 * j] = acc[j];
    if (lane == 0) {
        zs[wave] = z;
        ns[wave] = n;
    }
    __syncthreads();
    const int e = threadIdx.x;
    if (e < E) {
        out.prob[(size_t)b * E + e] = (sums[0][e] + sums[1][e]) + (sums[2][e] + sums[3][e]);
        out.count[(size_t)b * E + e] = hist[e];
    }
    if (e == 0) {
        out.z[b] = (zs[0] + zs[1]) + (zs[2] + zs[3]);
        out.tokens[b] = ns[0] + ns[1] + ns[2] + ns[3];
    }
}

__global__ __launch_bounds__(256) void balance_sequence_kernel(const int32_t* __restrict__ offsets, int T, int E, int chunks,
                                                               int n_seq, Partials in, int32_t* __restrict__ counts,
                                                               float* __restrict__ prob_sums,
                                                               int32_t* __restrict__ seq_tokens) {
    __shared__ double red[256];
    const int s = blockIdx.x, e = threadIdx.x;
    int b0 = 0, b1 = chunks;
    if (offsets) {
        b0 = min(first_chunk(offsets, s, T), chunks);
        b1 = min(first_chunk(offsets, s + 1, T), chunks);
    }
    double p = 0., z = 0.;
    int n = 0, tokens = 0;
    for (int b = b0; b < b1; ++b) {
        if (e < E) {
            p += in.prob[(size_t)b * E + e];
            n += in.count[(size_t)b * E + e];
        }
        z += in.z[b];
        tokens += in.tokens[b];
    }
    if (e < E) {
        counts[(size_t)s * E + e] = n;
        prob_sums[(size_t)s * E + e] = (float)p;
    }
    red[e] = (double)n * p;
    __syncthreads();
    for (int d = 128; d > 0; d >>= 1) {
        if (e < d) red[e] += red[e + d];
        __syncthreads();
    }
    if (e == 0) {
        seq_tokens[s] = tokens;
        in.seq_loss[s] = tokens ? red[0] / tokens : 0.;
        in.seq_z[s] = z;
    }
}

__global__ __launch_bounds__(256) void balance_total_kernel(int E, int K, int n_seq, float balance_coef, float z_coef,
                                                            Partials in, int32_t* __restrict__ seq_tokens,
                                                            float* __restrict__ losses) {
    __shared__ double red_l[256], red_z[256];
    __shared__ int red_n[256];
    const int i = threadIdx.x;
    double l = 0., z = 0.;
    int n = 0;
    for (int s = i; s < n_seq; s += 256) {
        l += in.seq_loss[s];
        z += in.seq_z[s];
        n += seq_tokens[s];
    }
    red_l[i] = l;
    red_z[i] = z;
    red_n[i] = n;
    __syncthreads();
    for (int d = 128; d > 0; d >>= 1) {
        if (i < d) {
            red_l[i] += red_l[i + d];
            red_z[i] += red_z[i + d];
            red_n[i] += red_n[i + d];
        }
        __syncthreads();
    }
    if (i == 0) {
        const int total = red_n[0];
        seq_tokens[n_seq] = total;
        losses[0] = total ? (float)(red_l[0] * balance_coef * E / ((double)K * total)) : 0.f;
        losses[1] = total ? (float)(red_z[0] * z_coef / total) : 0.f;
    }
}

__global__ __launch_bounds__(256) void balance_backward_kernel(const float* __restrict__ logits,
                                                               const uint8_t* __restrict__ mask,
                                                               const int32_t* __restrict__ offsets,
                                                               const int32_t* __restrict__ counts,
                                                               const int32_t* __restrict__ seq_tokens,
                                                               const float* __restrict__ dlosses, const float* addend, int T,
                                                               int E, int K, int n_seq, float balance_coef, float z_coef,
                                                               float* dlogits) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Chunk c = find_chunk(blockIdx.x, offsets, n_seq, T);
    const float n = (float)max(seq_tokens[n_seq], 1), n_s = (float)max(seq_tokens[c.seq], 1);
    const float db = dlosses ? dlosses[0] : 1.f, dz = dlosses ? dlosses[1] : 1.f;
    const float a = db * balance_coef * E / (K * n) / n_s, az = dz * 2.f * z_coef / n;
    float g[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = lane + 64 * j < E ? a * counts[(size_t)c.seq * E + lane + 64 * j] : 0.f;
    for (int t = c.t0 + wave; t < c.t1; t += 4) {
        float p[4] = {0.f, 0.f, 0.f, 0.f}, lse = 0.f;
        if (!mask || mask[t] != 0) lse = token_softmax(logits + (size_t)t * E, E, lane, p);
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) dot += p[j] * g[j];
        dot = wave_sum(dot);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = lane + 64 * j;
            if (e >= E) continue;
            const size_t at = (size_t)t * E + e;
            const float d = p[j] * (g[j] - dot + az * lse);
            dlogits[at] = addend ? d + addend[at] : d;
        }
    }
}

}  // namespace

size_t balance_loss_workspace_bytes(int T, int E, int n_seq) {
    // with offsets or without: the larger of the two numbers of chunks
    return carve(nullptr, max(chunk_count(T, n_seq, true), chunk_count(T, n_seq, false)), E, n_seq, nullptr);
}

void launch_balance_loss(const float* logits, const int32_t* idx, const uint8_t* mask, const int32_t* offsets, int T, int E,
                         int K, int n_seq, float balance_coef, float z_coef, int32_t* counts, float* prob_sums,
                         int32_t* seq_tokens, float* losses, void* ws, hipStream_t s) {
    const int chunks = chunk_count(T, n_seq, offsets != nullptr);
    Partials p;
    carve(ws, chunks, E, n_seq, &p);
    hipLaunchKernelGGL(balance_partial_kernel, dim3(chunks), dim3(256), 0, s, logits, idx, mask, offsets, T, E, K, n_seq, p);
    hipLaunchKernelGGL(balance_sequence_kernel, dim3(n_seq), dim3(256), 0, s, offsets, T, E, chunks, n_seq, p, counts,
                       prob_sums, seq_tokens);
    hipLaunchKernelGGL(balance_total_kernel, dim3(1), dim3(256), 0, s, E, K, n_seq, balance_coef, z_coef, p, seq_tokens,
                       losses);
}

void launch_balance_loss_backward(const float* logits, const uint8_t* mask, const int32_t* offsets, const int32_t* counts,
                                  const int32_t* seq_tokens, const float* dlosses, const float* addend, int T, int E, int K,
                                  int n_seq, float balance_coef, float z_coef, float* dlogits, hipStream_t s) {
    hipLaunchKernelGGL(balance_backward_kernel, dim3(chunk_count(T, n_seq, offsets != nullptr)), dim3(256), 0, s, logits, mask,
                       offsets, counts, seq_tokens, dlosses, addend, T, E, K, n_seq, balance_coef, z_coef, dlogits);
}

}  // namespace moe
