// Balance loss and z loss of a router, per-expert counts, and their gradient in the logits (formulas in include/moe.h).
//
//   balance_partial_kernel   a chunk of one sequence's tokens: sums of probabilities, counts, squares of the
//                            log-sum-exps and valid tokens of the chunk
//   balance_sequence_kernel  the chunks of one sequence added up in order (64 experts to a workgroup)
//   balance_total_kernel     the two losses from all sequences
//   balance_single_kernel    the last two in one, for one sequence
//   balance_backward_kernel  the gradient, token by token
//
// All are bound by memory: the forward reads the logits once, the backward reads and writes them once.  A token's logits lie
// four to a lane in as many lanes as its experts need (a power of two, LPT), so that 64 / LPT tokens share a wave, a lane
// always has the same experts and keeps its sums of probabilities in registers; four batches of tokens are in flight.
#include <type_traits>

#include "common.h"

namespace moe {

namespace {

constexpr int kBatches = 4;        // tokens a lane has in flight
constexpr int kSlab = 64;          // experts of a workgroup of balance_sequence_kernel

// Tokens of a chunk and threads of its workgroup: functions of T (and of whether there are sequences) only, so that the
// order of the sums is reproducible.  One sequence: up to 256 chunks, one to a compute unit, that one workgroup can add up.
__host__ __device__ inline int chunk_tokens(int T, bool packed) {
    if (packed) return T > 65536 ? 256 : 64;
    const int c = (T + 255) / 256;
    return c < 64 ? 64 : (c + 15) & ~15;
}

inline int chunk_count(int T, int n_seq, bool packed) {
    const int c = chunk_tokens(T, packed);
    return packed ? T / c + n_seq : (T + c - 1) / c + (T == 0);
}

__device__ __forceinline__ int clamp_token(int t, int T) { return min(max(t, 0), T); }

// Chunks of C tokens are numbered across the sequences without a table: sequence s starts at chunk offsets[s] / C + s, which
// leaves it ceil(length / C) of them or one more (floor((a + n) / C) + 1 - floor(a / C) >= ceil(n / C)).
__device__ __forceinline__ int first_chunk(const int32_t* offsets, int s, int T, int C) { return clamp_token(offsets[s], T) / C + s; }

struct Chunk {
    int seq, t0, t1;
};

__device__ __forceinline__ Chunk find_chunk(int b, const int32_t* offsets, int n_seq, int T, int C) {
    if (offsets == nullptr) return {0, b * C, b * C + min(T - b * C, C)};
    int lo = 0, hi = n_seq;   // the last sequence that starts at chunk b or before it
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first_chunk(offsets, mid, T, C) <= b) lo = mid;
        else hi = mid;
    }
    const int begin = clamp_token(offsets[lo], T), end = clamp_token(offsets[lo + 1], T);
    const long long t0 = begin + (long long)(b - first_chunk(offsets, lo, T, C)) * C;
    const int from = max((int)(t0 < end ? t0 : end), 0);
    return {lo, from, from + min(end - from, C)};
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// One number for each of a lane's kBatches tokens, the same in all lanes of a token.  With four lanes to a token or more each
// lane holds only that of token lane % 4, so that what is worked out from it (a reciprocal, a logarithm) is worked out once.
template <int LPT>
struct PerToken {
    static constexpr int N = LPT >= 4 ? 1 : kBatches;
    float v[N];

    template <int U>
    __device__ __forceinline__ float get() const {
        if constexpr (LPT >= 4) return dpp<0x55 * U>(v[0]);   // quad_perm U, U, U, U
        else return v[U];
    }
};

// Reduces each token's numbers over its LPT neighbouring lanes.  Within a quad the four tokens are dealt to the four lanes (two
// exchanges of halves instead of two reductions for every token), then quads are joined by rotations of a row of 16, rows and
// halves of the wave by swaps.
template <int LPT, typename F>
__device__ __forceinline__ PerToken<LPT> reduce(float (&a)[kBatches], F&& f) {
    static_assert(kBatches == 4, "a quad holds four tokens");
    PerToken<LPT> out;
    if constexpr (LPT < 4) {
#pragma unroll
        for (int u = 0; u < kBatches; ++u) out.v[u] = LPT == 2 ? f(a[u], dpp<0xb1>(a[u])) : a[u];
    } else {
        if constexpr (LPT == 8) {
#pragma unroll
            for (int u = 0; u < kBatches; ++u) a[u] = f(a[u], dpp<0x141>(a[u]));   // row_half_mirror: the other quad
        }
        const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
        const float lo = f(odd ? a[1] : a[0], dpp<0xb1>(odd ? a[0] : a[1]));       // quad_perm 1, 0, 3, 2
        const float hi = f(odd ? a[3] : a[2], dpp<0xb1>(odd ? a[2] : a[3]));
        float v = f(high ? hi : lo, dpp<0x4e>(high ? lo : hi));                    // quad_perm 2, 3, 0, 1
        if constexpr (LPT >= 16) {
            v = f(v, dpp<0x124>(v));                                               // row_ror 4, then 8
            v = f(v, dpp<0x128>(v));
        }
        if constexpr (LPT >= 32) {
            const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
        }
        if constexpr (LPT >= 64) {
            const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
        }
        out.v[0] = v;
    }
    return out;
}
template <int LPT>
__device__ __forceinline__ PerToken<LPT> reduce_sum(float (&a)[kBatches]) {
    return reduce<LPT>(a, [](float x, float y) { return x + y; });
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// A lane's four logits of a token; -inf past the last expert.
__device__ __forceinline__ f32x4 load_logits(const float* row, int e, int E, bool vec) {
    f32x4 x = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (vec) {
        if (e < E) x = *reinterpret_cast<const f32x4*>(row + e);
    } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (e + u < E) x[u] = row[e + u];
    }
    return x;
}

// A lane's logits of its next tokens, one in each of kBatches batches of `step` tokens.  ok: bit u is set where token u counts;
// what others hold is replaced, so that it cannot spread.
struct Batches {
    f32x4 x[kBatches];
    uint32_t ok;

    __device__ __forceinline__ void load(const float* logits, const uint8_t* mask, int t, int step, int end, int e, int E, bool vec) {
        ok = 0;
#pragma unroll
        for (int u = 0; u < kBatches; ++u) {
            const int tu = t + u * step;
            const bool in = tu < end;
            const size_t row = in ? tu : end - 1;
            x[u] = load_logits(logits + row * E, e, E, vec);
            ok |= (in && (mask == nullptr || mask[row] != 0) ? 1u : 0u) << u;
        }
    }
    __device__ __forceinline__ void hide_masked() {
#pragma unroll
        for (int u = 0; u < kBatches; ++u)
#pragma unroll
            for (int v = 0; v < 4; ++v) x[u][v] = ok >> u & 1 ? x[u][v] : 0.f;
    }
};

// x becomes exp(x - top), top being a token's largest logit, and `sums` the lane's sums of them.  All of -inf: zeros, top 0.
template <int LPT>
__device__ __forceinline__ PerToken<LPT> exponentials(f32x4 (&x)[kBatches], float (&sums)[kBatches]) {
    constexpr float kLog2E = 1.44269504f;
    float m[kBatches];
#pragma unroll
    for (int u = 0; u < kBatches; ++u) m[u] = fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3]));
    PerToken<LPT> top = reduce<LPT>(m, [](float a, float b) { return fmaxf(a, b); });
#pragma unroll
    for (int i = 0; i < PerToken<LPT>::N; ++i) top.v[i] = top.v[i] == -INFINITY ? 0.f : top.v[i];   // exp(-inf - 0) = 0, NaN stays
    auto one = [&](auto index) {
        constexpr int u = index.value;
        const float from = top.template get<u>();
#pragma unroll
        for (int v = 0; v < 4; ++v) x[u][v] = __builtin_amdgcn_exp2f((x[u][v] - from) * kLog2E);
        sums[u] = (x[u][0] + x[u][1]) + (x[u][2] + x[u][3]);
    };
    one(std::integral_constant<int, 0>());
    one(std::integral_constant<int, 1>());
    one(std::integral_constant<int, 2>());
    one(std::integral_constant<int, 3>());
    return top;
}

// Whether the token counts that entry i of a PerToken stands for.
template <int LPT>
__device__ __forceinline__ bool counts_at(uint32_t ok, int i) {
    return ok >> (LPT >= 4 ? threadIdx.x & 3 : i) & 1;
}

// log-sum-exp from the largest logit and the sum of exp(x - top), which is 1 at least; the instruction's own logarithm
__device__ __forceinline__ float log_sum(float top, float s) { return fmaf(__builtin_amdgcn_logf(s), 0.693147181f, top); }

// Workspace: what every chunk leaves, then what every sequence leaves.
struct Partials {
    float* prob;      // [chunks, E]
    int32_t* count;   // [chunks, E]
    float* z;         // [chunks]
    int32_t* tokens;  // [chunks]
    double* seq_loss; // [n_seq, slabs]
    double* seq_z;    // [n_seq]
};

inline int slabs_of(int E) { return (E + kSlab - 1) / kSlab; }

inline size_t carve(void* ws, int chunks, int E, int n_seq, Partials* out) {
    uint8_t* base = static_cast<uint8_t*>(ws);
    size_t o = 0;
    auto take = [&](size_t bytes) { uint8_t* p = base + o; o = up256(o + bytes); return p; };
    Partials p;
    p.prob = reinterpret_cast<float*>(take((size_t)chunks * E * 4));
    p.count = reinterpret_cast<int32_t*>(take((size_t)chunks * E * 4));
    p.z = reinterpret_cast<float*>(take((size_t)chunks * 4));
    p.tokens = reinterpret_cast<int32_t*>(take((size_t)chunks * 4));
    p.seq_loss = reinterpret_cast<double*>(take((size_t)n_seq * slabs_of(E) * 8));
    p.seq_z = reinterpret_cast<double*>(take((size_t)n_seq * 8));
    if (out) *out = p;
    return o;
}

// One chunk to a workgroup of up to 16 waves.
template <int LPT>
__global__ __launch_bounds__(1024) void balance_partial_kernel(const float* __restrict__ logits, const int32_t* __restrict__ idx,
                                                               const uint8_t* __restrict__ mask,
                                                               const int32_t* __restrict__ offsets, int T, int E, int K,
                                                               int n_seq, int C, Partials out) {
    constexpr int kTokens = 64 / LPT, kExperts = 4 * LPT;
    __shared__ int32_t hist[kExperts];
    __shared__ float sums[16][kExperts];
    __shared__ float zs[16];
    __shared__ int32_t ns[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, b = blockIdx.x;
    const int q = lane % LPT, e = 4 * q;
    const bool vec = E % 4 == 0;
    const Chunk c = find_chunk(b, offsets, n_seq, T, C);
    const int step = waves * kTokens, own = lane / LPT;
    int t = c.t0 + wave * kTokens;
    Batches next;
    if (t < c.t1) next.load(logits, mask, t + own, step, c.t1, e, E, vec);
    if (threadIdx.x < kExperts) hist[threadIdx.x] = 0;
    __syncthreads();
    // counts: every assignment of the chunk once, whole numbers in any order
    const int64_t a1 = (int64_t)c.t1 * K;
    for (int64_t a = (int64_t)c.t0 * K + threadIdx.x; a < a1; a += blockDim.x) {
        const int i = idx[a];
        if ((unsigned)i < (unsigned)E && (mask == nullptr || mask[(uint32_t)a / (uint32_t)K] != 0)) atomicAdd(&hist[i], 1);
    }
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float zsum = 0.f;
    int n = 0;
    while (t < c.t1) {
        Batches cur = next;
        t += kBatches * step;
        if (t < c.t1) next.load(logits, mask, t + own, step, c.t1, e, E, vec);
        if (mask) cur.hide_masked();
        float sums[kBatches];
        const PerToken<LPT> top = exponentials<LPT>(cur.x, sums);
        PerToken<LPT> s = reduce_sum<LPT>(sums);
#pragma unroll
        for (int i = 0; i < PerToken<LPT>::N; ++i) {
            // a token that does not count, or has no probability, adds nothing to either loss
            const bool ok = counts_at<LPT>(cur.ok, i) && s.v[i] != 0.f;
            const float lse = ok ? log_sum(top.v[i], s.v[i]) : 0.f;
            if (q < (LPT >= 4 ? 4 : 1)) zsum = fmaf(lse, lse, zsum);
            s.v[i] = ok ? __builtin_amdgcn_rcpf(s.v[i]) : 0.f;
        }
        if (q == 0) n += __popc(cur.ok);
        auto add = [&](auto index) {
            constexpr int u = index.value;
            const float r = s.template get<u>();
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[v] = fmaf(cur.x[u][v], r, acc[v]);
        };
        add(std::integral_constant<int, 0>());
        add(std::integral_constant<int, 1>());
        add(std::integral_constant<int, 2>());
        add(std::integral_constant<int, 3>());
    }
    // lanes with the same experts, then waves
#pragma unroll
    for (int off = LPT; off < 64; off <<= 1)
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[u] += __shfl_xor(acc[u], off, 64);
    zsum = wave_sum(zsum);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off, 64);
    if (lane < LPT) {
#pragma unroll
        for (int u = 0; u < 4; ++u) sums[wave][e + u] = acc[u];
    }
    if (lane == 0) {
        zs[wave] = zsum;
        ns[wave] = n;
    }
    __syncthreads();
    if (threadIdx.x < E) {
        float p = 0.f;
        for (int w = 0; w < waves; ++w) p += sums[w][threadIdx.x];
        out.prob[(size_t)b * E + threadIdx.x] = p;
        out.count[(size_t)b * E + threadIdx.x] = hist[threadIdx.x];
    }
    if (threadIdx.x == 0) {
        float z = 0.f;
        int tokens = 0;
        for (int w = 0; w < waves; ++w) {
            z += zs[w];
            tokens += ns[w];
        }
        out.z[b] = z;
        out.tokens[b] = tokens;
    }
}

// Sums over the workgroup's 1024 or 256 threads, in all of them; `red` holds one value a wave.
template <typename T>
__device__ __forceinline__ T workgroup_sum(T v, T* red) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    T s = 0;
    for (int w = 0; w < (int)blockDim.x >> 6; ++w) s += red[w];
    return s;
}

// What the chunks [b0, b1) leave for the experts [e0, e0 + width), added up by `rows` rows of threads of `width` each (a power
// of two) and written; returns sum_e count * prob of them in thread 0.
__device__ __forceinline__ double add_chunks(const Partials& in, int b0, int b1, int E, int e0, int width, int32_t* counts,
                                             float* prob_sums, double* red_p, int32_t* red_n) {
    const int col = threadIdx.x & (width - 1), row = threadIdx.x / width, rows = blockDim.x / width, e = e0 + col;
    double p = 0.;
    int n = 0;
    if (e < E) {
#pragma unroll 8
        for (int b = b0 + row; b < b1; b += rows) {
            p += in.prob[(size_t)b * E + e];
            n += in.count[(size_t)b * E + e];
        }
    }
    red_p[threadIdx.x] = p;
    red_n[threadIdx.x] = n;
    __syncthreads();
    for (int d = rows >> 1; d > 0; d >>= 1) {
        if (row < d) {
            red_p[threadIdx.x] += red_p[threadIdx.x + d * width];
            red_n[threadIdx.x] += red_n[threadIdx.x + d * width];
        }
        __syncthreads();
    }
    double loss = 0.;
    if (row == 0 && e < E) {
        counts[e] = red_n[col];
        prob_sums[e] = (float)red_p[col];
        loss = red_p[col] * red_n[col];
    }
    return workgroup_sum(loss, red_p);
}

__device__ __forceinline__ void chunk_totals(const Partials& in, int b0, int b1, double* red, int32_t* red_n, double& z, int& n) {
    z = 0.;
    n = 0;
    for (int b = b0 + threadIdx.x; b < b1; b += blockDim.x) {
        z += in.z[b];
        n += in.tokens[b];
    }
    z = workgroup_sum(z, red);
    n = workgroup_sum(n, red_n);
}

__device__ __forceinline__ void write_losses(double loss, double z, int n, int E, int K, float balance_coef, float z_coef,
                                             int32_t* all_tokens, float* losses) {
    *all_tokens = n;
    losses[0] = n ? (float)(loss * balance_coef * E / ((double)K * n)) : 0.f;
    losses[1] = n ? (float)(z * z_coef / n) : 0.f;
}

__global__ __launch_bounds__(1024) void balance_single_kernel(int E, int K, int chunks, int width, float balance_coef,
                                                              float z_coef, Partials in, int32_t* __restrict__ counts,
                                                              float* __restrict__ prob_sums, int32_t* __restrict__ seq_tokens,
                                                              float* __restrict__ losses) {
    __shared__ double red_p[1024];
    __shared__ int32_t red_n[1024];
    const double loss = add_chunks(in, 0, chunks, E, 0, width, counts, prob_sums, red_p, red_n);
    double z;
    int n;
    chunk_totals(in, 0, chunks, red_p, red_n, z, n);
    if (threadIdx.x == 0) {
        seq_tokens[0] = n;
        write_losses(n ? loss / n : 0., z, n, E, K, balance_coef, z_coef, seq_tokens + 1, losses);
    }
}

__global__ __launch_bounds__(256) void balance_sequence_kernel(const int32_t* __restrict__ offsets, int T, int E, int chunks,
                                                               int C, int width, Partials in, int32_t* __restrict__ counts,
                                                               float* __restrict__ prob_sums,
                                                               int32_t* __restrict__ seq_tokens) {
    __shared__ double red_p[256];
    __shared__ int32_t red_n[256];
    const int s = blockIdx.x, slab = blockIdx.y;
    const int b0 = min(first_chunk(offsets, s, T, C), chunks), b1 = min(first_chunk(offsets, s + 1, T, C), chunks);
    const double loss = add_chunks(in, b0, b1, E, slab * kSlab, width, counts + (size_t)s * E, prob_sums + (size_t)s * E, red_p, red_n);
    double z;
    int n;
    chunk_totals(in, b0, b1, red_p, red_n, z, n);
    if (threadIdx.x == 0) {
        in.seq_loss[(size_t)s * gridDim.y + slab] = n ? loss / n : 0.;
        if (slab == 0) {
            seq_tokens[s] = n;
            in.seq_z[s] = z;
        }
    }
}

__global__ __launch_bounds__(1024) void balance_total_kernel(int E, int K, int n_seq, int slabs, float balance_coef, float z_coef,
                                                             Partials in, int32_t* __restrict__ seq_tokens,
                                                             float* __restrict__ losses) {
    __shared__ double red[16];
    __shared__ int32_t red_n[16];
    double l = 0., z = 0.;
    int n = 0;
    for (int s = threadIdx.x; s < n_seq; s += 1024) {
        z += in.seq_z[s];
        n += seq_tokens[s];
    }
    for (int i = threadIdx.x; i < n_seq * slabs; i += 1024) l += in.seq_loss[i];
    l = workgroup_sum(l, red);
    z = workgroup_sum(z, red);
    n = workgroup_sum(n, red_n);
    if (threadIdx.x == 0) write_losses(l, z, n, E, K, balance_coef, z_coef, seq_tokens + n_seq, losses);
}

template <int LPT>
__global__ __launch_bounds__(256) void balance_backward_kernel(const float* __restrict__ logits,
                                                               const uint8_t* __restrict__ mask,
                                                               const int32_t* __restrict__ offsets,
                                                               const int32_t* __restrict__ counts,
                                                               const int32_t* __restrict__ seq_tokens,
                                                               const float* __restrict__ dlosses, const float* addend, int T,
                                                               int E, int K, int n_seq, int C, float balance_coef,
                                                               float z_coef, float* dlogits) {
    constexpr int kTokens = 64 / LPT;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int q = lane % LPT, e = 4 * q;
    const bool vec = E % 4 == 0;
    const Chunk c = find_chunk(blockIdx.x, offsets, n_seq, T, C);
    const float n = (float)max(seq_tokens[n_seq], 1), n_s = (float)max(seq_tokens[c.seq], 1);
    const float db = dlosses ? dlosses[0] : 1.f, dz = dlosses ? dlosses[1] : 1.f;
    const float a = db * balance_coef * E / (K * n) / n_s, az = dz * 2.f * z_coef / n;
    f32x4 g;
#pragma unroll
    for (int u = 0; u < 4; ++u) g[u] = e + u < E ? a * counts[(size_t)c.seq * E + e + u] : 0.f;
    const int step = 4 * kTokens;
    for (int t = c.t0 + wave * kTokens + lane / LPT; t - lane / LPT < c.t1; t += kBatches * step) {
        Batches b;
        b.load(logits, mask, t, step, c.t1, e, E, vec);
        f32x4 more[kBatches];
        if (addend) {
#pragma unroll
            for (int u = 0; u < kBatches; ++u) more[u] = load_logits(addend + (size_t)min(t + u * step, c.t1 - 1) * E, e, E, vec);
        } else {
#pragma unroll
            for (int u = 0; u < kBatches; ++u) more[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        if (mask) b.hide_masked();
        float sums[kBatches], dots[kBatches];
        const PerToken<LPT> top = exponentials<LPT>(b.x, sums);
#pragma unroll
        for (int u = 0; u < kBatches; ++u)
            dots[u] = (b.x[u][0] * g[0] + b.x[u][1] * g[1]) + (b.x[u][2] * g[2] + b.x[u][3] * g[3]);
        PerToken<LPT> r = reduce_sum<LPT>(sums), shift = reduce_sum<LPT>(dots);
#pragma unroll
        for (int i = 0; i < PerToken<LPT>::N; ++i) {
            // r = 0 where a token does not count or has no probability
            const bool ok = counts_at<LPT>(b.ok, i) && r.v[i] != 0.f;
            const float lse = log_sum(top.v[i], r.v[i]);
            r.v[i] = ok ? __builtin_amdgcn_rcpf(r.v[i]) : 0.f;
            shift.v[i] = ok ? fmaf(az, lse, -(shift.v[i] * r.v[i])) : 0.f;
        }
        auto write = [&](auto index) {
            constexpr int u = index.value;
            const float ru = r.template get<u>(), su = shift.template get<u>();
            f32x4 d;
#pragma unroll
            for (int v = 0; v < 4; ++v) d[v] = fmaf(b.x[u][v] * ru, g[v] + su, more[u][v]);
            if (t + u * step < c.t1) {
                float* row = dlogits + (size_t)(t + u * step) * E;
                if (vec) {
                    if (e < E) *reinterpret_cast<f32x4*>(row + e) = d;
                } else {
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (e + v < E) row[e + v] = d[v];
                }
            }
        };
        write(std::integral_constant<int, 0>());
        write(std::integral_constant<int, 1>());
        write(std::integral_constant<int, 2>());
        write(std::integral_constant<int, 3>());
    }
}

// Calls f with the lanes a token of E experts takes.
template <typename F>
void with_lanes(int E, F&& f) {
    if (E <= 4) f(std::integral_constant<int, 1>());
    else if (E <= 8) f(std::integral_constant<int, 2>());
    else if (E <= 16) f(std::integral_constant<int, 4>());
    else if (E <= 32) f(std::integral_constant<int, 8>());
    else if (E <= 64) f(std::integral_constant<int, 16>());
    else if (E <= 128) f(std::integral_constant<int, 32>());
    else f(std::integral_constant<int, 64>());
}

// the smallest power of two that is n or more
inline int power_of_two(int n) {
    int w = 1;
    while (w < n) w *= 2;
    return w;
}

}  // namespace

size_t balance_loss_workspace_bytes(int T, int E, int n_seq) {
    // with offsets or without: the larger of the two numbers of chunks
    return carve(nullptr, max(chunk_count(T, n_seq, true), chunk_count(T, n_seq, false)), E, n_seq, nullptr);
}

void launch_balance_loss(const float* logits, const int32_t* idx, const uint8_t* mask, const int32_t* offsets, int T, int E,
                         int K, int n_seq, float balance_coef, float z_coef, int32_t* counts, float* prob_sums,
                         int32_t* seq_tokens, float* losses, void* ws, hipStream_t s) {
    const bool packed = offsets != nullptr;
    const int chunks = chunk_count(T, n_seq, packed), C = chunk_tokens(T, packed);
    Partials p;
    carve(ws, chunks, E, n_seq, &p);
    with_lanes(E, [&](auto lanes) {
        hipLaunchKernelGGL(balance_partial_kernel<lanes.value>, dim3(chunks), dim3(packed ? 256 : 1024), 0, s, logits, idx, mask,
                           offsets, T, E, K, n_seq, C, p);
    });
    if (!packed) {
        hipLaunchKernelGGL(balance_single_kernel, dim3(1), dim3(1024), 0, s, E, K, chunks, power_of_two(E), balance_coef, z_coef,
                           p, counts, prob_sums, seq_tokens, losses);
        return;
    }
    const int slabs = slabs_of(E);
    hipLaunchKernelGGL(balance_sequence_kernel, dim3(n_seq, slabs), dim3(256), 0, s, offsets, T, E, chunks, C,
                       power_of_two(E < kSlab ? E : kSlab), p, counts, prob_sums, seq_tokens);
    hipLaunchKernelGGL(balance_total_kernel, dim3(1), dim3(1024), 0, s, E, K, n_seq, slabs, balance_coef, z_coef, p, seq_tokens,
                       losses);
}

void launch_balance_loss_backward(const float* logits, const uint8_t* mask, const int32_t* offsets, const int32_t* counts,
                                  const int32_t* seq_tokens, const float* dlosses, const float* addend, int T, int E, int K,
                                  int n_seq, float balance_coef, float z_coef, float* dlogits, hipStream_t s) {
    const bool packed = offsets != nullptr;
    const int C = 64, chunks = packed ? T / C + n_seq : (T + C - 1) / C;
    with_lanes(E, [&](auto lanes) {
        hipLaunchKernelGGL(balance_backward_kernel<lanes.value>, dim3(chunks), dim3(256), 0, s, logits, mask, offsets, counts,
                           seq_tokens, dlosses, addend, T, E, K, n_seq, C, balance_coef, z_coef, dlogits);
    });
}

}  // namespace moe
