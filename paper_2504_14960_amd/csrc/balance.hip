// Balance loss and z loss of a router, per-expert counts, and their gradient in the logits (formulas in include/moe.h).
//
//   balance_partial_kernel   a chunk of one sequence's tokens: sums of probabilities, counts, squares of the
//                            log-sum-exps and valid tokens of the chunk; a small call's only chunk writes the results
//   balance_finish_kernel    the chunks of one sequence added up in order (some experts to a workgroup); the last
//                            workgroup adds up the sequences
//   balance_total_kernel     the same, where there are many sequences
//   balance_backward_kernel  the gradient, token by token
//
// All are bound by memory: the forward reads the logits once, the backward reads and writes them once.  A token's logits lie
// four to a lane in as many lanes as its experts need (a power of two, LPT), so that 64 / LPT tokens share a wave, a lane
// always has the same experts and keeps its sums of probabilities in registers; four batches of tokens are in flight.  What a
// token needs from all its lanes (largest logit, sum of exponentials, the gradient's dot product) is reduced for four tokens
// at once, which leaves 57 instructions a token of 256 experts (101 in the backward); token by token it took 99 (131), and the
// vector units set the pace.
//
// Measured (fp32 logits, streamed past the caches: 10 % faster than through them): forward of 262144 tokens x 256 experts
// 46 us in the first launch (6.0 TB/s) and 6.7 in the second, of 32768 x 64 6.3 and 4.6, of 256 x 8 4.0 in the only one;
// gradient of 262144 x 256 87 us (6.2 TB/s), of 7777 x 60 in 23 sequences 5.1.
#include <type_traits>

#include "wave_sum.h"

namespace moe {

namespace {

constexpr int kBatches = 4;            // tokens a lane has in flight
constexpr int kGridGroups = 1 << 23;  // workgroups of 256 threads in a launch at most: a grid has less than 2^32 threads
constexpr int kTicketGroups = 64;      // workgroups of balance_finish_kernel of which the last one adds up the sequences

// How a call is cut, by its sizes alone, so that the order of the sums is reproducible.  The chunks of one sequence are added
// up by one workgroup for 64 experts; for more, 16 experts to a workgroup and a ticket for the last of them: 6.6 us instead
// of 11.4 for 256 chunks of 256 experts (one workgroup takes in some 50 B/ns), while the ticket costs 3 us where one is enough.
struct Cut {
    int chunk_tokens, chunks, threads;   // balance_partial_kernel
    int slab, slabs, finish_threads;     // balance_finish_kernel: experts of a workgroup, workgroups of a sequence
    bool direct, ticket;

    Cut(int T, int E, int n_seq, bool packed) {
        if (packed) {
            chunk_tokens = T > 65536 ? 256 : 64;
            chunks = T / chunk_tokens + n_seq;
            threads = 256;
        } else {
            // up to 256 chunks, one to a compute unit; a small call, of few logits and of few tokens, is one (us, one chunk / many:
            // 512 x 64 and 4096 x 8 logits 7.4 / 11.0 and 7.5 / 11.0, twice as many tokens 12.2 / 10.3 and 14.8 / 10.3; 8192 x 1, x 2
            // and x 4 11.0 / 10.9, 11.3 / 10.8 and 8.7 / 10.9, 16384 x 1 and x 2 19.0 / 10.9 and 19.6 / 10.9)
            const int c = (T + 255) / 256;
            const bool small = T <= 8192 && T * E <= 32768;
            chunk_tokens = small ? (T > 0 ? T : 1) : c < 64 ? 64 : (c + 15) & ~15;
            chunks = T > 0 ? (T + chunk_tokens - 1) / chunk_tokens : 1;
            threads = 1024;
        }
        direct = !packed && chunks == 1;
        slab = (packed ? chunks / n_seq <= 64 : E <= 64) ? 64 : 16;
        slabs = (E + slab - 1) / slab;
        finish_threads = chunks / n_seq > 32 ? 1024 : 256;
        ticket = n_seq * slabs <= kTicketGroups;
    }
};

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
    const int nth = b - first_chunk(offsets, lo, T, C);
    if (nth < 0) return {lo, begin, begin};   // tokens before the first sequence: nobody's
    const long long t0 = begin + (long long)nth * C;
    const int from = (int)(t0 < end ? t0 : end);
    return {lo, from, from + min(end - from, C)};
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
        if constexpr (LPT >= 32) v = with_swapped<false>(v, f);
        if constexpr (LPT >= 64) v = with_swapped<true>(v, f);
        out.v[0] = v;
    }
    return out;
}
template <int LPT>
__device__ __forceinline__ PerToken<LPT> reduce_sum(float (&a)[kBatches]) {
    return reduce<LPT>(a, [](float x, float y) { return x + y; });
}

// The experts of a lane: four neighbours, read as one piece, where rows are whole 16-byte pieces (WHOLE); else every LPT-th, so
// that neighbouring lanes read neighbouring values (262144 x 255 logits, the same ones again: gradient 184 us with four neighbours
// read one by one, 113 as pieces at odd addresses, 99 so).
template <int LPT, bool WHOLE>
__device__ __forceinline__ int expert_of(int q, int u) {
    return WHOLE ? 4 * q + u : q + u * LPT;
}

// A lane's four values of a token's row, -inf past its end.  Streamed past the caches, but for rows that are not whole pieces where
// nothing is written beside them, whose ends share lines with the next row (us through / past the caches, inputs in turn: forward of
// 262144 x 33 17.1 / 18.5, x 65 25.8 / 26.4, x 129 47.5 / 46.2, x 255 58.8 / 56.8, 32768 x 63 11.0 / 11.9 and x 129 14.8 / 15.5;
// gradient of 262144 x 129 74.1 / 73.1, x 255 114 / 114).
template <int LPT, bool WHOLE, bool STREAM>
__device__ __forceinline__ f32x4 load_row(const float* row, int q, int E) {
    f32x4 x = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if constexpr (WHOLE) {
        if (4 * q < E) x = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(row + 4 * q));
    } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (q + u * LPT < E) x[u] = STREAM ? __builtin_nontemporal_load(row + q + u * LPT) : row[q + u * LPT];
    }
    return x;
}
template <int LPT, bool WHOLE>
__device__ __forceinline__ void store_row(float* row, int q, int E, const f32x4& d) {
    if constexpr (WHOLE) {
        if (4 * q < E) __builtin_nontemporal_store(d, reinterpret_cast<f32x4*>(row + 4 * q));
    } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (q + u * LPT < E) row[q + u * LPT] = d[u];
    }
}

// A lane's logits of its next tokens, one in each of kBatches batches of `step` tokens, of which those below `end` exist.  load
// only asks for them: whether a token counts is looked at where they are used, or every load would be waited for at once.
template <int LPT, bool WHOLE, bool STREAM>
struct Batches {
    f32x4 x[kBatches];
    uint32_t keep[kBatches];   // bytes of the mask

    __device__ __forceinline__ void load(const float* logits, const uint8_t* mask, int t, int step, int end, int q, int E) {
#pragma unroll
        for (int u = 0; u < kBatches; ++u) {
            const size_t row = min(t + u * step, end - 1);
            x[u] = load_row<LPT, WHOLE, STREAM>(logits + row * E, q, E);
            keep[u] = mask ? mask[row] : 1;
        }
    }
    // Bit u is set where token u counts; what a masked one holds is replaced, so that it cannot spread.
    __device__ __forceinline__ uint32_t settle(bool masked, int t, int step, int end) {
        uint32_t ok = 0;
#pragma unroll
        for (int u = 0; u < kBatches; ++u) {
            ok |= (t + u * step < end && keep[u] != 0 ? 1u : 0u) << u;
            if (masked) {
#pragma unroll
                for (int v = 0; v < 4; ++v) x[u][v] = keep[u] ? x[u][v] : 0.f;
            }
        }
        return ok;
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
struct Cell {
    float prob;
    int32_t count;
};
struct Tail {
    double z;   // in 64 bits from the first square on: that of a row of the lowest fp32 value is 10^77
    int32_t tokens;
};
struct Partials {
    Cell* cell;       // [chunks, E]
    Tail* tail;       // [chunks]
    double* loss;     // [n_seq, slabs]
    double* z;        // [n_seq]
    uint32_t* ticket; // workgroups of balance_finish_kernel that are done; cleared by balance_partial_kernel
};

inline size_t carve(void* ws, int chunks, int slabs, int E, int n_seq, Partials* out) {
    uint8_t* base = static_cast<uint8_t*>(ws);
    size_t o = 0;
    auto take = [&](size_t bytes) { uint8_t* p = base + o; o = up256(o + bytes); return p; };
    Partials p;
    p.cell = reinterpret_cast<Cell*>(take((size_t)chunks * E * sizeof(Cell)));
    p.tail = reinterpret_cast<Tail*>(take((size_t)chunks * sizeof(Tail)));
    p.loss = reinterpret_cast<double*>(take((size_t)n_seq * slabs * 8));
    p.z = reinterpret_cast<double*>(take((size_t)n_seq * 8));
    p.ticket = reinterpret_cast<uint32_t*>(take(4));
    if (out) *out = p;
    return o;
}

struct Results {
    int32_t* counts;
    float* prob_sums;
    int32_t* seq_tokens;
    float* losses;
    float balance_coef, z_coef;
    int E, K, n_seq;

    // loss: sum over sequences of sum_e counts prob_sums / n_s
    __device__ __forceinline__ void write_losses(double loss, double z, int n) const {
        seq_tokens[n_seq] = n;
        losses[0] = n ? (float)(loss * balance_coef * E / ((double)K * n)) : 0.f;
        losses[1] = n ? (float)(z * z_coef / n) : 0.f;
    }
};

// Three sums over the workgroup in one exchange, valid in the first wave.
struct Three {
    double a[16], b[16];
    int32_t n[16];

    __device__ __forceinline__ void sum(double& x, double& y, int& m) {
        x = wave_sum(x);
        y = wave_sum(y);
        m = wave_sum(m);
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        if (lane == 0) {
            a[wave] = x;
            b[wave] = y;
            n[wave] = m;
        }
        __syncthreads();
        if (wave > 0) return;
        x = lane < waves ? a[lane] : 0.;
        y = lane < waves ? b[lane] : 0.;
        m = lane < waves ? n[lane] : 0;
        x = wave_sum(x);
        y = wave_sum(y);
        m = wave_sum(m);
    }
};

// One chunk to a workgroup of up to 16 waves.
template <int LPT, bool WHOLE, bool MASKED>
__global__ __launch_bounds__(1024) void balance_partial_kernel(const float* __restrict__ logits, const int32_t* __restrict__ idx,
                                                               const uint8_t* __restrict__ token_mask,
                                                               const int32_t* __restrict__ offsets, int T, int E, int K,
                                                               int n_seq, int C, bool direct, Partials out, Results res) {
    constexpr int kTokens = 64 / LPT, kExperts = 4 * LPT;
    __shared__ double parts[4];
    __shared__ int32_t hist[kExperts];
    __shared__ float sums[16][kExperts];
    __shared__ double zs[16];
    __shared__ int32_t ns[16];
    const uint8_t* mask = MASKED ? token_mask : nullptr;   // known at compile time: 52 instead of 54 us for 262144 x 256
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, b = blockIdx.x;
    const int q = lane % LPT;
    const Chunk c = find_chunk(b, offsets, n_seq, T, C);
    const int step = waves * kTokens, own = lane / LPT;
    int t = c.t0 + wave * kTokens;
    Batches<LPT, WHOLE, WHOLE> next;
    if (t < c.t1) next.load(logits, mask, t + own, step, c.t1, q, E);
    if (threadIdx.x < kExperts) hist[threadIdx.x] = 0;
    __syncthreads();
    // counts: every assignment of the chunk once, whole numbers in any order.  The token of a masked one: (a + 1/2) / K is at
    // least 1 / 2K away from a whole number, more than the roundings of a product below 2^22.
    const int assigned = max(c.t1 - c.t0, 0) * K;
    const int32_t* picked = idx + (size_t)c.t0 * K;
    const float per_token = 1.f / K;
    for (int a = threadIdx.x; a < assigned; a += 4 * blockDim.x) {
        int i[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int at = a + u * blockDim.x;
            bool in = at < assigned;
            const int safe = in ? at : assigned - 1;
            if (mask) in = in && mask[c.t0 + (assigned < 1 << 22 ? (int)((safe + 0.5f) * per_token) : safe / K)] != 0;
            i[u] = picked[safe];
            if (!in) i[u] = -1;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if ((unsigned)i[u] < (unsigned)E) atomicAdd(&hist[i[u]], 1);
    }
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    double zsum = 0.;
    int n = 0;
    while (t < c.t1) {
        Batches<LPT, WHOLE, WHOLE> cur = next;
        const int now = t + own;
        t += kBatches * step;
        if (t < c.t1) next.load(logits, mask, t + own, step, c.t1, q, E);
        const uint32_t counted = cur.settle(MASKED, now, step, c.t1);
        float sums[kBatches];
        const PerToken<LPT> top = exponentials<LPT>(cur.x, sums);
        PerToken<LPT> s = reduce_sum<LPT>(sums);
#pragma unroll
        for (int i = 0; i < PerToken<LPT>::N; ++i) {
            // a token that does not count, or has no probability, adds nothing to either loss
            const bool ok = counts_at<LPT>(counted, i) && s.v[i] != 0.f;
            const float lse = ok ? log_sum(top.v[i], s.v[i]) : 0.f;
            if (q < (LPT >= 4 ? 4 : 1)) zsum = fma((double)lse, (double)lse, zsum);
            s.v[i] = ok ? __builtin_amdgcn_rcpf(s.v[i]) : 0.f;
        }
        if (q == 0) n += __popc(counted);
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
    for (int u = 0; u < 4; ++u) acc[u] = sum_congruent<LPT>((float)acc[u]);
    zsum = wave_sum(zsum);
    n = wave_sum(n);
    if (lane < LPT) {
#pragma unroll
        for (int u = 0; u < 4; ++u) sums[wave][expert_of<LPT, WHOLE>(q, u)] = acc[u];
    }
    if (lane == 0) {
        zs[wave] = zsum;
        ns[wave] = n;
    }
    __syncthreads();
    float p = 0.f;
    int count = 0;
    if (threadIdx.x < E) {
#pragma unroll
        for (int w = 0; w < 16; ++w) p += w < waves ? sums[w][threadIdx.x] : 0.f;
        count = hist[threadIdx.x];
    }
    double z = 0., loss = 0.;
    int tokens = 0;
    if (wave == 0) {
        z = wave_sum(lane < waves ? zs[lane] : 0.);
        tokens = wave_sum(lane < waves ? ns[lane] : 0);
    }
    if (!direct) {
        if (threadIdx.x < E) out.cell[(size_t)b * E + threadIdx.x] = {p, count};
        if (threadIdx.x == 0) {
            out.tail[b] = {z, tokens};
            if (b == 0) *out.ticket = 0;
        }
        return;
    }
    if (threadIdx.x < E) {
        res.counts[threadIdx.x] = count;
        res.prob_sums[threadIdx.x] = p;
        loss = (double)p * count;
    }
    loss = wave_sum(loss);
    if (kExperts > 64) {
        if (lane == 0 && wave < 4) parts[wave] = loss;
        __syncthreads();
        loss = (parts[0] + parts[1]) + (parts[2] + parts[3]);
    }
    if (threadIdx.x == 0) {
        res.seq_tokens[0] = tokens;
        res.write_losses(tokens ? loss / tokens : 0., z, tokens);
    }
}

// The sums over sequences from what the workgroups of balance_finish_kernel left, in a fixed order.
__device__ __forceinline__ void add_sequences(const Partials& in, const Results& res, int slabs, Three& three) {
    double loss = 0., z = 0.;
    int n = 0;
    for (int s = threadIdx.x; s < res.n_seq; s += blockDim.x) {
        z += in.z[s];
        n += res.seq_tokens[s];
    }
    for (int i = threadIdx.x; i < res.n_seq * slabs; i += blockDim.x) loss += in.loss[i];
    three.sum(loss, z, n);
    if (threadIdx.x == 0) res.write_losses(loss, z, n);
}

// Workgroup (s, i): the chunks of sequence s for the experts [i slab, (i + 1) slab), one to a thread of a row of `width` (a power
// of two, slab or what holds all experts), the chunks dealt over the rows.
__global__ __launch_bounds__(1024) void balance_finish_kernel(const int32_t* __restrict__ offsets, int T, int C, int chunks,
                                                              int slab, int width, bool ticket, Partials in, Results res) {
    __shared__ double red_p[16][64], red_z[16];
    __shared__ int32_t red_n[16][64], red_tokens[16];
    __shared__ Three three;
    __shared__ bool last;
    const int s = blockIdx.x, E = res.E;
    int b0 = 0, b1 = chunks;
    if (offsets) {
        b0 = min(first_chunk(offsets, s, T, C), chunks);
        b1 = min(first_chunk(offsets, s + 1, T, C), chunks);
    }
    const int col = threadIdx.x & (width - 1), row = threadIdx.x / width, rows = blockDim.x / width;
    const int e = blockIdx.y * slab + col;
    double p = 0., z = 0.;
    int n = 0, tokens = 0;
    for (int b = b0 + threadIdx.x; b < b1; b += blockDim.x) {
        const Tail t = in.tail[b];
        z += t.z;
        tokens += t.tokens;
    }
    if (e < E) {
#pragma unroll 16
        for (int b = b0 + row; b < b1; b += rows) {
            const Cell c = in.cell[(size_t)b * E + e];
            p += c.prob;
            n += c.count;
        }
    }
    // lanes with the same expert, waves by way of the LDS, then the first wave
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    for (int off = width; off < 64; off <<= 1) {
        p += __shfl_xor(p, off, 64);
        n += __shfl_xor(n, off, 64);
    }
    z = wave_sum(z);
    tokens = wave_sum(tokens);
    if (lane < width) {
        red_p[wave][lane] = p;
        red_n[wave][lane] = n;
    }
    if (lane == 0) {
        red_z[wave] = z;
        red_tokens[wave] = tokens;
    }
    __syncthreads();
    double loss = 0.;
    if (wave == 0) {
        z = wave_sum(lane < waves ? red_z[lane] : 0.);
        tokens = wave_sum(lane < waves ? red_tokens[lane] : 0);
        if (lane < width && e < E) {
            p = 0.;
            n = 0;
#pragma unroll
            for (int w = 0; w < 16; ++w) {
                p += w < waves ? red_p[w][lane] : 0.;
                n += w < waves ? red_n[w][lane] : 0;
            }
            res.counts[(size_t)s * E + e] = n;
            res.prob_sums[(size_t)s * E + e] = (float)p;
            loss = p * n;
        }
        loss = wave_sum(loss);
    }
    if (gridDim.x * gridDim.y == 1) {
        if (threadIdx.x == 0) {
            res.seq_tokens[0] = tokens;
            res.write_losses(tokens ? loss / tokens : 0., z, tokens);
        }
        return;
    }
    if (threadIdx.x == 0) {
        in.loss[(size_t)s * gridDim.y + blockIdx.y] = tokens ? loss / tokens : 0.;
        if (blockIdx.y == 0) {
            res.seq_tokens[s] = tokens;
            in.z[s] = z;
        }
    }
    if (!ticket) return;
    // the workgroup that ends last sees what all others wrote, and adds it up in the order of the sequences
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(in.ticket, 1u) == gridDim.x * gridDim.y - 1;
        __threadfence();
    }
    __syncthreads();
    if (last) add_sequences(in, res, gridDim.y, three);
}

__global__ __launch_bounds__(1024) void balance_total_kernel(int slabs, Partials in, Results res) {
    __shared__ Three three;
    add_sequences(in, res, slabs, three);
}

template <int LPT, bool WHOLE>
__global__ __launch_bounds__(256) void balance_backward_kernel(const float* __restrict__ logits,
                                                               const uint8_t* __restrict__ mask,
                                                               const int32_t* __restrict__ offsets,
                                                               const int32_t* __restrict__ counts,
                                                               const int32_t* __restrict__ seq_tokens,
                                                               const float* __restrict__ dlosses, const float* addend, int T,
                                                               int E, int K, int n_seq, int C, int from_chunk,
                                                               float balance_coef, float z_coef, float* dlogits) {
    constexpr int kTokens = 64 / LPT;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int q = lane % LPT;
    const Chunk c = find_chunk(from_chunk + blockIdx.x, offsets, n_seq, T, C);
    const float n = (float)max(seq_tokens[n_seq], 1), n_s = (float)max(seq_tokens[c.seq], 1);
    const float db = dlosses ? dlosses[0] : 1.f, dz = dlosses ? dlosses[1] : 1.f;
    const float a = db * balance_coef * E / (K * n) / n_s, az = dz * 2.f * z_coef / n;
    f32x4 g;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int e = expert_of<LPT, WHOLE>(q, u);
        g[u] = e < E ? a * counts[(size_t)c.seq * E + e] : 0.f;
    }
    const int step = 4 * kTokens;
    const int t = c.t0 + wave * kTokens + lane / LPT;
    if (c.t0 + wave * kTokens >= c.t1) return;
    Batches<LPT, WHOLE, true> b;
    b.load(logits, mask, t, step, c.t1, q, E);
    f32x4 more[kBatches];
    if (addend) {
#pragma unroll
        for (int u = 0; u < kBatches; ++u) more[u] = load_row<LPT, WHOLE, true>(addend + (size_t)min(t + u * step, c.t1 - 1) * E, q, E);
    } else {
#pragma unroll
        for (int u = 0; u < kBatches; ++u) more[u] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const uint32_t counted = b.settle(mask != nullptr, t, step, c.t1);
    float sums[kBatches], dots[kBatches];
    const PerToken<LPT> top = exponentials<LPT>(b.x, sums);
#pragma unroll
    for (int u = 0; u < kBatches; ++u)
        dots[u] = (b.x[u][0] * g[0] + b.x[u][1] * g[1]) + (b.x[u][2] * g[2] + b.x[u][3] * g[3]);
    PerToken<LPT> r = reduce_sum<LPT>(sums), shift = reduce_sum<LPT>(dots);
#pragma unroll
    for (int i = 0; i < PerToken<LPT>::N; ++i) {
        // r = 0 where a token does not count or has no probability
        const bool ok = counts_at<LPT>(counted, i) && r.v[i] != 0.f;
        const float lse = log_sum(top.v[i], r.v[i]);
        r.v[i] = ok ? __builtin_amdgcn_rcpf(r.v[i]) : 0.f;
        shift.v[i] = ok ? fmaf(az, lse, -(shift.v[i] * r.v[i])) : 0.f;
    }
    auto write = [&](auto index) {
        constexpr int u = index.value;
        const float ru = r.template get<u>(), su = shift.template get<u>();
        f32x4 d;
        // not 0 * g where a token does not count: g is infinite or NaN where the losses' own gradient is
#pragma unroll
        for (int v = 0; v < 4; ++v) d[v] = ru != 0.f ? fmaf(b.x[u][v] * ru, g[v] + su, more[u][v]) : more[u][v];
        if (t + u * step < c.t1) store_row<LPT, WHOLE>(dlogits + (size_t)(t + u * step) * E, q, E, d);
    };
    write(std::integral_constant<int, 0>());
    write(std::integral_constant<int, 1>());
    write(std::integral_constant<int, 2>());
    write(std::integral_constant<int, 3>());
}

// Calls f with the lanes a token of E experts takes, and whether its rows are whole pieces.
template <typename F>
void with_lanes(int E, F&& f) {
    auto call = [&](auto lanes) {
        if (E % 4 == 0) f(lanes, std::true_type());
        else f(lanes, std::false_type());
    };
    if (E <= 4) call(std::integral_constant<int, 1>());
    else if (E <= 8) call(std::integral_constant<int, 2>());
    else if (E <= 16) call(std::integral_constant<int, 4>());
    else if (E <= 32) call(std::integral_constant<int, 8>());
    else if (E <= 64) call(std::integral_constant<int, 16>());
    else if (E <= 128) call(std::integral_constant<int, 32>());
    else call(std::integral_constant<int, 64>());
}

// the smallest power of two that is n or more
inline int power_of_two(int n) {
    int w = 1;
    while (w < n) w *= 2;
    return w;
}

}  // namespace

// Room for the chunks and slabs of any Cut of up to T tokens, E experts and n_seq sequences, with offsets or without, so that a
// workspace for the largest call serves every smaller one (chunks get longer above 65536 tokens, and fewer).
size_t balance_loss_workspace_bytes(int T, int E, int n_seq) {
    const int chunks = max(min(T, 65536) / 64, T / 256) + n_seq;
    return carve(nullptr, chunks, (E + 15) / 16, E, n_seq, nullptr);
}

void launch_balance_loss(const float* logits, const int32_t* idx, const uint8_t* mask, const int32_t* offsets, int T, int E,
                         int K, int n_seq, float balance_coef, float z_coef, int32_t* counts, float* prob_sums,
                         int32_t* seq_tokens, float* losses, void* ws, hipStream_t s) {
    const Cut cut(T, E, n_seq, offsets != nullptr);
    Partials p;
    carve(ws, cut.chunks, cut.slabs, E, n_seq, &p);
    const Results res = {counts, prob_sums, seq_tokens, losses, balance_coef, z_coef, E, K, n_seq};
    with_lanes(E, [&](auto lanes, auto whole) {
        auto kernel = mask ? balance_partial_kernel<lanes.value, whole.value, true> : balance_partial_kernel<lanes.value, whole.value, false>;
        hipLaunchKernelGGL(kernel, dim3(cut.chunks), dim3(cut.threads), 0, s, logits, idx, mask, offsets, T, E, K, n_seq,
                           cut.chunk_tokens, cut.direct, p, res);
    });
    if (cut.direct) return;
    hipLaunchKernelGGL(balance_finish_kernel, dim3(n_seq, cut.slabs), dim3(cut.finish_threads), 0, s, offsets, T,
                       cut.chunk_tokens, cut.chunks, cut.slab, power_of_two(E < cut.slab ? E : cut.slab), cut.ticket, p, res);
    if (!cut.ticket) hipLaunchKernelGGL(balance_total_kernel, dim3(1), dim3(1024), 0, s, cut.slabs, p, res);
}

void launch_balance_loss_backward(const float* logits, const uint8_t* mask, const int32_t* offsets, const int32_t* counts,
                                  const int32_t* seq_tokens, const float* dlosses, const float* addend, int T, int E, int K,
                                  int n_seq, float balance_coef, float z_coef, float* dlogits, hipStream_t s) {
    const bool packed = offsets != nullptr;
    with_lanes(E, [&](auto lanes, auto whole) {
        // one round of four waves: 2 rounds to a workgroup take 7.9 instead of 5.8 us for 65536 tokens x 16 experts and 10.5
        // instead of 7.7 for 65536 x 64, and save 2 of 90 us only for the largest call
        constexpr int C = kBatches * 4 * (64 / lanes.value);
        const int chunks = packed ? T / C + n_seq : (T + C - 1) / C;
        for (int first = 0; first < chunks; first += kGridGroups)
            hipLaunchKernelGGL((balance_backward_kernel<lanes.value, whole.value>), dim3(min(chunks - first, kGridGroups)), dim3(256), 0, s,
                               logits, mask, offsets, counts, seq_tokens, dlosses, addend, T, E, K, n_seq, C, first, balance_coef, z_coef,
                               dlogits);
    });
}

}  // namespace moe
