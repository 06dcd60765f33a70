// Routing by scores: experts and gates of every token from its logits, where what decides is not the logit but its score
// (softmax or sigmoid) plus a balancing bias, within the best groups of experts; the gradient of the gates; and the step of the
// bias.
//
// Scores decide what is selected, so they are rounded to fp32 once, from 64 bits: two programs that follow the definition then
// select the same experts.
#include <type_traits>

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

// What an expert or a group is ranked by, as one number: its value, and in the bits behind fp32's its index, so that of equal ones
// the lower index is the larger number.  Infinity as 2^128, which leaves those bits free.
__device__ __forceinline__ double rank_key(float value, int e) {
    uint64_t b = __builtin_bit_cast(uint64_t, fmin((double)(value + 0.f), 0x1p128));   // -0 to +0
    b |= (uint64_t)(value < 0.f ? e : 255 - e);
    return __builtin_bit_cast(double, b);
}
// score and bias; not NaN, -inf or the lowest number
__device__ __forceinline__ double select_key(float choice, int e) { return choice > -__FLT_MAX__ ? rank_key(choice, e) : kNever; }
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

// ---- any number of experts a token ----
constexpr int kSelectWaves = 4;

// Token t by a wave, any groups, scores in 64 bits.  Lane l holds experts l + 64 j; keys, best: LDS of this wave, 64 VPL each.
// Bound by the vector unit.  262144 tokens x 256 experts, us: 12 experts a token 447 (1057 vector instructions a token), 8 in 4 groups of
// 64 experts 672 (1346, and conflicts in LDS, where a lane reads a group), in 32 groups of 8 555; the bytes take 47 at 6 TB/s.
template <int VPL>
__device__ __forceinline__ void select_token(const SelectArgs& p, int t, int lane, double* keys, double* best) {
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
        for (int j = 0; j < VPL; ++j) keys[lane + 64 * j] = key[j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        double mine[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int g = lane + 64 * j;
            mine[j] = kNever;
            if (g < p.groups) {
                double first = kNever, second = kNever;
#pragma unroll 4
                for (int i = 0; i < size; ++i) {
                    const double k = keys[g * size + i];
                    second = k > first ? first : max_key(second, k);
                    first = max_key(first, k);
                }
                if (first > kNever) {
                    float sum = key_choice(first);
                    if (p.group_best > 1 && second > kNever) sum += key_choice(second);
                    mine[j] = rank_key(fmaxf(sum, -__FLT_MAX__), g);
                }
                best[g] = mine[j];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        int rank[VPL] = {};
        for (int g = 0; g < p.groups; ++g) {
            const double other = best[g];
#pragma unroll
            for (int j = 0; j < VPL; ++j) rank[j] += other > mine[j];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            if (lane + 64 * j < p.groups && rank[j] >= p.topk_groups) best[lane + 64 * j] = kNever;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int e = lane + 64 * j;
            if (e < p.E && !(best[e / size] > kNever)) key[j] = kNever;
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

template <int VPL>
__global__ __launch_bounds__(64 * kSelectWaves) void select_wave_kernel(SelectArgs p) {
    __shared__ double keys[kSelectWaves][64 * VPL], best[kSelectWaves][64 * VPL];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int t = blockIdx.x * kSelectWaves + wave; t < p.T; t += gridDim.x * kSelectWaves)
        select_token<VPL>(p, t, threadIdx.x & 63, keys[wave], best[wave]);
}

// In idx[t][0] of a token whose selection is left to this kernel
constexpr int kDoubtful = -2;

// 64 tokens for every wave; the workgroup's doubtful ones are dealt to its waves.  A chain of some 5 us for each.
template <int VPL>
__global__ __launch_bounds__(64 * kSelectWaves) void select_doubtful_kernel(SelectArgs p) {
    __shared__ double keys[kSelectWaves][64 * VPL], best[kSelectWaves][64 * VPL];
    __shared__ int tokens[64 * kSelectWaves], counts[kSelectWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = blockIdx.x * (64 * kSelectWaves) + (int)threadIdx.x;
    const bool doubtful = t < p.T && p.idx[(size_t)t * p.K] == kDoubtful;
    const uint64_t m = __ballot(doubtful);
    if (lane == 0) counts[wave] = __popcll(m);
    __syncthreads();
    int first = 0, n = 0;
    for (int w = 0; w < kSelectWaves; ++w) {
        first += w < wave ? counts[w] : 0;
        n += counts[w];
    }
    if (doubtful) tokens[first + __popcll(m & ((1ull << lane) - 1))] = t;
    __syncthreads();
    for (int i = wave; i < n; i += kSelectWaves)
        select_token<VPL>(p, __builtin_amdgcn_readfirstlane(tokens[i]), lane, keys[wave], best[wave]);
}

// ---- up to eight experts a token ----
// L lanes to a token, a run of `run` <= VPL experts to a lane (where there are groups: a group).  A lane sorts its keys in
// eights and merges them to its eight largest, and the lanes of a token merge theirs: bitonic networks of v_max_f64 and
// v_min_f64, which run at the full rate and carry the expert's index along in the key.
//
// Bound by the vector unit.  Scores in 64 bits would be half of its work, so they are first formed in fp32, and what was
// selected by them stands if no difference that decided it is within what they may be off; else the wave does it all again
// in 64 bits (a token in some hundreds, of logits that are hardly ever equal: equal keys are always in doubt.  Logits that were rounded
// to bf16 leave a third of the tokens in doubt where no bias tells their experts apart: 262144 x 256 then takes 319 us in 8 groups
// and 243 without, instead of 103 and 98).  LATER: in a launch behind this one, which finds them marked; the code that does it takes a
// fifth of this kernel's time by its registers alone.  262144 tokens x 256 experts in 8 groups, 8 of 4 groups: 101 us, some 160 vector
// instructions a token (75 us of issue; the bytes take 47 at 6 TB/s); with softmax scores 120, 203 instructions.  250 experts, whose
// rows are not read in fours, 172 with as many instructions, the rest of it waiting.  A token to a wave with all scores in 64 bits took 449.
// Keys up to here belong to experts that are not selected.  (Their low bits make them smaller.)
constexpr double kLow = -(double)__FLT_MAX__;

__device__ __forceinline__ double min_key(double a, double b) {
    double r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ void order(double& a, double& b) {   // the larger one first
    const double hi = max_key(a, b), lo = min_key(a, b);
    a = hi;
    b = lo;
}
// eight keys in descending order (odd-even merging: 19 comparisons)
__device__ __forceinline__ void sort8(double* v) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) order(v[i], v[i + 1]);
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        order(v[i], v[i + 2]);
        order(v[i + 1], v[i + 3]);
        order(v[i + 1], v[i + 2]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) order(v[i], v[i + 4]);
    order(v[2], v[4]);
    order(v[3], v[5]);
    order(v[1], v[2]);
    order(v[3], v[4]);
    order(v[5], v[6]);
}
// the eight largest of two descending eights, descending: a is the one, b the other; next: the largest key left out so far
__device__ __forceinline__ void merge8(double (&a)[8], const double (&b)[8], double& next) {
    double out[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        out[i] = min_key(a[i], b[7 - i]);
        a[i] = max_key(a[i], b[7 - i]);
    }
#pragma unroll
    for (int d = 4; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < d; ++i) out[i] = max_key(out[i], out[i + d]);
    next = max_key(next, out[0]);
#pragma unroll
    for (int d = 4; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((i & d) == 0) order(a[i], a[i + d]);
}
// the same of a lane's list and that of its partner: neighbouring lanes, pairs, fours and eights
template <int CTRL>
__device__ __forceinline__ void merge_lanes(double (&a)[8], double& next) {
    double b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = dpp<CTRL>(a[i]);
    next = max_key(next, dpp<CTRL>(next));
    merge8(a, b, next);
}

// How far apart two keys are that fp32 scores tell apart for certain: either bound is enough.
// A sigmoid 1 / (1 + x), x = 2^(c v): the product is off by 1.22 * 2^-24 of itself (its rounding and c's), which moves the score by
// s (1 - s) |v| of that, at most 0.28 * 2^-24; x by 2^-23 of itself, s (1 - s) of that, 0.5 * 2^-24; the sum by 2^-24; the reciprocal by
// 2^-23: together less than 2^-22, with the definition's rounding 1.13 * 2^-22.  Key = score + bias adds 2^-23 of itself, in
// both.  Two keys: 1.13 * 2^-21 + 2^-22 of the smaller one, for which stand 2^-20 and 2^-21.  (With 2^-18
// for both, which a softmax needs, one token in 180 was done again and not one in 900: 262144 x 256 119 us instead of 114.)  Far from 0 the score itself
// is small, and off by less than 2^-17 of itself (|v| up to 88).
// A softmax's probability is off by less than 2^-17 of itself (the rounding of the exponential's argument, and the sum's 32 terms), and by
// less than 2^-19 altogether.
// Equal keys are always in doubt, so a key carries its expert's number in any order.
template <bool SIGMOID>
struct Doubt {
    double part, least, own_part, own_least;
    __device__ __forceinline__ Doubt(bool biased)
        : part(SIGMOID ? 0x1p-21 : 0x1p-18), least(SIGMOID ? 0x1p-20 : 0x1p-18), own_part(biased ? part : 0x1p-16),
          own_least(biased ? least : 0x1p-126) {}
    __device__ __forceinline__ double of(double magnitude) const {
        return fmin(fma(magnitude, part, least), fma(magnitude, own_part, own_least));
    }
    __device__ __forceinline__ bool apart(double large, double small) const { return large - small > of(fabs(small)); }
};

// exp(d) for d <= 0 to about a unit in the last place: the product's rounding is made up for
__device__ __forceinline__ float exp_near(float d) {
    d = fmaxf(d, -150.f);   // 0 from there on, and the lines below would take infinities apart
    const float hi = d * 1.44269502f, lo = fmaf(d, 1.44269502f, -hi) + d * 1.92596303e-8f;
    const float e = __builtin_amdgcn_exp2f(hi);
    return fmaf(e, lo * 0.693147181f, e);
}

template <int VPL, int L, bool VEC, bool SIGMOID, bool LATER>
__global__ __launch_bounds__(256, 4) void select_lists_kernel(SelectArgs p, int run) {
    constexpr int TOKENS = 256 / L, SLOTS = (8 + L - 1) / L, LDB = VPL + 4;
    __shared__ __attribute__((aligned(16))) float biases[L * LDB];   // 4 more floats a lane: other banks
    __shared__ double keys[4][LATER ? 1 : kMaxExperts], best[4][LATER ? 1 : kMaxExperts];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int sub = lane & (L - 1), e0 = sub * run;
    const int mine = min(run, p.E - e0);   // experts of this lane; none, or fewer, in the last lanes
    const bool biased = p.bias != nullptr;
    for (int i = threadIdx.x; i < L * VPL; i += 256) {
        const int l = i / VPL, j = i % VPL, e = l * run + j;
        const float b = biased && j < run && e < p.E ? p.bias[e] : 0.f;
        biases[l * LDB + j] = b == b ? fminf(fmaxf(b, -__FLT_MAX__), __FLT_MAX__) : -__FLT_MAX__;   // a score adds nothing to these
    }
    const Doubt<SIGMOID> doubt(biased);
    __syncthreads();
    auto lanes = [](auto v, auto&& f) {
        if constexpr (L > 1) v = f(v, dpp<0xB1>(v));
        if constexpr (L > 2) v = f(v, dpp<0x4E>(v));
        if constexpr (L > 4) v = f(v, dpp<0x141>(v));
        if constexpr (L > 8) v = f(v, dpp<0x140>(v));
        return v;
    };
    auto add = [](auto a, auto b) { return a + b; };
    for (int t0 = blockIdx.x * TOKENS; t0 < p.T; t0 += gridDim.x * TOKENS) {   // uniform trip count: lanes work together
        const int t = t0 + (int)threadIdx.x / L;
        const bool valid = t < p.T;
        const float* const row = p.logits + (size_t)(valid ? t : p.T - 1) * p.E;
        float x[VPL];
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < VPL; j += 4) {
                f32x4 v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                if (j < mine) v = *reinterpret_cast<const f32x4*>(row + e0 + j);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[j + q] = v[q];
            }
        } else {
#pragma unroll
            for (int j = 0; j < VPL; ++j) x[j] = j < mine ? row[e0 + j] : -INFINITY;
        }
        // keys from scores in fp32
        float m = -INFINITY;
        double z = 1.;
        float rz = 1.f;
        if constexpr (!SIGMOID) {
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                x[j] = x[j] > -INFINITY ? fminf(x[j], __FLT_MAX__) : -INFINITY;   // of infinite ones the differences are 0
                m = fmaxf(m, x[j]);
            }
            m = lanes(m, [](float a, float b) { return fmaxf(a, b); });
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                const float e = exp_near(x[j] - m);          // 0 for -inf
                sum += e;
                x[j] = x[j] > -INFINITY ? e : -INFINITY;     // from here on
            }
            z = lanes((double)sum, add);
            rz = 1.f / (float)z;
            if (!p.renorm) {   // the gates' divisor: 32 terms of very different sizes lose too much in fp32
                z = 0.;
#pragma unroll
                for (int j = 0; j < VPL; ++j) z += (double)fmaxf(x[j], 0.f);
                z = lanes(z, add);
            }
        }
        int at = sub * LDB;
        asm volatile("" : "+v"(at));   // or the biases are kept in registers over all tokens
        // the lane's eight largest, and the largest behind them
        double list[8], next = kLow;
#pragma unroll
        for (int j = 0; j < VPL; j += 8) {
            __builtin_amdgcn_sched_barrier(0);   // eight keys at a time, not all of them: registers
            double key[8];
#pragma unroll
            for (int q = 0; q < 8; q += 4) {
                const f32x4 b = *reinterpret_cast<const f32x4*>(&biases[at + j + q]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v = x[j + q + i];
                    const float s = SIGMOID ? __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504f)) : v * rz;
                    float choice = s + b[i];
                    asm("" : "+v"(choice));              // a select below, and no branch around the exponential
                    choice = v > -INFINITY ? choice : -__FLT_MAX__;
                    key[q + i] = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, (double)choice) | (uint64_t)(j + q + i));
                }
            }
            sort8(key);
            if (j == 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) list[i] = key[i];
            } else {
                merge8(list, key, next);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)   // the lane beside the place in its run
            list[i] = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, list[i]) | (uint64_t)(sub * 32));
        // among infinite logits the largest finite one would count as infinite
        bool sure = SIGMOID || m < __FLT_MAX__, keep = true;
        if (p.groups > 1) {
            // this lane's group: its value, its rank, and the largest value that ranks behind it
            float total = key_choice(list[0]), size = list[0] > kLow ? fabsf(total) : 0.f;
            if (p.group_best > 1 && list[1] > kLow) {
                const float second = key_choice(list[1]);
                total += second;
                size += fabsf(second);
            }
            size = lanes(size, [](float a, float b) { return fmaxf(a, b); });
            sure &= size < 1e30f;                            // sums that may overflow
            if (!(list[0] > kLow)) total = -INFINITY;
            int rank = 0;
            float below = -INFINITY;
#pragma unroll
            for (int d = 1; d < L; ++d) {
                const float other = __shfl_xor(total, d, 64);
                const bool ahead = other > total || (other == total && (sub ^ d) < sub);
                rank += ahead;
                below = ahead ? below : fmaxf(below, other);
            }
            keep = rank < p.topk_groups && total > -INFINITY;
            // a sum may be far smaller than what was added up
            if (rank == p.topk_groups - 1 && below > -INFINITY)
                sure &= (double)total - (double)below > 2. * doubt.of((double)size);
            if (!keep) {
#pragma unroll
                for (int i = 0; i < 8; ++i) list[i] = kLow;
                next = kLow;
            }
        }
        if constexpr (L > 1) merge_lanes<0xB1>(list, next);
        if constexpr (L > 2) merge_lanes<0x4E>(list, next);
        if constexpr (L > 4) merge_lanes<0x141>(list, next);
        if constexpr (L > 8) merge_lanes<0x140>(list, next);
        // neighbours among the first K and the one behind them
#pragma unroll
        for (int k = 1; k <= 8; ++k) {
            const double key = k < 8 ? list[k] : next;
            if (k <= p.K && key > kLow) sure &= doubt.apart(list[k - 1], key);
        }
        const uint64_t unsure = __ballot(!sure && valid);
        // slot k in lane k mod L
        double g[SLOTS], sum = 0.;
        int e[SLOTS];
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            const int k = sub + L * i;
            double found = kLow;
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (q == k) found = list[q];
            const int place = (int)(__builtin_bit_cast(uint64_t, found) & 0x1ffu);   // 32 times the lane, and in its run
            e[i] = k < p.K && found > kLow ? (place >> 5) * run + (place & 31) : -1;
            g[i] = 0.;
            if (e[i] >= 0) g[i] = SIGMOID ? sigmoid64(row[e[i]]) : shifted_exp64(fminf(row[e[i]], __FLT_MAX__), m);
            sum += g[i];
        }
        if (p.renorm) z = lanes(sum, add);
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            const int k = sub + L * i;
            if (!valid || k >= p.K) continue;
            if (LATER && k == 0 && (unsure >> (lane & ~(L - 1)) & ((1ull << L) - 1))) e[i] = kDoubtful;
            p.idx[(size_t)t * p.K + k] = e[i];
            p.gate[(size_t)t * p.K + k] = z > 0. ? (float)(g[i] / z * (double)p.scale) : 0.f;
        }
        // tokens in doubt once more, by the whole wave and in 64 bits
        if constexpr (LATER) continue;
        for (int first = 0; unsure && first < 64; first += L)
            if (unsure >> first & ((1ull << L) - 1)) select_token<kMaxExperts / 64>(p, t0 + (wave * 64 + first) / L, lane, keys[wave], best[wave]);
    }
}

// From so many tokens and logits on the doubtful tokens get a launch of their own, which takes 5 to 8 us.  us, in the same launch / so,
// sigmoid: 256 experts in 8 groups, 65536 tokens 35.6 / 38.6, 131072 tokens 55.5 / 56.5, 262144 tokens 104 / 99; 64 experts, 65536 tokens 15.0
// / 15.2, 131072 tokens 23.6 / 22.3, 1048576 tokens 152 / 133; 8 experts, 131072 tokens 7.6 / 9.7, 1048576 tokens 22.0 / 20.3.  (Measured
// with a wave's doubtful tokens one after the other; dealt to the workgroup's waves, 262144 tokens of 256 take 7 us less.)
constexpr int kLaterTokens = 1 << 17;
constexpr int64_t kLaterLogits = 1 << 23;

template <int VPL, int L>
bool launch_lists_of(const SelectArgs& p, int run, hipStream_t s) {
    const int grid = min((p.T + 256 / L - 1) / (256 / L), 256 * 8);
    auto go = [&](auto vec, auto sigmoid, auto later) {
        hipLaunchKernelGGL((select_lists_kernel<VPL, L, decltype(vec)::value, decltype(sigmoid)::value, decltype(later)::value>), dim3(grid),
                           dim3(256), 0, s, p, run);
    };
    const std::true_type yes;
    const std::false_type no;
    if (run % 4 == 0 && p.E % 4 == 0) {
        if (p.T >= kLaterTokens && (int64_t)p.T * p.E >= kLaterLogits) {
            p.sigmoid ? go(yes, yes, yes) : go(yes, no, yes);
            const dim3 rest((p.T + 64 * kSelectWaves - 1) / (64 * kSelectWaves)), block(64 * kSelectWaves);
            if (p.E <= 64) hipLaunchKernelGGL(select_doubtful_kernel<1>, rest, block, 0, s, p);
            else hipLaunchKernelGGL(select_doubtful_kernel<4>, rest, block, 0, s, p);
        } else {
            p.sigmoid ? go(yes, yes, no) : go(yes, no, no);
        }
    } else {
        p.sigmoid ? go(no, yes, no) : go(no, no, no);
    }
    return true;
}

// false where the groups do not fit the lanes
bool launch_lists(const SelectArgs& p, hipStream_t s) {
    int L = 1, run;
    if (p.groups > 1) {
        while (L < p.groups) L <<= 1;
        run = p.E / p.groups;
    } else {
        while (L < 8 && p.E > 8 * L) L <<= 1;
        run = ((p.E + L - 1) / L + 3) & ~3;
    }
    if (L > 16 || run > 32) return false;
    auto of = [&](auto vpl) {
        constexpr int VPL = decltype(vpl)::value;
        return L <= 2 ? launch_lists_of<VPL, 2>(p, run, s) : L == 4 ? launch_lists_of<VPL, 4>(p, run, s)
             : L == 8 ? launch_lists_of<VPL, 8>(p, run, s) : launch_lists_of<VPL, 16>(p, run, s);
    };
    if (L == 1) return launch_lists_of<8, 1>(p, run, s);   // up to eight experts
    if (run <= 8) return of(std::integral_constant<int, 8>{});
    if (run <= 16) return of(std::integral_constant<int, 16>{});
    return of(std::integral_constant<int, 32>{});
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

// 2^64 exp(d) for d <= 0, as near: what the hardware's exponential would take for 0, fp32's denormal numbers, is there with all its bits
__device__ __forceinline__ float exp_lifted(float d) {
    d = fmaxf(d, -150.f);
    const float hi = d * 1.44269502f, up = hi + 64.f, lo = fmaf(d, 1.44269502f, -hi) + fmaf(d, 1.92596303e-8f, hi - (up - 64.f));
    const float e = __builtin_amdgcn_exp2f(up);
    return fmaf(e, lo * 0.693147181f, e);
}
__device__ __forceinline__ float exp_gradual(float d) { return exp_lifted(d) * 0x1p-64f; }

// Selected scores that are 0 in 64 bits, where sigmoid and softmax are formed forward: logits, and logits against the row's largest,
// from here down
constexpr float kNoSigmoid = -709.7827f, kNoSoftmax = -745.133f;

// f over N consecutive lanes (a power of two), in all of them
template <typename F>
__device__ __forceinline__ float lanes_fold(float v, int N, F&& f) {
    for (int d = 1; d < N; d <<= 1) v = f(v, __shfl_xor(v, d, 64));
    return v;
}

// TW tokens to a wave: 8 of up to 8 slots, 4 of up to 64.  The slots' work, of which there is little, is dealt over the wave, 64 / TW
// lanes to a token; the rows of dlogits are put together in LDS and written in one piece, which starts at a multiple of 16
// bytes whatever E is.  Bound by that write (softmax: and by the read of the logits).  262144 tokens x 256 experts, 8 slots, sigmoid: 74
// us for 294 MB, 420 with the 64-byte sectors around the logits it picks (5.7 TB/s); every lane storing for itself took 164.  Softmax: 180
// us for 554 MB, 244 vector instructions a token (112 us of issue) in four waves a SIMD, as many as LDS has room for.
template <bool SIGMOID, int TW, bool STREAM>
__global__ __launch_bounds__(256) void select_dlogits_kernel(SelectBackwardArgs p) {
    constexpr int PER = 64 / TW, SLOTS = TW == 8 ? 1 : 4;
    extern __shared__ __attribute__((aligned(16))) float rows_of_waves[];
    __shared__ float totals[4][TW], largest[4][TW];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t0 = (blockIdx.x * 4 + wave) * TW, E = p.E;
    if (t0 >= p.T) return;
    const int nt = min(TW, p.T - t0);
    float* const rows = rows_of_waves + wave * (TW * E);
    const size_t base = (size_t)t0 * E;
    auto add = [](float a, float b) { return a + b; };
    auto max_of = [](float a, float b) { return fmaxf(a, b); };
    auto sync = [] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    // softmax: probabilities, L lanes to a token, experts q + L i of lane q, 64 / L tokens at a time; 0 of experts that are not open
    constexpr int PASSES = SIGMOID ? 1 : TW;
    int L = 1;
    float prob[PASSES][4];
    if constexpr (!SIGMOID) {
        while (4 * L < E) L <<= 1;
        const int q = lane & (L - 1), at = lane / L, step = 64 / L;
#pragma unroll
        for (int s = 0; s < PASSES; ++s) {
            if (s * step >= TW) continue;
            const int t = s * step + at;
            const bool in = t < nt;                          // the same for the lanes of a token
            float m = -INFINITY, z = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                prob[s][i] = in && q + L * i < E ? p.logits[base + (size_t)t * E + q + L * i] : -INFINITY;
                m = fmaxf(m, prob[s][i]);                    // of NaN and a number the number
            }
            m = lanes_fold(m, L, max_of);
            if (q == 0 && t < TW) largest[wave][t] = m;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = prob[s][i];
                prob[s][i] = x > -INFINITY ? (x == m ? 0x1p64f : exp_lifted(x - m)) : 0.f;   // the sum cancels the factor
                z += prob[s][i];
            }
            z = lanes_fold(z, L, add);
            const float rz = z > 0.f ? 1.f / z : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                prob[s][i] *= rz;
                if (t < TW && q + L * i < E) rows[t * E + q + L * i] = prob[s][i];
            }
        }
        sync();
    }
    // slots sub, sub + PER, ..: expert, score, 1 - score (sigmoid), gradient of the gate
    const int tok = lane / PER, sub = lane % PER;
    int e[SLOTS];
    float l[SLOTS], s[SLOTS], rest[SLOTS], d[SLOTS], sum = 0.f, top = -INFINITY;
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        const int k = sub + PER * j;
        e[j] = -1;
        l[j] = -INFINITY;
        s[j] = d[j] = 0.f;
        rest[j] = 1.f;
        if (k < p.K && tok < nt) {
            const size_t slot = (size_t)(t0 + tok) * p.K + k;
            const int i = p.idx[slot];
            if ((unsigned)i < (unsigned)E) {
                l[j] = p.logits[base + (size_t)tok * E + i];
                if (l[j] > -INFINITY) {
                    e[j] = tok * E + i;
                    d[j] = p.dgate[slot] * p.scale;
                    top = fmaxf(top, l[j]);
                }
            }
        }
    }
    // Of renormalised gates only the scores' ratios count: they are formed against the largest of the token's, so that small ones,
    // which the forward has in 64 bits, keep theirs
    if (p.renorm) top = lanes_fold(top, PER, max_of);
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        if (e[j] >= 0) {
            if constexpr (SIGMOID) {
                const float x = exp_gradual(-fabsf(l[j])), r = 1.f / (1.f + x);
                s[j] = l[j] >= 0.f ? r : p.renorm ? exp_gradual(l[j] - fminf(top, 0.f)) * r : x * r;
                rest[j] = l[j] >= 0.f ? x * r : r;
                if (p.renorm && !(top > kNoSigmoid)) s[j] = 0.f;
            } else if (p.renorm) {
                const float m = largest[wave][tok];
                if (top == m || top - m > kNoSoftmax) s[j] = l[j] == top ? 1.f : exp_gradual(l[j] - top);
            } else {
                s[j] = rows[e[j]];
            }
        }
        sum += s[j];
    }
    // c: gradient of the logarithm of the score, times 1 - score (sigmoid)
    float c[SLOTS], total = 0.f, mean = 0.f;
    if (p.renorm) {
        sum = lanes_fold(sum, PER, add);
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
            s[j] = sum > 0.f ? s[j] / sum : 0.f;
            mean += d[j] * s[j];
        }
        mean = lanes_fold(mean, PER, add);
    }
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        c[j] = e[j] >= 0 ? (d[j] - mean) * s[j] : 0.f;
        total += c[j];
        c[j] *= rest[j];
    }
    // an expert named twice by a token: of the slots that leave their number at its place, one finds another's there
    sync();
#pragma unroll
    for (int j = 0; j < SLOTS; ++j)
        if (e[j] >= 0) rows[e[j]] = __int_as_float(lane * SLOTS + j);
    sync();
    bool twice = false;
#pragma unroll
    for (int j = 0; j < SLOTS; ++j)
        if (e[j] >= 0) twice |= __float_as_int(rows[e[j]]) != lane * SLOTS + j;
    sync();
    if constexpr (SIGMOID) {
        for (int i = lane; i < TW * E / 4; i += 64) reinterpret_cast<f32x4*>(rows)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    } else {
        total = lanes_fold(total, PER, add);
        if (sub == 0) totals[wave][tok] = total;
        sync();
        const int q = lane & (L - 1), at = lane / L, step = 64 / L;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int t = i * step + at;
            if (i * step >= TW || t >= TW) continue;
            const float of = totals[wave][t];
#pragma unroll
            for (int n = 0; n < 4; ++n)
                if (q + L * n < E) rows[t * E + q + L * n] = -prob[i][n] * of;
        }
    }
    sync();
    if (__ballot(twice) == 0) {
#pragma unroll
        for (int j = 0; j < SLOTS; ++j)
            if (e[j] >= 0) rows[e[j]] += c[j];
    } else {   // one after the other
#pragma unroll
        for (int j = 0; j < SLOTS; ++j)
            for (int k = 0; k < PER; ++k) {
                if (sub == k && e[j] >= 0) rows[e[j]] += c[j];
                sync();
            }
    }
    sync();
    const int n = nt * E;
    float* const out = p.dlogits + base;
    for (int i = 4 * lane; i < n; i += 256) {
        f32x4 v = *reinterpret_cast<const f32x4*>(rows + i);
        if (i + 4 <= n) {
            if (p.addend) v += *reinterpret_cast<const f32x4*>(p.addend + base + i);
            if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<f32x4*>(out + i));
            else *reinterpret_cast<f32x4*>(out + i) = v;
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (i + q < n) out[i + q] = v[q] + (p.addend ? p.addend[base + i + q] : 0.f);
        }
    }
}

// ---- the step of the bias ----
// A chain of loads: rows of counts are dealt to four groups of threads, and each has all its loads in flight (a row of 64 experts 2.7
// us in the kernel; 4096 rows of 256 4.8 and 3.6, one load after another 24 together).
constexpr int kBiasRows = 64;   // rows of counts that a workgroup adds up

// sum of rows [r0, r0 + kBiasRows) below n_rows of column e, for threads e < 256 (the first group)
template <typename N>
__device__ __forceinline__ int64_t column_sum(const N* __restrict__ rows, int r0, int n_rows, int E, int64_t (&part)[4][256]) {
    const int e = threadIdx.x & 255, g = threadIdx.x >> 8;
    N v[kBiasRows / 4];
#pragma unroll
    for (int i = 0; i < kBiasRows / 4; ++i) {
        const int r = r0 + 4 * i + g;
        v[i] = e < E && r < n_rows ? rows[(size_t)r * E + e] : 0;
    }
    int64_t n = 0;
#pragma unroll
    for (int i = 0; i < kBiasRows / 4; ++i) n += v[i];
    part[g][e] = n;
    __syncthreads();
    n = part[0][e] + part[1][e] + part[2][e] + part[3][e];
    __syncthreads();
    return n;
}

// sums[b][e] = sum of a workgroup's rows
__global__ __launch_bounds__(1024) void bias_sum_kernel(const int32_t* __restrict__ counts, int n_rows, int E,
                                                        int64_t* __restrict__ sums) {
    __shared__ int64_t part[4][256];
    const int64_t n = column_sum(counts, blockIdx.x * kBiasRows, n_rows, E, part);
    if ((int)threadIdx.x < E) sums[(size_t)blockIdx.x * E + threadIdx.x] = n;
}

// bias[e] += rate * sign(sum_j n_j - E n_e), n the sums of n_rows rows
template <typename N>
__global__ __launch_bounds__(1024) void bias_step_kernel(const N* __restrict__ rows, int n_rows, int E, float rate,
                                                         float* __restrict__ bias) {
    __shared__ int64_t part[4][256];
    const int e = threadIdx.x;
    const float before = e < E ? bias[e] : 0.f;
    int64_t n = 0;
    for (int r = 0; r < n_rows; r += kBiasRows) n += column_sum(rows, r, n_rows, E, part);
    const int64_t sum = wave_sum(e < E ? n : 0);
    if ((e & 63) == 0 && e < 256) part[0][e >> 6] = sum;
    __syncthreads();
    const int64_t off = part[0][0] + part[0][1] + part[0][2] + part[0][3] - (int64_t)E * n;
    if (e < E && off != 0) bias[e] = before + (off > 0 ? rate : -rate);
}

}  // namespace

void launch_select(const float* logits, const float* bias, int T, int E, int K, moe_score_t score, int groups, int topk_groups,
                   int group_best, int renorm, float scale, int32_t* idx, float* gate, hipStream_t s) {
    const SelectArgs p = {logits, bias, idx, gate, scale, T, E, K, score == MOE_SCORE_SIGMOID, groups, topk_groups, group_best, renorm};
    if (K <= 8 && launch_lists(p, s)) return;
    const dim3 grid(min((T + kSelectWaves - 1) / kSelectWaves, 1 << 20)), block(64 * kSelectWaves);
    if (E <= 64) hipLaunchKernelGGL(select_wave_kernel<1>, grid, block, 0, s, p);
    else if (E <= 128) hipLaunchKernelGGL(select_wave_kernel<2>, grid, block, 0, s, p);
    else hipLaunchKernelGGL(select_wave_kernel<4>, grid, block, 0, s, p);
}

void launch_select_dlogits(const float* logits, const int32_t* idx, const float* dgate, const float* addend, int T, int E, int K,
                           moe_score_t score, int renorm, float scale, float* dlogits, hipStream_t s) {
    // streamed where what follows would not find them in the 256 MB cache (262144 tokens x 256 experts: 84 us, streamed 74)
    const bool stream = (size_t)T * E * sizeof(float) > kCachedBytes;
    const SelectBackwardArgs p = {logits, idx, dgate, addend, dlogits, scale, T, E, K, score == MOE_SCORE_SIGMOID, renorm};
    const int tw = K <= 8 ? 8 : 4;
    auto pick = [&](auto st) {
        constexpr bool S = decltype(st)::value;
        return K <= 8 ? (p.sigmoid ? select_dlogits_kernel<true, 8, S> : select_dlogits_kernel<false, 8, S>)
                      : (p.sigmoid ? select_dlogits_kernel<true, 4, S> : select_dlogits_kernel<false, 4, S>);
    };
    const auto kern = stream ? pick(std::true_type{}) : pick(std::false_type{});
    hipLaunchKernelGGL(kern, dim3((unsigned)((T + 4ll * tw - 1) / (4 * tw))), dim3(256), (size_t)4 * tw * E * sizeof(float), s, p);
}

size_t bias_update_workspace_bytes(int n_rows, int E) {
    return n_rows <= kBiasRows ? 0 : (size_t)((n_rows + kBiasRows - 1) / kBiasRows) * E * sizeof(int64_t);
}

void launch_bias_update(const int32_t* counts, int n_rows, int E, float rate, float* bias, void* ws, hipStream_t s) {
    if (n_rows <= kBiasRows) {
        hipLaunchKernelGGL(bias_step_kernel<int32_t>, dim3(1), dim3(1024), 0, s, counts, n_rows, E, rate, bias);
        return;
    }
    const int parts = (n_rows + kBiasRows - 1) / kBiasRows;
    int64_t* part = static_cast<int64_t*>(ws);
    hipLaunchKernelGGL(bias_sum_kernel, dim3(parts), dim3(1024), 0, s, counts, n_rows, E, part);
    hipLaunchKernelGGL(bias_step_kernel<int64_t>, dim3(1), dim3(1024), 0, s, part, parts, E, rate, bias);
}

}  // namespace moe
