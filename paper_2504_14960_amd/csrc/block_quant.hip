// Quantisation to E4M3 with a scale for every block of 128 (fp8_block.h): rows (1 x 128), rows gathered by expert, weights
// (128 x 128) in the layouts of the forward and of the backward.  Bound by memory: every value is read once.
#include <type_traits>

#include "fp8_block.h"

namespace moe {

namespace {

template <bool BF16>
__global__ __launch_bounds__(256) void block_rows_quantize_kernel(const void* __restrict__ src, int rows, int C,
                                                                  uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    block_quantize_rows<BF16>(src, rows, C, codes, scales, blockIdx.x, gridDim.x);
}

// 512 values of a token to a wave, read and quantised once and stored to each of its rows of the expert order.  8192 tokens x 6144,
// 2 rows each: 37 us, 5.5 TB/s.
__global__ __launch_bounds__(256) void permute_copy_block_kernel(const bf16_t* __restrict__ x,
                                                                 const int32_t* __restrict__ row_of_assign, int T, int K, int H,
                                                                 int r_max, uint8_t* __restrict__ codes,
                                                                 uint8_t* __restrict__ scales) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int stride = block_scale_stride(H), pieces = (H + 511) / 512;
    const int64_t items = (int64_t)T * pieces;
    for (int64_t item = (int64_t)blockIdx.x * 4 + wave; item < items; item += (int64_t)gridDim.x * 4) {
        const int t = (int)(item / pieces), c = (int)(item - (int64_t)t * pieces) * 512 + 8 * lane;
        float f[8] = {};
        if (c < H) load8<true>(x, (size_t)t * H + c, f);
        int my_row = lane < K ? row_of_assign[(size_t)t * K + lane] : -1;
        if ((unsigned)my_row >= (unsigned)r_max) my_row = -1;
        uint32_t scale;
        const u32x2 q = quantize8(f, scale);
        for (uint64_t m = __ballot(my_row >= 0); m; m &= m - 1) {
            const int row = __shfl(my_row, __ffsll((unsigned long long)m) - 1, 64);
            if (c >= H) continue;
            *reinterpret_cast<u32x2*>(codes + (size_t)row * H + c) = q;
            if ((lane & 15) == 0) scales[(size_t)row * stride + c / kBlock] = (uint8_t)scale;
        }
    }
}

template <bool STREAM, typename V>
__device__ __forceinline__ void store_codes(uint8_t* to, const V& v) {
    if (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<V*>(to));
    else *reinterpret_cast<V*>(to) = v;
}

// A block of 128 x 128 to a workgroup: w [E, N, K] -> codes [E, N, K] and, transposed, at column t0 of [E, K, ldt]; either may
// be null.  A thread holds eight columns of eight rows.  Bound by HBM.
// A layer's three in one launch, streamed ones in three (us, in three / in one: 12 experts, 1024 x 1408, fp32 72 / 60 (5.2 TB/s); 64,
// 4096 x 1408, bf16, streamed 792 / 817).
// STREAM, past the caches, where the codes that a call writes are more than the memory-side cache keeps: the stores, and the
// loads of bf16 weights (an fp32 thread's two loads share a line, which the first would drop).  The call, us, not streamed /
// so, and with the FFN of 64 rows per expert behind it: 12 experts, 1024 x 1408, fp32 (104 MB of codes) 72 / 67 and 100 / 101;
// 8, 2048 x 2048, bf16 (201 MB) with it 131 / 132; 16, 2048 x 2048, bf16 (403 MB) with it 234 / 216; 8, 4096 x 4096, fp32
// (805 MB) with it 577 / 554, streamed loads too 564; 64, 4096 x 1408, bf16 (2.2 GB) 845 / 788 (5.6 TB/s) and 1080 / 1024.
template <bool BF16, bool STREAM>
__global__ __launch_bounds__(256) void block_weights_kernel(LayerWeights p, int E, int first) {
    __shared__ uint32_t tops[4];
    __shared__ __attribute__((aligned(16))) uint8_t tile[128][128 + 16];   // transposed
    const int z = first + (int)blockIdx.z, which = (z >= E) + (z >= 2 * E), e = z - which * E;
    const auto [w, N, K, codes, scales, codes_t, scales_t, ldt, t0] = p.of[which];
    const bool turned = (int)(gridDim.x * kBlock) != K;   // the down projection in the others' grid
    const int nb = turned ? blockIdx.x : blockIdx.y, kb = turned ? blockIdx.y : blockIdx.x, n0 = nb * kBlock, k0 = kb * kBlock;
    const int cv = threadIdx.x % 16, rv = threadIdx.x / 16;
    float f[8][8];
    uint32_t top = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) load8<BF16, BF16 && STREAM>(w, ((size_t)e * N + n0 + 8 * rv + r) * K + k0 + 8 * cv, f[r]);
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude(f[r][j]));
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    const uint32_t scale = block_scale(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
    const float inv = block_inverse(scale);
    u32x2 q[8];
#pragma unroll
    for (int r = 0; r < 8; ++r)
        q[r] = u32x2{block_codes(f[r][0], f[r][1], f[r][2], f[r][3], inv, scale),
                     block_codes(f[r][4], f[r][5], f[r][6], f[r][7], inv, scale)};
    if (codes) {
#pragma unroll
        for (int r = 0; r < 8; ++r)
            store_codes<STREAM>(codes + ((size_t)e * N + n0 + 8 * rv + r) * K + k0 + 8 * cv, q[r]);
        if (threadIdx.x == 0) scales[((size_t)e * (N / kBlock) + nb) * block_scale_stride(K) + kb] = (uint8_t)scale;
    }
    if (!codes_t) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        u32x2 v = {0u, 0u};
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r / 4] |= (q[r][j / 4] >> (8 * (j % 4)) & 0xffu) << (8 * (r % 4));
        *reinterpret_cast<u32x2*>(&tile[8 * cv + j][8 * rv]) = v;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = 32 * i + threadIdx.x / 8, at = threadIdx.x % 8 * 16;
        store_codes<STREAM>(codes_t + ((size_t)e * K + k0 + c) * ldt + t0 + n0 + at, *reinterpret_cast<const u32x4*>(&tile[c][at]));
    }
    if (threadIdx.x == 0)
        scales_t[((size_t)e * (K / kBlock) + kb) * block_scale_stride(ldt) + t0 / kBlock + nb] = (uint8_t)scale;
}

}  // namespace

void launch_block_quantize(const void* src, moe_dtype_t dt, int rows, int C, void* codes, uint8_t* scales, hipStream_t s) {
    auto kern = dt == MOE_BF16 ? block_rows_quantize_kernel<true> : block_rows_quantize_kernel<false>;
    hipLaunchKernelGGL(kern, dim3(block_quantize_grid(rows)), dim3(256), 0, s, src, rows, C, static_cast<uint8_t*>(codes), scales);
}

void launch_block_weights(moe_dtype_t dt, int E, int H, int F, const LayerWeights& p, hipStream_t s) {
    const size_t codes = (size_t)3 * E * H * F * ((p.of[0].codes != nullptr) + (p.of[0].codes_t != nullptr));
    const bool stream = codes > kCachedBytes;
    auto pick = [&](auto bf16) {
        return stream ? block_weights_kernel<decltype(bf16)::value, true> : block_weights_kernel<decltype(bf16)::value, false>;
    };
    auto kern = dt == MOE_BF16 ? pick(std::true_type{}) : pick(std::false_type{});
    if (stream) {
        for (int i = 0; i < 3; ++i)
            hipLaunchKernelGGL(kern, dim3(p.of[i].K / kBlock, p.of[i].N / kBlock, E), dim3(256), 0, s, p, E, i * E);
    } else {
        hipLaunchKernelGGL(kern, dim3(H / kBlock, F / kBlock, 3 * E), dim3(256), 0, s, p, E, 0);
    }
}

void launch_permute_block(const void* x, const int32_t* idx, int T, int H, int E, int K, int capacity, int r_max, void* codes,
                          uint8_t* scales, int32_t* counts, int32_t* offsets, int32_t* row_of_assign, int32_t* assign_of_row,
                          void* ws, hipStream_t s) {
    if (launch_permute_block_small(x, idx, T, H, E, K, capacity, r_max, codes, scales, counts, offsets, row_of_assign, assign_of_row, s))
        return;
    launch_permute(nullptr, idx, T, H, E, K, capacity, r_max, MOE_BF16, nullptr, counts, offsets, row_of_assign, assign_of_row, ws, s);
    hipLaunchKernelGGL(permute_copy_block_kernel, dim3((unsigned)min(((long long)T * ((H + 511) / 512) + 3) / 4, 256ll * 32)), dim3(256), 0, s,
                       static_cast<const bf16_t*>(x), row_of_assign, T, K, H, r_max, static_cast<uint8_t*>(codes), scales);
}

}  // namespace moe
