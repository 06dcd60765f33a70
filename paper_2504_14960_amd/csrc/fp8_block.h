// E4M3 with a scale for every block of 128: a power of two, as E8M0 (a byte b stands for 2^(b-127), 255 for NaN).
//
// Powers of two, because the scaled matrix instruction multiplies both operands' E8M0 scales in on the way: a block of 128 along
// the contraction is the instruction's whole depth, so scaling costs no vector instruction, where any other scale would cost
// a fused multiply-add for every accumulator and block.  And what a code and its scale stand for has four significant bits, so
// it is a bf16 value too, and the weight gradients multiply exactly what the forward did: from a scale of 2^-124 on, with which the
// smallest code is bf16's smallest value, 2^-133.  With 2^-125 and 2^-126 what lies below that is rounded.
#pragma once

#include "common.h"
#include "wave_sum.h"

namespace moe {

constexpr int kBlock = 128;
typedef __attribute__((ext_vector_type(8))) int i32x8;

// Bytes of a row of scales for C values: whole words, so that four of them are one load.
__host__ __device__ inline int block_scale_stride(int C) { return (C / kBlock + 3) & ~3; }

constexpr uint32_t kNotFinite = 0x7f800000u;   // magnitudes as bits from here on are infinity or NaN

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The scale of a block whose largest magnitude has these bits: the smallest power of two, from 2^-126, that leaves at most 448
// (1.75 * 2^8: the exponent goes up where the fraction is above 0.75); 255 where a value is not finite.
__device__ __forceinline__ uint32_t block_scale(uint32_t top) {
    const int b = (int)((top + 0x1fffffu) >> 23) - 8;
    return top >= kNotFinite ? 255u : (uint32_t)max(b, 1);
}
// what the block's values are multiplied with; any number for 255
__device__ __forceinline__ float block_inverse(uint32_t scale) { return __uint_as_float((254u - min(scale, 254u)) << 23); }
// what a scale stands for; infinity for 255, whose codes are NaN
__device__ __forceinline__ float block_value(uint32_t scale) { return __uint_as_float(scale ? scale << 23 : 0x400000u); }

// four values of a block to their nearest codes, ties to even (the scale leaves at most 448: nothing to clamp)
__device__ __forceinline__ uint32_t block_codes(float a, float b, float c, float d, float inverse, uint32_t scale) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, r, true);
    return scale == 255u ? 0x7f7f7f7fu : (uint32_t)r;
}

// 16 bytes of bf16 as eight floats
__device__ __forceinline__ void bf16x8_to_f32(const u32x4& v, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[2 * j] = __uint_as_float(v[j] << 16);
        f[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
    }
}

// the largest magnitude over the 16 lanes of a row of the wave, in all of them
__device__ __forceinline__ uint32_t max16(uint32_t v) {
    v = max(v, dpp<0x121>(v));   // row_ror 1, 2, 4, 8
    v = max(v, dpp<0x122>(v));
    v = max(v, dpp<0x124>(v));
    return max(v, dpp<0x128>(v));
}

// the largest magnitude over the lanes that are congruent modulo 16, in all of them
__device__ __forceinline__ uint32_t max_rows(uint32_t v) {
    auto larger = [](uint32_t a, uint32_t b) { return max(a, b); };
    return with_swapped<true>(with_swapped<false>(v, larger), larger);
}

// eight values of a block that 16 neighbouring lanes hold: their codes, and the block's scale
__device__ __forceinline__ u32x2 quantize8(const float (&f)[8], uint32_t& scale) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, magnitude(f[j]));
    scale = block_scale(max16(top));
    const float inv = block_inverse(scale);
    return u32x2{block_codes(f[0], f[1], f[2], f[3], inv, scale), block_codes(f[4], f[5], f[6], f[7], inv, scale)};
}

template <bool BF16, bool STREAM = false>
__device__ __forceinline__ void load8(const void* src, size_t at, float (&f)[8]) {
    if constexpr (BF16) {
        const u32x4* from = reinterpret_cast<const u32x4*>(static_cast<const bf16_t*>(src) + at);
        bf16x8_to_f32(STREAM ? __builtin_nontemporal_load(from) : *from, f);
    } else {
        const f32x4 lo = *reinterpret_cast<const f32x4*>(static_cast<const float*>(src) + at);
        const f32x4 hi = *reinterpret_cast<const f32x4*>(static_cast<const float*>(src) + at + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f[j] = lo[j];
            f[4 + j] = hi[j];
        }
    }
}

// Rows 0 .. n - 1, one to a wave, 512 values at a time, by workgroup `block` of `blocks` of four waves (16384 rows of 6144 bf16, in
// block_prepare_kernel: 54 us, 5.6 TB/s)
template <bool BF16>
__device__ __forceinline__ void block_quantize_rows(const void* __restrict__ src, int n, int C, uint8_t* __restrict__ codes,
                                                    uint8_t* __restrict__ scales, int block, int blocks) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, stride = block_scale_stride(C);
    for (int r = block * 4 + wave; r < n; r += blocks * 4)
        for (int c0 = 0; c0 < C; c0 += 512) {   // uniform trip count: shuffles inside
            const int c = c0 + 8 * lane;
            float f[8] = {};
            if (c < C) load8<BF16>(src, (size_t)r * C + c, f);
            uint32_t scale;
            const u32x2 q = quantize8(f, scale);
            if (c >= C) continue;
            *reinterpret_cast<u32x2*>(codes + (size_t)r * C + c) = q;
            if ((lane & 15) == 0) scales[(size_t)r * stride + c / kBlock] = (uint8_t)scale;
        }
}
inline int block_quantize_grid(int rows) { return (int)min((rows + 3ll) / 4, 256ll * 16); }

// What the grouped products of the block-scaled expert FFN work on: C = A [rows, K] . B[e]^T over the rows of every expert
struct BlockGemm {
    const uint8_t* A;             // codes [rows, K]
    const uint8_t* a_scales;      // [rows, stride(K)]
    const int32_t* offsets;
    const uint8_t *B0, *B1;       // codes [E, N, K]; B1: the up projection
    const uint8_t *b0_scales, *b1_scales;   // [E, N / 128, stride(K)]
    void* C;                      // kBlockPlain: bf16 [rows, N]; kBlockSwiglu: codes [rows, N]; kBlockGrad: codes [rows, 2 N]
    uint8_t* c_scales;            // of the codes
    bf16_t* gu;                   // kBlockSwiglu: g | u [rows, 2 N] out, or null; kBlockGrad: in
    bf16_t* dgu;                  // kBlockGrad: dg | du [rows, 2 N] out
    int E, N, K, r_max;
};
// y = A B0^T; h = silu(A B0^T) * (A B1^T) quantised; dg | du from dh = A B0^T and g | u, in bf16 and quantised
enum { kBlockPlain = 0, kBlockSwiglu = 1, kBlockGrad = 2 };

constexpr int kMaxBlockRow = 1 << 22;   // values of an operand's row: 32-bit offsets inside a tile

void launch_block_gemm(int mode, const BlockGemm& p, hipStream_t s);      // the choice of the kernel
void launch_block_persist(int mode, const BlockGemm& p, hipStream_t s);   // gemm_persist_block.hip: many rows per expert, K >= 256

}  // namespace moe
