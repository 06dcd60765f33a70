// Grouped products of the expert FFN on E4M3 operands with a scale for every block of 128 (fp8_block.h): the weights streamed
// from memory to registers, a few rows per expert at a time.
//
//   C[r, n] = sum_b 2^(sa[r,b] + sb[n/128,b]) sum_{k in b} A[r,k] B[n,k]         (b: blocks of 128 along the contraction)
//
// One 16x16x128 scaled matrix instruction per 16 rows, 16 weight rows and block.
#include "fp8_block.h"
#include "stream_tile.h"

namespace moe {

namespace {

// c += 2^(sa + sb) a . b: the weight fragment comes first, so that a lane holds row lane % 16 of the activations and four
// neighbouring columns of the result
__device__ __forceinline__ f32x4 mfma_block(const Piece& w, const Piece& a, f32x4 c, uint32_t sw, uint32_t sa) {
    i32x8 wv, av;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        wv[i] = (int)w.lo[i];
        wv[4 + i] = (int)w.hi[i];
        av[i] = (int)a.lo[i];
        av[4 + i] = (int)a.hi[i];
    }
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av, c, 0, 0, 0, (int)sw, 0, (int)sa);
}

// Tile of 16 MB rows x 32 CW columns.  A wave has 32 of the columns (of gate and of up); KS waves share them and take the blocks
// along the contraction in turn.
template <int MODE, int MB, int CW, int KS>
__global__ __launch_bounds__(64 * CW * KS) void block_rows_kernel(BlockGemm p) {
    static_assert(MODE == kBlockPlain || CW == 4, "a block of the quantised result");
    constexpr int BM = 16 * MB, FO = 2, FN = MODE == kBlockSwiglu ? 2 * FO : FO;
    __shared__ uint32_t tops[2][4][BM];   // largest magnitude of a wave's columns of every row (kBlockGrad: dg and du)
    __shared__ __attribute__((aligned(16))) f32x4 parts[KS > 1 ? KS - 1 : 1][KS > 1 ? CW * MB * FN : 1][64];
    const int lane = threadIdx.x & 63, id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = id % CW, kpart = id / CW;
    const Tile t = locate_tile<BM>(p.offsets, p.E, p.N / (32 * CW), blockIdx.x);
    if (!t.valid) return;
    const int fr = lane & 15, fk = lane >> 4;
    const int KT = p.K / kBlock, ks = block_scale_stride(p.K);
    const int col0 = (t.ntile * CW + wave) * 32;

    const uint8_t *a[MB], *as[MB], *b[FN];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int r = t.row0 + min(16 * i + fr, t.rows - 1);
        a[i] = p.A + (size_t)r * p.K + 32 * fk;
        as[i] = p.a_scales + (size_t)r * ks;
    }
    const size_t wrow = (size_t)t.expert * p.N + col0 + fr;
#pragma unroll
    for (int j = 0; j < FN; ++j) b[j] = (j < FO ? p.B0 : p.B1) + (wrow + 16 * (j % FO)) * p.K + 32 * fk;
    const size_t srow = ((size_t)t.expert * (p.N / kBlock) + col0 / kBlock) * ks;
    const uint8_t *const bs0 = p.b0_scales + srow, *const bs1 = MODE == kBlockSwiglu ? p.b1_scales + srow : nullptr;

    f32x4 acc[MB][FN];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct Step {
        Piece a[MB], b[FN];
        uint32_t sa[MB], sb[2];
    };
    const int first = rotation(t, KT);   // see there: the order of a row's sum is that of its weight tile and expert
    auto load = [&](Step& s, int n) {
        int k = n + first;
        k = k >= KT ? k - KT : k;
#pragma unroll
        for (int j = 0; j < FN; ++j) s.b[j] = {ld16(b[j] + (size_t)k * kBlock), ld16(b[j] + (size_t)k * kBlock + 16)};
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            s.a[i] = {ld16(a[i] + (size_t)k * kBlock), ld16(a[i] + (size_t)k * kBlock + 16)};
            s.sa[i] = as[i][k];
        }
        s.sb[0] = bs0[k];
        s.sb[1] = MODE == kBlockSwiglu ? bs1[k] : 0u;
    };
    Step cur, next;
    if (kpart < KT) load(cur, kpart);
    for (int n = kpart; n < KT; n += KS) {
        if (n + KS < KT) load(next, n + KS);
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < MB; ++i) acc[i][j] = mfma_block(cur.b[j], cur.a[i], acc[i][j], cur.sb[j / FO], cur.sa[i]);
        cur = next;
    }
    if constexpr (KS > 1) {
        if (kpart > 0) {
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) parts[kpart - 1][(wave * MB + i) * FN + j][lane] = acc[i][j];
        }
        __syncthreads();
        if (kpart > 0 && MODE == kBlockPlain) return;
#pragma unroll
        for (int q = 0; q < KS - 1; ++q)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] += parts[q][(wave * MB + i) * FN + j][lane];
    }
    const bool writes = kpart == 0;   // the other waves go along to the barrier

    // a lane's values: row fr of block i, columns col0 + 16 j + 4 fk .. + 3
    if constexpr (MODE == kBlockPlain) {
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            const int r = 16 * i + fr;
            if (r >= t.rows) continue;
            bf16_t* const c = static_cast<bf16_t*>(p.C) + (size_t)(t.row0 + r) * p.N + col0 + 4 * fk;
#pragma unroll
            for (int j = 0; j < FO; ++j) {
                const f32x4& v = acc[i][j];
                *reinterpret_cast<u32x2*>(c + 16 * j) = u32x2{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
            }
        }
    } else {
        constexpr int PARTS = MODE == kBlockGrad ? 2 : 1;
        f32x4 out[MB][PARTS][FO];
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            const int r = 16 * i + fr;
            const bool in = r < t.rows && writes;
            uint32_t top[PARTS] = {};
#pragma unroll
            for (int j = 0; j < FO; ++j) {
                const size_t at = (size_t)(t.row0 + (in ? r : 0)) * (2 * p.N) + col0 + 16 * j + 4 * fk;
                if constexpr (MODE == kBlockSwiglu) {
                    const f32x4 g = acc[i][j], u = acc[i][j + FO];
                    if (p.gu && in) {
                        *reinterpret_cast<u32x2*>(p.gu + at) = u32x2{pack2_bf16(g[0], g[1]), pack2_bf16(g[2], g[3])};
                        *reinterpret_cast<u32x2*>(p.gu + at + p.N) = u32x2{pack2_bf16(u[0], u[1]), pack2_bf16(u[2], u[3])};
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) out[i][0][j][q] = g[q] * __builtin_amdgcn_rcpf(1.f + __expf(-g[q])) * u[q];
                } else {
                    const u32x2 gv = *reinterpret_cast<const u32x2*>(p.gu + at), uv = *reinterpret_cast<const u32x2*>(p.gu + at + p.N);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float g = __uint_as_float(q & 1 ? gv[q / 2] & 0xffff0000u : gv[q / 2] << 16);
                        const float u = __uint_as_float(q & 1 ? uv[q / 2] & 0xffff0000u : uv[q / 2] << 16);
                        const float sg = __builtin_amdgcn_rcpf(1.f + __expf(-g)), dh = acc[i][j][q];
                        out[i][0][j][q] = dh * u * sg * (1.f + g * (1.f - sg));
                        out[i][1][j][q] = dh * g * sg;
                    }
                    if (in) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const f32x4& v = out[i][h][j];
                            *reinterpret_cast<u32x2*>(p.dgu + at + h * p.N) = u32x2{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
                        }
                    }
                }
#pragma unroll
                for (int h = 0; h < PARTS; ++h)
#pragma unroll
                    for (int q = 0; q < 4; ++q) top[h] = max(top[h], magnitude(out[i][h][j][q]));
            }
#pragma unroll
            for (int h = 0; h < PARTS; ++h) {
                const uint32_t m = max_rows(top[h]);
                if (fk == 0 && writes) tops[h][wave][r] = m;
            }
        }
        __syncthreads();
        const int ldc = PARTS * p.N, lds = block_scale_stride(ldc);
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            const int r = 16 * i + fr;
            if (r >= t.rows || !writes) continue;
#pragma unroll
            for (int h = 0; h < PARTS; ++h) {
                const uint32_t m = max(max(tops[h][0][r], tops[h][1][r]), max(tops[h][2][r], tops[h][3][r]));
                const uint32_t scale = block_scale(m);
                const float inv = block_inverse(scale);
                uint8_t* const c = static_cast<uint8_t*>(p.C) + (size_t)(t.row0 + r) * ldc + h * p.N + col0 + 4 * fk;
#pragma unroll
                for (int j = 0; j < FO; ++j) {
                    const f32x4& v = out[i][h][j];
                    *reinterpret_cast<uint32_t*>(c + 16 * j) = block_codes(v[0], v[1], v[2], v[3], inv, scale);
                }
                if (wave == 0 && fk == 0) p.c_scales[(size_t)(t.row0 + r) * lds + h * (p.N / kBlock) + t.ntile] = (uint8_t)scale;
            }
        }
    }
}

template <int MODE, int MB, int CW, int KS>
void launch_rows(const BlockGemm& p, hipStream_t s) {
    hipLaunchKernelGGL((block_rows_kernel<MODE, MB, CW, KS>), dim3(grid_for(p.r_max, p.E, 16 * MB, p.N / (32 * CW))),
                       dim3(64 * CW * KS), 0, s, p);
}

// The persistent tiles from more than kFewRows rows for every expert that can have any: they stream the weights as well, but a
// tile's 128 rows are multiplied whatever they hold, and with few tiles they leave compute units without one.  us, gate/up and down,
// rows / tiles: 64 experts, 3584 x 2560, 32 tokens (4 rows each) 189 and 94 / 195 and 93, 64 tokens 218 and 122 / 202 and 115, 512 tokens 508
// and 334 / 231 and 132; 8 experts, 4096 x 14336, 1 token 38 and 20 / 40 and 74, 16 tokens (4 rows each) 172 and 83 / 204 and 110, 64 tokens 203
// and 114 / 206 and 112; 64 experts, 4096 x 1408, 64 tokens (6 rows each) 130 and 67 / 135 and 70.  The weights alone take 165 and
// 83, 187 and 93; 39 and 20, 157 and 78; 115 and 58 at 6 TB/s.
constexpr int kFewRows = 6;
// One product with up to so many tiles of 128 columns is cut into columns of 32, its contraction dealt to eight waves (us, 128
// columns and two waves / so: 8 experts, 4096 x 14336, down, 1 token 59 / 20, 4 tokens 69 / 53; 64 experts, 3584 x 2560, 32 tokens, with
// 1792 tiles, 94 / 96).
constexpr int kFewTiles = 256;

template <int MODE>
void launch_block(const BlockGemm& p, hipStream_t s) {
    const int taken = min(p.E, p.r_max);   // experts that can have rows
    if (p.K < 256) launch_rows<MODE, 4, 4, 1>(p, s);   // one block along the contraction: nothing to pipeline
    else if (p.r_max > kFewRows * taken) launch_block_persist(MODE, p, s);
    else if (MODE == kBlockPlain && (long long)taken * (p.N / kBlock) <= kFewTiles) launch_rows<kBlockPlain, 1, 1, 8>(p, s);
    else launch_rows<MODE, 1, 4, 2>(p, s);
}

}  // namespace

void launch_block_gemm(int mode, const BlockGemm& p, hipStream_t s) {
    if (mode == kBlockPlain) launch_block<kBlockPlain>(p, s);
    else if (mode == kBlockSwiglu) launch_block<kBlockSwiglu>(p, s);
    else launch_block<kBlockGrad>(p, s);
}

}  // namespace moe
