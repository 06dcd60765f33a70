// Grouped expert GEMM (a3) on FP8 operands with per-tensor delayed scaling
// (Section 4.5, "FP8 Training Performance").
//
// The engine is gemm_persist_fp8.h's.  The epilogues: the gate/up GEMM
// dequantises g and u, applies SwiGLU, records max |h| for the next step's scale
// and writes h as E4M3 with this step's (delayed) scale; the down GEMM
// dequantises into bf16.  Bound by power with many rows (see gemm_persist.hip).
// Measured, gate/up and down, us, 32x32x64 / this: 8 experts of 16384 rows, 6144 x
// 16384, 2550 and 1262 / 2458 and 1191 (2.7 and 2.8 PFLOP/s); 8 x 4096 rows, 6144 x
// 2048, 645 and 372 / 605 and 350; 64 skewed experts of 82000 rows, 4096 x 1408, 822
// and 502 / 783 and 479.
#include "fp8_convert.h"
#include "gemm_persist_fp8.h"
#include "gemm_stream.h"

namespace moe {

namespace {

// Epilogue of the gate/up GEMM: h = silu(g) * u from the dequantised
// accumulators, one byte per value.  Staged through a wave-private LDS patch of
// W = 16*FO bytes per row (16-byte granules XOR-swizzled by the row) so that the
// global stores are whole 16-byte pieces along the rows.
template <int FM, int FN, int WM>
__device__ __forceinline__ float store_h_fp8(f32x4 (&acc)[FM][FN], int t_row0, int t_rows, int t_n0, uint8_t* C,
                                             int N, int wm, int wn, int lane, uint8_t* stage, float dq_gate,
                                             float dq_up, float scale_h, float amax) {
    constexpr int FO = FN / 2;
    constexpr int W = FO * 16;        // bytes per staged row
    constexpr int GPR = W / 16;       // granules per row: a fragment's columns are one
    constexpr int RP256 = 256 / W;    // rows per 256 bytes
    constexpr int RPI = 1024 / W;     // rows per 64-lane read
    static_assert(W <= 256 && 256 % W == 0 && 32 % RPI == 0, "staged row must divide the bank window");
    asm volatile("" : "+v"(lane));    // keeps the addresses below from being hoisted out of the tile loop
    const int fr = lane & 15, fk = lane >> 4;
    static_assert((16 / RP256) % GPR == 0, "both row blocks of a patch have the same swizzle");
    const int xw = (fr / RP256) & (GPR - 1);
    uint8_t* wrow = stage + fr * W + 4 * fk;
    const int rl = lane / GPR, gl = lane % GPR;
    const int col = t_n0 + wn * (FO * 16) + gl * 16;
#pragma unroll
    for (int i = 0; i < FM / 2; ++i) {   // 32 rows at a time
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[2 * i + q][j]));   // see gemm_persist.hip
#pragma unroll
            for (int j = 0; j < FO; ++j) {
                float hv[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float g = acc[2 * i + q][j][u] * dq_gate;
                    const float up = acc[2 * i + q][j + FO][u] * dq_up;
                    hv[u] = g * __builtin_amdgcn_rcpf(1.f + __expf(-g)) * up;   // silu(g) * up
                    amax = fmaxf(amax, fabsf(hv[u]));
                }
                const uint32_t packed = f32x4_to_e4m3(hv[0] * scale_h, hv[1] * scale_h, hv[2] * scale_h,
                                                      hv[3] * scale_h);
                // lane's 4 columns: bytes 16j + 4fk .. +3 of the row
                *reinterpret_cast<uint32_t*>(wrow + q * (16 * W) + ((j ^ xw) << 4)) = packed;
                asm volatile("" : "+v"(amax));   // now, or the values wait for it in scratch memory
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const int first = wm * WM + i * 32;
#pragma unroll
        for (int it = 0; it < 32 / RPI; ++it) {
            const int row = it * RPI + rl;
            const int xr = (row / RP256) & (GPR - 1);
            const u32x4 v = *reinterpret_cast<const u32x4*>(stage + row * W + ((gl ^ xr) << 4));
            const int grow = first + row;
            if (grow < t_rows && col < N) *reinterpret_cast<u32x4*>(C + (size_t)(t_row0 + grow) * N + col) = v;
        }
    }
    return amax;
}

// Epilogue of the down GEMM: y = acc * dq as bf16, staged like the bf16 kernel's.
template <int FM, int FN, int WM>
__device__ __forceinline__ void store_y_bf16(f32x4 (&acc)[FM][FN], int t_row0, int t_rows, int t_n0, bf16_t* C,
                                             int N, int wm, int wn, int lane, uint8_t* stage, float dq) {
    constexpr int W = FN * 32;
    constexpr int GPR = W / 16;
    constexpr int RP256 = 256 / W;
    constexpr int RPI = 1024 / W;
    static_assert(W <= 256 && 256 % W == 0, "staged row must divide the bank window");
    asm volatile("" : "+v"(lane));
    const int fr = lane & 15, fk = lane >> 4;
    static_assert((16 / RP256) % GPR == 0, "both row blocks of a patch have the same swizzle");
    const int xw = (fr / RP256) & (GPR - 1);
    uint8_t* wrow = stage + fr * W + 8 * (fk & 1);
    const int gw = fk >> 1;           // a fragment is two granules wide
    const int rl = lane / GPR, gl = lane % GPR;
    const int col = t_n0 + wn * (FN * 16) + gl * 8;
#pragma unroll
    for (int i = 0; i < FM / 2; ++i) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[2 * i + q][j]));
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const f32x4& a = acc[2 * i + q][j];
                u32x2 o;
                o[0] = pack2_bf16(a[0] * dq, a[1] * dq);
                o[1] = pack2_bf16(a[2] * dq, a[3] * dq);
                *reinterpret_cast<u32x2*>(wrow + q * (16 * W) + (((2 * j + gw) ^ xw) << 4)) = o;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const int first = wm * WM + i * 32;
#pragma unroll
        for (int it = 0; it < 32 / RPI; ++it) {
            const int row = it * RPI + rl;
            const int xr = (row / RP256) & (GPR - 1);
            const u32x4 v = *reinterpret_cast<const u32x4*>(stage + row * W + ((gl ^ xr) << 4));
            const int grow = first + row;
            if (grow < t_rows && col < N) *reinterpret_cast<u32x4*>(C + (size_t)(t_row0 + grow) * N + col) = v;
        }
    }
}

// h as E4M3 (s0, s1 dequantise g and u, s2 scales h) with max |h| to *amax_out, or null; y as bf16 (s0 dequantises it)
template <bool SWIGLU>
struct TensorStore {
    void* C;
    float* amax_out;
    float s0, s1, s2, amax;
    int N;

    template <int FM, int FN>
    __device__ __forceinline__ void tile(f32x4 (&acc)[FM][FN], int row0, int rows, int n0, int wm, int wn, int lane, uint8_t* stage,
                                         uint8_t*, bool wave_idle) {
        constexpr int WM = FM * 16;
        if constexpr (SWIGLU) {
            const float m = store_h_fp8<FM, FN, WM>(acc, row0, rows, n0, static_cast<uint8_t*>(C), N, wm, wn, lane, stage, s0, s1, s2, amax);
            if (!wave_idle) amax = m;
        } else {
            store_y_bf16<FM, FN, WM>(acc, row0, rows, n0, static_cast<bf16_t*>(C), N, wm, wn, lane, stage, s0);
        }
    }

    __device__ __forceinline__ void finish(int lane) {
        if constexpr (SWIGLU) {
            if (!amax_out) return;
            // max |h| over the wave, then one atomic per wave; h >= 0 as a float compares like its bit pattern.
            // Rows past the tile's valid rows may have contributed garbage: they were computed from re-read valid
            // rows of the same expert, so they are values h takes anyway.
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor(amax, off, 64));
            if (lane == 0 && amax > __builtin_nontemporal_load(amax_out))   // *amax_out only grows; NaN compares false
                atomicMax(reinterpret_cast<int*>(amax_out), __float_as_int(amax));
        }
    }
};

// Tiles of 256, 192 or 128 rows, chosen on the device from the rows that every expert really has; `rows` != 0: those.
template <bool SWIGLU, bool IDLE_SKIP, bool DEEP_B>
__global__ __launch_bounds__(256) void gemm_fp8_persist_kernel(
    const uint8_t* __restrict__ A, const int32_t* __restrict__ offsets, int E, int N, int K,
    const uint8_t* __restrict__ B0, const uint8_t* __restrict__ B1, void* __restrict__ C, int ntn, float s0,
    float s1, float s2, float* __restrict__ amax_out, int rows) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const TensorStore<SWIGLU> store = {C, amax_out, s0, s1, s2, 0.f, N};
    if constexpr (!DEEP_B) {
        fp8_body<256, SWIGLU, IDLE_SKIP, DEEP_B>(A, offsets, E, N, K, B0, B1, ntn, NoScales{}, store, smem);
    } else {
        const int height = rows != 0 ? rows : pick_height(kCostFp8, offsets, E, ntn, K / 128, threadIdx.x & 63);
        if (height == 256)
            fp8_body<256, SWIGLU, IDLE_SKIP, DEEP_B>(A, offsets, E, N, K, B0, B1, ntn, NoScales{}, store, smem);
        else if (height == 192)
            fp8_body<192, SWIGLU, IDLE_SKIP, DEEP_B>(A, offsets, E, N, K, B0, B1, ntn, NoScales{}, store, smem);
        else
            fp8_body<128, SWIGLU, IDLE_SKIP, DEEP_B>(A, offsets, E, N, K, B0, B1, ntn, NoScales{}, store, smem);
    }
}

static int g_fp8_deep_b = 1;   // three LDS stages for the weight tile (0: for the activation tile)

template <bool SWIGLU>
void launch_fp8(const void* A, const int32_t* offsets, int r_max, int E, int N, int K, const void* B0, const void* B1,
                void* C, float s0, float s1, float s2, float* amax, hipStream_t s) {
    constexpr int OUTN = SWIGLU ? 128 : 256;
    constexpr size_t smem = (size_t)(3 * 256 + 2 * 256) * 128;
    const int ntn = (N + OUTN - 1) / OUTN;
    const bool idle_skip = persist_idle_skip(E);
    const bool deep = g_fp8_deep_b != 0;
    auto kern = deep ? (idle_skip ? gemm_fp8_persist_kernel<SWIGLU, true, true> : gemm_fp8_persist_kernel<SWIGLU, false, true>)
                     : (idle_skip ? gemm_fp8_persist_kernel<SWIGLU, true, false> : gemm_fp8_persist_kernel<SWIGLU, false, false>);
    static OncePerDevice lds[2][2];
    allow_lds(lds[deep][idle_skip], reinterpret_cast<const void*>(kern), (int)smem);
    const int grid = min(persist_grid(), grid_for(r_max, E, deep ? 128 : 256, ntn));
    hipLaunchKernelGGL(kern, dim3(grid), dim3(256), smem, s, static_cast<const uint8_t*>(A), offsets, E, N, K,
                       static_cast<const uint8_t*>(B0), static_cast<const uint8_t*>(B1), C, ntn, s0, s1, s2, amax,
                       persist_tile_rows());
}

}  // namespace

void set_fp8_deep_b(int v) { g_fp8_deep_b = v; }

bool fp8_ffn_supported(int H, int F) { return H % 128 == 0 && F % 128 == 0 && H >= 256 && F >= 256; }

void launch_expert_ffn_fp8(const void* x_perm, const int32_t* offsets, int r_max, int H, int F, int E,
                           const void* w_gate, const void* w_up, const void* w_down, float dq_gate, float dq_up,
                           float scale_h, float dq_down, void* h, float* amax_h, void* y_perm, int phase,
                           hipStream_t s) {
    if (phase & 1) {
        const StreamPlan plan = plan_stream(kStreamFp8, r_max, E, F, H, true, true, 0);
        if (plan.kind != kPlanLarge)
            launch_stream(plan, kStreamFp8, x_perm, offsets, r_max, E, F, H, w_gate, w_up, h, nullptr, dq_gate, dq_up, scale_h,
                          amax_h, nullptr, s);
        else
            launch_fp8<true>(x_perm, offsets, r_max, E, F, H, w_gate, w_up, h, dq_gate, dq_up, scale_h, amax_h, s);
    }
    if (phase & 2) {
        const StreamPlan plan = plan_stream(kStreamFp8, r_max, E, H, F, false, true, 0);
        if (plan.kind != kPlanLarge)
            launch_stream(plan, kStreamFp8, h, offsets, r_max, E, H, F, w_down, nullptr, y_perm, nullptr, dq_down, 0.f, 0.f,
                          nullptr, nullptr, s);
        else
            launch_fp8<false>(h, offsets, r_max, E, H, F, w_down, nullptr, y_perm, dq_down, 0.f, 0.f, nullptr, s);
    }
}

}  // namespace moe
