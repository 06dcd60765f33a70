// Grouped expert GEMMs on E4M3 operands with a scale for every block of 128 (fp8_block.h): many rows per expert, on the engine of
// gemm_persist_fp8.h.
//
// A k-tile is a block along the contraction, so the scaled matrix instruction takes the operands' scales as it takes their
// codes: no instruction is added for any accumulator.  A lane needs one byte for every row of its activation fragments and, the
// weights' blocks being 128 wide, one (gate and up: two) for all its weight rows.  A wave loads the bytes
// of four k-tiles of each of its rows once, a row to a lane, and the quarters of the wave exchange them in registers; the
// loads are issued two k-tiles ahead of their use, in front of those whose end the k loop's own wait leaves open, so that no
// wait is added either.
//
// Bound by the matrix units and the power they draw.  8 experts x 2048 rows, 6144 x 16384: gate/up 2570 us (2.57 PFLOP/s), with g | u
// stored 2750 to 2810 (1.07 GB more to write), down 1260 to 1290 (2.6 PFLOP/s); with one scale a tensor, on the same engine, 2390 and
// 1190.  A scale loaded for every k-tile in front of its use took 2767 and 1509.
#include "fp8_block.h"
#include "gemm_persist_fp8.h"

namespace moe {

namespace {

// FM row fragments and, along the weight rows, NB blocks of a wave (gate and up, or one)
template <int FM, int NB>
struct BlockScales {
    static constexpr int NR = (FM + 3) / 4;   // loads of 64 rows
    const uint8_t *A, *B0, *B1;               // scales of all rows, and of the weights' blocks: at most a 64th of the codes (K is
    int stride, n_blocks;                     // 256 and more), so less than 4 GiB.  Bytes of a row of scales; blocks along N

    struct Rows {
        uint32_t a, b;                        // where the tile's scales start
        int bytes;                            // of its rows of scales
    };
    Rows cur, next, from;
    int at[NR];                               // lane l loads for the wave's rows l and l + 64
    uint32_t ra[NR], rb[NB];                  // as loaded: four k-tiles
    uint32_t wa[NR], wb[NB];                  // the byte of the k-tile behind the one that is multiplied comes first
    uint32_t half[NR][2];
    uint32_t sa[FM], na[FM], sb[NB], loaded[NB];
    int k;
    bool fresh, wanted;

    __device__ __forceinline__ Rows rows_of(const PTile& t, int wn) const {
        // behind the last block the last one again: those columns are not stored
        const int block = min(t.n0 / kBlock + (NB == 1 ? wn : 0), n_blocks - 1);
        return {uni((uint32_t)t.row0 * (uint32_t)stride), uni((uint32_t)(t.expert * n_blocks + block) * (uint32_t)stride),
                uni(t.rows * stride)};
    }
    // a word of a buffer; of one without bytes 0, which no memory is asked for
    static __device__ __forceinline__ uint32_t word(const uint8_t* base, int bytes, int lane_at, int from) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, bytes, 0x00027000);
        return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rsrc, lane_at, from, 0);
    }
    __device__ __forceinline__ void load_a(int i) { ra[i] = word(A + from.a, wanted ? from.bytes : 0, at[i], wanted ? k : 0); }
    __device__ __forceinline__ void load_b(int i) { rb[i] = word((i ? B1 : B0) + from.b, wanted ? stride : 0, 0, wanted ? k : 0); }
    // na[i] of a lane: what the lane of row 16 i + lane % 16 holds.  The quarters of 16 lanes, each in all four
    __device__ __forceinline__ void spread_half(int i) {
        const auto h = __builtin_amdgcn_permlane32_swap(wa[i], wa[i], false, false);
        half[i][0] = h[0];
        half[i][1] = h[1];
    }
    __device__ __forceinline__ void spread_quarter(int i, int h) {
        if (4 * i + 2 * h >= FM) return;
        const auto q = __builtin_amdgcn_permlane16_swap(half[i][h], half[i][h], false, false);
        na[4 * i + 2 * h] = q[0];
        na[4 * i + 2 * h + 1] = q[1];
    }
    __device__ __forceinline__ void start(const PTile& t, int first_row, int lane, int wn) {
        cur = next = from = rows_of(t, wn);
        wanted = true;
        k = 0;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            at[i] = (first_row + lane + 64 * i) * stride;
            load_a(i);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            load_b(i);
            wb[i] = sb[i] = uni(rb[i]);
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            wa[i] = ra[i];
            spread_half(i);
            spread_quarter(i, 0);
            spread_quarter(i, 1);
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] = na[i];
    }
    // t is the tile after the one that begins
    __device__ __forceinline__ void next_tile(const PTile& t, int wn) {
        cur = next;
        if (t.valid) next = rows_of(t, wn);
    }
    __device__ __forceinline__ f32x4 mfma(const i32x8& w, const i32x8& a, const f32x4& c, int i, int h) const {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, c, 0, 0, 0, (int)sb[NB == 2 ? h : 0], 0, (int)sa[i]);
    }
    // What there is to do in the second half of k-tile kt, in pieces of a few instructions, so that each is covered by a matrix
    // instruction: the next k-tile's scales to their lanes, and the load for the one behind it if it is the first of four (or of
    // the next tile).  No branches: they split the k loop, and what is loaded is then copied, and waited for, at the split.
    static constexpr int PIECES = 16;
    __device__ __forceinline__ void piece(int p, int kt, int KT) {
        if (p == 0) fresh = kt + 1 == KT || ((kt + 1) & 3) == 0;
        if (p == 1 || (p == 2 && NR == 2)) wa[p - 1] = fresh ? ra[p - 1] : wa[p - 1] >> 8;
        if (p == 3) {
#pragma unroll
            for (int i = 0; i < NB; ++i) loaded[i] = uni(rb[i]);
        }
        if (p == 4) {
#pragma unroll
            for (int i = 0; i < NB; ++i) wb[i] = fresh ? loaded[i] : wb[i] >> 8;
        }
        if (p == 5 || (p == 8 && NR == 2)) spread_half((p - 5) / 3);
        if (p == 6 || (p == 9 && NR == 2)) spread_quarter((p - 6) / 3, 0);
        if (p == 7 || (p == 10 && NR == 2)) spread_quarter((p - 7) / 3, 1);
        if (p == 11) {
            const bool over = kt + 2 >= KT;
            from.a = over ? next.a : cur.a;
            from.b = over ? next.b : cur.b;
            from.bytes = over ? next.bytes : cur.bytes;
            k = over ? kt + 2 - KT : kt + 2;
            wanted = (k & 3) == 0;
        }
        if (p == 12 || (p == 13 && NR == 2)) load_a(p - 12);
        if (p == 14 || (p == 15 && NB == 2)) load_b(p - 14);
    }
    __device__ __forceinline__ void step_row(int i) {
        sa[i] = na[i];
        asm volatile("" : "+v"(sa[i]));       // here, between matrix instructions, and not at the loop's end
    }
    // behind matrix instruction `slot` of `slots`, four to a row
    __device__ __forceinline__ void behind(int slot, int slots, int kt, int KT) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
            if (p * slots / PIECES == slot) piece(p, kt, KT);
        const int all = 10 * slots / PIECES + 1;   // na is complete
#pragma unroll
        for (int i = 0; i < FM; ++i)
            if (min(max(4 * i + 4, all + i), slots - 1) == slot && 4 * i + 4 <= slots - 1) step_row(i);
    }
    __device__ __forceinline__ void end_step() {
#pragma unroll
        for (int i = 0; i < FM; ++i)
            if (4 * i + 4 > 4 * FM - 1) step_row(i);
#pragma unroll
        for (int i = 0; i < NB; ++i) sb[i] = wb[i];
    }
    // a k-tile whose products are left out
    __device__ __forceinline__ void skip(int kt, int KT) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) piece(p, kt, KT);
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] = na[i];
#pragma unroll
        for (int i = 0; i < NB; ++i) sb[i] = wb[i];
    }
};

// rows of a wave's patch, 16-byte granules at places that neither side's accesses share a bank at: granule g of row r at
// g ^ (r / rows per 256 bytes)
template <int W>
__device__ __forceinline__ int granule(int row, int g) {
    constexpr int GPR = W / 16, RP256 = W >= 256 ? 1 : 256 / W;
    return row * W + ((g ^ ((row / RP256) & (GPR - 1))) << 4);
}

// y = acc in bf16, 32 rows at a time through the patch
struct PlainStore {
    BlockGemm p;

    template <int FM, int FN>
    __device__ __forceinline__ void tile(f32x4 (&acc)[FM][FN], int row0, int rows, int n0, int wm, int wn, int lane, uint8_t* stage,
                                         uint8_t*, bool) {
        constexpr int WM = FM * 16, W = FN * 32, GPR = W / 16, RPI = 1024 / W;
        asm volatile("" : "+v"(lane));    // keeps the addresses below from being hoisted out of the tile loop
        const int fr = lane & 15, fk = lane >> 4, rl = lane / GPR, gl = lane % GPR;
        const int col = n0 + wn * (FN * 16) + gl * 8;
#pragma unroll
        for (int i = 0; i < FM / 2; ++i) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[2 * i + q][j]));   // see gemm_persist.hip
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const f32x4& a = acc[2 * i + q][j];
                    *reinterpret_cast<u32x2*>(stage + granule<W>(16 * q + fr, 2 * j + (fk >> 1)) + 8 * (fk & 1)) =
                        u32x2{pack2_bf16(a[0], a[1]), pack2_bf16(a[2], a[3])};
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int it = 0; it < 32 / RPI; ++it) {
                const int row = it * RPI + rl, grow = wm * WM + i * 32 + row;
                const u32x4 v = *reinterpret_cast<const u32x4*>(stage + granule<W>(row, gl));
                if (grow < rows && col < p.N)
                    *reinterpret_cast<u32x4*>(static_cast<bf16_t*>(p.C) + (size_t)(row0 + grow) * p.N + col) = v;
            }
        }
    }
    __device__ __forceinline__ void finish(int) {}
};

// h = silu(g) * u as codes.  A wave has 64 of a block's 128 columns, the wave beside it the others: the rows' largest magnitudes
// go through LDS, and the codes are formed behind a barrier.
struct SwigluStore {
    BlockGemm p;

    template <int FM, int FN>
    __device__ __forceinline__ void tile(f32x4 (&acc)[FM][FN], int row0, int rows, int n0, int wm, int wn, int lane, uint8_t* stage,
                                         uint8_t* slot, bool) {
        constexpr int FO = FN / 2, WM = FM * 16;
        asm volatile("" : "+v"(lane));
        const int fr = lane & 15, fk = lane >> 4;
        const int col0 = n0 + wn * (FO * 16);
        // the last 512 bytes of every wave's 8 KiB: its rows' largest magnitudes
        uint32_t* const mine = reinterpret_cast<uint32_t*>(slot + (2 * wm + wn + 1) * 8192 - 512);
        const uint32_t* const other = reinterpret_cast<const uint32_t*>(slot + (2 * wm + 1 - wn + 1) * 8192 - 512);
        static_assert(WM * 4 <= 512 && FN * 32 * 32 == 8192, "patch");
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[i][j]));
            if (p.gu) {
                // g | u of 16 rows, 128 bytes each
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const f32x4& a = acc[i][j];
                    *reinterpret_cast<u32x2*>(stage + granule<256>(fr, 2 * j + (fk >> 1)) + 8 * (fk & 1)) =
                        u32x2{pack2_bf16(a[0], a[1]), pack2_bf16(a[2], a[3])};
                }
                const int rl = lane >> 4, gl = lane & 15;
                const int col = col0 + (gl & 7) * 8 + (gl >> 3) * p.N;
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int row = 4 * it + rl, grow = wm * WM + i * 16 + row;
                    const u32x4 v = *reinterpret_cast<const u32x4*>(stage + granule<256>(row, gl));
                    if (grow < rows) *reinterpret_cast<u32x4*>(p.gu + (size_t)(row0 + grow) * (2 * p.N) + col) = v;
                }
            }
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < FO; ++j)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float g = acc[i][j][u], up = acc[i][j + FO][u];
                    const float h = g * __builtin_amdgcn_rcpf(1.f + __expf(-g)) * up;
                    acc[i][j][u] = h;
                    top = max(top, magnitude(h));
                }
            top = max_rows(top);
            if (fk == 0) mine[16 * i + fr] = top;
#pragma unroll
            for (int j = 0; j < FO; ++j) asm volatile("" : "+a"(acc[i][j]));
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        const int stride = block_scale_stride(p.N);
        constexpr int W = FO * 16;            // 64 bytes a row, 32 rows at a time
#pragma unroll
        for (int i = 0; i < FM / 2; ++i) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                __builtin_amdgcn_sched_barrier(0);
                const int r = 32 * i + 16 * q + fr, grow = wm * WM + r;
                const uint32_t scale = block_scale(max(mine[r], other[r]));
                const float inv = block_inverse(scale);
                if (wn == 0 && fk == 0 && grow < rows) p.c_scales[(size_t)(row0 + grow) * stride + n0 / kBlock] = (uint8_t)scale;
#pragma unroll
                for (int j = 0; j < FO; ++j) {
                    const f32x4& h = acc[2 * i + q][j];
                    *reinterpret_cast<uint32_t*>(stage + granule<W>(16 * q + fr, j) + 4 * fk) = block_codes(h[0], h[1], h[2], h[3], inv, scale);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            const int rl = lane >> 2, gl = lane & 3;
#pragma unroll
            for (int it = 0; it < 2; ++it) {
                const int row = 16 * it + rl, grow = wm * WM + 32 * i + row;
                const u32x4 v = *reinterpret_cast<const u32x4*>(stage + granule<W>(row, gl));
                if (grow < rows) *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(p.C) + (size_t)(row0 + grow) * p.N + col0 + gl * 16) = v;
            }
        }
    }
    __device__ __forceinline__ void finish(int) {}
};

// dg | du from dh and the saved g | u, in bf16 and as codes.  16 rows of dh at a time go through the patch in fp32, so that a
// lane then has eight neighbouring columns of a row, sixteen lanes a block.  The next 16 rows' g | u are asked for as these are
// used up.  Buffer accesses, which leave out what is not in the tile without a branch: nothing waits for the stores.  (Asked for when
// needed, behind branches: 12 experts, 2331 rows, 1024 x 1408, 28 us instead of 24; 64 experts, 16384 rows, 6144 x 2048, 350 instead
// of 325.)
struct GradStore {
    BlockGemm p;

    static constexpr int kFlags = 0x00027000;

    template <int FM, int FN>
    __device__ __forceinline__ void tile(f32x4 (&acc)[FM][FN], int row0, int rows, int n0, int wm, int wn, int lane, uint8_t* stage,
                                         uint8_t*, bool) {
        constexpr int WM = FM * 16, W = 512;
        static_assert(FN == 8 && 16 * W == FN * 32 * 32, "patch");
        asm volatile("" : "+v"(lane));
        const int fr = lane & 15, fk = lane >> 4, rl = lane >> 4, gl = lane & 15;
        const int col = n0 + wn * 128 + 8 * gl;
        const uint32_t pitch = 4u * (uint32_t)p.N, stride = (uint32_t)block_scale_stride(2 * p.N);   // bytes
        auto rows_of = [&](const void* base, uint32_t bytes) {
            return __builtin_amdgcn_make_buffer_rsrc(static_cast<uint8_t*>(const_cast<void*>(base)) + (size_t)row0 * bytes, 0,
                                                     (int)((uint32_t)rows * bytes), kFlags);
        };
        const auto gu = rows_of(p.gu, pitch), dgu = rows_of(p.dgu, pitch), codes = rows_of(p.C, pitch / 2),
                   scales = rows_of(p.c_scales, stride);
        const uint32_t first = (uint32_t)(col < p.N ? wm * WM + rl : rows);   // rows from `rows` on are none
        u32x4 gv[4], uv[4];
        auto load = [&](int i, int it) {
            const uint32_t at = (first + 16 * i + 4 * it) * pitch + 2u * (uint32_t)col;
            gv[it] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(gu, (int)at, 0, 0));
            uv[it] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(gu, (int)(at + 2u * (uint32_t)p.N), 0, 0));
        };
#pragma unroll
        for (int it = 0; it < 4; ++it) load(0, it);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[i][j]));
#pragma unroll
            for (int j = 0; j < FN; ++j) *reinterpret_cast<f32x4*>(stage + fr * W + (((4 * j + fk) ^ (2 * fr & 31)) << 4)) = acc[i][j];
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                __builtin_amdgcn_sched_barrier(0);
                const int row = 4 * it + rl;
                float g[8], u[8], dg[8], du[8];
                bf16x8_to_f32(gv[it], g);
                bf16x8_to_f32(uv[it], u);
                if (i + 1 < FM) load(i + 1, it);
                uint32_t tg = 0, tu = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 dh = *reinterpret_cast<const f32x4*>(stage + row * W + (((2 * gl + h) ^ (2 * row & 31)) << 4));
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int e = 4 * h + q;
                        const float sg = __builtin_amdgcn_rcpf(1.f + __expf(-g[e]));
                        dg[e] = dh[q] * u[e] * sg * (1.f + g[e] * (1.f - sg));
                        du[e] = dh[q] * g[e] * sg;
                        tg = max(tg, magnitude(dg[e]));
                        tu = max(tu, magnitude(du[e]));
                    }
                }
                tg = max16(tg);
                tu = max16(tu);
                const uint32_t grow = first + 16 * i + 4 * it;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float(&v)[8] = h ? du : dg;
                    const uint32_t scale = block_scale(h ? tu : tg), c = (uint32_t)(col + h * p.N);
                    const float inv = block_inverse(scale);
                    __builtin_amdgcn_raw_buffer_store_b128(
                        u32x4{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])}, dgu,
                        (int)(grow * pitch + 2 * c), 0, 0);
                    __builtin_amdgcn_raw_buffer_store_b64(
                        u32x2{block_codes(v[0], v[1], v[2], v[3], inv, scale), block_codes(v[4], v[5], v[6], v[7], inv, scale)}, codes,
                        (int)(grow * (pitch / 2) + c), 0, 0);
                    __builtin_amdgcn_raw_buffer_store_b8((uint8_t)scale, scales, (int)((gl == 0 ? grow : (uint32_t)rows) * stride + c / kBlock),
                                                         0, 0);
                }
            }
        }
    }
    __device__ __forceinline__ void finish(int) {}
};

template <int MODE>
struct StoreOf;
template <>
struct StoreOf<kBlockPlain> {
    using type = PlainStore;
};
template <>
struct StoreOf<kBlockSwiglu> {
    using type = SwigluStore;
};
template <>
struct StoreOf<kBlockGrad> {
    using type = GradStore;
};

template <int MODE, int BM, bool IDLE_SKIP>
__device__ __forceinline__ void block_body(const BlockGemm& p, int ntn, uint8_t* smem) {
    BlockScales<BM / 32, MODE == kBlockSwiglu ? 2 : 1> scales;
    scales.A = p.a_scales;
    scales.B0 = p.b0_scales;
    scales.B1 = p.b1_scales;
    scales.stride = block_scale_stride(p.K);
    scales.n_blocks = p.N / kBlock;
    fp8_body<BM, MODE == kBlockSwiglu, IDLE_SKIP, true>(p.A, p.offsets, p.E, p.N, p.K, p.B0, p.B1, ntn, scales,
                                                        typename StoreOf<MODE>::type{p}, smem);
}

// Tiles of 256, 192 or 128 rows, chosen on the device from the rows that every expert really has; `rows` != 0: those.
template <int MODE, bool IDLE_SKIP>
__global__ __launch_bounds__(256) void block_persist_kernel(BlockGemm p, int ntn, int rows) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int height = rows != 0 ? rows : pick_height(kCostFp8, p.offsets, p.E, ntn, p.K / 128, threadIdx.x & 63);
    if (height == 256) block_body<MODE, 256, IDLE_SKIP>(p, ntn, smem);
    else if (height == 192) block_body<MODE, 192, IDLE_SKIP>(p, ntn, smem);
    else block_body<MODE, 128, IDLE_SKIP>(p, ntn, smem);
}

template <int MODE>
void launch_persist(const BlockGemm& p, hipStream_t s) {
    constexpr int OUTN = MODE == kBlockSwiglu ? 128 : 256;
    constexpr size_t smem = (size_t)(3 * 256 + 2 * 256) * 128;
    const int ntn = (p.N + OUTN - 1) / OUTN;
    const bool idle_skip = persist_idle_skip(p.E);
    auto kern = idle_skip ? block_persist_kernel<MODE, true> : block_persist_kernel<MODE, false>;
    static OncePerDevice lds[2];
    allow_lds(lds[idle_skip], reinterpret_cast<const void*>(kern), (int)smem);
    const int grid = min(persist_grid(), grid_for(p.r_max, p.E, 128, ntn));
    hipLaunchKernelGGL(kern, dim3(grid), dim3(256), smem, s, p, ntn, persist_tile_rows());
}

}  // namespace

void launch_block_persist(int mode, const BlockGemm& p, hipStream_t s) {
    if (mode == kBlockPlain) launch_persist<kBlockPlain>(p, s);
    else if (mode == kBlockSwiglu) launch_persist<kBlockSwiglu>(p, s);
    else launch_persist<kBlockGrad>(p, s);
}

}  // namespace moe
