// Products with a device's weights: x W^T with W in 4 bits (tpq_linear4), and the feed-forward block's
// act(x Wg^T) * (x Wu^T) with both matrices in BF16 or in 4 bits (tpq_gated), in one kernel for one token and for thousands.
//
// The OUTPUTS are the rows of the tensor cores' tile and the tokens its columns (tcgen05, M = 128, N = 16 .. 256 tokens, K = 16): few tokens
// then cost few columns, and weights are read once whatever T is.  Gate and up are two accumulators over the same tokens, so the
// activation and the product are the epilogue's, in binary32, with one rounding.
//
// Weights in 4 bits become BF16 operands in TENSOR memory: a thread is a row of the tile (an output), takes 64 codes of it from shared
// memory and stores the 64 values with one tcgen05.st; nothing is written to shared memory again.  A step has 5 significant bits and a code
// is -8 .. 7, so step * code IS a BF16 number: (16 + u) s - 24 s with u = code + 8 in the mantissa of 16.0, one fused operation for
// two values (24 s has 7 significant bits), exact.  An output's power of two multiplies its sum at the end.
//
//   warp 0       copies (one lane): blocks of weights (4 bits: as they lie, 128 outputs x 128 inputs) and the tokens' inputs
//   warp 1       tensor memory, MMA issue (one elected lane)
//   4 bits: warps 2-17 codes to operands: 4 rows of 32 x 4 parts of a stage's (or of two stages') 64-wide pieces; warps 18-21 epilogue
//   BF16:   warps 2-9  epilogue
//
// Few tokens: a tile's inputs are split over the blocks of a cluster, so that all SMs read weights; the partial sums meet in the
// cluster's shared memory and are added in the order of the blocks (the same call gives the same bits).
// Every wait is bounded: on expiry the block records TPQ_ERR_TIMEOUT, skips its stores, frees its tensor memory and returns.
#include <cuda_bf16.h>

#include "block_internal.h"

namespace {

constexpr int BM = 128, MOST_STAGES = 16, MOST_SLOTS = 8;
constexpr int WAIT_LIMIT = 1 << 24;                     // try_wait attempts (each suspends for a hardware time slice) ...
constexpr unsigned long long WAIT_NS = 1000000000ull;   // ... and one second, whichever ends first
constexpr uint32_t SMEM_MAX = 227u * 1024u;
constexpr uint32_t BAR_BYTES = 512;                     // barriers and the tensor-memory address
constexpr uint32_t W_BF16_BYTES = BM * 64 * 2;

__host__ __device__ constexpr int threads_of(bool w4) { return w4 ? 22 * 32 : 10 * 32; }

struct params {
    int64_t T;
    int n, tiles_n, tiles_t, N, pitch;  // N: tokens of a tile; pitch: columns of an accumulator
    int kblocks;                        // stages of a tile: 128 inputs (4 bits) or 64 (BF16)
    int split, stages, bufs, depth;     // blocks of a tile; ring; accumulator sets; stages whose operands fit tensor memory
    uint32_t w_block, x_at, stage, tmem_cols;
    int group_shift;
    const uint8_t *w4[2];
    const float *factor[2];
    void *out;
    int64_t out_stride;
    int out_fp32, act;
    int *status;
};

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity)
{
    unsigned long long t0 = 0;
    for (int i = 0; i < WAIT_LIMIT; ++i) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        if (ok) return true;
        if ((i & 63) == 63) {
            unsigned long long t;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (t0 == 0) t0 = t;
            else if (t - t0 > WAIT_NS) return false;
        }
    }
    return false;
}
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)); }

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool elect()
{
    uint32_t one;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xFFFFFFFF;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(one));
    return one != 0;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// operands of 128-byte rows with the 128-byte swizzle, 8-row groups of 1024 bytes; a step of 16 along K is 32 bytes
__device__ __forceinline__ uint64_t operand(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// FP32 accumulator, BF16 operands, both K-major, M = 128
__device__ __forceinline__ uint32_t instr(int N) { return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(BM >> 4) << 24); }

#define L4(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3])
#define S4(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3])
#define U4(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3])
// 16 columns of the thread's row (the values are there after ld_wait)
__device__ __forceinline__ void ld16(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : L4(r, 0), L4(r, 4), L4(r, 8), L4(r, 12)
                 : "r"(addr)
                 : "memory");
}
// (the registers pass through, so that nothing that uses them moves ahead of the wait)
__device__ __forceinline__ void ld_wait(uint32_t (&r)[16]) { asm volatile("tcgen05.wait::ld.sync.aligned;" : U4(r, 0), U4(r, 4), U4(r, 8), U4(r, 12)::"memory"); }
__device__ __forceinline__ void st32(uint32_t addr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::S4(r, 0), S4(r, 4), S4(r, 8), S4(r, 12), S4(r, 16), S4(r, 20), S4(r, 24), S4(r, 28), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ float lds_cluster(uint32_t addr, uint32_t rank)
{
    uint32_t a;
    float v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// 8 codes (a word of the layout) times the step: pairs (2i, 2i + 1) as BF16
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t step2, uint32_t bias2, uint32_t *r)
{
    const uint32_t at[4] = {w, w >> 4, w >> 8, __funnelshift_r(w, w, 12)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t u = (at[i] & 0x00780078u) | 0x41804180u;  // 16 + u
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r[i]) : "r"(u), "r"(step2), "r"(bias2));
    }
}

// The activation in binary32.  Exponentials and quotients are CUDA's approximate ones (errors of a few 2^-23 of an activation that is
// rounded to BF16 behind the product); a gate below -80 or so, whose activation is under 2^-100, may come out as 0.
__device__ __forceinline__ float activation(float g, int act)
{
    if (act == TPQ_ACT_SILU) return __fdividef(g, 1.0f + __expf(-g));
    if (act == TPQ_ACT_GELU_TANH) {  // (1 + tanh z) / 2 = 1 / (1 + exp(-2z)): no cancellation for negative gates
        const float z = 1.5957691216057308f * g * fmaf(0.044715f * g, g, 1.0f);
        return __fdividef(g, 1.0f + __expf(-z));
    }
    return 0.5f * g * erfcf(-0.70710678118654752f * g);  // (1 + erf z) = erfc(-z), without the cancellation
}

template <bool W4, int NW>
__device__ __forceinline__ void store(const params &p, int64_t t, int col, float v)
{
    if (p.out_fp32) static_cast<float *>(p.out)[t * p.out_stride + col] = v;
    else static_cast<__nv_bfloat16 *>(p.out)[t * p.out_stride + col] = __float2bfloat16_rn(v);
}

struct ring {  // a stage and its parity
    int s = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int n)
    {
        if (++s == n) {
            s = 0;
            phase ^= 1;
        }
    }
};

template <bool W4, int NW>
__global__ void __launch_bounds__(threads_of(W4), 1)
product(const params p, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1)
{
    extern __shared__ uint8_t raw[];
    constexpr int SPS = 2 * NW;                      // 64-wide operand pieces of a stage (4 bits)
    constexpr int EPI = W4 ? 18 : 2, EPI_WARPS = W4 ? 4 : 8;
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t bars = base + p.stages * p.stage;
    uint8_t *const gen = raw + (base - smem_u32(raw));
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(gen + p.stages * p.stage + BAR_BYTES - 16);
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (MOST_STAGES + s); };
    auto a_full = [&](int s) { return bars + 8u * (2 * MOST_STAGES + s); };
    auto a_empty = [&](int s) { return bars + 8u * (2 * MOST_STAGES + MOST_SLOTS + s); };
    auto acc_full = [&](int b) { return bars + 8u * (2 * MOST_STAGES + 2 * MOST_SLOTS + b); };
    auto acc_empty = [&](int b) { return bars + 8u * (2 * MOST_STAGES + 2 * MOST_SLOTS + 2 + b); };

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tiles = p.tiles_n * p.tiles_t, places = gridDim.x / p.split;
    const int rank = p.split > 1 ? (int)(blockIdx.x % p.split) : 0, first_tile = blockIdx.x / p.split;
    const int kb0 = (int)((int64_t)p.kblocks * rank / p.split), kb1 = (int)((int64_t)p.kblocks * (rank + 1) / p.split);
    // tiles in bands of 16 tiles of tokens, in a band output by output: blocks that run together share weights
    auto origin = [&](int tile, int &tn, int &tt) {
        const int per = 16 * p.tiles_n, band = tile / per, in = tile - band * per;
        const int rows = p.tiles_t - 16 * band < 16 ? p.tiles_t - 16 * band : 16;
        tn = in / rows;
        tt = band * 16 + in - tn * rows;
    };

    if (tid == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int s = 0; s < MOST_SLOTS; ++s) {
            mbar_init(a_full(s), 4);
            mbar_init(a_empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), EPI_WARPS);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(p.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp == 0 && lane == 0 && first_tile < tiles) {
        // Into L2 ahead of the kernel before: a hint, the copies proper come after the wait.
        int tn, tt;
        origin(first_tile, tn, tt);
        const int n = kb1 - kb0 < p.stages ? kb1 - kb0 : p.stages;
        for (int i = 0; i < n; ++i) {
            if (W4) {
                for (int a = 0; a < NW; ++a)
                    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p.w4[a] + ((int64_t)tn * p.kblocks + kb0 + i) * p.w_block), "r"(p.w_block) : "memory");
            } else {
                asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(&map_w0), "r"((kb0 + i) * 64), "r"(tn * BM) : "memory");
                if (NW == 2)
                    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(&map_w1), "r"((kb0 + i) * 64), "r"(tn * BM) : "memory");
            }
        }
    }
    fence_before();
    tpq_grid_dep_wait();
    __syncthreads();
    tpq_grid_dep_launch();
    fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t a_at = tmem + (uint32_t)(p.bufs * NW * p.pitch);  // operands behind the accumulators
    bool ok = true;

    if (warp == 0) {
        if (lane == 0) {
            ring r;
            int64_t it = 0;
            for (int tile = first_tile; tile < tiles && ok; tile += places) {
                int tn, tt;
                origin(tile, tn, tt);
                for (int kb = kb0; kb < kb1; ++kb, ++it, r.next(p.stages)) {
                    if (it >= p.stages && !wait(empty(r.s), r.phase ^ 1)) {
                        ok = false;
                        break;
                    }
                    const uint32_t at = base + r.s * p.stage, bar = full(r.s);
                    if (W4) {
                        mbar_expect_tx(bar, NW * p.w_block + 2 * (uint32_t)p.N * 128);
                        for (int a = 0; a < NW; ++a) bulk_g2s(at + a * p.w_block, p.w4[a] + ((int64_t)tn * p.kblocks + kb) * p.w_block, p.w_block, bar);
                        tma_load_2d(at + p.x_at, &map_x, kb * 128, tt * p.N, bar);
                        tma_load_2d(at + p.x_at + p.N * 128, &map_x, kb * 128 + 64, tt * p.N, bar);
                    } else {
                        mbar_expect_tx(bar, NW * W_BF16_BYTES + (uint32_t)p.N * 128);
                        tma_load_2d(at, &map_w0, kb * 64, tn * BM, bar);
                        if (NW == 2) tma_load_2d(at + W_BF16_BYTES, &map_w1, kb * 64, tn * BM, bar);
                        tma_load_2d(at + p.x_at, &map_x, kb * 64, tt * p.N, bar);
                    }
                }
            }
            if (!ok) {  // giving up: let the copies already issued land before the shared memory is released
                ring l = r;
                for (int j = 0; j < p.stages; ++j) {
                    (void)wait(full(l.s), l.phase ^ 1);
                    l.next(p.stages);
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t idesc = instr(p.N);
        ring r;
        int64_t it = 0;
        int n_tile = 0;
        for (int tile = first_tile; tile < tiles && ok; tile += places, ++n_tile) {
            const int b = p.bufs == 2 ? n_tile & 1 : 0, use = p.bufs == 2 ? n_tile >> 1 : n_tile;
            if (use >= 1) ok = wait_warp(acc_empty(b), (use - 1) & 1);
            if (!ok) break;
            fence_after();
            const uint32_t d = tmem + (uint32_t)(b * NW * p.pitch);
            for (int kb = kb0; kb < kb1; ++kb, ++it, r.next(p.stages)) {
                ok = wait_warp(full(r.s), r.phase);
                if (!ok) break;
                const uint32_t at = base + r.s * p.stage;
                if (W4) {
                    const int turn = p.depth == 2 ? (int)(it & 1) : 0;
                    const uint32_t parity = (uint32_t)(p.depth == 2 ? it >> 1 : it) & 1;
#pragma unroll
                    for (int j = 0; j < SPS; ++j) {  // piece j / NW of the inputs, weight j % NW
                        const int slot = turn * SPS + j;
                        ok = ok && wait_warp(a_full(slot), parity);
                        if (!ok) break;
                        fence_after();
                        if (elect()) {
                            const uint64_t x = operand(at + p.x_at + (j / NW) * p.N * 128);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                mma_ts(d + (uint32_t)((j % NW) * p.pitch), a_at + (uint32_t)(slot * 32 + k * 8), x + 2 * k, idesc, kb != kb0 || j >= NW || k != 0);
                            commit(a_empty(slot));
                            if (j == SPS - 1) {
                                commit(empty(r.s));
                                if (kb == kb1 - 1) commit(acc_full(b));
                            }
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                } else {
                    fence_after();
                    if (elect()) {
                        const uint64_t x = operand(at + p.x_at), w = operand(at);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int a = 0; a < NW; ++a)
                                mma_ss(d + (uint32_t)(a * p.pitch), w + a * (W_BF16_BYTES >> 4) + 2 * k, x + 2 * k, idesc, kb != kb0 || k != 0);
                        commit(empty(r.s));
                        if (kb == kb1 - 1) commit(acc_full(b));
                    }
                    __syncwarp();
                }
            }
        }
    } else if (W4 && warp < EPI) {
        // ---------------- codes to operands.  Two weights: a warp has (piece, weight) of every stage.  One: a piece of every other stage.
        const int q = warp & 3, cls = (warp - 2) >> 2;
        const int piece = NW == 2 ? cls >> 1 : cls & 1, a = NW == 2 ? cls & 1 : 0;
        const uint32_t row = (uint32_t)(q * 32 + lane);
        const uint32_t codes = a * p.w_block + piece * (2 * BM * 16) + row * 16;
        const uint32_t step0 = a * p.w_block + W4_CODE_BYTES + ((piece * 64) >> p.group_shift) * BM + row;
        const uint32_t step1 = a * p.w_block + W4_CODE_BYTES + ((piece * 64 + 32) >> p.group_shift) * BM + row;
        const uint32_t to = a_at + ((uint32_t)(q * 32) << 16);
        ring r;
        int64_t it = 0;
        for (int tile = first_tile; tile < tiles && ok; tile += places) {
            for (int kb = kb0; kb < kb1; ++kb, ++it, r.next(p.stages)) {
                if (NW == 1 && (int)(it & 1) != cls >> 1) continue;
                const int turn = p.depth == 2 ? (int)(it & 1) : 0;
                const int64_t use = p.depth == 2 ? it >> 1 : it;
                const int slot = turn * SPS + (NW == 2 ? cls : piece);
                if (!wait(full(r.s), r.phase)) ok = false;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t at = base + r.s * p.stage;
                const uint4 c0 = lds128(at + codes), c1 = lds128(at + codes + BM * 16);
                const uint32_t s0 = lds8(at + step0), s1 = lds8(at + step1);
                uint32_t v[32];
                uint32_t step2 = ((s0 << 3) + (119u << 7)) * 0x00010001u, bias2;
                asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(bias2) : "r"(step2), "r"(0xC1C0C1C0u));  // -24
                unpack8(c0.x, step2, bias2, v);
                unpack8(c0.y, step2, bias2, v + 4);
                unpack8(c0.z, step2, bias2, v + 8);
                unpack8(c0.w, step2, bias2, v + 12);
                step2 = ((s1 << 3) + (119u << 7)) * 0x00010001u;
                asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(bias2) : "r"(step2), "r"(0xC1C0C1C0u));
                unpack8(c1.x, step2, bias2, v + 16);
                unpack8(c1.y, step2, bias2, v + 20);
                unpack8(c1.z, step2, bias2, v + 24);
                unpack8(c1.w, step2, bias2, v + 28);
                if (use >= 1 && !wait(a_empty(slot), (uint32_t)(use - 1) & 1)) ok = false;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                fence_after();
                st32(to + slot * 32, v);
                st_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(a_full(slot));
            }
        }
    } else {
        // ---------------- epilogue
        const int q = warp & 3, part = (warp - EPI) >> 2;
        int n_tile = 0;
        for (int tile = first_tile; tile < tiles; tile += places, ++n_tile) {
            const int b = p.bufs == 2 ? n_tile & 1 : 0, use = p.bufs == 2 ? n_tile >> 1 : n_tile;
            int tn, tt;
            origin(tile, tn, tt);
            const int col = tn * BM + q * 32 + lane;
            float f0 = 1.0f, f1 = 1.0f;
            if (W4) {
                f0 = p.factor[0][col];
                if (NW == 2) f1 = p.factor[1][col];
            }
            ok = wait_warp(acc_full(b), (uint32_t)use & 1);
            if (!ok) break;
            fence_after();
            const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(b * NW * p.pitch);
            const int64_t t0 = (int64_t)tt * p.N;
            for (int c = 16 * part; c < p.N; c += 16 * (EPI_WARPS / 4)) {
                if (t0 + c >= p.T) break;
                uint32_t y0[16], y1[16];
                ld16(from + c, y0);
                if (NW == 2) ld16(from + p.pitch + c, y1);
                ld_wait(y0);
                if (NW == 2) ld_wait(y1);
                if (p.split > 1) {
                    float *const part_sums = reinterpret_cast<float *>(gen) + q * 32 + lane;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        part_sums[(c + j) * BM] = __uint_as_float(y0[j]);
                        if (NW == 2) part_sums[(p.N + c + j) * BM] = __uint_as_float(y1[j]);
                    }
                } else if (col < p.n) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        if (t0 + c + j >= p.T) break;
                        float v = __uint_as_float(y0[j]) * f0;
                        if (NW == 2) v = activation(v, p.act) * (__uint_as_float(y1[j]) * f1);
                        store<W4, NW>(p, t0 + c + j, col, v);
                    }
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty(b));
        }
    }
    if (!ok) atomicExch(p.status, (int)TPQ_ERR_TIMEOUT);
    if (p.split > 1) {
        // the cluster's partial sums, in the order of its blocks; each block ends with its share of the tile's tokens
        cluster_sync();
        int tn, tt;
        origin(first_tile, tn, tt);
        const int64_t t0 = (int64_t)tt * p.N;
        const int cells = (int)(p.T - t0 < p.N ? p.T - t0 : p.N) * BM;
        const int from = (int)((int64_t)cells * rank / p.split), to = (int)((int64_t)cells * (rank + 1) / p.split);
        for (int i = from + tid; i < to; i += blockDim.x) {
            const int col = tn * BM + (i & (BM - 1));
            float v = 0.0f, u = 0.0f;
            for (int k = 0; k < p.split; ++k) {
                v += lds_cluster(base + 4u * i, k);
                if (NW == 2) u += lds_cluster(base + 4u * (p.N * BM + i), k);
            }
            if (col >= p.n || !ok) continue;
            if (W4) v *= p.factor[0][col];
            if (NW == 2) {
                if (W4) u *= p.factor[1][col];
                v = activation(v, p.act) * u;
            }
            store<W4, NW>(p, t0 + i / BM, col, v);
        }
        cluster_sync();  // nobody reads this block's shared memory any more
    }
    fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.tmem_cols) : "memory");
    }
}

// [rows][K] BF16 with a row stride -> boxes of box_rows rows x 64 inputs with the 128-byte swizzle; what lies outside reads as 0
bool make_map(const void *ptr, int64_t rows, int64_t K, int64_t stride, int box_rows, CUtensorMap *out)
{
    tpq_encode_tiled_fn fn = tpq_tensor_map_encoder();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, one[2] = {1, 1};
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(ptr), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool W4, int NW>
cudaError_t launch(params p, const product_call &c, const tpq_block *b, cudaStream_t st)
{
    // the tile's tokens
    const int most = W4 ? (NW == 2 ? 96 : 192) : 256;
    p.tiles_t = (int)((c.T + most - 1) / most);
    p.N = (int)(((c.T + p.tiles_t - 1) / p.tiles_t + 15) / 16 * 16);
    p.tiles_t = (int)((c.T + p.N - 1) / p.N);
    p.pitch = (p.N + 31) / 32 * 32;
    p.tiles_n = (int)((c.n + BM - 1) / BM);
    p.kblocks = (int)((c.K + (W4 ? 127 : 63)) / (W4 ? 128 : 64));
    p.w_block = W4 ? w4_block_bytes(c.group) : W_BF16_BYTES;
    p.x_at = (NW * p.w_block + 1023) / 1024 * 1024;
    p.stage = p.x_at + (W4 ? 2 : 1) * p.N * 128;
    p.stages = (int)((SMEM_MAX - 1024 - BAR_BYTES) / p.stage);
    if (p.stages > MOST_STAGES) p.stages = MOST_STAGES;
    const int64_t tiles = (int64_t)p.tiles_n * p.tiles_t;
    // few tiles: the inputs of each split over a cluster
    p.split = 1;
    for (int s = 2; s <= 8 && s <= p.kblocks; ++s)
        if (tiles <= b->clusters[s] && (uint64_t)NW * p.N * BM * 4 <= (uint64_t)p.stages * p.stage) p.split = s;
    const int a_cols = W4 ? 64 * NW : 0;
    p.bufs = tiles * p.split > b->sm_count && 2 * NW * p.pitch + a_cols * (NW == 2 ? 1 : 2) <= 512 ? 2 : 1;
    p.depth = W4 && p.bufs * NW * p.pitch + 2 * a_cols <= 512 ? 2 : 1;
    const int cols = p.bufs * NW * p.pitch + p.depth * a_cols;
    p.tmem_cols = cols <= 32 ? 32 : cols <= 64 ? 64 : cols <= 128 ? 128 : cols <= 256 ? 256 : 512;
    CUtensorMap mx, mw[2];
    if (!make_map(c.x, c.T, c.K, c.x_stride, p.N, &mx)) return cudaErrorNotSupported;
    for (int a = 0; a < 2; ++a) {
        mw[a] = mx;
        if (!W4 && a < NW && !make_map(c.w[a], c.n, c.K, c.w_stride[a], BM, &mw[a])) return cudaErrorNotSupported;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.split > 1 ? tiles * p.split : tiles < b->sm_count ? tiles : b->sm_count));
    cfg.blockDim = dim3(threads_of(W4));
    cfg.dynamicSmemBytes = 1024 + (size_t)p.stages * p.stage + BAR_BYTES;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = p.split;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = p.split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, product<W4, NW>, p, mx, mw[0], mw[1]);
}

template <bool W4, int NW>
cudaError_t prepare(tpq_block *b)
{
    return cudaFuncSetAttribute(product<W4, NW>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_MAX);
}

}  // namespace

// Once per handle: the kernels' shared memory, and how many clusters of each size run side by side (one block an SM).
cudaError_t product_prepare(tpq_block *b)
{
    cudaError_t e = prepare<true, 1>(b);
    if (e == cudaSuccess) e = prepare<true, 2>(b);
    if (e == cudaSuccess) e = prepare<false, 2>(b);
    for (int s = 2; s <= 8 && e == cudaSuccess; ++s) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)s);
        cfg.blockDim = dim3(threads_of(true));
        cfg.dynamicSmemBytes = SMEM_MAX;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = s;
        at[0].val.clusterDim.y = 1;
        at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&b->clusters[s], product<true, 2>, &cfg);
    }
    return e;
}

cudaError_t product_launch(const product_call &c, const tpq_block *b, cudaStream_t st, int64_t *launches)
{
    params p = {};
    p.T = c.T;
    p.n = (int)c.n;
    p.out = c.out;
    p.out_stride = c.out_stride;
    p.out_fp32 = c.out_fp32;
    p.act = c.act;
    p.status = b->status;
    p.group_shift = c.group == 32 ? 5 : c.group == 64 ? 6 : 7;
    if (c.group)
        for (int a = 0; a < c.n_weights; ++a) {
            p.w4[a] = static_cast<const uint8_t *>(c.w[a]);
            p.factor[a] = reinterpret_cast<const float *>(p.w4[a] + w4_factors_at(c.n, c.K, c.group));
        }
    cudaError_t e;
    if (!c.group) e = launch<false, 2>(p, c, b, st);
    else if (c.n_weights == 2) e = launch<true, 2>(p, c, b, st);
    else e = launch<true, 1>(p, c, b, st);
    if (e == cudaSuccess) ++*launches;
    return e;
}
