// Products with a device's weights: x W^T with W in 4 bits (tpq_linear4), and the feed-forward block's
// act(x Wg^T) * (x Wu^T) with both matrices in BF16 or in 4 bits (tpq_gated), in one kernel for one token and for thousands.
//
// The OUTPUTS are the rows of the tensor cores' tile and the tokens its columns (tcgen05, M = 128, N = 16 .. 256 tokens, K = 16): few tokens
// then cost few columns, and a tile of tokens reads the weights once: up to 256 tokens (128 with two weights in 4 bits, 192 for FP32 outputs) all do.  Gate and up are two accumulators over the same tokens, so the
// activation and the product are the epilogue's, in binary32, with one rounding.
//
// Weights in 4 bits become BF16 operands in TENSOR memory: a thread is a row of the tile (an output), takes 64 codes of it from shared
// memory and stores the 64 values with one tcgen05.st; nothing is written to shared memory again.  A step has 5 significant bits and a code
// is -8 .. 7, so step * code IS a BF16 number (products.h).  An output's power of two multiplies its sum at the end.
//
//   warp 0      copies (one lane): blocks of weights (4 bits: as they lie, 128 outputs x 128 inputs) and the tokens' inputs
//   warp 1      tensor memory, MMA issue (one elected lane)
//   warps 2-17  4 bits: codes to operands, two groups of warps in turns, of which one waits and loads while the other computes; a warp has 32 rows x
//               half of a stage's inputs (few tokens: 8 warps, one group); then, as with BF16, the epilogue
//
// One accumulator set (for FP32 outputs see ADD): the epilogue, which all 16 warps share, is 1 to 3 % of a large tile's time, and wider tiles save more
// than a second set would.  The first stages of the next tile are unpacked ahead of it.  One commit a stage frees its shared memory and its operands: a
// commit costs the tensor pipe about 300 clocks (with one for each 64-wide piece, one token's head of 32000 outputs x 5120 took 49 us).
//
// Few tokens: a tile's inputs are split over the blocks of a cluster, so that all SMs read weights; each block stores its part of the sums to the
// block of the cluster that ends with them, which adds them in the order of the blocks (the same call gives the same bits).
//
// What bounds it (B200; products of other work in turn, so that weights come from memory).  Many tokens: the tensor pipe (67 % of all cycles active at the clock
// that the power limit leaves): gated 1999 x 5120 x 3456 in 4 bits 103 us (1370 TFLOP/s) in passes one behind the other in a graph, 124 in a program under that limit; 2048 in
// BF16 106 and 125 us, where shared memory is as close.  Few tokens,
// 4 bits: unpacking (9 instructions for 8 codes of 32 outputs, 20 with all that goes round it) and what is left over when tiles of 128 outputs
// are dealt out: 32000 x 5120, one token, BF16 out 22.7 to 24 us (3.5 to 3.8 TB/s); without unpacking, stores to tensor memory and MMAs it would be 18.6.  BF16: memory, 18 us of
// 2 x 4608 x 4608, one token (4.7 TB/s).  One token of 5120 x 1728: 5.5 us, latency (2.7 us from the first copy to the sums, 1.7 us cluster and stores).
// Tried for few tokens and not kept: mma.sync (16 outputs x 16 inputs x 8 tokens) with weights unpacked in registers, no barriers and no tensor memory:
// 32 to 38 us of the 32000 x 5120 whatever was done to it, 66 with 16 tokens, 138 with 32: one takes 33 clocks of a scheduler.
// Every wait is bounded.  A warp whose wait expires records TPQ_ERR_TIMEOUT and tells its block and its cluster: a split tile is then not stored at all,
// of others what has its sums is; the copies and MMAs that are under way end before the block's memory is given back.
#include <cuda_bf16.h>

#include "block_internal.h"
#include "products.h"

namespace {

constexpr int BM = 128, MOST_STAGES = 16, MOST_DEPTH = 4, ADD_STAGES = 4;
constexpr int WAIT_LIMIT = 1 << 24;                     // try_wait attempts (each suspends for a hardware time slice) ...
constexpr unsigned long long WAIT_NS = 1000000000ull;   // ... and one second, whichever ends first
#ifdef TPQ_GIVE_UP  // (a test's build: bit p of it has waits for parity p expire that are not over at the first look, the others after 10 ms)
constexpr unsigned GIVE_UP = TPQ_GIVE_UP;
constexpr unsigned long long PATIENCE_NS = 10000000ull;
#else
constexpr unsigned GIVE_UP = 0;
constexpr unsigned long long PATIENCE_NS = WAIT_NS;
#endif
constexpr uint32_t SMEM_MAX = 227u * 1024u, SMEM_HALF = 112u * 1024u;  // of a block that has an SM for itself, of two beside one another
constexpr uint32_t BAR_BYTES = 512;                     // barriers, the tensor-memory address, whether a wait expired
constexpr uint32_t W_BF16_BYTES = BM * 64 * 2;

struct params {
    int64_t T;
    int n, tiles_n, tiles_t, N, pitch;  // N: tokens of a tile; pitch: columns of an accumulator
    int kstages, blocks;                // stages of a tile, blocks (4 bits) of a row of tiles
    int split, stages, depth;           // blocks of a tile; ring; stages whose operands fit tensor memory
    uint32_t w_block, x_at, stage, tmem_cols;
    int turns;                          // ADD with sums in tensor memory: 1 where two accumulators take turns, 0 where there is one
    uint32_t sums_at;                   // of a split tile: where the cluster's partial sums go, from the first stage on (0: over the stages)
    int group_shift;
    const uint8_t *w4[2];
    const float *factor[2];
    void *out;
    int64_t out_stride;
    int out_fp32, act;
    int *status;
};

__device__ __forceinline__ uint32_t try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok;
}
// (out of line: most waits end at the first attempt, and the loop's code would cost them 30 of their 90 clocks)
template <unsigned long long NS>
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity)
{
    unsigned long long t0 = 0;
    bool ok = false;
    for (int i = 0; i < WAIT_LIMIT; ++i) {
        ok = try_wait(bar, parity);
        if (ok) break;
        if ((i & 63) == 63) {
            unsigned long long t;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (t0 == 0) t0 = t;
            else if (t - t0 > NS) break;
        }
    }
    return __all_sync(0xffffffffu, ok);
}
template <unsigned long long NS = WAIT_NS>
__device__ __forceinline__ bool wait_end(uint32_t bar, uint32_t parity)
{
    return __all_sync(0xffffffffu, try_wait(bar, parity)) || wait_long<NS>(bar, parity);
}
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity)  // by a whole warp
{
    if (GIVE_UP >> (parity & 1) & 1) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        return __all_sync(0xffffffffu, ok);
    }
    return wait_end<PATIENCE_NS>(bar, parity);
}

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
// Operands in shared memory: descriptors' low words; the high word is the same for all.  Rows of 128 bytes with the 128-byte swizzle, 8-row groups
// of 1024 bytes; a step of 16 along K is 32 bytes.
__device__ __forceinline__ uint32_t operand_low(uint32_t addr) { return ((addr & 0x3FFFFu) >> 4) | 1u << 16; }
constexpr uint32_t OPERAND_HIGH = (1024 >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 x, {%1, %3};\n\t"
        "mov.b64 y, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b), "r"(OPERAND_HIGH), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 y, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b), "r"(OPERAND_HIGH), "r"(idesc), "r"(accumulate)
        : "memory");
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
__device__ __forceinline__ void st(uint32_t addr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::S4(r, 0), S4(r, 4), S4(r, 8), S4(r, 12), S4(r, 16), S4(r, 20), S4(r, 24), S4(r, 28), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void st(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::S4(r, 0), S4(r, 4), S4(r, 8),
        S4(r, 12), "r"(addr)
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
// 32 codes (a 16-byte piece of the layout) times their step: pairs (2i, 2i + 1) as BF16
__device__ __forceinline__ void unpack32(const uint4 &c, uint32_t byte, uint32_t *r)
{
    const uint32_t words[4] = {c.x, c.y, c.z, c.w};
    const w4_step step = w4_load_step(byte);
#pragma unroll
    for (int q = 0; q < 4; ++q) w4_unpack(words[q], step, r + 4 * q);
}

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

// NW weights.  KB: inputs of a stage, 128 KB; 0: BF16 weights, 64 inputs.  WORKERS: 8 or 16.  HALF: of an SM, for two blocks.
// (An SM's registers are given to warps by fours: 10 warps cost as much as 12.)
// ADD (FP32 outputs): the tensor cores cut off what does not fit their binary32 sums, 4e-9 of the norm for every 16 inputs.  So they add up at most 512 inputs, and
// the warps that unpack add these sums up, rounded to nearest:
//   few tokens (KB = 2)   a stage's, in registers, ahead of handing over the next one's operands: it is complete when these have room.
//   more (KB = 1)         those of 4 stages (a chunk), in tensor memory: 32 sums of a thread in registers made unpacking 15 % slower.  Up to 128 tokens two accumulators
//                         take turns; beyond, and with two blocks on an SM, there is room for one, and the tensor cores wait while a chunk is drained.
// Logits of 5120 inputs are off by 0.8 to 1.1e-7 of their norm (sums of binary32 products: 0.9e-7), cut off over all inputs by 1.3e-6; 32000 outputs of 5120 in FP32 take 27.0 us
// for one token (BF16 24.2), 34.5 for 64 (28.0), 45 for 128 (42), 151 for 512 (125); 2048 x 3456 x 5120 63 us (56.5).
template <int NW, int KB, int WORKERS, bool HALF, bool ADD>
__global__ void __launch_bounds__(HALF ? 384 : (2 + WORKERS) * 32, HALF ? 2 : 1)
product(const params p, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1)
{
    extern __shared__ uint8_t raw[];
    constexpr bool W4 = KB > 0;
    constexpr int KX = W4 ? 2 * KB : 1;          // 64-wide pieces of the inputs in a stage
    constexpr uint32_t A_COLS = KX * NW * 32;    // of tensor memory for a stage's operands
    constexpr bool IN_REGS = ADD && KB == 2, IN_TMEM = ADD && KB == 1;
    constexpr int CHUNK = IN_TMEM ? ADD_STAGES : 1 << 30;  // stages that the tensor cores add up
    const int turns = HALF ? 0 : p.turns, accs = IN_TMEM ? 2 + turns : NW;  // accumulators (IN_TMEM: and the sums)
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t bars = base + p.stages * p.stage;
    uint8_t *const gen = raw + (base - smem_u32(raw));
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(gen + p.stages * p.stage + BAR_BYTES - 16);
    volatile uint32_t *const expired = tmem_slot + 1;  // a wait of this block or of its cluster
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (MOST_STAGES + s); };
    auto a_full = [&](int s) { return bars + 8u * (2 * MOST_STAGES + s); };
    auto acc_full = [&](int b) { return bars + 8u * (2 * MOST_STAGES + MOST_DEPTH + b); };  // (IN_TMEM: of the two accumulators; else 0)
    auto acc_empty = [&](int b) { return bars + 8u * (2 * MOST_STAGES + MOST_DEPTH + 2 + b); };
    // the accumulator of the n-th set of sums, and its barriers' parity
    auto which = [&](uint32_t n) { return IN_TMEM ? n & turns : 0u; };
    auto parity = [&](uint32_t n) { return IN_TMEM ? n >> turns & 1 : n & 1; };

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tiles = p.tiles_n * p.tiles_t, places = gridDim.x / p.split;
    const int rank = p.split > 1 ? (int)(blockIdx.x % p.split) : 0, first_tile = blockIdx.x / p.split;
    const int kb0 = (int)((int64_t)p.kstages * rank / p.split), kb1 = (int)((int64_t)p.kstages * (rank + 1) / p.split);
    // tiles in bands of 16 tiles of tokens, in a band output by output: blocks that run together share weights
    auto origin = [&](int tile, int &tn, int &tt) {
        const int per = 16 * p.tiles_n, band = tile / per, in = tile - band * per;
        const int rows = p.tiles_t - 16 * band < 16 ? p.tiles_t - 16 * band : 16;
        tn = in / rows;
        tt = band * 16 + in - tn * rows;
    };
    // pieces of stage kb (with two blocks a stage, the last one of a row may have one)
    auto pieces = [&](int kb) { return KB == 2 && 2 * kb + 1 == p.blocks ? 2 : KX; };

    if (tid == 0) *expired = 0;
    __syncwarp();
    if (p.split > 1 && p.sums_at) cluster_arrive();  // (the blocks' memory is there: waited for ahead of the first store to it)
    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int s = 0; s < MOST_DEPTH; ++s) mbar_init(a_full(s), 8);  // one arrival per warp of a group
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), WORKERS);
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
        for (int i = kb0; i < kb0 + n; ++i) {
            if (W4) {
                for (int a = 0; a < NW; ++a)
                    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p.w4[a] + ((int64_t)tn * p.blocks + KB * i) * p.w_block), "r"(pieces(i) / 2 * p.w_block)
                                 : "memory");
            } else {
                asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(&map_w0), "r"(i * 64), "r"(tn * BM) : "memory");
                if (NW == 2) asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(&map_w1), "r"(i * 64), "r"(tn * BM) : "memory");
            }
        }
    }
    fence_before();
    tpq_grid_dep_wait();
    __syncthreads();
    tpq_grid_dep_launch();
    fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t a_at = tmem + (uint32_t)(accs * p.pitch);  // operands behind the accumulators
    bool ok = true;
    ring last;      // warp 0: behind the last stage copied; warp 1: the last stage multiplied
    int issued = 0;  // stages, warp 0 up to the ring's length
    uint32_t complete = 0;  // warp 1: commits of the accumulators
    float sum[IN_REGS ? 16 : 1];  // of columns 16 * part .. of the warp's rows

    if (warp == 0) {
        // the copies of a stage leave from as many lanes
        ring r;
        for (int tile = first_tile; tile < tiles && ok; tile += places) {
            int tn, tt;
            origin(tile, tn, tt);
            const uint8_t *w = W4 && lane < NW ? p.w4[lane] + ((int64_t)tn * p.blocks + KB * kb0) * p.w_block : nullptr;
            for (int kb = kb0; kb < kb1; ++kb, r.next(p.stages)) {
                if (issued == p.stages) ok = wait_warp(empty(r.s), r.phase ^ 1);
                else ++issued;
                if (!ok) break;
                const uint32_t at = base + r.s * p.stage, bar = full(r.s);
                const int kx = pieces(kb);
                if (lane == 0) mbar_expect_tx(bar, (W4 ? NW * KB * p.w_block / KX * kx : NW * W_BF16_BYTES) + kx * (uint32_t)p.N * 128);
                __syncwarp();
                if (W4) {
                    const uint32_t bytes = KB * p.w_block / KX * kx;
                    if (lane < NW) bulk_g2s(at + lane * p.w_block, w, bytes, bar);
                    w += KB * p.w_block;
                } else if (lane < NW) {
                    tma_load_2d(at + lane * W_BF16_BYTES, lane ? &map_w1 : &map_w0, kb * 64, tn * BM, bar);
                }
                if (lane < kx) tma_load_2d(at + p.x_at + lane * (p.N * 128), &map_x, (kb * KX + lane) * 64, tt * p.N, bar);
            }
        }
        last = r;
    } else if (warp == 1) {
        const uint32_t idesc = instr(p.N), tmem1 = tmem + (uint32_t)p.pitch, x_piece = (uint32_t)p.N * 128 >> 4;
        ring r, t;  // of shared memory and of the operands in tensor memory
        for (int tile = first_tile; tile < tiles && ok; tile += places) {
            for (int kb = kb0; kb < kb1; ++kb, r.next(p.stages)) {
                const int in_chunk = IN_TMEM ? (kb - kb0) % CHUNK : kb - kb0;
                const bool first = IN_REGS || in_chunk == 0, end = !IN_REGS && (kb == kb1 - 1 || in_chunk == CHUNK - 1);
                if (!IN_REGS && first) {  // (ahead of an accumulator's first set there is nothing to wait for)
                    ok = wait_warp(acc_empty(which(complete)), parity(complete) ^ 1);
                    if (!ok) break;
                }
                // (operands in tensor memory are there: so is the rest of their stage, which their warps waited for)
                ok = W4 ? wait_warp(a_full(t.s), t.phase) : wait_warp(full(r.s), r.phase);
                if (!ok) break;
                fence_after();
                if (elect()) {
                    const uint32_t at = base + r.s * p.stage, x = operand_low(at + p.x_at);
                    if (W4) {
                        const int kx = pieces(kb);
                        const uint32_t a0 = a_at + t.s * A_COLS, d = which(complete) ? tmem1 : tmem;
#pragma unroll
                        for (int j = 0; j < KX; ++j) {
                            if (j >= kx) break;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
#pragma unroll
                                for (int a = 0; a < NW; ++a)
                                    mma_ts(a ? tmem1 : d, a0 + (uint32_t)((j * NW + a) * 32 + k * 8), x + j * x_piece + 2 * k, idesc, j + k ? 1u : (uint32_t)!first);
                        }
                    } else {
                        const uint32_t w = operand_low(at);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int a = 0; a < NW; ++a)
                                mma_ss(a ? tmem1 : tmem, w + a * (W_BF16_BYTES >> 4) + 2 * k, x + 2 * k, idesc, k ? 1u : (uint32_t)!first);
                    }
                    commit(empty(r.s));
                    if (end) commit(acc_full(which(complete)));
                }
                __syncwarp();
                last = r;
                issued = 1;
                complete += end;
                if (W4) t.next(p.depth);
            }
        }
    } else {
        const int q = warp & 3, part = (warp - 2) >> 2;  // rows q * 32 .. of a tile (the quarter of tensor memory that this warp reaches)
        const uint32_t from = tmem + ((uint32_t)(q * 32) << 16);
        const uint32_t sums_or_up = (uint32_t)((IN_TMEM ? 1 + turns : 1) * p.pitch);
        uint32_t filled = 0;  // sets of sums drained
        // What the tensor cores have added up: the oldest chunk that is not drained, of tile `undrained`.
        const int nk = kb1 - kb0, chunks = IN_TMEM ? (nk + CHUNK - 1) / CHUNK : 1;
        int undrained = first_tile, chunk = 0;
        // one that is not its tile's last: to the tile's sums
        auto gather = [&]() {
            ok = wait_warp(acc_full(which(filled)), parity(filled));
            if (!ok) return;
            fence_after();
            const uint32_t acc = from + which(filled) * p.pitch + 16 * part, sums = from + sums_or_up + 16 * part;
#pragma unroll
            for (int c = 0; c < (HALF ? 64 : 192); c += 4 * WORKERS) {
                if (16 * part + c >= p.N) break;
                uint32_t y[16], z[16];
                ld16(acc + c, y);
                if (chunk) {
                    ld16(sums + c, z);
                    ld_wait(y);
                    ld_wait(z);
#pragma unroll
                    for (int j = 0; j < 16; ++j) y[j] = __float_as_uint(__uint_as_float(z[j]) + __uint_as_float(y[j]));
                } else ld_wait(y);
                st(sums + c, y);
            }
            st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty(which(filled)));
            ++filled;
            ++chunk;
        };
        // The last one, and with it its tile's sums: scaled, through the activation, to memory.  (A split tile's is left for the cluster.)
        auto epilogue = [&]() {
            int tn, tt;
            origin(undrained, tn, tt);
            const int col = tn * BM + q * 32 + lane;
            float f0 = 1.0f, f1 = 1.0f;
            if (W4) {
                f0 = W4_SCALE * p.factor[0][col];
                if (NW == 2) f1 = W4_SCALE * p.factor[1][col];
            }
            ok = wait_warp(acc_full(which(filled)), parity(filled));
            if (!ok) return;
            fence_after();
            const int64_t t0 = (int64_t)tt * p.N;
            for (int c = 16 * part; c < p.N; c += 4 * WORKERS) {
                if (t0 + c >= p.T) break;
                uint32_t y0[16], y1[16];
                ld16(from + which(filled) * p.pitch + c, y0);
                if (NW == 2 || (IN_TMEM && chunk)) ld16(from + sums_or_up + c, y1);
                ld_wait(y0);
                if (NW == 2 || (IN_TMEM && chunk)) ld_wait(y1);
                if (col < p.n) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        if (t0 + c + j >= p.T) break;
                        float v = __uint_as_float(y0[j]);
                        if (IN_TMEM && chunk) v += __uint_as_float(y1[j]);
                        v *= f0;
                        if (NW == 2) v = activation(v, p.act) * (__uint_as_float(y1[j]) * f1);
                        store(p, t0 + c + j, col, v);
                    }
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty(which(filled)));
            ++filled;
            undrained += places;
            chunk = 0;
        };
        auto drain = [&]() {
            if (IN_TMEM && chunk < chunks - 1) gather();
            else epilogue();
        };
        // IN_REGS: a stage's sums to its tile's, and those to memory
        const uint32_t my_sums = from + 16 * part;
        const bool summing = IN_REGS && 16 * part < p.N;
        auto add = [&]() {
            uint32_t y[16];
            ld16(my_sums, y);
            ld_wait(y);
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[IN_REGS ? j : 0] += __uint_as_float(y[j]);
        };
        auto finish = [&](int tile) {
            int tn, tt;
            origin(tile, tn, tt);
            const int col = tn * BM + q * 32 + lane;
            const int64_t t0 = (int64_t)tt * p.N + 16 * part;
            const float f = W4_SCALE * p.factor[0][col];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                if (IN_REGS && summing && col < p.n && t0 + j < p.T) store(p, t0 + j, col, sum[IN_REGS ? j : 0] * f);
                sum[IN_REGS ? j : 0] = 0.0f;
            }
        };
        if (!W4) {
            if (p.split == 1)
                while (undrained < tiles && ok) drain();
        } else {
            // A warp of the stage's group has half of its 64-wide pieces: of one weight consecutive ones, of two weights one of each.
            constexpr int MINE = KX * NW / 2;
            const int half = part & 1, turn = part >> 1;  // (8 warps: one group)
            const uint32_t row = (uint32_t)(q * 32 + lane);
            uint32_t codes[MINE], steps[MINE];
#pragma unroll
            for (int m = 0; m < MINE; ++m) {
                const int j = NW == 2 ? half : half * MINE + m;  // the piece along the inputs
                const uint32_t block = (uint32_t)(NW == 2 ? m : j >> 1) * p.w_block;
                codes[m] = block + (j & 1) * (2 * BM * 16) + row * 16;
                steps[m] = block + W4_CODE_BYTES + (((j & 1) * 64) >> p.group_shift) * BM + row;
            }
            const uint32_t second = (uint32_t)((32 >> p.group_shift) * BM);  // from the step of a piece's first 32 inputs to that of the others
            const uint32_t to = a_at + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * MINE * 32);
            ring r, t, done;  // done: the stage whose operands lay in the same place, `depth` stages ago
            // Stages until the next chunk is drained.  That is ahead of the one whose operands take the place of those that wait for it, `depth` stages behind
            // the chunk; sums of parts of a tile are drained a stage behind it, with two accumulators two (they are complete by then).
            int left = (IN_TMEM && chunks > 1 ? CHUNK : nk) + (IN_TMEM ? 1 + turns : p.depth);
            int fresh = p.depth, skip = turn;                 // places that held no operands yet; whether the next stage is the other group's
            if (IN_REGS)
#pragma unroll
                for (int j = 0; j < 16; ++j) sum[IN_REGS ? j : 0] = 0.0f;
            for (int tile = first_tile; tile < tiles && ok; tile += places) {
                for (int kb = kb0; kb < kb1; ++kb, r.next(p.stages), t.next(p.depth)) {
                    if (!IN_REGS && left-- == 0) {
                        drain();
                        if (!ok) break;
                        left = (chunk == chunks - 1 ? nk - chunk * (IN_TMEM ? CHUNK : 0) : CHUNK) - 1;
                    }
                    const ring free = done;
                    const bool used = fresh == 0;
                    if (used) done.next(p.stages);
                    else --fresh;
                    if (WORKERS == 16) {
                        skip ^= 1;
                        if (!skip) continue;
                    }
                    ok = wait_warp(full(r.s), r.phase);
                    if (!ok) break;
                    const uint32_t at = base + r.s * p.stage;
                    const bool there = KB < 2 || half == 0 || pieces(kb) == KX;
#pragma unroll
                    for (int m = 0; m < MINE; ++m) {
                        uint32_t v[32];
                        if (there) {
                            const uint32_t s0 = lds8(at + steps[m]), s1 = lds8(at + steps[m] + second);
                            const uint4 c0 = lds128(at + codes[m]), c1 = lds128(at + codes[m] + BM * 16);
                            unpack32(c0, s0, v);
                            unpack32(c1, s1, v + 16);
                        }
                        if (m == 0) {
                            if (used) ok = wait_warp(empty(free.s), free.phase);
                            if (!ok) break;
                            fence_after();
                        }
                        if (there) st(to + t.s * A_COLS + m * 32, v);
                        if (IN_REGS && m == MINE - 1 && used && summing) add();  // (the stage before this one's, complete as its operands are free: depth is 1)
                    }
                    if (!ok) break;
                    if (IN_REGS && used && kb == kb0 && p.split == 1) finish(tile - places);
                    st_wait();
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(a_full(t.s));
                }
            }
            if (IN_REGS) {
                ok = ok && wait_warp(empty(done.s), done.phase);
                if (ok) {
                    fence_after();
                    if (summing) add();
                    if (p.split == 1) finish(first_tile + (tiles - 1 - first_tile) / places * places);
                }
            } else if (p.split == 1) {
                while (undrained < tiles && ok) drain();
            } else {
                while (chunk < chunks - 1 && ok) gather();
            }
        }
        if (p.split > 1 && !IN_REGS) ok = ok && wait_warp(acc_full(which(filled)), parity(filled));
    }
    if (!ok) {
        atomicExch(p.status, (int)TPQ_ERR_TIMEOUT);
        *expired = 1;
    }
    if (p.split > 1) {
        // Every block ends with a share of the tile's cells (token, output): the others store theirs of it to its memory, [block][weight][cell],
        // and it adds them in the order of the blocks.
        int tn, tt;
        origin(first_tile, tn, tt);
        const int64_t t0 = (int64_t)tt * p.N;
        const int tokens = (int)(p.T - t0 < p.N ? p.T - t0 : p.N);
        const int share = ((tokens + p.split - 1) / p.split) * BM, from = rank * share;
        const int mine = tokens * BM - from < share ? tokens * BM - from : share;
        const float *const sums = reinterpret_cast<const float *>(gen + p.sums_at);
        const int first_col = tn * BM + (tid & (BM - 1));
        float f0 = 1.0f, f1 = 1.0f;
        if (W4 && tid < mine) {
            f0 = W4_SCALE * p.factor[0][first_col];
            if (NW == 2) f1 = W4_SCALE * p.factor[1][first_col];
        }
        if (!p.sums_at) cluster_arrive();  // (this block's stages are free)
        cluster_wait();
        if (!ok && lane < p.split) st_cluster(map_cluster(smem_u32(tmem_slot + 1), lane), 1u);
        __syncwarp();
        if (warp >= 2 && ok) {
            fence_after();
            const int q = warp & 3, part = (warp - 2) >> 2, per = (tokens + p.split - 1) / p.split;
            const uint32_t at = tmem + ((uint32_t)(q * 32) << 16), cell0 = base + p.sums_at + 4u * (uint32_t)(rank * NW * share + q * 32 + lane);
            for (int c = 16 * part; c < tokens; c += 4 * WORKERS) {
                uint32_t y0[16], y1[16];
                if (IN_REGS) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) y0[j] = __float_as_uint(sum[IN_REGS ? j : 0]);
                } else {
                    const int chunk = IN_TMEM ? (kb1 - kb0 - 1) / CHUNK : 0;  // the last one
                    const bool added = chunk > 0;
                    ld16(at + which(chunk) * p.pitch + c, y0);
                    if (NW == 2 || added) ld16(at + (IN_TMEM ? 1 + turns : 1) * p.pitch + c, y1);
                    ld_wait(y0);
                    if (NW == 2 || added) ld_wait(y1);
                    if (added)
#pragma unroll
                        for (int j = 0; j < 16; ++j) y0[j] = __float_as_uint(__uint_as_float(y1[j]) + __uint_as_float(y0[j]));
                }
                int owner = c / per, in = c - owner * per;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    if (c + j >= tokens) break;
                    const uint32_t to = map_cluster(cell0 + 4u * (uint32_t)(in * BM), owner);
                    st_cluster(to, y0[j]);
                    if (NW == 2) st_cluster(to + 4u * (uint32_t)share, y1[j]);
                    if (++in == per) in = 0, ++owner;
                }
            }
        }
        cluster_arrive();
        cluster_wait();
        const bool all_there = *expired == 0;
        for (int i = tid; i < mine; i += blockDim.x) {
            const int cell = from + i, col = tn * BM + (cell & (BM - 1));
            float v = 0.0f, u = 0.0f;
#pragma unroll 8
            for (int k = 0; k < p.split; ++k) {
                v += sums[k * NW * share + i];
                if (NW == 2) u += sums[(k * NW + 1) * share + i];
            }
            if (col >= p.n || !all_there) continue;
            if (W4 && i != tid) {
                f0 = W4_SCALE * p.factor[0][col];
                if (NW == 2) f1 = W4_SCALE * p.factor[1][col];
            }
            v *= f0;
            if (NW == 2) v = activation(v, p.act) * (u * f1);
            store(p, t0 + cell / BM, col, v);
        }
    }
    fence_before();
    __syncthreads();
    if (*expired) {
        // giving up: what was issued ends before shared and tensor memory are given back (the rest of a whole walk has been waited for)
        if (warp == 0) {
            if (issued < p.stages) last = ring{0, 1};
            for (int j = 0; j < issued; ++j, last.next(p.stages)) (void)wait_end(full(last.s), last.phase ^ 1);
        } else if (warp == 1 && issued) {
            (void)wait_end(empty(last.s), last.phase);
            if (complete) (void)wait_end(acc_full(which(complete - 1)), parity(complete - 1));
        }
    }
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

template <int NW, int KB, int WORKERS, bool HALF, bool ADD = false>
cudaError_t launch(params p, const product_call &c, const tpq_block *b, cudaStream_t st)
{
    constexpr bool W4 = KB > 0;
    constexpr int KX = W4 ? 2 * KB : 1, TMEM = HALF ? 256 : 512;
    const int places = b->sm_count * (HALF ? 2 : 1);
    p.kstages = (int)((c.K + KX * 64 - 1) / (KX * 64));
    p.blocks = (int)((c.K + 127) / 128);
    p.w_block = W4 ? w4_block_bytes(c.group) : W_BF16_BYTES;
    p.x_at = ((W4 ? NW * KB : NW) * p.w_block + 1023) / 1024 * 1024;
    p.stage = p.x_at + KX * p.N * 128;
    p.stages = (int)(((HALF ? SMEM_HALF : SMEM_MAX) - 1024 - BAR_BYTES) / p.stage);
    if (p.stages > MOST_STAGES) p.stages = MOST_STAGES;
    const int64_t tiles = (int64_t)p.tiles_n * p.tiles_t;
    // The partial sums' place is beside the ring, or, where the ring would lose half of itself, in it.
    const uint32_t sums = p.split > 1 ? (uint32_t)(p.split * NW * ((p.N + p.split - 1) / p.split) * BM * 4) : 0;
    const int most = p.stages, walk = (p.kstages + p.split - 1) / p.split;
    // (no more of the ring than a single tile fills: the next kernel's blocks then start beside this one's)
    if (tiles * p.split <= places && p.stages > walk) p.stages = walk;
    bool beside = false;
    if (sums) {
        const uint32_t room = (HALF ? SMEM_HALF : SMEM_MAX) - 1024 - BAR_BYTES;
        const int with = (int)((room - sums) / p.stage);
        beside = with >= p.stages || 2 * with > most;
        if (beside && with < p.stages) p.stages = with;
        if (!beside && p.stages * p.stage < sums) p.stages = (int)((sums + p.stage - 1) / p.stage);
    }
    p.sums_at = beside ? p.stages * p.stage + BAR_BYTES : 0;
    const int a_cols = KX * NW * 32;
    p.turns = ADD && KB == 1 && !HALF && p.N <= 128;
    const int accs = ADD && KB == 1 ? 2 + p.turns : NW;
    p.depth = W4 ? (TMEM - accs * p.pitch) / a_cols : 1;
    if (ADD && KB == 2) p.depth = 1;  // (the sums of a stage are read ahead of the next one's)
    if (p.depth > MOST_DEPTH) p.depth = MOST_DEPTH;
    if (p.depth > p.stages) p.depth = p.stages;
    const int cols = accs * p.pitch + (W4 ? p.depth * a_cols : 0);
    p.tmem_cols = cols <= 32 ? 32 : cols <= 64 ? 64 : cols <= 128 ? 128 : cols <= 256 ? 256 : 512;
    CUtensorMap mx, mw[2];
    if (!make_map(c.x, c.T, c.K, c.x_stride, p.N, &mx)) return cudaErrorNotSupported;
    for (int a = 0; a < 2; ++a) {
        mw[a] = mx;
        if (!W4 && a < NW && !make_map(c.w[a], c.n, c.K, c.w_stride[a], BM, &mw[a])) return cudaErrorNotSupported;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.split > 1 ? tiles * p.split : tiles < places ? tiles : places));
    cfg.blockDim = dim3((2 + WORKERS) * 32);
    cfg.dynamicSmemBytes = 1024 + (size_t)p.stages * p.stage + BAR_BYTES + (beside ? sums : 0);
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
    return cudaLaunchKernelEx(&cfg, product<NW, KB, WORKERS, HALF, ADD>, p, mx, mw[0], mw[1]);
}

template <int NW, int KB, int WORKERS, bool HALF, bool ADD = false>
cudaError_t prepare()
{
    return cudaFuncSetAttribute(product<NW, KB, WORKERS, HALF, ADD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(HALF ? SMEM_HALF : SMEM_MAX));
}

// (What a block of half an SM takes, for the question of how many clusters run side by side.  Of the product kernels it is answered as if
// one block filled an SM; two do: 15.8 warps were active on average, where one block has 10.)
__global__ void __launch_bounds__(384, 2) half_block() {}

// clusters of `split` blocks that run side by side
template <bool HALF>
cudaError_t count_clusters(int split, int *n)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(split * 148));
    cfg.blockDim = dim3((2 + (HALF ? 8 : 16)) * 32);
    cfg.dynamicSmemBytes = HALF ? SMEM_HALF : SMEM_MAX;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = split;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (HALF) return cudaOccupancyMaxActiveClusters(n, half_block, &cfg);
    return cudaOccupancyMaxActiveClusters(n, product<2, 1, 16, false, false>, &cfg);
}

}  // namespace

// Once per handle: the kernels' shared memory, and how many clusters of each size run side by side.
cudaError_t product_prepare(tpq_block *b)
{
    cudaError_t e = prepare<1, 1, 16, false>();
    if (e == cudaSuccess) e = prepare<1, 1, 16, false, true>();
    if (e == cudaSuccess) e = prepare<2, 1, 16, false>();
    if (e == cudaSuccess) e = prepare<2, 0, 16, false>();
    if (e == cudaSuccess) e = prepare<1, 1, 8, true>();
    if (e == cudaSuccess) e = prepare<1, 1, 8, true, true>();
    if (e == cudaSuccess) e = prepare<1, 2, 8, true>();
    if (e == cudaSuccess) e = prepare<1, 2, 8, true, true>();
    if (e == cudaSuccess) e = prepare<2, 1, 8, true>();
    if (e == cudaSuccess) e = cudaFuncSetAttribute(half_block, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_HALF);
    for (int s = 2; s <= 8 && e == cudaSuccess; ++s) {
        e = count_clusters<false>(s, &b->clusters[s]);
        if (e == cudaSuccess) e = count_clusters<true>(s, &b->clusters_half[s]);
    }
    return e;
}

namespace {

enum kernel_kind { BF16_GATED, GATED, GATED_HALF, LINEAR, LINEAR_HALF, LINEAR_HALF_DEEP };
struct plan {
    kernel_kind kind;
    int N, split;
};

// The kernel, the tokens of a tile and the blocks that share one: the least estimated time, in clocks.  A stage's (`one` or, for two tokens of the tile,
// `token`, whichever is more; sums of FP32 outputs cost 7 % more, and 25 % of 64 tokens) are measured: 4 bits and many tokens are what the tensor cores take under the power limit (256 tokens 1500, with
// two weights 128 tokens 1640); few are what unpacking takes, more where a second block is on the SM (`beside`); BF16 weights are bound by shared
// memory, 128 bytes a clock for the copies in and the operands out (512 + 3 a token), or by memory.
// 2048 x 3456 x 5120 in 4 bits: tiles of 192 tokens 58 us (three rounds), of 256 63.5 (three, the third a sixth full); gated 2048 x 5120 x 3456 in
// BF16: of 208 106 us, of 256 111.  32000 outputs of 5120, one token: 22.7 us with two blocks on an SM, 27.3 with one; 64 tokens 27.2 and 30.8; but
// two weights of 4608 x 4608 and 61 tokens 21.0 and 15.1.  One token of 4608 x 4608, gated: 11.1 us with 7 blocks to a tile, 13.0 with 4.
plan choose(const product_call &c, const tpq_block *b, int tiles_n)
{
    const bool two = c.n_weights == 2;
    const int most = c.group && two ? 128 : c.out_fp32 ? 192 : 256;
    const int64_t t0 = (c.T + most - 1) / most;
    plan best = {};
    int64_t best_cost = 0;
    for (int64_t t = t0; t < t0 + (c.T > 64 ? 8 : 1); ++t) {
        const int N = (int)(((c.T + t - 1) / t + 15) / 16 * 16);
        const int64_t tiles = tiles_n * ((c.T + N - 1) / N);
        const kernel_kind kind = !c.group ? BF16_GATED : two ? N <= 32 ? GATED_HALF : GATED : N <= 32 ? LINEAR_HALF_DEEP : N <= 64 ? LINEAR_HALF : LINEAR;
        const bool half = kind == GATED_HALF || kind == LINEAR_HALF || kind == LINEAR_HALF_DEEP;
        const int deep = kind == BF16_GATED ? 64 : kind == LINEAR_HALF_DEEP ? 256 : 128;
        const int kstages = (int)((c.K + deep - 1) / deep);
        int64_t one, token = 0, beside = 0;  // token: of two tokens; beside: with a second block on the SM
        switch (kind) {
        case BF16_GATED: one = 512 + 3 * N > 1100 ? 512 + 3 * N : 1100; break;
        case GATED: one = 1450, token = 26; break;
        case LINEAR: one = c.out_fp32 ? 960 : 900, token = c.out_fp32 ? 15 : 12; break;
        case GATED_HALF: one = 1700, beside = 1900; break;
        case LINEAR_HALF: one = c.out_fp32 ? 950 : 750, beside = c.out_fp32 ? 1350 : 1100; break;
        default: one = 1170, beside = 1800; break;
        }
        if (token * N / 2 > one) one = token * N / 2;
        const int64_t end = 800 + (two ? 7 : 4) * N;
        const int *const clusters = half ? b->clusters_half : b->clusters;
        for (int s = 1; s <= 8 && s <= kstages; ++s) {
            if (s > 1 && tiles > clusters[s]) continue;
            if (s > 1 && (int64_t)s * c.n_weights * ((N + s - 1) / s) * BM * 4 > 128 * 1024) continue;  // (partial sums that no ring has room for)
            const int64_t blocks = tiles * s, places = (int64_t)b->sm_count * (half ? 2 : 1), rounds = (blocks + places - 1) / places;
            const int64_t stage = half && blocks > b->sm_count ? beside : one;
            const int64_t cost = rounds * ((kstages + s - 1) / s * stage + end) + (s > 1 ? 2000 + 150 * s : 0);
            if (best_cost && cost >= best_cost) continue;
            best_cost = cost;
            best = {kind, N, s};
        }
    }
    return best;
}

}  // namespace

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
    p.tiles_n = (int)((c.n + BM - 1) / BM);
    const plan best = choose(c, b, p.tiles_n);
    p.N = best.N;
    p.tiles_t = (int)((c.T + p.N - 1) / p.N);
    p.pitch = (p.N + 31) / 32 * 32;
    p.split = best.split;
    cudaError_t e;
    switch (best.kind) {
    case BF16_GATED: e = launch<2, 0, 16, false>(p, c, b, st); break;
    case GATED: e = launch<2, 1, 16, false>(p, c, b, st); break;
    case GATED_HALF: e = launch<2, 1, 8, true>(p, c, b, st); break;
    case LINEAR: e = c.out_fp32 ? launch<1, 1, 16, false, true>(p, c, b, st) : launch<1, 1, 16, false>(p, c, b, st); break;
    case LINEAR_HALF: e = c.out_fp32 ? launch<1, 1, 8, true, true>(p, c, b, st) : launch<1, 1, 8, true>(p, c, b, st); break;
    default: e = c.out_fp32 ? launch<1, 2, 8, true, true>(p, c, b, st) : launch<1, 2, 8, true>(p, c, b, st); break;
    }
    if (e == cudaSuccess) ++*launches;
    return e;
}
