// Products with a device's weights: x W^T with W in 4 bits (tpq_linear4), and the feed-forward block's
// act(x Wg^T) * (x Wu^T) with both matrices in BF16 or in 4 bits (tpq_gated), in one kernel for one token and for thousands.
//
// The OUTPUTS are the rows of the tensor cores' tile and the tokens its columns (tcgen05, M = 128, N = 16 .. 256 tokens, K = 16): few tokens
// then cost few columns, and weights are read once whatever T is.  Gate and up are two accumulators over the same tokens, so the
// activation and the product are the epilogue's, in binary32, with one rounding.
//
// Weights in 4 bits become BF16 operands in TENSOR memory: a thread is a row of the tile (an output), takes 64 codes of it from shared
// memory and stores the 64 values with one tcgen05.st; nothing is written to shared memory again.  A step has 5 significant bits and a code
// is -8 .. 7, so step * code IS a BF16 number (products.h).  An output's power of two multiplies its sum at the end.
//
//   warp 0      copies (one lane): blocks of weights (4 bits: as they lie, 128 outputs x 128 inputs) and the tokens' inputs
//   warp 1      tensor memory, MMA issue (one elected lane)
//   warps 2-17  4 bits: codes to operands, two groups of warps in turns, of which one waits and loads while the other computes; a warp has 32 rows x
//               half of a stage's inputs; then, as with BF16, the epilogue
//
// One accumulator set: the epilogue, which all 16 warps share, is 1 to 3 % of a large tile's time, and wider tiles save more than a second
// set would.  The first stages of the next tile are unpacked ahead of it.  One commit a stage frees its shared memory and its operands: a
// commit costs the tensor pipe about 300 clocks (with one for each 64-wide piece, one token's head of 32000 outputs x 5120 took 49 us).
//
// Few tokens: a tile's inputs are split over the blocks of a cluster, so that all SMs read weights; the partial sums meet in the
// cluster's shared memory and are added in the order of the blocks (the same call gives the same bits).
// Every wait is bounded: on expiry the block records TPQ_ERR_TIMEOUT, skips its stores, frees its tensor memory and returns.
#include <cuda_bf16.h>

#include "block_internal.h"
#include "products.h"

namespace {

constexpr int BM = 128, MOST_STAGES = 16, MOST_DEPTH = 4, WORKERS = 16, THREADS = (2 + WORKERS) * 32;
constexpr int WAIT_LIMIT = 1 << 24;                     // try_wait attempts (each suspends for a hardware time slice) ...
constexpr unsigned long long WAIT_NS = 1000000000ull;   // ... and one second, whichever ends first
constexpr uint32_t SMEM_MAX = 227u * 1024u;
constexpr uint32_t BAR_BYTES = 512;                     // barriers and the tensor-memory address
constexpr uint32_t W_BF16_BYTES = BM * 64 * 2;

struct params {
    int64_t T;
    int n, tiles_n, tiles_t, N, pitch;  // N: tokens of a tile; pitch: columns of an accumulator
    int kstages, blocks;                // stages of a tile, blocks (4 bits) of a row of tiles
    int split, stages, depth;           // blocks of a tile; ring; stages whose operands fit tensor memory
    uint32_t w_block, x_at, stage, tmem_cols;
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
            else if (t - t0 > WAIT_NS) break;
        }
    }
    return __all_sync(0xffffffffu, ok);
}
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity)  // by a whole warp
{
    return __all_sync(0xffffffffu, try_wait(bar, parity)) || wait_long(bar, parity);
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

// NW weights.  KB: inputs of a stage, 128 KB; 0: BF16 weights, 64 inputs.
template <int NW, int KB>
__global__ void __launch_bounds__(THREADS, 1)
product(const params p, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1)
{
    extern __shared__ uint8_t raw[];
    constexpr bool W4 = KB > 0;
    constexpr int KX = W4 ? 2 * KB : 1;          // 64-wide pieces of the inputs in a stage
    constexpr uint32_t A_COLS = KX * NW * 32;    // of tensor memory for a stage's operands
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t bars = base + p.stages * p.stage;
    uint8_t *const gen = raw + (base - smem_u32(raw));
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(gen + p.stages * p.stage + BAR_BYTES - 16);
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (MOST_STAGES + s); };
    auto a_full = [&](int s) { return bars + 8u * (2 * MOST_STAGES + s); };
    const uint32_t acc_full = bars + 8u * (2 * MOST_STAGES + MOST_DEPTH), acc_empty = acc_full + 8u;

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

    if (tid == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int s = 0; s < MOST_DEPTH; ++s) mbar_init(a_full(s), WORKERS / 2);  // one arrival per warp of a group
        mbar_init(acc_full, 1);
        mbar_init(acc_empty, WORKERS);
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
    const uint32_t a_at = tmem + (uint32_t)(NW * p.pitch);  // operands behind the accumulators
    bool ok = true;

    if (warp == 0) {
        // the copies of a stage leave from as many lanes
        ring r;
        int used = 0;  // stages issued so far, up to the ring's length
        for (int tile = first_tile; tile < tiles && ok; tile += places) {
            int tn, tt;
            origin(tile, tn, tt);
            const uint8_t *w = W4 && lane < NW ? p.w4[lane] + ((int64_t)tn * p.blocks + KB * kb0) * p.w_block : nullptr;
            for (int kb = kb0; kb < kb1; ++kb, r.next(p.stages)) {
                if (used == p.stages) ok = wait_warp(empty(r.s), r.phase ^ 1);
                else ++used;
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
        if (!ok) {  // giving up: let the copies already issued land before the shared memory is released
            ring l = r;
            for (int j = 0; j < p.stages; ++j) {
                (void)wait_warp(full(l.s), l.phase ^ 1);
                l.next(p.stages);
            }
        }
    } else if (warp == 1) {
        const uint32_t idesc = instr(p.N), tmem1 = tmem + (uint32_t)p.pitch, x_piece = (uint32_t)p.N * 128 >> 4;
        ring r, t;  // of shared memory and of the operands in tensor memory
        bool more = false;
        uint32_t drained = 0;
        for (int tile = first_tile; tile < tiles && ok; tile += places) {
            if (more) {
                ok = wait_warp(acc_empty, drained);
                drained ^= 1;
            }
            more = true;
            if (!ok) break;
            for (int kb = kb0; kb < kb1; ++kb, r.next(p.stages)) {
                // (operands in tensor memory are there: so is the rest of their stage, which their warps waited for)
                ok = W4 ? wait_warp(a_full(t.s), t.phase) : wait_warp(full(r.s), r.phase);
                if (!ok) break;
                fence_after();
                if (elect()) {
                    const uint32_t at = base + r.s * p.stage, x = operand_low(at + p.x_at);
                    if (W4) {
                        const int kx = pieces(kb);
                        const uint32_t a0 = a_at + t.s * A_COLS;
#pragma unroll
                        for (int j = 0; j < KX; ++j) {
                            if (j >= kx) break;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
#pragma unroll
                                for (int a = 0; a < NW; ++a)
                                    mma_ts(a ? tmem1 : tmem, a0 + (uint32_t)((j * NW + a) * 32 + k * 8), x + j * x_piece + 2 * k, idesc, j + k ? 1u : (uint32_t)(kb != kb0));
                        }
                    } else {
                        const uint32_t w = operand_low(at);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int a = 0; a < NW; ++a)
                                mma_ss(a ? tmem1 : tmem, w + a * (W_BF16_BYTES >> 4) + 2 * k, x + 2 * k, idesc, k ? 1u : (uint32_t)(kb != kb0));
                    }
                    commit(empty(r.s));
                    if (kb == kb1 - 1) commit(acc_full);
                }
                __syncwarp();
                if (W4) t.next(p.depth);
            }
        }
    } else {
        const int q = warp & 3, part = (warp - 2) >> 2;  // rows q * 32 .. of a tile (the quarter of tensor memory that this warp reaches)
        uint32_t filled = 0;
        // The tile's sums: scaled, through the activation, to memory; or, of a split tile, to this block's shared memory.
        auto epilogue = [&](int tile) {
            int tn, tt;
            origin(tile, tn, tt);
            const int col = tn * BM + q * 32 + lane;
            float f0 = 1.0f, f1 = 1.0f;
            if (W4) {
                f0 = W4_SCALE * p.factor[0][col];
                if (NW == 2) f1 = W4_SCALE * p.factor[1][col];
            }
            ok = wait_warp(acc_full, filled);
            filled ^= 1;
            if (!ok) return;
            fence_after();
            const uint32_t from = tmem + ((uint32_t)(q * 32) << 16);
            const int64_t t0 = (int64_t)tt * p.N;
            for (int c = 16 * part; c < p.N; c += 4 * WORKERS) {
                if (t0 + c >= p.T) break;
                uint32_t y0[16], y1[16];
                ld16(from + c, y0);
                if (NW == 2) ld16(from + p.pitch + c, y1);
                ld_wait(y0);
                if (NW == 2) ld_wait(y1);
                if (p.split > 1) {
                    float *const sums = reinterpret_cast<float *>(gen) + q * 32 + lane;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        sums[(c + j) * BM] = __uint_as_float(y0[j]);
                        if (NW == 2) sums[(p.N + c + j) * BM] = __uint_as_float(y1[j]);
                    }
                } else if (col < p.n) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        if (t0 + c + j >= p.T) break;
                        float v = __uint_as_float(y0[j]) * f0;
                        if (NW == 2) v = activation(v, p.act) * (__uint_as_float(y1[j]) * f1);
                        store(p, t0 + c + j, col, v);
                    }
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty);
        };
        if (!W4) {
            for (int tile = first_tile; tile < tiles && ok; tile += places) epilogue(tile);
        } else {
            // A warp of the stage's group has half of its 64-wide pieces: of one weight consecutive ones, of two weights one of each.
            constexpr int MINE = KX * NW / 2;
            const int half = part & 1, turn = part >> 1;
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
            const int nk = kb1 - kb0;
            int undrained = first_tile;                       // the oldest tile that is not drained yet ...
            int64_t it = 0, drain = (int64_t)nk + p.depth;    // ... and the stage ahead of which it is
            for (int tile = first_tile; tile < tiles && ok; tile += places) {
                for (int kb = kb0; kb < kb1; ++kb, ++it, r.next(p.stages), t.next(p.depth)) {
                    if (it == drain) {
                        epilogue(undrained);
                        if (!ok) break;
                        undrained += places;
                        drain += nk;
                    }
                    const ring free = done;
                    if (it >= p.depth) done.next(p.stages);
                    if ((int)(it & 1) != turn) continue;
                    ok = wait_warp(full(r.s), r.phase);
                    if (!ok) break;
                    const uint32_t at = base + r.s * p.stage;
                    const bool there = KB < 2 || half == 0 || pieces(kb) == KX;
#pragma unroll
                    for (int m = 0; m < MINE; ++m) {
                        uint32_t v[32];
                        if (there) {
                            const uint4 c0 = lds128(at + codes[m]), c1 = lds128(at + codes[m] + BM * 16);
                            const uint32_t s0 = lds8(at + steps[m]), s1 = lds8(at + steps[m] + second);
                            unpack32(c0, s0, v);
                            unpack32(c1, s1, v + 16);
                        }
                        if (m == 0) {
                            if (it >= p.depth) ok = wait_warp(empty(free.s), free.phase);
                            if (!ok) break;
                            fence_after();
                        }
                        if (there) st(to + t.s * A_COLS + m * 32, v);
                    }
                    if (!ok) break;
                    st_wait();
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(a_full(t.s));
                }
            }
            for (; undrained < tiles && ok; undrained += places) epilogue(undrained);
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
            if (KB > 0) v *= W4_SCALE * p.factor[0][col];
            if (NW == 2) {
                if (KB > 0) u *= W4_SCALE * p.factor[1][col];
                v = activation(v, p.act) * u;
            }
            store(p, t0 + i / BM, col, v);
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

template <int NW, int KB>
cudaError_t launch(params p, const product_call &c, const tpq_block *b, cudaStream_t st)
{
    constexpr bool W4 = KB > 0;
    constexpr int KX = W4 ? 2 * KB : 1;
    p.kstages = (int)((c.K + KX * 64 - 1) / (KX * 64));
    p.blocks = (int)((c.K + 127) / 128);
    p.w_block = W4 ? w4_block_bytes(c.group) : W_BF16_BYTES;
    p.x_at = ((W4 ? NW * KB : NW) * p.w_block + 1023) / 1024 * 1024;
    p.stage = p.x_at + KX * p.N * 128;
    p.stages = (int)((SMEM_MAX - 1024 - BAR_BYTES) / p.stage);
    if (p.stages > MOST_STAGES) p.stages = MOST_STAGES;
    const int64_t tiles = (int64_t)p.tiles_n * p.tiles_t;
    // few tiles: the inputs of each split over a cluster
    p.split = 1;
    for (int s = 2; s <= 8 && s <= p.kstages; ++s)
        if (tiles <= b->clusters[s] && (uint64_t)NW * p.N * BM * 4 <= (uint64_t)p.stages * p.stage) p.split = s;
    const int a_cols = KX * NW * 32;
    p.depth = W4 ? (512 - NW * p.pitch) / a_cols : 1;
    if (p.depth > MOST_DEPTH) p.depth = MOST_DEPTH;
    if (p.depth > p.stages) p.depth = p.stages;
    const int cols = NW * p.pitch + (W4 ? p.depth * a_cols : 0);
    p.tmem_cols = cols <= 32 ? 32 : cols <= 64 ? 64 : cols <= 128 ? 128 : cols <= 256 ? 256 : 512;
    CUtensorMap mx, mw[2];
    if (!make_map(c.x, c.T, c.K, c.x_stride, p.N, &mx)) return cudaErrorNotSupported;
    for (int a = 0; a < 2; ++a) {
        mw[a] = mx;
        if (!W4 && a < NW && !make_map(c.w[a], c.n, c.K, c.w_stride[a], BM, &mw[a])) return cudaErrorNotSupported;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.split > 1 ? tiles * p.split : tiles < b->sm_count ? tiles : b->sm_count));
    cfg.blockDim = dim3(THREADS);
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
    return cudaLaunchKernelEx(&cfg, product<NW, KB>, p, mx, mw[0], mw[1]);
}

template <int NW, int KB>
cudaError_t prepare()
{
    return cudaFuncSetAttribute(product<NW, KB>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_MAX);
}

}  // namespace

// Once per handle: the kernels' shared memory, and how many clusters of each size run side by side (one block an SM).
cudaError_t product_prepare(tpq_block *b)
{
    cudaError_t e = prepare<1, 1>();
    if (e == cudaSuccess) e = prepare<1, 2>();
    if (e == cudaSuccess) e = prepare<2, 1>();
    if (e == cudaSuccess) e = prepare<2, 0>();
    for (int s = 2; s <= 8 && e == cudaSuccess; ++s) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)s);
        cfg.blockDim = dim3(THREADS);
        cfg.dynamicSmemBytes = SMEM_MAX;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = s;
        at[0].val.clusterDim.y = 1;
        at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&b->clusters[s], product<2, 1>, &cfg);
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
    // the tile's tokens
    const int most = c.group && c.n_weights == 2 ? 128 : 256;
    p.tiles_t = (int)((c.T + most - 1) / most);
    p.N = (int)(((c.T + p.tiles_t - 1) / p.tiles_t + 15) / 16 * 16);
    p.tiles_t = (int)((c.T + p.N - 1) / p.N);
    p.pitch = (p.N + 31) / 32 * 32;
    p.tiles_n = (int)((c.n + BM - 1) / BM);
    cudaError_t e;
    if (!c.group) e = launch<2, 0>(p, c, b, st);
    else if (c.n_weights == 2) e = launch<2, 1>(p, c, b, st);
    else if (p.N <= 64) e = launch<1, 2>(p, c, b, st);
    else e = launch<1, 1>(p, c, b, st);
    if (e == cudaSuccess) ++*launches;
    return e;
}
