// Attention over the 4-bit cache (tpq_kv_attention) for sequences that bring many rows: prompts and chunks of them.
//
// Scores S = Q K^T of 128 rows x 128 positions and sums O += P V run on tcgen05, P from tensor memory.  What a row's thread does per
// element decides the speed, so that here, unlike in kv_attention.cu, keys and values are formed, in FP16: with 2^F the scale of a
// block of 16 positions' values (their largest magnitude M is 2^14 .. 2^15 of it), v_t 2^-F is rounded once, to 11 bits where it is at
// least 2^-28 of that magnitude; keys likewise with 2^Fk, and a row of Q with its own power of two, which is exact.  (F is also the
// block's for rows that see only some of it: P of theirs is that much larger, and where M is 2^21 times what they see, other positions'
// P fall below FP16's normal numbers; 2^-31 M a position in all.)  A row (query head
// x new position) of S is one thread's, which finds
//   y_t = S_t (2^Fk 2^Fq scale log2 e) + F,   P_t = 2^(y_t - m + 7) in FP16,
//   l = sum over blocks of 2^-F sum P_t,   out = O / l.
// m moves only when a row's maximum has grown by more than 8 (P stays below 2^15): O is rescaled in tensor memory then, which
// after a sequence's first tiles hardly happens.
//
// A block has 256 rows (two tiles of 128, A and B) of one key head and walks tiles of 128 positions.  Tensor memory holds S_A, S_B
// (P in their place) and O_A, O_B, all of it.  While the exponentials of one row tile run, the tensor cores work for the other:
//   ... P_A E(j), Q_A C(j+1), P_B E(j), Q_B C(j+1), P_A E(j+1), ...
//   warp 0       copies: blocks of 16 positions as they lie in the pages, 64 positions a stage
//   warp 1       tensor memory, MMA issue (one elected lane)
//   warps 2-9    unpack: codes to the two operands' tiles (128-byte swizzle), words to the terms of a block
//   warps 10-17  softmax: a thread per row; the rows themselves into shared memory at the start, the output at the end
// Unpacking a tile costs as much however many rows use it: 256 rows, which the query heads of a key head share.
//
// Work.  attention_plan lists the (sequence, 256 rows) pairs and adds up their tiles (causal, window); a run of tiles in that order
// goes to each block, all of the same length.  A run that begins or ends inside a pair's key head leaves a partial result, at
// most two a block, which attention_prompt_join puts together.
//
// What bounds it.  4800 clocks for 256 rows x 128 positions, 2080 of them on the tensor pipe (without contention for shared memory): of each
// row tile the scores, the walk over them (650 clocks to the maximum, 2000 of exponentials) and the products follow each other, and only
// the two row tiles overlap.  Two limits lie close behind: a product of scores reads 64 KB of operands in its 520 clocks, all that shared memory
// gives (128 bytes a clock), while the unpacking writes 64 KB a tile into it; and the tile's 32 768 exponentials are 2048 clocks at 16 a clock.
// 2 x 8191 tokens, 32 heads of 128 on 16, window 4096: 1112 to 1135 us, 727 to 742 TFLOP/s of what is visible; 2048 tokens, 10 heads: 46 us, of which
// the plan, the first and last tiles and the joining are half.  Heads of 64 leave half of the sums' columns unused.  Measured (against 1100 us then) and not kept: scores in two halves of 64 positions a step ahead (a
// product of 64 columns takes as long as one of 128, whose rows of Q are what is read: 1463 us), both softmax warpgroups on one row tile (the
// exchange of maxima costs more than it hides: 1405 us), an MMA thread for each row tile (1235 us), blocks of 16 scores
// loaded while the one before is worked on (1209 us against 1104: more and smaller loads and stores of tensor memory), codes instead of formed keys and values as operands (five
// terms a position to load per row: 2750 us at the time, against 2285 with formed values), 128 scores in registers (89 KB of code: a
// quarter of the warps' time went into fetching instructions).
// Every wait is bounded: on expiry the block records TPQ_ERR_TIMEOUT, frees its tensor memory and returns.
#include "kv_internal.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace {

constexpr int BM = 256, TILE = 128, HALF = 64;  // rows of a block, positions of a tile, of a copy stage
constexpr int RAW = 4;                          // copy stages
constexpr int THREADS = 18 * 32;
constexpr int UNPACK = 2, SOFTMAX = 10;         // first warps of those roles (eight each: two on every scheduler)
constexpr int PLAN_THREADS = 1024;
// Runs are dealt out in units: a (256 rows, key head) pair is its tiles and EXTRA more, which stand for its beginning and end (13 700
// clocks against 4800 of a tile: fitted to the blocks' times.  2 x 8191 tokens, 32 heads on 16, window 4096: 1098 us; with 2 extra ones
// 1266, 4: 1103, 6: 1122).
constexpr int EXTRA = 3;

// A sequence's rows row0 .. row0 + rows - 1 (row: new position x query head of a key head).
struct alignas(16) plan_item {
    int seq, before, tiles, rows;   // before: units (below) of the items ahead
    int first, from;                // tiles that any row sees: [0, first) and [from, ...), `tiles` in all
    int lo[2], hi[2];               // positions of the first and last row of row tiles A and B (hi < lo: it has none)
    int tok, head, row0, len;       // of the first row: row of the step's tensors and query head in its group; the sequence's length
    int pad[2];
};
static_assert(sizeof(plan_item) == 64, "four vector loads");
struct alignas(16) plan_head {
    int items, total, pad[2];
};
struct prompt_params {
    kv_batch b;
    kv_attention_call c;
    plan_head *head;
    plan_item *items;
    int *seq_items;  // [sequences] items ahead of a sequence's
    int most_items;
    int4 *headers;  // as in attention_split
    float *parts;   // [blocks][2][BM][D + 4]
    float scale2;
    int group, group_inv, few;  // group_inv: 2^20 / group rounded up; sequences of up to `few` rows are attention_split's
};

__device__ __forceinline__ plan_item item_of(const kv_seq &s, const kv_attention_call &c, int group, int block)
{
    plan_item t{};
    t.row0 = block * BM;
    const int left = s.n * group - t.row0;  // (rows of a sequence fit 31 bits: checked by the host)
    t.rows = left < BM ? left : BM;
    const int p0 = s.len - s.n, tok = t.row0 / group;
    t.tok = s.start + tok;
    t.head = t.row0 - tok * group;
    t.len = s.len;
    for (int k = 0; k < 2; ++k) {
        const int rows = t.rows - 128 * k;
        t.lo[k] = p0 + (t.row0 + 128 * k) / group;
        t.hi[k] = rows > 0 ? p0 + (t.row0 + 128 * k + (rows < 128 ? rows : 128) - 1) / group : t.lo[k] - 1;
    }
    if (c.window) {
        const int from = t.lo[0] - c.window + 1;
        if (from > 0) {
            t.from = from / TILE;
            const int first = ((c.n_first < from ? c.n_first : from) + TILE - 1) / TILE;
            t.first = first < t.from ? first : t.from;
        }
    }
    t.tiles = t.first + (t.rows > 128 ? t.hi[1] : t.hi[0]) / TILE + 1 - t.from;
    return t;
}

__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t *warps, int64_t &total)  // inclusive; PLAN_THREADS threads
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, x, m);
        if (lane >= m) x += o;
    }
    __syncthreads();
    if (lane == 31) warps[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int64_t y = warps[lane];
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) {
            const int64_t o = __shfl_up_sync(0xffffffffu, y, m);
            if (lane >= m) y += o;
        }
        warps[lane] = y;
    }
    __syncthreads();
    total = warps[31];
    return x + (warp ? warps[warp - 1] : 0);
}

// One block: the list of items, and the tiles ahead of each.  Sums in 64 bits: 1024 items may have 2^33 tiles.
__global__ void __launch_bounds__(PLAN_THREADS) attention_plan(const prompt_params p)
{
    __shared__ int64_t warps[32];
    tpq_grid_dep_wait();
    tpq_grid_dep_launch();
    const kv_batch &b = p.b;
    int64_t items = 0;
    for (int s0 = 0; s0 < b.n_seqs; s0 += PLAN_THREADS) {
        const int s = s0 + threadIdx.x;
        int n = 0;
        if (s < b.n_seqs) {
            const kv_seq q = kv_load_seq(b, s);
            if (q.n * p.group > p.few) n = (q.n * p.group + BM - 1) / BM;
        }
        int64_t total;
        const int64_t at = items + block_scan(n, warps, total) - n;
        items += total;
        if (s < b.n_seqs && items <= p.most_items) p.seq_items[s] = (int)at;
        if (items > p.most_items) break;  // (uniform)
    }
    if (items > p.most_items) {  // starts that overlap: more rows than there are
        if (threadIdx.x == 0) {
            kv_report(b);
            *p.head = plan_head{0, 0, {0, 0}};
        }
        return;
    }
    __syncthreads();
    int64_t before = 0;
    for (int i0 = 0; i0 < items; i0 += PLAN_THREADS) {
        const int i = i0 + threadIdx.x;
        int n = 0;
        plan_item it{};
        if (i < items) {
            int lo = 0, hi = b.n_seqs;  // the last sequence whose items begin at or before i
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (p.seq_items[mid] <= i) lo = mid;
                else hi = mid;
            }
            it = item_of(kv_load_seq(b, lo), p.c, p.group, i - p.seq_items[lo]);
            it.seq = lo;
            n = it.tiles + EXTRA;
        }
        int64_t total;
        const int64_t at = before + (block_scan(n, warps, total) - n) * b.n_kv_heads;
        before += total * b.n_kv_heads;
        if (i < items) {
            it.before = (int)at;  // (used only if all of them fit)
            p.items[i] = it;
        }
    }
    if (threadIdx.x == 0) {
        if (before > KV_MOST_UNITS) {
            kv_report(b);
            before = 0;
        }
        *p.head = plan_head{(int)items, (int)before, {0, 0}};
    }
}

// ---- waits, tensor memory, MMA

constexpr int WAIT_LIMIT = 1 << 24;
constexpr unsigned long long WAIT_NS = 1000000000ull;
__device__ __forceinline__ bool arrived(uint32_t bar, uint32_t parity)
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
// (out of line: two dozen waits' loops would not leave the instruction cache room for the arithmetic)
__device__ __noinline__ bool wait_more(uint32_t bar, uint32_t parity)
{
    unsigned long long t0 = 0;
#pragma unroll 1
    for (int i = 0; i < WAIT_LIMIT; ++i) {
        if (arrived(bar, parity)) return true;
        if ((i & 63) == 63) {
            unsigned long long t;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (t0 == 0) t0 = t;
            else if (t - t0 > WAIT_NS) return false;
        }
    }
    return false;
}
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) { return arrived(bar, parity) || wait_more(bar, parity); }
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
// (the descriptors' high halves are constants: only the low ones are held)
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 x, {%1, %3};\n\t"
        "mov.b64 y, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b), "r"(high), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 y, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b), "r"(high), "r"(idesc), "r"(accumulate)
        : "memory");
}
#define R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define W8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of the thread's row (the values are there after ld_wait)
__device__ __forceinline__ void ld32(uint32_t addr, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : R8(r, 0), R8(r, 8), R8(r, 16), R8(r, 24)
        : "r"(addr)
        : "memory");
}
#define T8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
// (the loaded registers pass through: nothing that uses them comes ahead of the wait; `loaded`: of another 32, behind the same wait)
__device__ __forceinline__ void ld_wait(uint32_t *r) { asm volatile("tcgen05.wait::ld.sync.aligned;" : T8(r, 0), T8(r, 8), T8(r, 16), T8(r, 24)::"memory"); }
__device__ __forceinline__ void loaded(uint32_t *r) { asm volatile("" : T8(r, 0), T8(r, 8), T8(r, 16), T8(r, 24)::"memory"); }
__device__ __forceinline__ void st32(uint32_t addr, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::W8(r, 0), W8(r, 8), W8(r, 16), W8(r, 24), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void st16(uint32_t addr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::W8(r, 0), W8(r, 8), "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Operands of 128-byte rows with the 128-byte swizzle, 8-row groups of 1024 bytes.  Depth along the row (Q, keys): a step of 16 is 32
// bytes of the row, 64-deep sub-tiles lie behind each other.  Depth along the rows (values: a row is a position, along it the head's
// values): a step of 16 is 16 rows, the next 64 values are `lead` bytes on.
__device__ __forceinline__ uint32_t operand(uint32_t addr, uint32_t lead) { return ((addr & 0x3FFFFu) >> 4) | ((lead >> 4) << 16); }
constexpr uint32_t OPERAND_HIGH = (1024 >> 4) | (1u << 14) | (2u << 29);  // 1024 bytes from 8 rows to the next; version; 128-byte swizzle
// FP32 sums of 128 rows x n columns of FP16 products; `rows_deep`: B's depth runs along its rows
__host__ __device__ constexpr uint32_t instr(int n, bool rows_deep)
{
    return (1u << 4) | (rows_deep ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t bits)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(a), "r"(mask), "r"(bits));
    return r;
}
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }
// two binary32 operations an instruction
typedef unsigned long long f2;
__device__ __forceinline__ f2 pack2(float a, float b)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f2 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c)
{
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b)
{
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ float4 lds4(uint32_t addr)
{
    float4 r;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(r.x), "=f"(r.y), "=f"(r.z), "=f"(r.w) : "r"(addr));
    return r;
}
// Terms of a block of 16 positions: 2^Fk, F, 2^-F (Fk, F: exponents of its keys' and values' scales).
constexpr uint32_t TERM_BYTES = TILE / KV_BLOCK * 16;
// FP16 step and low of a position for a scale that puts the block's largest magnitude in [2^14, 2^15); e: that one's exponent field.
// Called by a warp, lane <-> position lane % 16; a vector of nobody counts as zeros.
__device__ __forceinline__ uint32_t to_scale(float step, float low, bool on, int &e)
{
    float big = on ? fminf(fmaxf(fabsf(low), fabsf(fmaf(15.0f, step, low))), 3.4e38f) : 0.0f;
    const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(big));  // (not negative: in the order of its bits)
    e = top < 0x21800000u ? 67 : (int)(top >> 23);  // (nothing is below 2^-57 but zeros)
    const float inv = __uint_as_float((uint32_t)(268 - e) << 23);  // 2^(141 - e)
    const __half2 h = __floats2half2_rn(on ? step * inv : 0.0f, on ? low * inv : 0.0f);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// 8 codes -> low + step * code in the order 0 4 1 5 2 6 3 7, one rounding
__device__ __forceinline__ uint4 values(uint32_t w, uint32_t step_low)
{
    const __half2 sl = *reinterpret_cast<const __half2 *>(&step_low), step = __low2half2(sl), low = __high2half2(sl);
    const uint32_t hi = w >> 8;
    uint32_t u[4] = {and_or(w, 0x000f000fu, 0x64006400u), and_or(w, 0x00f000f0u, 0x64006400u), and_or(hi, 0x000f000fu, 0x64006400u), and_or(hi, 0x00f000f0u, 0x64006400u)};
#pragma unroll
    for (int z = 0; z < 4; ++z) {  // 1024 + c, 1024 + 16 c -> c, exactly
        const __half2 c = *reinterpret_cast<const __half2 *>(&u[z]);
        const __half2 y = __hfma2(z & 1 ? __hfma2(c, __float2half2_rn(0.0625f), __float2half2_rn(-64.0f)) : __hadd2(c, __float2half2_rn(-1024.0f)), step, low);
        u[z] = *reinterpret_cast<const uint32_t *>(&y);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

template <int D>
struct Smem {
    static constexpr uint32_t TILE_BYTES = TILE * D * 2;  // an operand tile
    static constexpr uint32_t Q = 0, K = Q + 2 * TILE_BYTES, V = K + 2 * TILE_BYTES, RAWS = V + 2 * TILE_BYTES;
    static constexpr uint32_t RAW_BYTES = HALF / KV_BLOCK * kv_block_bytes(D);
    static constexpr uint32_t TERM = RAWS + RAW * RAW_BYTES;
    static constexpr uint32_t BARS = TERM + 3 * TERM_BYTES;
    static constexpr uint32_t BYTES = BARS + 304;
    static_assert(BYTES <= 227 * 1024, "shared memory of a block");
};
// barriers, 8 bytes each from BARS
enum { B_RAW_FULL = 0, B_RAW_EMPTY = B_RAW_FULL + RAW, B_K_FULL = B_RAW_EMPTY + RAW, B_V_FULL = B_K_FULL + 2, B_K_EMPTY = B_V_FULL + 2, B_V_EMPTY = B_K_EMPTY + 2,
       B_Q_FULL = B_V_EMPTY + 2, B_S_FULL = B_Q_FULL + 2, B_P_FULL = B_S_FULL + 2 /* 2 x half + row tile */, B_O_FULL = B_P_FULL + 4, B_O_EMPTY = B_O_FULL + 2, B_T_FULL = B_O_EMPTY + 2,
       B_COUNT = B_T_FULL + 3 };
static_assert(8 * B_COUNT + 4 * RAW + 4 <= 304, "barriers");

// A block's run of units, one (item, key head) after the other.
struct run {
    int unit, end, item;
};
struct segment {
    const plan_item *item;
    int kh, t0, nt;  // tiles t0 .. t0 + nt - 1 of the item's
    int first, skip; // (for base)
    __device__ __forceinline__ int base(int j) const  // first position of tile j of the segment
    {
        const int t = t0 + j;
        return (t < first ? t : t + skip) * TILE;
    }
};
// The next segment with a tile in it; false at the run's end.
__device__ __forceinline__ bool next_segment(const prompt_params &p, run &r, segment &g)
{
#pragma unroll 1
    while (r.unit < r.end) {
        const plan_item *it = p.items + r.item;
        const int4 q = *reinterpret_cast<const int4 *>(it);  // seq, before, tiles, rows
        const int weight = q.z + EXTRA, off = r.unit - q.y;
        if (off >= weight * p.b.n_kv_heads) {
            ++r.item;
            continue;
        }
        const int kh = off / weight, o = off - kh * weight, n = weight - o < r.end - r.unit ? weight - o : r.end - r.unit;
        r.unit += n;
        const int t0 = o > EXTRA ? o - EXTRA : 0, t1 = o + n - EXTRA;
        if (t1 <= t0) continue;
        const int2 f = *reinterpret_cast<const int2 *>(&it->first);
        g = segment{it, kh, t0, t1 - t0, f.x, f.y - f.x};
        return true;
    }
    return false;
}
// Positions of a row tile's first and last row (hi < lo: it has none).
struct reach {
    int lo, hi;
};
__device__ __forceinline__ reach reach_of(const segment &g, int t) { return reach{g.item->lo[t], g.item->hi[t]}; }
// Whether a row tile sees any position of a tile that starts at `base`; whether all of its rows see all of it.
__device__ __forceinline__ bool sees(const prompt_params &p, const reach &r, int base)
{
    return r.hi >= r.lo && base <= r.hi && (p.c.window == 0 || base + TILE - 1 > r.lo - p.c.window || base < p.c.n_first);
}
__device__ __forceinline__ bool sees_all(const prompt_params &p, const reach &r, int base)
{
    return base + TILE - 1 <= r.lo && (p.c.window == 0 || base > r.hi - p.c.window || base + TILE <= p.c.n_first);
}

// 16 positions' codes to rows row0 .. of an operand tile; scaled: step and low of position lane % 16
template <int D>
__device__ __forceinline__ void unpack(const uint8_t *codes, uint8_t *tile, int row0, uint32_t scaled, int lane)
{
    uint4 c[D / 64];
    uint32_t sl[D / 64];
#pragma unroll
    for (int k = 0; k < D / 64; ++k) {
        // 16 bytes (32 codes) of position `row`; eight lanes read and write 128 different bytes of banks
        const int row = D == 128 ? (lane & 7) + 8 * k : lane & 15, q = D == 128 ? ((lane >> 3) + (row >> 1)) & 3 : lane >> 4;
        c[k] = *reinterpret_cast<const uint4 *>(codes + row * (D / 2) + 16 * q);
        sl[k] = __shfl_sync(0xffffffffu, scaled, row);
    }
#pragma unroll
    for (int k = 0; k < D / 64; ++k) {
        const int row = D == 128 ? (lane & 7) + 8 * k : lane & 15, q = D == 128 ? ((lane >> 3) + (row >> 1)) & 3 : lane >> 4;
        uint8_t *const line = tile + (q >> 1) * (TILE * 128) + (row0 + row) * 128;
        const uint32_t w[4] = {c[k].x, c[k].y, c[k].z, c[k].w};
#pragma unroll
        for (int jw = 0; jw < 4; ++jw) *reinterpret_cast<uint4 *>(line + ((((q & 1) * 4 + jw) ^ (row & 7)) * 16)) = values(w[jw], sl[k]);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1) attention_prompt(const prompt_params p)
{
    using L = Smem<D>;
    extern __shared__ __align__(1024) uint8_t raw_smem[];
    const uint32_t smem = smem_u32(raw_smem);
    uint8_t *const gen = raw_smem;
    if (smem & 1023u) {  // (dynamic shared memory begins on such a boundary where there is no other; the swizzle needs it)
        tpq_grid_dep_wait();
        if (threadIdx.x == 0) {
            p.headers[blockIdx.x] = make_int4(0, 0, 0, 0);  // nothing to join
            atomicExch(p.b.status, (int)TPQ_ERR_ALIGN);
        }
        return;
    }
    const uint32_t bars = smem + L::BARS;
    auto bar = [&](int i) { return bars + 8u * i; };
    uint32_t *const there = reinterpret_cast<uint32_t *>(gen + L::BARS + 8 * B_COUNT);  // [RAW]: blocks of a copy stage that were copied
    uint32_t *const tmem_slot = there + RAW;
    const kv_batch &b = p.b;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < 3; ++i) mbar_init(bar(B_T_FULL + i), TILE / KV_BLOCK);
        for (int i = 0; i < RAW; ++i) {
            mbar_init(bar(B_RAW_FULL + i), 1);
            mbar_init(bar(B_RAW_EMPTY + i), HALF / KV_BLOCK);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(B_K_FULL + i), TILE / KV_BLOCK);
            mbar_init(bar(B_V_FULL + i), TILE / KV_BLOCK);
            mbar_init(bar(B_K_EMPTY + i), 1);
            mbar_init(bar(B_V_EMPTY + i), 1);
            mbar_init(bar(B_Q_FULL + i), 4);
            mbar_init(bar(B_S_FULL + i), 1);
            mbar_init(bar(B_P_FULL + i), 4);
            mbar_init(bar(B_P_FULL + 2 + i), 4);
            mbar_init(bar(B_O_FULL + i), 1);
            mbar_init(bar(B_O_EMPTY + i), 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    tpq_grid_dep_wait();
    __syncthreads();
    tpq_grid_dep_launch();
    fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;

    // ---- this block's run
    run r0;
    {
        const plan_head h = *p.head;
        const int share = (int)(((int64_t)h.total + gridDim.x - 1) / gridDim.x);
        r0.unit = (int)min((int64_t)blockIdx.x * share, (int64_t)h.total);
        r0.end = h.total - r0.unit > share ? r0.unit + share : h.total;
        int lo = 0, n = h.items;  // the last item that begins at or before the unit (every warp for itself): as in kv_find_seq
        while (n > 0) {
            const int step = (n + 31) / 32, at = (lane + 1) * step - 1 < n ? (lane + 1) * step - 1 : n - 1;
            const int c = __popc(__ballot_sync(0xffffffffu, p.items[lo + at].before <= r0.unit));
            const int skip = c * step < n ? c * step : n;
            lo += skip;
            n = c == 32 ? 0 : (n - skip < step - 1 ? n - skip : step - 1);
        }
        r0.item = lo > 0 ? lo - 1 : 0;
    }
    run r = r0;

    if (warp == 0) {
        // ---------------- copies
        int stage = 0;  // copy stages so far
        segment g;
        while (ok && next_segment(p, r, g)) {
            const int seq = g.item->seq, len = g.item->len, from = g.item->lo[0] - p.c.window + 1, hi = g.item->rows > 128 ? g.item->hi[1] : g.item->hi[0];
            auto page_of = [&](int h) {  // page of this lane's block (of four) of copy stage h of the segment, -1: not copied
                if (h >= 2 * g.nt || lane >= HALF / KV_BLOCK) return -1;
                const int pos = g.base(h >> 1) + (h & 1) * HALF + lane * KV_BLOCK;
                if (pos >= len || pos > hi) return -1;
                if (p.c.window && pos >= p.c.n_first && pos + KV_BLOCK <= from) return -1;  // no row sees it
                const int page = b.table[seq * b.table_stride + (pos >> b.page_shift)];
                if (page >= 0 && page < b.n_pages) return page;
                kv_report(b);
                return -1;
            };
            int next = -1;
#pragma unroll 1
            for (int h = -1; h < 2 * g.nt; ++h) {
                const int page = next, st = stage % RAW;
                next = page_of(h + 1);  // a step ahead of its use
                if (h < 0) continue;
                if (stage >= RAW) ok = __all_sync(0xffffffffu, wait(bar(B_RAW_EMPTY + st), (stage / RAW - 1) & 1));
                if (!ok) break;
                const uint32_t have = __ballot_sync(0xffffffffu, page >= 0);
                if (lane == 0) {
                    there[st] = have;
                    mbar_expect_tx(bar(B_RAW_FULL + st), __popc(have) * kv_block_bytes(D));
                }
                __syncwarp();
                if (page >= 0) {
                    const int pos = g.base(h >> 1) + (h & 1) * HALF + lane * KV_BLOCK, blocks = b.page_size / KV_BLOCK;
                    const uint8_t *src = b.cache + (((int64_t)page * b.n_kv_heads + g.kh) * blocks + (pos & (b.page_size - 1)) / KV_BLOCK) * kv_block_bytes(D);
                    bulk_g2s(smem + L::RAWS + st * L::RAW_BYTES + lane * kv_block_bytes(D), src, kv_block_bytes(D), bar(B_RAW_FULL + st));
                }
                ++stage;
            }
        }
        if (!ok)  // let the copies in flight land before the shared memory is released
            for (int k = stage > RAW ? stage - RAW : 0; k < stage; ++k) (void)wait(bar(B_RAW_FULL + k % RAW), (k / RAW) & 1);
    } else if (warp == 1) {
        // ---------------- MMA: one thread, known to the compiler as such
        if (elect()) {
            constexpr uint32_t qk_instr = instr(TILE, false), pv_instr = instr(D, true);
            int it = 0;                             // tiles so far: operand buffer it % 2
            // a bit for each row tile: phase of its scores' barrier, of its rows' and sums' barriers, whether it has had sums before
            uint32_t p_phase = 0, q_phase = 0, begun = 0;
            segment g;
            while (ok && next_segment(p, r, g)) {
                const reach re_a = reach_of(g, 0), re_b = reach_of(g, 1);
                int last_a = -1, last_b = -1;
#pragma unroll 1
                for (int j = g.nt - 1; j >= 0 && last_a < 0; --j)
                    if (sees(p, re_a, g.base(j))) last_a = j;
#pragma unroll 1
                for (int j = g.nt - 1; j >= 0 && last_b < 0; --j)
                    if (sees(p, re_b, g.base(j))) last_b = j;
                uint32_t any = 0;  // row tiles with sums of this segment
                // step j: P_t V(j) for both row tiles, each followed by Q_t K(j + 1); step -1 has the first scores only
#pragma unroll 1
                for (int j = -1; j < g.nt && ok; ++j) {
                    const int i = it + j;
                    const bool more = j + 1 < g.nt;
                    if (j >= 0) ok = wait(bar(B_V_FULL + (i & 1)), (i >> 1) & 1);
#pragma unroll 1
                    for (int t = 0; t < 2 && ok; ++t) {
                        if (j >= 0 && sees(p, t ? re_b : re_a, g.base(j))) {
                            if (!(any >> t & 1) && (begun >> t & 1)) ok = wait(bar(B_O_EMPTY + t), (q_phase >> t & 1) ^ 1);
#pragma unroll 1
                            for (int half = 0; half < 2 && ok; ++half) {
                                ok = wait(bar(B_P_FULL + 2 * half + t), p_phase >> t & 1);
                                if (!ok) break;
                                fence_after();
                                const uint32_t v = operand(smem + L::V + (i & 1) * L::TILE_BYTES + half * (HALF * 128), TILE * 128);
#pragma unroll
                                for (int x = 0; x < HALF / 16; ++x)
                                    mma_ts(tmem + 256 + t * 128, tmem + t * TILE + half * (HALF / 2) + 8 * x, v + x * (2048 >> 4), OPERAND_HIGH, pv_instr, (any >> t & 1) | half | (x != 0));
                                if (half == 1 && j == (t ? last_b : last_a)) commit(bar(B_O_FULL + t));
                            }
                            if (!ok) break;
                            any |= 1u << t;
                            p_phase ^= 1u << t;
                        }
                        if (more) {
                            if (j < 0 && (t ? last_b : last_a) >= 0) ok = wait(bar(B_Q_FULL + t), q_phase >> t & 1);
                            if (t == 0 && ok) ok = wait(bar(B_K_FULL + ((i + 1) & 1)), ((i + 1) >> 1) & 1);
                            if (!ok) break;
                            fence_after();
                            if (sees(p, t ? re_b : re_a, g.base(j + 1))) {
                                const uint32_t a = operand(smem + L::Q + t * L::TILE_BYTES, 16), k = operand(smem + L::K + ((i + 1) & 1) * L::TILE_BYTES, 16);
#pragma unroll
                                for (int x = 0; x < D / 16; ++x) {
                                    const uint32_t at = (x / 4) * (128 * 128 >> 4) + 2 * (x % 4);
                                    mma_ss(tmem + t * TILE, a + at, k + at, OPERAND_HIGH, qk_instr, x != 0);
                                }
                                commit(bar(B_S_FULL + t));
                            }
                        }
                    }
                    if (!ok) break;
                    if (j >= 0) commit(bar(B_V_EMPTY + (i & 1)));
                    if (more) commit(bar(B_K_EMPTY + ((i + 1) & 1)));
                }
                it += g.nt;
                begun |= any;
                q_phase ^= any;
            }
        }
        __syncwarp();
    } else if (warp < SOFTMAX) {
        // ---------------- unpack: block warp - UNPACK of every tile
        const int block = warp - UNPACK, at = block & 3, n = lane & 15;
        int it = 0;
        segment g;
        while (ok && next_segment(p, r, g)) {
            const int len = g.item->len;
#pragma unroll 1
            for (int j = 0; j < g.nt; ++j, ++it) {
                const int stage = 2 * it + block / 4, st = stage % RAW;
                ok = __all_sync(0xffffffffu, wait(bar(B_RAW_FULL + st), (stage / RAW) & 1));
                if (!ok) break;
                const uint8_t *const blk = gen + L::RAWS + st * L::RAW_BYTES + at * kv_block_bytes(D);
                const bool have = (there[st] >> at) & 1u, on = have && g.base(j) + block * KV_BLOCK + n < len;
                const uint32_t kw = reinterpret_cast<const uint32_t *>(blk + kv_k_words(D))[n], vw = reinterpret_cast<const uint32_t *>(blk + kv_v_words(D))[n];
                const float ks = __uint_as_float(kw << 16), kl = __uint_as_float(kw & 0xffff0000u);
                const float vs = __uint_as_float(vw << 16), vl = __uint_as_float(vw & 0xffff0000u);
                // (a key or value vector that is no number makes the rows that see it NaN by way of their scores: a weight of
                // 0 times NaN would reach the others)
                const bool bad = !(fabsf(vl) < INFINITY) || !(vs >= 0.0f && vs < INFINITY) || !(fabsf(kl) < INFINITY) || !(fabsf(ks) < INFINITY);
                int ek, ev;
                uint32_t k_scaled = to_scale(ks, kl, on && !bad, ek);
                const uint32_t v_scaled = to_scale(vs, vl, on && !bad, ev);
                if (on && bad) k_scaled = 0x7fff0000u;
                if (it >= 2) ok = __all_sync(0xffffffffu, wait(bar(B_K_EMPTY + (it & 1)), ((it >> 1) - 1) & 1));
                if (!ok) break;
                if (lane == 0)
                    *reinterpret_cast<float4 *>(gen + L::TERM + (it % 3) * TERM_BYTES + block * 16) =
                        have ? make_float4(__uint_as_float((uint32_t)(ek - 14) << 23), (float)(ev - 141), __uint_as_float((uint32_t)(268 - ev) << 23), 0.0f)
                             : make_float4(1.0f, -INFINITY, 0.0f, 0.0f);
                unpack<D>(blk, gen + L::K + (it & 1) * L::TILE_BYTES, block * KV_BLOCK, k_scaled, lane);
                if (lane == 0) {
                    mbar_arrive(bar(B_T_FULL + it % 3));
                    mbar_arrive(bar(B_K_FULL + (it & 1)));
                }
                if (it >= 2) ok = __all_sync(0xffffffffu, wait(bar(B_V_EMPTY + (it & 1)), ((it >> 1) - 1) & 1));
                if (!ok) break;
                unpack<D>(blk + kv_v_codes(D), gen + L::V + (it & 1) * L::TILE_BYTES, block * KV_BLOCK, v_scaled, lane);
                if (lane == 0) {
                    mbar_arrive(bar(B_V_FULL + (it & 1)));
                    mbar_arrive(bar(B_RAW_EMPTY + st));
                }
            }
        }
    } else {
        // ---------------- softmax: thread <-> row `row` of row tile t
        const int t = (warp - SOFTMAX) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem + t * TILE + lanes, o_addr = tmem + 256 + t * 128 + lanes;
        int it = 0, s_count = 0, segs = 0;
        if (tid == SOFTMAX * 32) p.headers[blockIdx.x] = make_int4(0, 0, 0, 0);
        // Of a warp's 32 rows, the 16 bytes that lane l has of step k (D/8 lanes a row).  Rows behind the item's last: that one.
        auto row_chunk = [&](const segment &g, int rows, int k, const uint16_t *x, int64_t stride) {
            const int w_row = t * 128 + (warp & 3) * 32 + k * (256 / D) + lane / (D / 8), in = w_row < rows ? w_row : rows - 1;
            const int local = g.item->head + in, dt = (local * p.group_inv) >> 20;  // local / group: exact below 2^12
            return reinterpret_cast<const uint4 *>(x + (int64_t)(g.item->tok + dt) * stride + (int64_t)(g.kh * p.group + local - dt * p.group) * D) + lane % (D / 8);
        };
        segment g;
        while (ok && next_segment(p, r, g)) {
            const reach re = reach_of(g, t);
            bool works = false;
#pragma unroll 1
            for (int j = 0; j < g.nt && !works; ++j) works = sees(p, re, g.base(j));
            int pos = -1;  // of this thread's row
            float m = -INFINITY, row_scale = 0.0f;
            f2 l2 = 0;
            bool any = false;
            uint8_t *const q_tile = gen + L::Q + t * L::TILE_BYTES;
            if (works) {
                // (position of the first row) + (rows behind it) / group
                if (t * 128 + row < g.item->rows) pos = g.item->lo[0] + (((g.item->head + t * 128 + row) * p.group_inv) >> 20);
                // the warp's 32 rows as they are, D/8 lanes a row, eight loads at a time
                const int rows = g.item->rows;
#pragma unroll 1
                for (int k0 = 0; k0 < D / 8; k0 += 8) {
                    uint4 x[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = *row_chunk(g, rows, k0 + k, p.c.q.p, p.c.q.stride);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int w_row = (warp & 3) * 32 + (k0 + k) * (256 / D) + lane / (D / 8), c = lane % (D / 8);
                        *reinterpret_cast<uint4 *>(q_tile + (c / 8) * (128 * 128) + w_row * 128 + (((c & 7) ^ (w_row & 7)) * 16)) = x[k];
                    }
                }
                __syncwarp();
                // a thread's own row in FP16, scaled so that its largest magnitude is in [2^14, 2^15) (BF16's 8 bits stay exact down to
                // 2^-31 of that), in the codes' order; a negative scale goes into the sign
                auto chunk = [&](int c) { return reinterpret_cast<uint4 *>(q_tile + (c / 8) * (128 * 128) + row * 128 + (((c & 7) ^ (row & 7)) * 16)); };
                uint32_t big = 0;  // magnitudes as integers, in both halves
#pragma unroll 2
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 x = *chunk(c);
                    big = __vmaxu2(__vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)), big);
                }
                big = max(big & 0xffffu, big >> 16);
                int e = (int)(big >> 7);
                const bool bad = e == 255;  // infinite or NaN: so is the row's answer
                if (e < 16 || bad) e = 16;
                const float up = __uint_as_float((uint32_t)(268 - e) << 23);
                row_scale = fabsf(p.scale2) * __uint_as_float((uint32_t)(e - 14) << 23);
                const uint32_t sign = p.scale2 < 0.0f ? 0x80008000u : 0u;
#pragma unroll 2
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 x = *chunk(c);
                    const uint32_t pairs[4] = {__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632)};
                    uint32_t u[4];
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        const __half2 h = __floats2half2_rn(__uint_as_float(pairs[z] << 16) * up, __uint_as_float(pairs[z] & 0xffff0000u) * up);
                        u[z] = (bad ? 0x7fff7fffu : *reinterpret_cast<const uint32_t *>(&h)) ^ sign;
                    }
                    *chunk(c) = make_uint4(u[0], u[1], u[2], u[3]);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B_Q_FULL + t));
            }
            for (int j = 0; j < g.nt; ++j) {
                const int base = g.base(j), i = it + j;
                if (!sees(p, re, base)) continue;
                // (the terms: there ahead of the scores, and not written again before this row tile is done with them)
                ok = __all_sync(0xffffffffu, wait(bar(B_S_FULL + t), s_count & 1)) && __all_sync(0xffffffffu, wait(bar(B_T_FULL + i % 3), (i / 3) & 1));
                if (!ok) break;
                ++s_count;
                fence_after();
                const uint32_t term = smem + L::TERM + (i % 3) * TERM_BYTES;
                if (!sees_all(p, re, base)) {  // scores of positions that this row does not see
#pragma unroll 1
                    for (int c = 0; c < TILE; c += 32) {
                        uint32_t x[32];
                        ld32(s_addr + c, x);
                        ld_wait(x);
                        const int at = base + c;
                        const uint32_t see = low_bits(pos - at + 1) & (p.c.window ? ~low_bits(pos - p.c.window + 1 - at) | low_bits(p.c.n_first - at) : 0xffffffffu);
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] = see >> k & 1u ? x[k] : 0xff800000u;
                        st32(s_addr + c, x);
                    }
                    st_wait();
                }
                // Twice over the scores, 64 and 32 columns at a time (they stay in tensor memory, and the code in the instruction cache: with all
                // 128 in registers and no loop, half of the warps' time went into fetching instructions)
                float top[2] = {-INFINITY, -INFINITY};
#pragma unroll 1
                for (int c = 0; c < TILE; c += 64) {
                    uint32_t x[64];
                    ld32(s_addr + c, x);
                    ld32(s_addr + c + 32, x + 32);
                    ld_wait(x);
                    loaded(x + 32);
#pragma unroll
                    for (int k = 0; k < 64; k += KV_BLOCK) {
                        const float4 tm = lds4(term + (c + k) / KV_BLOCK * 16);
                        float y[4];
#pragma unroll
                        for (int z = 0; z < 4; ++z)
                            y[z] = fmaxf(fmaxf(__uint_as_float(x[k + z]), __uint_as_float(x[k + 4 + z])), fmaxf(__uint_as_float(x[k + 8 + z]), __uint_as_float(x[k + 12 + z])));
                        top[k / KV_BLOCK & 1] = fmaxf(top[k / KV_BLOCK & 1], fmaf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(tm.x * row_scale, 0x1p-120f), tm.y));
                    }
                }
                const float tile_top = fmaxf(top[0], top[1]);
                if (!any) {
                    m = tile_top;
                } else if (__any_sync(0xffffffffu, tile_top > m + 8.0f)) {
                    const float m2 = fmaxf(m, tile_top), a = ex2(m - (m2 == -INFINITY ? 0.0f : m2));
                    m = m2;
                    const f2 a2 = pack2(a, a);
                    l2 = fma2(l2, a2, 0);
                    // (the scores of this tile were computed behind the products that O holds)
#pragma unroll 1
                    for (int k = 0; k < D; k += 32) {
                        uint32_t o[32];
                        ld32(o_addr + k, o);
                        ld_wait(o);
#pragma unroll
                        for (int z = 0; z < 32; ++z) o[z] = __float_as_uint(__uint_as_float(o[z]) * a);
                        st32(o_addr + k, o);
                    }
                    st_wait();
                }
                any = true;
                const float from = (m == -INFINITY ? 0.0f : m) - 7.0f;
#pragma unroll 1
                for (int c = 0; c < TILE; c += 32) {
                    uint32_t x[32], h[16];
                    ld32(s_addr + c, x);
                    ld_wait(x);
#pragma unroll
                    for (int b0 = 0; b0 < 32; b0 += KV_BLOCK) {
                        const float4 tm = lds4(term + (c + b0) / KV_BLOCK * 16);
                        const float sc = fmaxf(tm.x * row_scale, 0x1p-120f), of = tm.y - from;  // (not 0: -inf * 0)
                        const f2 sc2 = pack2(sc, sc), of2 = pack2(of, of);
                        f2 sum[2] = {0, 0};
#pragma unroll
                        for (int k = b0; k < b0 + KV_BLOCK; k += 4) {
                            float y[4];
                            unpack2(fma2(pack2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), sc2, of2), y[0], y[1]);
                            unpack2(fma2(pack2(__uint_as_float(x[k + 2]), __uint_as_float(x[k + 3])), sc2, of2), y[2], y[3]);
#pragma unroll
                            for (int z = 0; z < 4; ++z) y[z] = ex2(y[z]);
                            sum[0] = add2(sum[0], pack2(y[0], y[1]));
                            sum[1] = add2(sum[1], pack2(y[2], y[3]));
                            const __half2 h0 = __floats2half2_rn(y[0], y[1]), h1 = __floats2half2_rn(y[2], y[3]);
                            h[k / 2] = *reinterpret_cast<const uint32_t *>(&h0);
                            h[k / 2 + 1] = *reinterpret_cast<const uint32_t *>(&h1);
                        }
                        l2 = fma2(add2(sum[0], sum[1]), pack2(tm.z, tm.z), l2);
                    }
                    st16(s_addr + c / 2, h);  // (columns c/2 .. c/2 + 15: scores that have been read)
                    if (c & 32) {  // half of the weights: their products may begin
                        st_wait();
                        fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(B_P_FULL + 2 * (c >> 6) + t));
                    }
                }
            }
            it += g.nt;
            if (!ok) break;
            float l_a, l_b;
            unpack2(l2, l_a, l_b);
            const float l = l_a + l_b;
            if (works) {
                ok = __all_sync(0xffffffffu, wait(bar(B_O_FULL + t), segs & 1));
                if (!ok) break;
                ++segs;
                fence_after();
            }
            const int rows = g.item->rows;
            const bool mine = t * 128 + row < rows, whole = g.t0 == 0 && g.nt == g.item->tiles;
            float *part = p.parts + (((int64_t)blockIdx.x * 2 + (g.t0 == 0 ? 1 : 0)) * BM + t * 128 + row) * (D + 4);
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll 1
            for (int k = 0; k < D; k += 32) {
                uint32_t o[32];
                if (works) {
                    ld32(o_addr + k, o);
                    ld_wait(o);
                } else {
#pragma unroll
                    for (int z = 0; z < 32; ++z) o[z] = 0;
                }
#pragma unroll
                for (int c = 0; c < 32; c += 8) {
                    const int from[8] = {0, 2, 4, 6, 1, 3, 5, 7};  // value d of a chunk is column from[d]
                    float y[8];
#pragma unroll
                    for (int z = 0; z < 8; ++z) y[z] = __uint_as_float(o[c + from[z]]);
                    if (whole) {  // through shared memory (the rows' own place), so that a warp's stores are of whole rows
                        uint32_t u[4];
#pragma unroll
                        for (int z = 0; z < 4; ++z) {
                            const __nv_bfloat162 v = __floats2bfloat162_rn(y[2 * z] * inv, y[2 * z + 1] * inv);
                            u[z] = *reinterpret_cast<const uint32_t *>(&v);
                        }
                        const int ch = (k + c) / 8;
                        *reinterpret_cast<uint4 *>(q_tile + (ch / 8) * (128 * 128) + row * 128 + (((ch & 7) ^ (row & 7)) * 16)) = make_uint4(u[0], u[1], u[2], u[3]);
                    } else if (mine) {
                        reinterpret_cast<float4 *>(part + k + c)[0] = make_float4(y[0], y[1], y[2], y[3]);
                        reinterpret_cast<float4 *>(part + k + c)[1] = make_float4(y[4], y[5], y[6], y[7]);
                    }
                }
                __syncwarp();
            }
            if (whole) {
#pragma unroll 2
                for (int k = 0; k < D / 8; ++k) {
                    const int w_row = (warp & 3) * 32 + k * (256 / D) + lane / (D / 8), c = lane % (D / 8);
                    const uint4 x = *reinterpret_cast<const uint4 *>(q_tile + (c / 8) * (128 * 128) + w_row * 128 + (((c & 7) ^ (w_row & 7)) * 16));
                    if (t * 128 + w_row < rows) *const_cast<uint4 *>(row_chunk(g, rows, k, p.c.out, p.c.out_stride)) = x;
                }
                __syncwarp();
            }
            if (mine && !whole) *reinterpret_cast<float2 *>(part + D) = make_float2(m, l);
            if (works) {
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B_O_EMPTY + t));
            }
            if (tid == SOFTMAX * 32 && g.t0 == 0 && !whole) {  // the runs behind this one have `share` units each of what is left
                const int share = (int)(((int64_t)p.head->total + gridDim.x - 1) / gridDim.x);
                p.headers[blockIdx.x] = make_int4(1 + (g.item->tiles - g.nt + share - 1) / share, (int)(g.item - p.items), g.kh, 0);
            }
        }
    }
    if (!ok) atomicExch(b.status, (int)TPQ_ERR_TIMEOUT);
    fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// Puts the partial results together that run blockIdx.x ends with the first part of: a warp per row, JOIN_BLOCKS blocks.
constexpr int JOIN_BLOCKS = 8;
template <int D>
__global__ void __launch_bounds__(256) attention_prompt_join(const prompt_params p)
{
    constexpr int V = D / 32;  // values of a lane
    tpq_grid_dep_wait();
    const int4 head = p.headers[blockIdx.x];  // parts, item, key head
    const int lane = threadIdx.x & 31;
    if (head.x == 0) return;
    const plan_item &it = p.items[head.y];
    const int rows = it.rows;
#pragma unroll 1
    for (int r = blockIdx.y * (BM / JOIN_BLOCKS) + (threadIdx.x >> 5); r < min(rows, (int)(blockIdx.y + 1) * (BM / JOIN_BLOCKS)); r += 8) {
        float m = -INFINITY, l = 0.0f, o[V] = {};
        for (int i = 0; i < head.x; ++i) {
            const float *part = p.parts + ((((int64_t)blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * BM + r) * (D + 4);
            const float2 v = __ldcg(reinterpret_cast<const float2 *>(part + D));
            float z[V];
            if (V == 4) {
                const float4 q = __ldcg(reinterpret_cast<const float4 *>(part) + lane);
                z[0] = q.x, z[1] = q.y, z[V - 2] = q.z, z[V - 1] = q.w;
            } else {
                const float2 q = __ldcg(reinterpret_cast<const float2 *>(part) + lane);
                z[0] = q.x, z[1] = q.y;
            }
            const float top = fmaxf(m, v.x), from = top == -INFINITY ? 0.0f : top, a = ex2(m - from), f = ex2(v.x - from);
            m = top;
            l = fmaf(v.y, f, l * a);
#pragma unroll
            for (int k = 0; k < V; ++k) o[k] = fmaf(z[k], f, o[k] * a);
        }
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const int local = it.head + r, dt = local / p.group, h = head.z * p.group + (local - dt * p.group);
        uint32_t *dst = reinterpret_cast<uint32_t *>(p.c.out + (int64_t)(it.tok + dt) * p.c.out_stride + (int64_t)h * D + V * lane);
#pragma unroll
        for (int k = 0; k < V / 2; ++k) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(o[2 * k] * inv, o[2 * k + 1] * inv);
            dst[k] = *reinterpret_cast<const uint32_t *>(&v);
        }
    }
}

int64_t most_items(int64_t n_seqs, int64_t n_tokens, int64_t group)  // full items and one more of every sequence with rows
{
    const int64_t rows = n_tokens * group;
    return rows / BM + (rows < n_seqs ? rows : n_seqs) + 1;
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

}  // namespace

size_t kv_prompt_workspace(int D, int group, int sm_count, int64_t n_seqs, int64_t n_tokens)
{
    return up16(sizeof(plan_head)) + up16(sizeof(plan_item) * most_items(n_seqs, n_tokens, group)) + up16(4 * (size_t)n_seqs) + 16 * (size_t)sm_count +
           (size_t)sm_count * 2 * BM * (D + 4) * 4;
}

cudaError_t kv_launch_prompt(const kv_batch &b, int D, const kv_attention_call &c, int few, void *workspace, int sm_count, cudaStream_t st, int64_t *launches)
{
    const int group = b.n_heads / b.n_kv_heads;
    const int64_t items = most_items(b.n_seqs, b.n_tokens, group);
    uint8_t *w = static_cast<uint8_t *>(workspace);
    prompt_params p{b, c};
    p.head = reinterpret_cast<plan_head *>(w);
    w += up16(sizeof(plan_head));
    p.items = reinterpret_cast<plan_item *>(w);
    w += up16(sizeof(plan_item) * items);
    p.seq_items = reinterpret_cast<int *>(w);
    w += up16(4 * (size_t)b.n_seqs);
    p.headers = reinterpret_cast<int4 *>(w);
    w += 16 * (size_t)sm_count;
    p.parts = reinterpret_cast<float *>(w);
    p.most_items = (int)items;
    p.scale2 = c.scale * 1.4426950408889634f;
    p.group = group;
    p.group_inv = (1 << 20) / group + 1;
    p.few = few;
    cudaError_t e = tpq_launch_pdl(attention_plan, dim3(1), dim3(PLAN_THREADS), 0, st, p);
    if (e != cudaSuccess) return e;
    ++*launches;
    auto main = [&](auto kern, size_t smem) {
        cudaError_t f = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        return f != cudaSuccess ? f : tpq_launch_pdl(kern, dim3(sm_count), dim3(THREADS), smem, st, p);
    };
    e = D == 128 ? main(attention_prompt<128>, Smem<128>::BYTES) : main(attention_prompt<64>, Smem<64>::BYTES);
    if (e != cudaSuccess) return e;
    ++*launches;
    e = D == 128 ? tpq_launch_pdl(attention_prompt_join<128>, dim3(sm_count, JOIN_BLOCKS), dim3(256), 0, st, p)
                 : tpq_launch_pdl(attention_prompt_join<64>, dim3(sm_count, JOIN_BLOCKS), dim3(256), 0, st, p);
    if (e == cudaSuccess) ++*launches;
    return e;
}
