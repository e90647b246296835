// Attention over the 4-bit cache (tpq_kv_attention) for sequences that bring few rows: decoding, drafts to verify.
//
// Mathematics.  With keys k_t = a_t + s_t c_t (a: low, s: step, c: codes) and values v_t = b_t + r_t e_t,
//   x_t = scale log2(e) (s_t q.c_t + a_t sum(q)),  out = sum_t 2^x_t (b_t + r_t e_t) / sum_t 2^x_t.
// The products with codes run on the tensor cores with the codes themselves as operands: no key or value is ever formed.
// The values' steps go into the exponent, P_t = 2^(x_t + log2 r_t - m), so that a product P_t e_t needs no scale of its own
// and P_t is at most 2^15 whatever the steps are; then
//   out = sum_t P_t (e_t - 8) + sum_t P_t (b_t / r_t + 8)   over   sum_t P_t / r_t,
// m 7 below the maximum of x_t + log2 r_t when it last moved, which it does where that has grown by more than 8: P_t of the largest is
// 2^7 .. 2^15, within FP16.
//
// Codes become operands with little more than one logic instruction for two: a code in the low mantissa bits of FP16 1024
// (0x6400 | c) is 1024 + c, in bits 4 .. 7 (0x6400 | 16 c) it is 16 (64 + c), both exact; the sums of offsets are what the
// accumulators start from.  The keys use both forms, with a 16th of the row's value for the second one (a row has a power of two
// of its own that makes its BF16 values FP16 ones).  The values use the second form alone, whose offset is small beside the
// codes: their 72 x 16 = 1152 is taken off by one more product, of P with a constant, from which the sums of a chunk start:
// they are sums of P (e - 8), and what is added up in binary32 over a whole sequence has no common offset to lose digits to.  P is
// rounded to FP16 (11 bits; below 2^-21 of the largest one, with fewer), Q and the codes are exact.
//
// Operands.  Rows (query heads of one key head x new positions) are the 8 columns of an m16n8k16 product, positions (for the
// values: a head's values) its 16 rows, so that 8 query heads per key head leave nothing of the instruction unused.  The scores come
// out with positions along the lanes' groups; movmatrix turns them into the second product's operand.  Which code is which row
// or column of a fragment is free as long as both sides agree: lanes read 16 (keys) and 8 (values) contiguous bytes of a
// position, conflict-free and two-way.  mma.sync and not tcgen05: 16 positions x 8 rows are an eighth of the smallest
// tcgen05 tile, and what bounds this kernel is the memory that the codes come from and the instructions that unpack them
// (282 per warp and 16 positions of 2176 bytes).
//
// Work.  The positions of all sequences and key heads are cut into tiles of 256 (128 for more than 8 rows) and dealt out evenly, in order, to as many
// blocks as the GPU holds at a time, whatever the lengths are (a graph with this call replays for others).  A block whose
// run begins or ends inside a (sequence, key head) leaves a partial result, at most two in all; attention_join puts them
// together.  A warp takes a quarter of a tile, by itself: its copies (16 positions = one
// contiguous block of the cache), its barriers, its running maximum; the warps meet at the end of a (sequence, key head).
//
// What bounds it: instructions, 53 % of the issue slots (three warps a scheduler, whose 168 registers a thread fill the register file; the rest
// is their latency).  32 sequences of 16 to 32 thousand positions, 64 heads of 128 on 8: 210 to 222 us, 4.0 to 4.2 TB/s (two blocks of positions at a
// time 245 us against 205 then: copies' bookkeeping and maxima cost as much again); 64 of up to 8000, 4 heads on 2: 35 us, half of it beginnings
// and ends of runs; one sequence of 777: 11 us, the host's two launches.  Of the four kernels one spills: heads of 128, 16 rows at a time, 22 words.
#include "kv_internal.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace {

constexpr int WARPS = 4;
// Rows (new positions x query heads of a key head) of a sequence here: in groups of 8 NT, one after the other.  A sequence of more goes to the
// kernels of kv_prompt.cu, whose 256 rows take about as long for 40 as for 128.  Both, us (theirs with these launched for nothing, as in a
// batch of several), for rows of                          32   40   48   64   96  128  256
//   24 sequences of 2000 to 4000, 4 key heads of 128      51   67   68   82  116  145  271   here, whatever the rows
//                                                               69   69   69   69   70   84   there
//   the same with heads of 64                             40   52   53   63   88  109  203   here
//                                                               60   61   61   61   61   72   there
//   8 of 10 000 to 20 000, 8 key heads of 128            117  166  168  215  309  407  790   here
//                                                              155  155  156  157  158  180   there
//   2 of 1000 to 2000, 10 key heads of 128                19   20   20   23   27   33   49   here
//                                                               32   32   33   34   35   39   there
constexpr int MAX_ROWS = 32;

// Runs are dealt out in units: a (sequence, key head, group of rows) is its tiles and EXTRA more, which stand for its beginning and end
// (24 sequences of 16 to 32 rows, ragged: 54.8 us with none, 50.2 with one, 44.4 with two or three; 64 of one row: 33.5, 32.7, 32.5, 32.3).
constexpr int EXTRA = 2;

// NT: groups of 8 rows.  Blocks of 16 positions that a warp takes at a time: what is done once for them (the copies' bookkeeping, the
// maxima, adding the sums up) costs less the more they are; four where registers allow.  Stages of a warp's ring and blocks of an SM: what
// shared memory and registers (32 NT sums and as much besides) allow.
__host__ __device__ constexpr int chunk_blocks(int NT) { return NT == 1 ? 4 : 2; }
__host__ __device__ constexpr int chunk(int NT) { return KV_BLOCK * chunk_blocks(NT); }
__host__ __device__ constexpr int tile(int NT) { return WARPS * chunk(NT); }  // positions of a tile: a chunk of each warp
__host__ __device__ constexpr int stages(int D, int NT) { return NT == 1 ? (D == 64 ? 3 : 2) : D == 64 ? 4 : 3; }
constexpr int BLOCKS_PER_SM = 3;
__host__ __device__ constexpr int chunk_bytes(int D, int NT) { return chunk_blocks(NT) * kv_block_bytes(D); }
// floats of a partial result's row: sums of D values, maximum, normaliser, padded to 16 bytes
__host__ __device__ constexpr int part_row(int D) { return D + 4; }

template <int D, int NT>
struct Shared {
    uint8_t ring[WARPS][stages(D, NT)][chunk_bytes(D, NT)];  // (at a segment's end, a warp's sums: [8 NT][D + 4] floats)
    float4 words[WARPS][chunk(NT)];                          // per position: key step and low, log2 of the value step, its reciprocal
    float lows[WARPS][chunk(NT)];                            // (value low) / (value step) + 8
    uint2 q[NT == 1 ? 1 : NT * (D / 16) * 32];               // (NT > 1) the rows as operands
    float m[WARPS][8 * NT], l[WARPS][8 * NT];
    uint64_t full[WARPS][stages(D, NT)];
    uint32_t there[WARPS][stages(D, NT)];                    // bit b: block b of the chunk was copied
    int64_t scan[WARPS];
    int begin[2];                                            // where the block's run begins: sequence, tile of that sequence
};

struct split_params {
    kv_batch b;
    kv_attention_call c;
    float *parts;   // [blocks][2][8 NT][part_row]
    int4 *headers;  // [blocks]: of the part that the block's run ends with: parts in all, the sequence's first row, first row and rows, key head
    float scale2;   // scale * log2(e)
    int group;      // query heads of a key head
};

constexpr float NONE = -1e30f;  // m of rows that have seen nothing: below every score, and finite, so that differences are numbers

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float lg2(float x)
{
    float r;
    asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t bits)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(a), "r"(mask), "r"(bits));
    return r;
}
// d = a b + c, FP16 products, FP32 sums
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float c0, float c1, float c2, float c3)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// Tiles of a sequence that any of its rows sees: [0, first) and [from, end); its groups of rows.
struct tiles_of {
    int first, from, count, groups;
    __device__ int units() const { return count ? count + EXTRA : 0; }  // of a (sequence, key head, group of rows)
};
__device__ __forceinline__ tiles_of visible_tiles(const kv_seq &s, const kv_attention_call &c, int group, int tile, int rows)
{
    tiles_of t{0, 0, 0, 0};
    if (s.n <= 0 || s.n * group > MAX_ROWS) return t;
    if (c.window) {
        const int from = s.len - s.n - c.window + 1;  // of the first row
        if (from > 0) {
            t.from = from / tile;
            const int first = ((c.n_first < from ? c.n_first : from) + tile - 1) / tile;
            t.first = first < t.from ? first : t.from;
        }
    }
    t.count = t.first + (s.len + tile - 1) / tile - t.from;
    t.groups = rows == 8 ? 1 : (s.n * group + rows - 1) / rows;  // (groups of 8 are for sequences that have no more)
    return t;
}

template <int D, int NT>
__global__ void __launch_bounds__(WARPS * 32, BLOCKS_PER_SM)
attention_split(const split_params p)
{
    constexpr int NS = stages(D, NT), R = 8 * NT, C = chunk_blocks(NT), CHUNK = chunk(NT), TILE = tile(NT);
    constexpr int KW = D / 32;  // words of a key row that a lane reads
    extern __shared__ __align__(16) uint8_t raw[];
    Shared<D, NT> &sh = *reinterpret_cast<Shared<D, NT> *>(raw);
    const kv_batch &b = p.b;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, i4 = lane & 3;
    if (lane == 0)
        for (int s = 0; s < NS; ++s) mbar_init(smem_u32(&sh.full[warp][s]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tpq_grid_dep_wait();
    tpq_grid_dep_launch();

    // ---- where this block's run begins
    const int per = (b.n_seqs + WARPS * 32 - 1) / (WARPS * 32);
    const int s0 = tid * per, s1 = s0 + per < b.n_seqs ? s0 + per : b.n_seqs;
    int64_t want = 0;
    for (int s = s0; s < s1; ++s) {
        const tiles_of t = visible_tiles(kv_load_seq(b, s), p.c, p.group, tile(NT), 8 * NT);
        want += (int64_t)t.units() * t.groups * b.n_kv_heads;
    }
    int64_t sum = want;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, sum, m);
        if (lane >= m) sum += o;
    }
    if (lane == 31) sh.scan[warp] = sum;
    __syncthreads();
    int64_t all = 0, ahead = sum - want;
    for (int w = 0; w < WARPS; ++w) {
        if (w < warp) ahead += sh.scan[w];
        all += sh.scan[w];
    }
    if (all > KV_MOST_UNITS) {  // the same in every block: nothing is done, and nothing joined
        if (tid == 0) kv_report(b);
        all = 0;
    }
    const int total = (int)all, mine = (int)want, before = (int)ahead;  // (numbers of units from here on: none is larger than the total)
    const int share = (total + (int)gridDim.x - 1) / (int)gridDim.x;
    int unit = (int)blockIdx.x * share;
    const int unit_end = total - unit > share ? unit + share : total;
    if (unit >= unit_end) {
        if (tid == 0) p.headers[blockIdx.x] = make_int4(0, 0, 0, 0);
        return;
    }
    if (unit >= before && unit < before + mine) {
        int off = unit - before, s = s0;
        for (;; ++s) {
            const tiles_of t = visible_tiles(kv_load_seq(b, s), p.c, p.group, tile(NT), 8 * NT);
            const int n = t.units() * t.groups * b.n_kv_heads;
            if (off < n) break;
            off -= n;
        }
        sh.begin[0] = s;
        sh.begin[1] = off;
    }
    __syncthreads();
    int s = sh.begin[0], off = sh.begin[1];
    int phase = 0;  // chunks of the segments before (a warp's own): chunk j is in stage (phase + j) % NS
    int issued = 0;
    bool ok = true;
    int4 header = make_int4(0, 0, 0, 0);

    while (unit < unit_end) {
        const kv_seq seq = kv_load_seq(b, s);
        const tiles_of tl = visible_tiles(seq, p.c, p.group, tile(NT), 8 * NT);
        const int units = tl.units(), all_units = units * tl.groups * b.n_kv_heads;
        if (off >= all_units) {
            off -= all_units;
            ++s;
            continue;
        }
        const int pair = off / units, kh = NT == 1 ? pair : pair / tl.groups, row0 = NT == 1 ? 0 : (pair - kh * tl.groups) * R, u0 = off - pair * units;
        const int nu = units - u0 < unit_end - unit ? units - u0 : unit_end - unit;
        const int t0 = u0 > EXTRA ? u0 - EXTRA : 0, nt = u0 + nu - EXTRA - t0;
        unit += nu;
        off += nu;
        if (nt <= 0) continue;  // (the run begins or ends inside the extra units)
        const int rows = seq.n * p.group - row0 < R ? seq.n * p.group - row0 : R, p0 = seq.len - seq.n;

        // ---- copies: chunk j of the segment, block `lane` (below C) of it; the first ones are under way while the rows are fetched
        auto base_of = [&](int j) {
            const int t = t0 + j;
            return (t < tl.first ? t : tl.from + t - tl.first) * TILE + warp * CHUNK;
        };
        auto page_of = [&](int j) {  // page of this lane's block of chunk j, -1: none to copy
            if (j >= nt || lane >= C) return -1;
            const int pos = base_of(j) + lane * KV_BLOCK;
            if (pos >= seq.len) return -1;
            if (p.c.window && pos >= p.c.n_first && pos + KV_BLOCK <= p0 - p.c.window + 1) return -1;  // no row sees it
            const int page = b.table[s * b.table_stride + (pos >> b.page_shift)];
            if (page >= 0 && page < b.n_pages) return page;
            kv_report(b);
            return -1;
        };
        auto issue = [&](int j, int page) {
            const int st = (phase + j) % NS;
            const uint32_t bar = smem_u32(&sh.full[warp][st]);
            const uint32_t there = __ballot_sync(0xffffffffu, page >= 0);
            issued = phase + j + 1;
            if (lane == 0) {
                sh.there[warp][st] = there;
                mbar_expect_tx(bar, __popc(there) * kv_block_bytes(D));
            }
            __syncwarp();
            if (page >= 0) {
                const int pos = base_of(j) + lane * KV_BLOCK, blocks = b.page_size / KV_BLOCK;
                const uint8_t *src = b.cache + (((int64_t)page * b.n_kv_heads + kh) * blocks + (pos & (b.page_size - 1)) / KV_BLOCK) * kv_block_bytes(D);
                bulk_g2s(smem_u32(&sh.ring[warp][st][lane * kv_block_bytes(D)]), src, kv_block_bytes(D), bar);
            }
        };
#pragma unroll
        for (int j = 0; j < NS - 1; ++j)
            if (j < nt) issue(j, page_of(j));
        int next_page = page_of(NS - 1);


        // ---- the rows as operands: column n = lane / 4 of a group of 8, values 8 KW i4 .. of the head in the order (0 4)(1 5)(2 6)(3 7),
        // in FP16, scaled so that the row's largest magnitude is in [2^14, 2^15) (BF16's 8 bits stay exact down to 2^-27 of that),
        // a 16th of it where the codes come 16-fold
        uint2 qf[NT == 1 ? D / 16 : 1];
        float qsum[NT][2], qoff[NT][2], qscale[NT][2];  // of columns 2 i4 and 2 i4 + 1: sum of the row; what the codes' offsets add; its scale
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = 8 * n + g, tok = (row0 + r) / p.group, h = kh * p.group + (row0 + r - tok * p.group);
            const uint4 *src = reinterpret_cast<const uint4 *>(p.c.q.p + (int64_t)(seq.start + tok) * p.c.q.stride + (int64_t)h * D + 8 * KW * i4);
            uint4 x[KW];
            uint32_t big = 0;
#pragma unroll
            for (int j = 0; j < KW; ++j) {
                x[j] = r < rows ? src[j] : make_uint4(0, 0, 0, 0);
                big = __vmaxu2(__vmaxu2(__vmaxu2(x[j].x & 0x7fff7fffu, x[j].y & 0x7fff7fffu), __vmaxu2(x[j].z & 0x7fff7fffu, x[j].w & 0x7fff7fffu)), big);
            }
            big = max(big & 0xffffu, big >> 16);
            big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
            big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
            int e = (int)(big >> 7);
            const bool bad = e == 255;  // infinite or NaN: so is the row's answer
            if (e < 16 || bad) e = 16;
            const float up = __uint_as_float((uint32_t)(268 - e) << 23);
            float sum_q = 0.0f, off_q = 0.0f;
#pragma unroll
            for (int j = 0; j < KW; ++j) {
                const uint32_t pair[4] = {__byte_perm(x[j].x, x[j].z, 0x5410), __byte_perm(x[j].x, x[j].z, 0x7632), __byte_perm(x[j].y, x[j].w, 0x5410), __byte_perm(x[j].y, x[j].w, 0x7632)};
                uint32_t u[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float f0 = __uint_as_float(pair[k] << 16) * up, f1 = __uint_as_float(pair[k] & 0xffff0000u) * up;
                    const __half2 h2 = __floats2half2_rn(k & 1 ? f0 * 0.0625f : f0, k & 1 ? f1 * 0.0625f : f1);
                    u[k] = *reinterpret_cast<const uint32_t *>(&h2);
                    sum_q += f0 + f1;
                    off_q += (__low2float(h2) + __high2float(h2)) * -1024.0f;
                }
                const uint2 f0 = make_uint2(u[0], u[1]), f1 = make_uint2(u[2], u[3]);
                if (NT == 1) {
                    qf[2 * j] = f0;
                    qf[2 * j + 1] = f1;
                } else if (n == warp) {  // (every warp has them all; one stores)
                    sh.q[(n * (D / 16) + 2 * j) * 32 + lane] = f0;
                    sh.q[(n * (D / 16) + 2 * j + 1) * 32 + lane] = f1;
                }
            }
            float sc = p.scale2 * __uint_as_float((uint32_t)(e - 14) << 23);
            if (bad) sc = NAN;
            sum_q += __shfl_xor_sync(0xffffffffu, sum_q, 1);
            sum_q += __shfl_xor_sync(0xffffffffu, sum_q, 2);
            off_q += __shfl_xor_sync(0xffffffffu, off_q, 1);
            off_q += __shfl_xor_sync(0xffffffffu, off_q, 2);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                qsum[n][c] = __shfl_sync(0xffffffffu, sum_q, 8 * i4 + 4 * c) * __shfl_sync(0xffffffffu, sc, 8 * i4 + 4 * c);
                qoff[n][c] = __shfl_sync(0xffffffffu, off_q, 8 * i4 + 4 * c);
                qscale[n][c] = __shfl_sync(0xffffffffu, sc, 8 * i4 + 4 * c);
            }
        }
        if (NT > 1) __syncthreads();
        // m: 2^-7 of the running maximum's power, as an exponent (P = 2^(y - m) <= 2^15: below)
        float m[NT][2], l[NT][2], w[NT][2], o[NT][D / 16][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int k = 0; k < 2; ++k) m[n][k] = NONE, l[n][k] = 0.0f, w[n][k] = 0.0f;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) o[n][k][0] = o[n][k][1] = o[n][k][2] = o[n][k][3] = 0.0f;
        }

        for (int j = 0; j < nt && ok; ++j) {
            __syncwarp();  // every lane has read the stage that the next copy overwrites
            if (j + NS - 1 < nt) issue(j + NS - 1, next_page);
            next_page = page_of(j + NS);
            const int st = (phase + j) % NS;
            ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.full[warp][st]), ((phase + j) / NS) & 1));
            if (!ok) break;
            const uint8_t *chunk = sh.ring[warp][st];
            const int base = base_of(j);
            const uint32_t there = sh.there[warp][st];
            if (there == 0) continue;
#pragma unroll
            for (int at = lane; at < CHUNK; at += 32) {  // a position: what its words say
                const int pos = base + at;
                const uint32_t *ws = reinterpret_cast<const uint32_t *>(chunk + (at / KV_BLOCK) * kv_block_bytes(D)) + at % KV_BLOCK;
                const uint32_t kw = ws[kv_k_words(D) / 4], vw = ws[kv_v_words(D) / 4];
                const float ks = __uint_as_float(kw << 16), kl = __uint_as_float(kw & 0xffff0000u);
                const float vs = __uint_as_float(vw << 16), vl = __uint_as_float(vw & 0xffff0000u);
                const bool on = pos < seq.len && ((there >> (at / KV_BLOCK)) & 1u);
                // (the terms divide by the step.  Append writes none below 2^-60 or 2^-16 of `low`; in others' words a step below 2^-60 or
                // 2^-24 of `low` counts as that, which is 15 codes of 2^-24, or of next to nothing, off: 1/0 would make a weight of 0 NaN)
                const float r = fmaxf(vs, fmaxf(0x1p-60f, fabsf(vl) * 0x1p-24f));
                float inv;
                asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(r));
                // (positions of nobody: whatever their bytes are, NaN among them, weight 0 and finite terms.  A key or value vector that
                // is no number makes the rows that see it NaN by way of their scores: a weight of 0 times NaN would reach the others)
                const bool bad = !(fabsf(vl) < INFINITY) || !(vs >= 0.0f && vs < INFINITY) || !(fabsf(kl) < INFINITY) || !(fabsf(ks) < INFINITY);
                sh.words[warp][at] = on ? make_float4(ks, bad ? NAN : kl, lg2(r), inv) : make_float4(0.0f, 0.0f, -INFINITY, 0.0f);
                sh.lows[warp][at] = on && !bad ? fmaf(vl, inv, 8.0f) : 0.0f;
            }
            __syncwarp();

            // ---- scores: x[n][block][2 x position half + column]
            float x[NT][C][4];
#pragma unroll
            for (int k = 0; k < C; ++k) {
                // position of row r of the product: (r >> 1) + 4 (r & 1), and 8 more for rows 8 .. 15 (the values' reads below
                // then hit few banks twice)
                const uint8_t *rows_k = chunk + k * kv_block_bytes(D) + ((g >> 1) + 4 * (g & 1)) * (D / 2) + 4 * KW * i4;
                uint32_t ca[KW], cb[KW];
                if (KW == 4) {
                    *reinterpret_cast<uint4 *>(ca) = *reinterpret_cast<const uint4 *>(rows_k);
                    *reinterpret_cast<uint4 *>(cb) = *reinterpret_cast<const uint4 *>(rows_k + 8 * (D / 2));
                } else {
                    *reinterpret_cast<uint2 *>(ca) = *reinterpret_cast<const uint2 *>(rows_k);
                    *reinterpret_cast<uint2 *>(cb) = *reinterpret_cast<const uint2 *>(rows_k + 8 * (D / 2));
                }
#pragma unroll
                for (int jw = 0; jw < KW; ++jw) {
                    const uint32_t ha = ca[jw] >> 8, hb = cb[jw] >> 8;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t za = half ? ha : ca[jw], zb = half ? hb : cb[jw];
                        const uint32_t a0 = and_or(za, 0x000f000fu, 0x64006400u), a2 = and_or(za, 0x00f000f0u, 0x64006400u);
                        const uint32_t a1 = and_or(zb, 0x000f000fu, 0x64006400u), a3 = and_or(zb, 0x00f000f0u, 0x64006400u);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint2 f = NT == 1 ? qf[2 * jw + half] : sh.q[(n * (D / 16) + 2 * jw + half) * 32 + lane];
                            if (jw == 0 && half == 0) mma(x[n][k], a0, a1, a2, a3, f.x, f.y, qoff[n][0], qoff[n][1], qoff[n][0], qoff[n][1]);
                            else mma(x[n][k], a0, a1, a2, a3, f.x, f.y, x[n][k][0], x[n][k][1], x[n][k][2], x[n][k][3]);
                        }
                    }
                }
            }
            // every row sees every position of the chunk (that there is)?
            const bool all = base + CHUNK - 1 <= p0 && (p.c.window == 0 || base > seq.len - 1 - p.c.window || base + CHUNK <= p.c.n_first);
            auto at_of = [&](int k, int e) { return k * KV_BLOCK + (g >> 1) + 4 * (g & 1) + 8 * e; };
            float top[NT][2];
            bool more = false;
#pragma unroll
            for (int n = 0; n < NT; ++n) top[n][0] = top[n][1] = -INFINITY;
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float4 wd = sh.words[warp][at_of(k, e)];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float y = fmaf(x[n][k][2 * e + c], wd.x * qscale[n][c], fmaf(qsum[n][c], wd.y, wd.z));
                            if (!all) {
                                const int pos = base + at_of(k, e), at = p0 + (row0 + 8 * n + 2 * i4 + c) / p.group;
                                const bool see = pos <= at && (p.c.window == 0 || pos > at - p.c.window || pos < p.c.n_first);
                                if (!see) y = -INFINITY;
                            }
                            x[n][k][2 * e + c] = y;
                            top[n][c] = fmaxf(top[n][c], y);
                        }
                }
            // m moves only where a column's maximum has grown by more than 2^8
#pragma unroll
            for (int n = 0; n < NT; ++n) more = more || top[n][0] > m[n][0] + 15.0f || top[n][1] > m[n][1] + 15.0f;
            if (__any_sync(0xffffffffu, more)) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float alpha[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float t = top[n][c];
                        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
                        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
                        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
                        t = fmaxf(t - 7.0f, m[n][c]);
                        alpha[c] = ex2(m[n][c] - t);
                        m[n][c] = t;
                        l[n][c] *= alpha[c];
                        w[n][c] *= alpha[c];
                    }
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][k][e] *= alpha[e & 1];
                }
            }
            uint32_t pf[NT][C][2];
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float inv = sh.words[warp][at_of(k, e)].w, low = sh.lows[warp][at_of(k, e)];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float pr[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            pr[c] = ex2(x[n][k][2 * e + c] - m[n][c]);
                            l[n][c] = fmaf(pr[c], inv, l[n][c]);
                            w[n][c] = fmaf(pr[c], low, w[n][c]);
                        }
                        const __half2 h = __floats2half2_rn(pr[0], pr[1]);
                        pf[n][k][e] = transposed(*reinterpret_cast<const uint32_t *>(&h));
                    }
                }
            // ---- values: -1152 sum of P first, then the codes
            float start[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                mma(start[n], 0xe480e480u, 0xe480e480u, 0xe480e480u, 0xe480e480u, pf[n][0][0], pf[n][0][1], 0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int k = 1; k < C; ++k)
                    mma(start[n], 0xe480e480u, 0xe480e480u, 0xe480e480u, 0xe480e480u, pf[n][k][0], pf[n][k][1], start[n][0], start[n][1], start[n][2], start[n][3]);
            }
#pragma unroll
            for (int jw = 0; jw < D / 64; ++jw) {
                uint32_t lo[C][2], hi[C][2];  // of block k: positions i4, i4 + 4 (e = 0) and i4 + 8, i4 + 12 (e = 1); codes 0-3 and 4-7 of both
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint8_t *row = chunk + k * kv_block_bytes(D) + kv_v_codes(D) + (i4 + 8 * e) * (D / 2) + (D / 16) * g + 4 * jw;
                        const uint32_t u = *reinterpret_cast<const uint32_t *>(row), v = *reinterpret_cast<const uint32_t *>(row + 4 * (D / 2));
                        lo[k][e] = __byte_perm(u, v, 0x5410);
                        hi[k][e] = __byte_perm(u, v, 0x7632);
                    }
#pragma unroll
                for (int q = 0; q < 4; ++q) {  // codes 2q, 2q + 1 of the word
                    float acc[NT][4];
#pragma unroll
                    for (int k = 0; k < C; ++k) {
                        uint32_t a[2][2];  // [code][e]
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t z = q < 2 ? lo[k][e] : hi[k][e];
                            a[0][e] = and_or(q & 1 ? z >> 4 : z << 4, 0x00f000f0u, 0x64006400u);
                            a[1][e] = and_or(q & 1 ? z >> 8 : z, 0x00f000f0u, 0x64006400u);
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            if (k == 0) mma(acc[n], a[0][0], a[1][0], a[0][1], a[1][1], pf[n][0][0], pf[n][0][1], start[n][0], start[n][1], start[n][0], start[n][1]);
                            else mma(acc[n], a[0][0], a[1][0], a[0][1], a[1][1], pf[n][k][0], pf[n][k][1], acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][4 * jw + q][e] += acc[n][e];
                }
            }
        }
        phase += nt;

        // ---- the four warps' results of this (sequence, key head)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int k = 4; k < 32; k <<= 1) {
                    l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], k);
                    w[n][c] += __shfl_xor_sync(0xffffffffu, w[n][c], k);
                }
        if (g == 0)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    sh.m[warp][8 * n + 2 * i4 + c] = m[n][c];
                    sh.l[warp][8 * n + 2 * i4 + c] = l[n][c];
                }
        float *mine_o = reinterpret_cast<float *>(sh.ring[warp][0]);
        __syncwarp();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
                for (int c = 0; c < 2; ++c)  // values (D/8) g + 2k, + 1 of row 8n + 2 i4 + c; the factor 16 of the codes goes
                    *reinterpret_cast<float2 *>(mine_o + (8 * n + 2 * i4 + c) * (D + 4) + (D / 8) * g + 2 * k) =
                        make_float2(fmaf(o[n][k][c], 0.0625f, w[n][c]), fmaf(o[n][k][2 + c], 0.0625f, w[n][c]));
        const bool any_bad = __syncthreads_or(!ok);
        if (any_bad) break;
        const bool whole = t0 == 0 && nt == tl.count;
        float *part = p.parts + ((int64_t)blockIdx.x * 2 + (t0 == 0 ? 1 : 0)) * R * part_row(D);
        for (int at = tid; at < R * (D / 8); at += WARPS * 32) {
            const int r = at / (D / 8), d = at % (D / 8) * 8;
            if (r >= rows) break;
            float top = NONE;
#pragma unroll
            for (int v = 0; v < WARPS; ++v) top = fmaxf(top, sh.m[v][r]);
            float sum_l = 0.0f, y[8] = {};
#pragma unroll
            for (int v = 0; v < WARPS; ++v) {
                const float f = ex2(sh.m[v][r] - top);
                sum_l = fmaf(sh.l[v][r], f, sum_l);
                const float4 *z = reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(sh.ring[v][0]) + r * (D + 4) + d);
                const float4 z0 = z[0], z1 = z[1];
                const float zz[8] = {z0.x, z0.y, z0.z, z0.w, z1.x, z1.y, z1.z, z1.w};
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = fmaf(zz[k], f, y[k]);
            }
            if (whole) {
                const int tok = (row0 + r) / p.group, h = kh * p.group + (row0 + r - tok * p.group);
                const float inv = sum_l == 0.0f ? 0.0f : 1.0f / sum_l;
                uint32_t u[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const __nv_bfloat162 v2 = __floats2bfloat162_rn(y[2 * k] * inv, y[2 * k + 1] * inv);
                    u[k] = *reinterpret_cast<const uint32_t *>(&v2);
                }
                *reinterpret_cast<uint4 *>(p.c.out + (int64_t)(seq.start + tok) * p.c.out_stride + (int64_t)h * D + d) = make_uint4(u[0], u[1], u[2], u[3]);
            } else {
                float4 *dst = reinterpret_cast<float4 *>(part + r * part_row(D) + d);
                dst[0] = make_float4(y[0], y[1], y[2], y[3]);
                dst[1] = make_float4(y[4], y[5], y[6], y[7]);
                if (d == 0) *reinterpret_cast<float2 *>(part + r * part_row(D) + D) = make_float2(top, sum_l);
            }
        }
        if (t0 == 0 && nt < tl.count)  // begun here, ended by a later block (share tiles each)
            header = make_int4(1 + (tl.count - nt + share - 1) / share, seq.start, row0 << 16 | rows, kh);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the sums were written where copies go next
        __syncthreads();
    }
    if (!ok && lane == 0) {  // giving up: let the copies in flight land before the shared memory is released
        atomicExch(b.status, (int)TPQ_ERR_TIMEOUT);
        for (int k = issued > NS ? issued - NS : 0; k < issued; ++k) (void)mbar_wait(smem_u32(&sh.full[warp][k % NS]), (k / NS) & 1);
    }
    if (tid == 0) p.headers[blockIdx.x] = header;
}

// Puts partial results together, for the ones that run i ends with the first part of: a block takes the (run, row) pairs in turn, of
// which most have nothing to do.
constexpr int JOIN_PAIRS = 8;  // (their headers are loaded at once)
template <int D, int NT>
__global__ void __launch_bounds__(8 * D / 4)
attention_join(const split_params p, int runs)
{
    constexpr int GROUPS = 8, LANES = D / 4;  // parts in flight, threads of a row
    __shared__ float4 sums[GROUPS][LANES];
    __shared__ float2 ml[GROUPS];
    __shared__ int4 heads[JOIN_PAIRS];
    tpq_grid_dep_wait();
    const int lane = threadIdx.x % LANES, grp = threadIdx.x / LANES;
    if (threadIdx.x < JOIN_PAIRS) {
        const int pair = blockIdx.x + threadIdx.x * gridDim.x;
        heads[threadIdx.x] = pair < runs * 8 * NT ? __ldcg(p.headers + pair / (8 * NT)) : make_int4(0, 0, 0, 0);
    }
    __syncthreads();
    for (int k = 0; k < JOIN_PAIRS; ++k) {
        const int4 head = heads[k];  // parts, first row of the sequence, first row and rows, key head
        const int pair = blockIdx.x + k * gridDim.x, first = pair / (8 * NT), r = pair - first * (8 * NT);
        if (head.x == 0 || r >= (head.z & 0xffff)) continue;
        float m = NONE, l = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
        for (int i = grp; i < head.x; i += GROUPS) {
            // the first part is this run's last result, the others are the following runs' first
            const float *part = p.parts + (((int64_t)first + i) * 2 + (i == 0 ? 1 : 0)) * (8 * NT) * part_row(D) + r * part_row(D);
            const float2 v = __ldcg(reinterpret_cast<const float2 *>(part + D));
            const float4 z = __ldcg(reinterpret_cast<const float4 *>(part) + lane);
            const float top = fmaxf(m, v.x), a = ex2(m - top), f = ex2(v.x - top);
            m = top;
            l = fmaf(v.y, f, l * a);
            o = make_float4(fmaf(z.x, f, o.x * a), fmaf(z.y, f, o.y * a), fmaf(z.z, f, o.z * a), fmaf(z.w, f, o.w * a));
        }
        sums[grp][lane] = o;
        if (lane == 0) ml[grp] = make_float2(m, l);
        __syncthreads();
        if (grp == 0) {
            float top = NONE, sum_l = 0.0f;
#pragma unroll
            for (int v = 0; v < GROUPS; ++v) top = fmaxf(top, ml[v].x);
            float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int v = 0; v < GROUPS; ++v) {
                const float f = ex2(ml[v].x - top);
                const float4 z = sums[v][lane];
                sum_l = fmaf(ml[v].y, f, sum_l);
                y = make_float4(fmaf(z.x, f, y.x), fmaf(z.y, f, y.y), fmaf(z.z, f, y.z), fmaf(z.w, f, y.w));
            }
            const float inv = sum_l == 0.0f ? 0.0f : 1.0f / sum_l;
            const int row = (head.z >> 16) + r, tok = row / p.group, h = head.w * p.group + (row - tok * p.group);
            const __nv_bfloat162 a = __floats2bfloat162_rn(y.x * inv, y.y * inv), c = __floats2bfloat162_rn(y.z * inv, y.w * inv);
            *reinterpret_cast<uint2 *>(p.c.out + (int64_t)(head.y + tok) * p.c.out_stride + (int64_t)h * D + 4 * lane) =
                make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&c));
        }
        __syncthreads();
    }
}

// Groups of 8 rows that a warp takes at a time: one where no sequence has more rows, else two (24 sequences of 16 to 32 rows, heads of 64,
// before the runs were weighed: 55 us; four groups at once, with spilled registers and two blocks an SM, 81; one at a time 63).  A batch whose
// max_new allows more than 8 rows pays for it where its sequences bring 8 or fewer: 32 of 16 to 32 thousand positions 328 us instead of 210, 64 of up
// to 8000 44 instead of 33.
int row_groups(int64_t max_rows) { return max_rows <= 8 ? 1 : 2; }

template <int D, int NT>
cudaError_t launch_split(const split_params &p, int sm_count, cudaStream_t st, int64_t *launches)
{
    constexpr size_t smem = sizeof(Shared<D, NT>);
    static_assert(8 * NT * (D + 4) * 4 <= stages(D, NT) * chunk_bytes(D, NT), "a warp's sums fit its ring");
    cudaError_t e = cudaFuncSetAttribute(attention_split<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const int blocks = sm_count * BLOCKS_PER_SM;
    e = tpq_launch_pdl(attention_split<D, NT>, dim3(blocks), dim3(WARPS * 32), smem, st, p);
    if (e != cudaSuccess) return e;
    ++*launches;
    e = tpq_launch_pdl(attention_join<D, NT>, dim3((blocks * 8 * NT + JOIN_PAIRS - 1) / JOIN_PAIRS), dim3(8 * D / 4), 0, st, p, blocks);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace

size_t kv_attention_workspace(int D, int n_heads, int n_kv_heads, int sm_count, int64_t n_seqs, int64_t max_new, int64_t n_tokens)
{
    const int64_t group = n_heads / n_kv_heads;
    const int nt = row_groups(max_new * group);
    const size_t blocks = (size_t)sm_count * BLOCKS_PER_SM;
    return blocks * 16 + blocks * 2 * 8 * nt * part_row(D) * 4 +
           (max_new * group > MAX_ROWS ? kv_prompt_workspace(D, (int)group, sm_count, n_seqs, n_tokens) : 0);
}

cudaError_t kv_launch_attention(const kv_batch &b, int D, const kv_attention_call &c, int sm_count, cudaStream_t st, int64_t *launches)
{
    const int group = b.n_heads / b.n_kv_heads;
    const int64_t max_rows = (int64_t)b.max_new * group;
    const int nt = row_groups(max_rows);
    split_params p{b, c, nullptr, static_cast<int4 *>(c.workspace), c.scale * 1.4426950408889634f, group};
    const size_t blocks = (size_t)sm_count * BLOCKS_PER_SM;
    p.parts = reinterpret_cast<float *>(p.headers + blocks);
    if (max_rows > MAX_ROWS) {
        // (Of one sequence the kernels for many rows take whatever it brings: two launches less.  10 heads of 128, us, with and without these two:
        // 2048 new 50.0 and 44.8, 100 of 777 30.7 and 25.3, one of 777 where max_new is 128 25.0 and 17.8, but one of 32 000 there 35 and 58.)
        const cudaError_t e = kv_launch_prompt(b, D, c, b.n_seqs == 1 ? 0 : MAX_ROWS, p.parts + blocks * 2 * 8 * nt * part_row(D), sm_count, st, launches);
        if (e != cudaSuccess || b.n_seqs == 1) return e;
    }
    if (D == 128) return nt == 1 ? launch_split<128, 1>(p, sm_count, st, launches) : launch_split<128, 2>(p, sm_count, st, launches);
    return nt == 1 ? launch_split<64, 1>(p, sm_count, st, launches) : launch_split<64, 2>(p, sm_count, st, launches);
}
