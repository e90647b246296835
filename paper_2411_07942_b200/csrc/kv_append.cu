// Keys and values into the pages of the 4-bit cache, queries and keys rotated on the way (tpq_kv_append), and back out
// (tpq_kv_read).
//
// A vector is one head of one row.  D/8 lanes hold it, 8 adjacent values each: one 16-byte load, and the lane's 8 codes
// are one 32-bit word of the cache.  A warp takes one row and up to ITER * 256/D heads of one kind (queries, keys or values:
// no lane of a warp does another's work), all loads ahead of the arithmetic.  Nothing is read twice; what bounds a long prompt is
// memory (7652 rows of 64 query and 2 x 8 key and value heads of 128, and reading them back: 70 us, 4.7 TB/s; the division per value
// that was there first 80 us), what bounds one token is the chain token start -> length -> page number -> store (12 us with the read, all
// of it launches).  Four heads a lane at a time: two 91 us, eight 110; several jobs a warp one after the other: 76.
#include "kv_internal.h"

#include <cuda_bf16.h>

namespace {

constexpr int KV_WARPS = 4;

struct rotation {
    const float *table;
    const int32_t *positions;
    int64_t n_positions;
    int dim, interleaved;
};

__device__ __forceinline__ float min_nan(float a, float b)  // NaN if either is
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void widen(const uint4 &w, float (&x)[8])
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 narrow(const float (&x)[8])
{
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

// Codes of the 8 values of a lane and the word of the vector (the same in all its lanes).
template <int LANES>
__device__ __forceinline__ uint32_t quantise(const float (&x)[8], uint32_t &word)
{
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        lo = min_nan(lo, x[i]);
        hi = max_nan(hi, x[i]);
    }
#pragma unroll
    for (int m = LANES / 2; m > 0; m >>= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, m));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, m));
    }
    const float low = __bfloat162float(__float2bfloat16_rn(lo));
    const float d = __fsub_rn(hi, low);
    const float top = fmaxf(fabsf(lo), fabsf(hi));
    // (2^-16 of the largest magnitude: a finer step than that says nothing beside `low`, whose rounding may be 2^-9 of it;
    // 2^-60: the attention kernels divide by the steps)
    const float want = fmaxf(fmaxf(__fmul_rn(d, 1.0f / 15.0f), __fmul_rn(top, 0x1p-16f)), 0x1p-60f);
    const float step = __bfloat162float(__float2bfloat16_rn(want));
    if (!(d < INFINITY) || !isfinite(low)) {
        word = 0x7fc03f80u;  // low NaN, step 1
        return 0;
    }
    word = (__float_as_uint(low) & 0xffff0000u) | (__float_as_uint(step) >> 16);
    // The quotients, correctly rounded, from one reciprocal (Markstein's theorem: q + r y is, where y is the correctly rounded
    // reciprocal of the divisor, q = a y and r = a - q step exactly; with a divisor of 8 bits r is exact also where q is more than
    // a unit off, and no quotient comes within 2^-9 units of halfway between two numbers): a division per value took most of this kernel's
    // time.  Adding 1.5 x 2^23 rounds half to even.
    const float y = __frcp_rn(step);
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = __fsub_rn(x[i], low), q = __fmul_rn(a, y), u = __fmaf_rn(__fmaf_rn(-q, step, a), y, q);
        codes |= (__float_as_uint(__fadd_rn(fminf(fmaxf(u, 0.0f), 15.0f), 12582912.0f)) & 15u) << (4 * i);
    }
    return codes;
}

// The entry of a position: base of its block for key head 0, or NULL (status set) where its page is outside the pool.
__device__ __forceinline__ uint8_t *entry_block(const kv_batch &b, int s, int pos, int block_bytes)
{
    const int page = b.table[s * b.table_stride + (pos >> b.page_shift)];
    if (page < 0 || page >= b.n_pages) {
        kv_report(b);
        return nullptr;
    }
    const int blocks = b.page_size / KV_BLOCK;
    return b.cache + ((int64_t)page * b.n_kv_heads * blocks + ((pos & (b.page_size - 1)) / KV_BLOCK)) * block_bytes;
}

// ITER vectors a lane holds at a time; a warp's job is ITER * 256/D heads of one kind of one row.
template <int D, int ITER>
__global__ void __launch_bounds__(KV_WARPS * 32)
append_kernel(const kv_batch b, const rotation rot, const kv_rows k, const kv_rows v, const kv_rows q, uint16_t *q_out, int64_t q_out_stride)
{
    constexpr int LANES = D / 8, PER = 32 / LANES;  // lanes of a vector, vectors of a warp
    const int lane = threadIdx.x & 31, li = lane % LANES, sub = lane / LANES;
    const int q_jobs = q.p ? (b.n_heads + ITER * PER - 1) / (ITER * PER) : 0, kv_jobs = (b.n_kv_heads + ITER * PER - 1) / (ITER * PER);
    const int jobs = q_jobs + 2 * kv_jobs;
    const int64_t id = (int64_t)blockIdx.x * KV_WARPS + (threadIdx.x >> 5);
    const int64_t row = id / jobs;
    int job = (int)(id - row * jobs);
    tpq_grid_dep_wait();
    tpq_grid_dep_launch();
    if (row >= b.n_tokens) return;
    const int kind = job < q_jobs ? 0 : job < q_jobs + kv_jobs ? 1 : 2;  // queries, keys, values
    if (kind) job -= kind == 1 ? q_jobs : q_jobs + kv_jobs;
    const int heads = kind ? b.n_kv_heads : b.n_heads, h0 = job * ITER * PER + sub;
    const kv_rows in = kind == 0 ? q : kind == 1 ? k : v;
    const uint16_t *x_row = in.p + row * in.stride;
    uint4 raw[ITER];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {  // (rows that belong to nobody are the caller's memory too: n_tokens of them)
        const int h = h0 + i * PER;
        raw[i] = h < heads ? __ldcs(reinterpret_cast<const uint4 *>(x_row + (int64_t)h * D) + li) : make_uint4(0, 0, 0, 0);
    }
    const int s = kv_find_seq(b, row, lane);
    if (s < 0) return;
    const kv_seq seq = kv_load_seq(b, s);
    if (seq.n < 0 || !kv_owns(b, seq, row)) return;
    const int pos = seq.len - seq.n + (int)(row - seq.start);

    float cs[8], sn[8];  // of this lane's values; (half pairs) the partner's value times the signed sine is added
    int partner = lane;
    const bool turn = kind != 2 && rot.table != nullptr;
    const int p = rot.table && rot.positions ? rot.positions[row] : pos;
    if (rot.table && (p < 0 || p >= rot.n_positions)) {  // (the whole row is left out: queries, keys and values)
        if (lane == 0) kv_report(b);
        return;
    }
    if (turn) {
        const int half = rot.dim / 2, d = li * 8;
        const float *t = rot.table + (int64_t)p * rot.dim;
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[i] = 1.0f, sn[i] = 0.0f;
        if (d < rot.dim) {
            const int j = rot.interleaved ? d / 2 : d < half ? d : d - half;  // first pair of the lane
            const int n = rot.interleaved ? 4 : 8;
#pragma unroll
            for (int i = 0; i < 8; i += 4)
                if (i < n) {
                    const float4 c4 = __ldcg(reinterpret_cast<const float4 *>(t + j + i)), s4 = __ldcg(reinterpret_cast<const float4 *>(t + half + j + i));
                    cs[i] = c4.x, cs[i + 1] = c4.y, cs[i + 2] = c4.z, cs[i + 3] = c4.w;
                    sn[i] = s4.x, sn[i + 1] = s4.y, sn[i + 2] = s4.z, sn[i + 3] = s4.w;
                }
            if (!rot.interleaved) {
                partner = sub * LANES + (d < half ? li + half / 8 : li - half / 8);
                if (d < half)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sn[i] = -sn[i];  // a cos - b sin = a cos + b (-sin), rounding for rounding
            }
        }
    }
    uint8_t *block = kind ? entry_block(b, s, pos, kv_block_bytes(D)) : nullptr;
    if (kind && !block) return;
    const int64_t head_bytes = (int64_t)(b.page_size / KV_BLOCK) * kv_block_bytes(D);
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int h = h0 + i * PER;
        float x[8];
        widen(raw[i], x);
        if (turn) {
            if (rot.interleaved) {
                if (li * 8 < rot.dim) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float a = x[2 * j], c = x[2 * j + 1];
                        x[2 * j] = __fsub_rn(__fmul_rn(a, cs[j]), __fmul_rn(c, sn[j]));
                        x[2 * j + 1] = __fadd_rn(__fmul_rn(c, cs[j]), __fmul_rn(a, sn[j]));
                    }
                }
            } else {
                uint4 other;
                other.x = __shfl_sync(0xffffffffu, raw[i].x, partner);
                other.y = __shfl_sync(0xffffffffu, raw[i].y, partner);
                other.z = __shfl_sync(0xffffffffu, raw[i].z, partner);
                other.w = __shfl_sync(0xffffffffu, raw[i].w, partner);
                if (li * 8 < rot.dim) {
                    float y[8];
                    widen(other, y);
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = __fadd_rn(__fmul_rn(x[j], cs[j]), __fmul_rn(y[j], sn[j]));
                }
            }
        }
        if (kind == 0) {
            if (h < heads) __stcs(reinterpret_cast<uint4 *>(q_out + row * q_out_stride + (int64_t)h * D) + li, narrow(x));
        } else {
            uint32_t word;
            const uint32_t codes = quantise<LANES>(x, word);
            if (h < heads) {
                uint8_t *p = block + h * head_bytes;
                const int r = pos % KV_BLOCK;
                reinterpret_cast<uint32_t *>(p + (kind == 1 ? 0 : kv_v_codes(D)) + r * (D / 2))[li] = codes;
                if (li == 0) reinterpret_cast<uint32_t *>(p + (kind == 1 ? kv_k_words(D) : kv_v_words(D)))[r] = word;
            }
        }
    }
}

template <int D, int ITER>
__global__ void __launch_bounds__(KV_WARPS * 32)
read_kernel(const kv_batch b, uint16_t *k_out, int64_t k_stride, uint16_t *v_out, int64_t v_stride)
{
    constexpr int LANES = D / 8, PER = 32 / LANES;
    const int lane = threadIdx.x & 31, li = lane % LANES, sub = lane / LANES;
    const int half_jobs = (b.n_kv_heads + ITER * PER - 1) / (ITER * PER), jobs = (k_out ? half_jobs : 0) + (v_out ? half_jobs : 0);
    const int64_t id = (int64_t)blockIdx.x * KV_WARPS + (threadIdx.x >> 5);
    const int64_t row = id / jobs;
    int job = (int)(id - row * jobs);
    tpq_grid_dep_wait();
    tpq_grid_dep_launch();
    if (row >= b.n_tokens) return;
    const bool keys = k_out && job < half_jobs;
    if (k_out && !keys) job -= half_jobs;
    const int s = kv_find_seq(b, row, lane);
    if (s < 0) return;
    const kv_seq seq = kv_load_seq(b, s);
    if (seq.n < 0 || !kv_owns(b, seq, row)) return;
    const int pos = seq.len - seq.n + (int)(row - seq.start), r = pos % KV_BLOCK, h0 = job * ITER * PER + sub;
    const uint8_t *block = entry_block(b, s, pos, kv_block_bytes(D));
    if (!block) return;
    const int64_t head_bytes = (int64_t)(b.page_size / KV_BLOCK) * kv_block_bytes(D);
    uint32_t codes[ITER], word[ITER];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int h = h0 + i * PER;
        const uint8_t *p = block + h * head_bytes;
        codes[i] = word[i] = 0;
        if (h < b.n_kv_heads) {
            codes[i] = __ldcg(reinterpret_cast<const uint32_t *>(p + (keys ? 0 : kv_v_codes(D)) + r * (D / 2)) + li);
            word[i] = __ldcg(reinterpret_cast<const uint32_t *>(p + (keys ? kv_k_words(D) : kv_v_words(D))) + r);
        }
    }
    uint16_t *out = keys ? k_out + row * k_stride : v_out + row * v_stride;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int h = h0 + i * PER;
        const float step = __uint_as_float(word[i] << 16), low = __uint_as_float(word[i] & 0xffff0000u);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __fmaf_rn(step, (float)((codes[i] >> (4 * j)) & 15u), low);  // (the product is exact)
        if (h < b.n_kv_heads) __stcs(reinterpret_cast<uint4 *>(out + (int64_t)h * D) + li, narrow(x));
    }
}

// Heads of a warp's job: as many as leave every SM a dozen warps, at most four loads in flight per lane.
int job_heads(int64_t vectors, int per, int sm_count) { return vectors / per / 4 >= 12 * (int64_t)sm_count ? 4 : 1; }

}  // namespace

cudaError_t kv_launch_append(const kv_batch &b, int D, const tpq_kv_rotation *rot, kv_rows k, kv_rows v, kv_rows q, uint16_t *q_out,
                             int64_t q_out_stride, int sm_count, cudaStream_t st, int64_t *launches)
{
    rotation r{nullptr, nullptr, 0, 0, 0};
    if (rot) r = rotation{rot->table_dev, rot->positions_dev, rot->n_positions, rot->rot_dim, rot->interleaved};
    const int per = 256 / D;
    const int iter = job_heads(b.n_tokens * (2 * b.n_kv_heads + (q.p ? b.n_heads : 0)), per, sm_count);
    auto up = [&](int heads) { return (int64_t)(heads + iter * per - 1) / (iter * per); };
    const int64_t warps = b.n_tokens * (2 * up(b.n_kv_heads) + (q.p ? up(b.n_heads) : 0)), blocks = (warps + KV_WARPS - 1) / KV_WARPS;
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    auto go = [&](auto kern) { return tpq_launch_pdl(kern, dim3((unsigned)blocks), dim3(KV_WARPS * 32), 0, st, b, r, k, v, q, q_out, q_out_stride); };
    const cudaError_t e = D == 128 ? (iter == 4 ? go(append_kernel<128, 4>) : go(append_kernel<128, 1>))
                                   : (iter == 4 ? go(append_kernel<64, 4>) : go(append_kernel<64, 1>));
    if (e == cudaSuccess) ++*launches;
    return e;
}

cudaError_t kv_launch_read(const kv_batch &b, int D, uint16_t *k_out, int64_t k_stride, uint16_t *v_out, int64_t v_stride, int sm_count,
                           cudaStream_t st, int64_t *launches)
{
    const int per = 256 / D, kinds = (k_out ? 1 : 0) + (v_out ? 1 : 0);
    const int iter = job_heads(b.n_tokens * kinds * b.n_kv_heads, per, sm_count);
    const int64_t warps = b.n_tokens * kinds * ((b.n_kv_heads + iter * per - 1) / (iter * per)), blocks = (warps + KV_WARPS - 1) / KV_WARPS;
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    auto go = [&](auto kern) { return tpq_launch_pdl(kern, dim3((unsigned)blocks), dim3(KV_WARPS * 32), 0, st, b, k_out, k_stride, v_out, v_stride); };
    const cudaError_t e = D == 128 ? (iter == 4 ? go(read_kernel<128, 4>) : go(read_kernel<128, 1>))
                                   : (iter == 4 ? go(read_kernel<64, 4>) : go(read_kernel<64, 1>));
    if (e == cudaSuccess) ++*launches;
    return e;
}
