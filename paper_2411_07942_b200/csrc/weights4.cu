// Weights in 4 bits: BF16 rows -> blocks of codes and steps (tpq_quantize_weight), and back (tpq_read_weight).
//
// Both stream: 2 bytes in and half a byte out a value, or the other way round; memory is the bound.  A warp takes 8 rows x 128 inputs, a block
// of the layout's: lane (r, q) has of each 16-byte piece of codes word q, 8 values.  So a warp reads or writes 64 adjacent bytes of each row and
// 128 adjacent bytes of the pieces at a time.  A row's steps share a factor that depends on all of the row (its largest step's exponent): a first
// walk over the rows finds the groups' largest magnitudes; for the second one rows of up to 5120 stay in registers, longer ones are read again,
// from L2.
// 32000 x 5120 (412 MB): 97 us to 4 bits (4.3 TB/s; 10 instructions a value, 57 % of the issue slots and 54 % of the ALU's: latency as much), 67 to 71 back (6 TB/s).  With a thread to 32 values of a row (16-byte loads and stores 64 bytes apart) and
// quotients by __fdiv_rn they took 153 and 101, with the second walk
// from L2 the first took 119, with one value at a time 110.
#include <cuda_bf16.h>

#include "block_internal.h"

namespace {

constexpr int ROWS = 8, WARPS = 8, THREADS = WARPS * 32;

// 8 values of a row from k0 on (zeros behind its end) as 4 BF16 pairs
__device__ __forceinline__ uint4 load8(const uint16_t *row, int64_t k0, int64_t K, bool wide)
{
    if (wide && k0 + 8 <= K) return *reinterpret_cast<const uint4 *>(row + k0);
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t k = k0 + 2 * i;
        v[i] = (k < K ? row[k] : 0u) | (k + 1 < K ? (uint32_t)row[k + 1] : 0u) << 16;
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// 2a/15 rounded up to 5 significant bits, as the bits of a binary32; a: a BF16 magnitude's bits
__device__ __forceinline__ uint32_t step_bits(uint32_t a) { return (__float_as_uint(__fdiv_rn(2.0f * __uint_as_float(a << 16), 15.0f)) + 0x7FFFFu) & ~0x7FFFFu; }

// Of two magnitudes each the larger (NaN above all), and of two numbers each the smaller
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
{
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    return a;
}
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b)
{
    asm("min.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    return a;
}
// The codes of a pair x / step plus 8, in the low halves' low bits.  x has 8 significant bits and the step 5: where their quotient
// is at least a half, it is a tie or further than 2^-10 from every tie, so rounding the product with the reciprocal (off by 2^-19 at most)
// to multiples of 2^-14 first leaves exactly the ties; the second sum, with 1.5 * 2^23, rounds to integers.  (Above 7 steps, an exact BF16 number, is 7;
// nothing is below -8: the step is no smaller than 2/15 of the magnitude.)
__device__ __forceinline__ uint32_t code_pair(uint32_t x, uint32_t most, uint64_t inv)
{
    const uint32_t v = min2(x, most);
    uint64_t u;
    asm("mov.b64 %0, {%1, %2};" : "=l"(u) : "r"(v << 16), "r"(v & 0xFFFF0000u));
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(u) : "l"(inv));
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(u) : "l"(0x4442000044420000ull));  // 768 + 8
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(u) : "l"(0x4B3FFD004B3FFD00ull));  // 1.5 * 2^23 - 768
    uint32_t lo, hi;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(u));
    return __byte_perm(lo, hi, 0x5410);
}

// KEEP: blocks of a warp that stay in registers between the walks (0: as many as there are, read again)
template <int GROUP, int KEEP>
__global__ void __launch_bounds__(THREADS) quantize_weight(const uint16_t *w, int64_t stride, int64_t n, int64_t K, int wide, uint8_t *w4, float *factors)
{
    extern __shared__ uint16_t largest[];  // [ROWS][groups], bits of BF16 magnitudes (ordered like the numbers, NaN above infinity above those)
    __shared__ uint32_t tops[WARPS][ROWS];
    constexpr int GROUPS = W4_TILE / GROUP, BLOCK = W4_CODE_BYTES + W4_TILE * GROUPS;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, r = lane / 4, q = lane % 4;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;  // (the grid covers whole tiles of rows)
    const int kb = (int)((K + W4_TILE - 1) / W4_TILE);
    tpq_grid_dep_wait();
    const uint16_t *in = w + row * stride;
    const bool there = row < n;
    uint32_t top = 0;
    uint4 kept[KEEP ? KEEP : 1][4];
    auto fetch = [&](int b, uint4 (&v)[4]) {
#pragma unroll
        for (int p = 0; p < 4; ++p) v[p] = there && b < kb ? load8(in, (int64_t)b * W4_TILE + p * 32 + q * 8, K, wide) : make_uint4(0, 0, 0, 0);
    };
    auto measure = [&](int b, const uint4 (&values)[4]) {
        uint32_t m[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint4 &v = values[p];
            uint32_t a = max2(max2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), max2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
            a = max2(a, __shfl_xor_sync(0xffffffffu, a, 1));
            a = max2(a, __shfl_xor_sync(0xffffffffu, a, 2));
            m[p] = max(a & 0xFFFFu, a >> 16);
        }
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            uint32_t a = m[g * (4 / GROUPS)];
#pragma unroll
            for (int i = 1; i < 4 / GROUPS; ++i) a = max(a, m[g * (4 / GROUPS) + i]);
            if (q == 0) largest[(b * GROUPS + g) * ROWS + r] = (uint16_t)a;
            top = max(top, a);
        }
    };
    if (KEEP) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i) fetch(warp + i * WARPS, kept[i]);
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (warp + i * WARPS < kb) measure(warp + i * WARPS, kept[i]);
    } else {
        for (int b = warp; b < kb; b += WARPS) {
            fetch(b, kept[0]);
            measure(b, kept[0]);
        }
    }
    if (q == 0) tops[warp][r] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WARPS; ++i) top = max(top, tops[i][r]);
    // The row's exponent E: its largest step's, at least -87.  A step is 2^(E - 15) 2^e (1 + m/16) with e, m in 4 bits.
    const int E = max((int)(step_bits(top) >> 23), 40);
    const bool bad = top >= (127u + 120u) << 7;  // NaN, infinity, 2^120 and more: the row is NaN
    if (warp == 0 && q == 0) factors[row] = bad ? __uint_as_float(0x7FC00000u) : __uint_as_float((uint32_t)(E - 7) << 23);
    uint8_t *const tile = w4 + (row / W4_TILE) * (int64_t)kb * BLOCK;
    const int in_tile = (int)(row % W4_TILE);
    auto encode = [&](int b, const uint4 (&values)[4]) {
        uint8_t *const block = tile + (int64_t)b * BLOCK;
        uint64_t inv[GROUPS];
        uint32_t most[GROUPS];  // 7 steps
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const uint32_t bits = bad ? 0u : step_bits(largest[(b * GROUPS + g) * ROWS + r]);
            const int e = (int)(bits >> 23) - E + 15;
            const float step = __uint_as_float(e < 0 ? (uint32_t)(bad ? 127 : E - 15) << 23 : bits);
            const uint32_t inverse = __float_as_uint(__frcp_rn(step));
            inv[g] = (uint64_t)inverse << 32 | inverse;
            most[g] = (__float_as_uint(7.0f * step) >> 16) * 0x00010001u;
            if (q == 0) block[W4_CODE_BYTES + g * W4_TILE + in_tile] = (uint8_t)(e < 0 ? 0u : (uint32_t)e << 4 | (bits >> 19 & 15u));
        }
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint4 &v = values[p];
            const uint32_t pairs[4] = {v.x, v.y, v.z, v.w};
            uint32_t word = 0;
#pragma unroll
            for (int i = 3; i >= 0; --i) word = word * 16 + code_pair(pairs[i], most[p / (4 / GROUPS)], inv[p / (4 / GROUPS)]);  // pair i in bits 4i and 16 + 4i
            *reinterpret_cast<uint32_t *>(block + p * (W4_TILE * 16) + in_tile * 16 + q * 4) = bad ? 0x88888888u : word;
        }
    };
    if (KEEP) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (warp + i * WARPS < kb) encode(warp + i * WARPS, kept[i]);
    } else {
        for (int b = warp; b < kb; b += WARPS) {
            fetch(b, kept[0]);
            encode(b, kept[0]);
        }
    }
}

template <int GROUP>
__global__ void __launch_bounds__(THREADS) read_weight(const uint8_t *w4, const float *factors, int64_t n, int64_t K, uint16_t *out, int64_t stride, int wide)
{
    constexpr int GROUPS = W4_TILE / GROUP, BLOCK = W4_CODE_BYTES + W4_TILE * GROUPS;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, r = lane / 4, q = lane % 4;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    const int kb = (int)((K + W4_TILE - 1) / W4_TILE);
    tpq_grid_dep_wait();
    if (row >= n) return;
    const float factor = factors[row];
    const uint8_t *const tile = w4 + (row / W4_TILE) * (int64_t)kb * BLOCK;
    const int in_tile = (int)(row % W4_TILE);
#pragma unroll 2
    for (int b = warp; b < kb; b += WARPS) {
        const uint8_t *const block = tile + (int64_t)b * BLOCK;
        uint32_t words[4], bytes[GROUPS];
#pragma unroll
        for (int p = 0; p < 4; ++p) words[p] = *reinterpret_cast<const uint32_t *>(block + p * (W4_TILE * 16) + in_tile * 16 + q * 4);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) bytes[g] = block[W4_CODE_BYTES + g * W4_TILE + in_tile];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const float step = factor * __uint_as_float((bytes[p / (4 / GROUPS)] << 19) + (119u << 23));
            uint32_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t u = words[p] >> (4 * i);
                // (u in the mantissa of 2^23: a difference, exact)
                const float c0 = __uint_as_float((u & 15u) | 0x4B000000u) - 8388616.0f, c1 = __uint_as_float((u >> 16 & 15u) | 0x4B000000u) - 8388616.0f;
                const __nv_bfloat162 h = __floats2bfloat162_rn(step * c0, step * c1);
                v[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
            const int64_t k0 = (int64_t)b * W4_TILE + p * 32 + q * 8;
            uint16_t *const o = out + row * stride + k0;
            if (wide && k0 + 8 <= K) *reinterpret_cast<uint4 *>(o) = make_uint4(v[0], v[1], v[2], v[3]);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (k0 + i < K) o[i] = (uint16_t)(v[i / 2] >> (16 * (i % 2)));
        }
    }
}

bool wide_rows(const void *p, int64_t stride) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride % 8 == 0; }

size_t shared_bytes(int64_t K, int group) { return (size_t)ROWS * w4_tiles(K) * (W4_TILE / group) * 2; }

}  // namespace

// Once per handle.  The limit of shared memory belongs to the kernel on this device and not to a handle, so it is the same whoever sets it: what the
// longest rows take (64 KB; the other kernels stay below the 48 KB that need no leave).
cudaError_t w4_prepare()
{
    return cudaFuncSetAttribute(quantize_weight<32, 0>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared_bytes(W4_MOST_INPUTS, 32));
}

cudaError_t w4_launch_quantize(const uint16_t *w, int64_t stride, int64_t n, int64_t K, int group, uint8_t *w4, cudaStream_t st, int64_t *launches)
{
    const int64_t each = (w4_tiles(K) + WARPS - 1) / WARPS;  // blocks of a warp
#define KERNEL(KEEP) (group == 32 ? quantize_weight<32, KEEP> : group == 64 ? quantize_weight<64, KEEP> : quantize_weight<128, KEEP>)
    auto kern = each <= 2 ? KERNEL(2) : each <= 5 ? KERNEL(5) : KERNEL(0);
#undef KERNEL
    const cudaError_t e = tpq_launch_pdl(kern, dim3((unsigned)(w4_tiles(n) * (W4_TILE / ROWS))), dim3(THREADS), shared_bytes(K, group), st, w, stride, n, K,
                                         (int)wide_rows(w, stride), w4, reinterpret_cast<float *>(w4 + w4_factors_at(n, K, group)));
    if (e == cudaSuccess) ++*launches;
    return e;
}

cudaError_t w4_launch_read(const uint8_t *w4, int64_t n, int64_t K, int group, uint16_t *out, int64_t stride, cudaStream_t st, int64_t *launches)
{
    auto kern = group == 32 ? read_weight<32> : group == 64 ? read_weight<64> : read_weight<128>;
    cudaError_t e = tpq_launch_pdl(kern, dim3((unsigned)((n + ROWS - 1) / ROWS)), dim3(THREADS), 0, st, w4,
                                   reinterpret_cast<const float *>(w4 + w4_factors_at(n, K, group)), n, K, out, stride, (int)wide_rows(out, stride));
    if (e == cudaSuccess) ++*launches;
    return e;
}
