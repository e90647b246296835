// Weights in 4 bits: BF16 rows -> blocks of codes and steps (tpq_quantize_weight), and back (tpq_read_weight).
//
// Both stream: 2 bytes in and half a byte out a value, or the other way round; memory is the bound.  A block of threads takes 8 rows, a
// thread pieces of 32 adjacent values: 64 bytes of a row in, one 16-byte piece of codes out; the 8 rows' pieces are 128 adjacent
// bytes of the layout.  A row's steps share a factor that depends on all of the row (its largest step's exponent), so a first walk over the
// row finds the pieces' largest magnitudes; the second one reads the row again, from L2.
#include <cuda_bf16.h>

#include "block_internal.h"

namespace {

constexpr int ROWS = 8, THREADS = 256, PIECE = 32;
constexpr int LANES = THREADS / ROWS;  // pieces of a row at a time

// codes 8q .. 8q + 7 as a word: pair i (codes 2i, 2i + 1) in bits 4i and 16 + 4i
__device__ __forceinline__ uint32_t pack8(const uint32_t (&c)[8])
{
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= c[2 * i] << (4 * i) | c[2 * i + 1] << (16 + 4 * i);
    return w;
}

// 32 values of a row from k0 on (zeros behind its end) as 16 words of BF16 pairs
__device__ __forceinline__ void load_piece(const uint16_t *row, int64_t k0, int64_t K, bool wide, uint32_t (&v)[16])
{
    if (wide && k0 + PIECE <= K) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 q = reinterpret_cast<const uint4 *>(row + k0)[i];
            v[4 * i] = q.x;
            v[4 * i + 1] = q.y;
            v[4 * i + 2] = q.z;
            v[4 * i + 3] = q.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t k = k0 + 2 * i;
        v[i] = (k < K ? row[k] : 0u) | (k + 1 < K ? (uint32_t)row[k + 1] : 0u) << 16;
    }
}
__device__ __forceinline__ float lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

// 2a/15 rounded up to 5 significant bits, as the bits of a binary32
__device__ __forceinline__ uint32_t step_bits(uint32_t a) { return (__float_as_uint(__fdiv_rn(2.0f * __uint_as_float(a), 15.0f)) + 0x7FFFFu) & ~0x7FFFFu; }

template <int GROUP>
__global__ void __launch_bounds__(THREADS) quantize_weight(const uint16_t *w, int64_t stride, int64_t n, int64_t K, int wide, uint8_t *w4, float *factors)
{
    extern __shared__ uint32_t largest[];  // [ROWS][pieces], bits of magnitudes (ordered like the numbers)
    __shared__ uint32_t row_top[ROWS];
    constexpr int BLOCK = W4_CODE_BYTES + W4_TILE * (W4_TILE / GROUP), PER = GROUP / PIECE;
    const int r = threadIdx.x / LANES, lane = threadIdx.x % LANES;  // a warp is a row (the grid covers whole tiles of rows)
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    const int kb = (int)((K + W4_TILE - 1) / W4_TILE), pieces = kb * (W4_TILE / PIECE);
    tpq_grid_dep_wait();
    const uint16_t *in = w + row * stride;
    uint32_t top = 0;
    for (int p = lane; p < pieces; p += LANES) {
        uint32_t a = 0;
        if (row < n) {
            uint32_t v[16], m = 0;
            load_piece(in, (int64_t)p * PIECE, K, wide, v);
#pragma unroll
            for (int i = 0; i < 16; ++i) m = __vmaxu2(m, v[i] & 0x7FFF7FFFu);  // (magnitudes: NaN above infinity above numbers)
            a = max(m & 0xFFFFu, m >> 16) << 16;
        }
        largest[r * pieces + p] = a;
        top = max(top, a);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) row_top[r] = top;
    __syncthreads();
    // The row's exponent E: its largest step's, at least -87.  A step is 2^(E - 15) 2^e (1 + m/16) with e, m in 4 bits.
    const uint32_t top_bits = step_bits(top);
    const int E = max((int)(top_bits >> 23), 40);
    const bool bad = top >= (127u + 120u) << 23;  // NaN, infinity, 2^120 and more: the row is NaN
    if (lane == 0) factors[row] = bad ? __uint_as_float(0x7FC00000u) : __uint_as_float((uint32_t)(E - 7) << 23);
    uint8_t *const tile = w4 + (row / W4_TILE) * (int64_t)kb * BLOCK;
    const int in_tile = (int)(row % W4_TILE);
    for (int p = lane; p < pieces; p += LANES) {
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) a = max(a, largest[r * pieces + p / PER * PER + i]);
        const uint32_t bits = step_bits(a);
        const int e = (int)(bits >> 23) - E + 15;
        const uint32_t byte = e < 0 || bad ? 0u : (uint32_t)e << 4 | (bits >> 19 & 15u);
        const float step = bad ? 1.0f : __uint_as_float(e < 0 ? (uint32_t)(E - 15) << 23 : bits);
        uint32_t v[16];
        if (row < n && !bad) {
            load_piece(in, (int64_t)p * PIECE, K, wide, v);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = 0;
        }
        uint4 out;
        uint32_t *const words = reinterpret_cast<uint32_t *>(&out);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = i & 1 ? hi(v[4 * q + i / 2]) : lo(v[4 * q + i / 2]);
                c[i] = (uint32_t)(__float2int_rn(fminf(fmaxf(__fdiv_rn(x, step), -8.0f), 7.0f)) + 8);
            }
            words[q] = pack8(c);
        }
        uint8_t *const block = tile + (int64_t)(p / 4) * BLOCK;
        *reinterpret_cast<uint4 *>(block + (p % 4) * (W4_TILE * 16) + in_tile * 16) = out;
        if (p % PER == 0) block[W4_CODE_BYTES + (p % 4) / PER * W4_TILE + in_tile] = (uint8_t)byte;
    }
}

template <int GROUP>
__global__ void __launch_bounds__(THREADS) read_weight(const uint8_t *w4, const float *factors, int64_t n, int64_t K, uint16_t *out, int64_t stride, int wide)
{
    constexpr int BLOCK = W4_CODE_BYTES + W4_TILE * (W4_TILE / GROUP), PER = GROUP / PIECE;
    // a warp: 8 rows x 4 pieces (one block of the layout), so that both sides are runs of 128 bytes and more
    const int r = threadIdx.x % ROWS, p0 = threadIdx.x / ROWS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    const int kb = (int)((K + W4_TILE - 1) / W4_TILE), pieces = (int)((K + PIECE - 1) / PIECE);
    tpq_grid_dep_wait();
    if (row >= n) return;
    const float factor = factors[row];
    const uint8_t *const tile = w4 + (row / W4_TILE) * (int64_t)kb * BLOCK;
    const int in_tile = (int)(row % W4_TILE);
    for (int p = p0; p < pieces; p += THREADS / ROWS) {
        const uint8_t *const block = tile + (int64_t)(p / 4) * BLOCK;
        const uint4 q = *reinterpret_cast<const uint4 *>(block + (p % 4) * (W4_TILE * 16) + in_tile * 16);
        const uint32_t byte = block[W4_CODE_BYTES + (p % 4) / PER * W4_TILE + in_tile];
        const float step = factor * __uint_as_float((byte << 19) + (119u << 23));
        const uint32_t words[4] = {q.x, q.y, q.z, q.w};
        uint32_t v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t w = words[i / 4] >> (4 * (i % 4));
            const __nv_bfloat162 b = __floats2bfloat162_rn(step * (float)((int)(w & 15u) - 8), step * (float)((int)(w >> 16 & 15u) - 8));
            v[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        const int64_t k0 = (int64_t)p * PIECE;
        uint16_t *const o = out + row * stride + k0;
        if (wide && k0 + PIECE <= K) {
#pragma unroll
            for (int i = 0; i < 4; ++i) reinterpret_cast<uint4 *>(o)[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < PIECE; ++i)
                if (k0 + i < K) o[i] = (uint16_t)(v[i / 2] >> (16 * (i % 2)));
        }
    }
}

bool wide_rows(const void *p, int64_t stride) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride % 8 == 0; }

}  // namespace

cudaError_t w4_launch_quantize(const uint16_t *w, int64_t stride, int64_t n, int64_t K, int group, uint8_t *w4, cudaStream_t st, int64_t *launches)
{
    auto kern = group == 32 ? quantize_weight<32> : group == 64 ? quantize_weight<64> : quantize_weight<128>;
    const size_t smem = (size_t)ROWS * w4_tiles(K) * (W4_TILE / PIECE) * 4;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    e = tpq_launch_pdl(kern, dim3((unsigned)(w4_tiles(n) * (W4_TILE / ROWS))), dim3(THREADS), smem, st, w, stride, n, K, (int)wide_rows(w, stride), w4,
                       reinterpret_cast<float *>(w4 + w4_factors_at(n, K, group)));
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
