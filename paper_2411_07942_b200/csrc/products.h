// What the product kernels share on the device (not installed).
#pragma once

#include "block_internal.h"

// 4-bit weights as BF16, exactly.  A pattern below 256 read as BF16 (a subnormal, or a number of the smallest exponent) is 2^-133 of it as an
// integer, so u = code + 8 needs no exponent of its own, and no shift in either half of a byte: with s the step over the row's factor,
//   (u 2^-133) (s 2^119) - 8 s 2^-14  =  (u 2^-129) (s 2^115) - 8 s 2^-14  =  code s 2^-14,
// at most 8 significant bits in one rounding that has nothing to round; the 2^14 go into the factor.
constexpr float W4_SCALE = 16384.0f;
struct w4_step {  // of a step byte, twice each
    uint32_t low, high, bias;
};
__device__ __forceinline__ w4_step w4_load_step(uint32_t byte)
{
    return {byte * 0x00080008u + 0x77007700u, byte * 0x00080008u + 0x75007500u, byte * 0x00080008u + 0xB600B600u};
}
// 8 codes (a word of the layout) times the step: pairs (2i, 2i + 1)
__device__ __forceinline__ void w4_unpack(uint32_t w, const w4_step &s, uint32_t *r)
{
    const uint32_t v = w >> 8;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r[0]) : "r"(w & 0x000F000Fu), "r"(s.low), "r"(s.bias));
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r[1]) : "r"(w & 0x00F000F0u), "r"(s.high), "r"(s.bias));
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r[2]) : "r"(v & 0x000F000Fu), "r"(s.low), "r"(s.bias));
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r[3]) : "r"(v & 0x00F000F0u), "r"(s.high), "r"(s.bias));
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

// the same place in the shared memory of block `rank` of the cluster
__device__ __forceinline__ uint32_t map_cluster(uint32_t addr, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
__device__ __forceinline__ void st_cluster(uint32_t a, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
