// Attention over the 4-bit cache (tpq_kv_attention): a warp per row and query head walks the visible positions with the
// running maximum and sum of the softmax.
#include "kv_internal.h"

#include <cuda_bf16.h>

namespace {

template <int D>
__global__ void __launch_bounds__(128)
attention_rows(const kv_batch b, const kv_attention_call c)
{
    constexpr int V = D / 32;  // values of a lane
    const int lane = threadIdx.x & 31;
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5), row = id / b.n_heads;
    const int h = (int)(id - row * b.n_heads), kh = h / (b.n_heads / b.n_kv_heads);
    tpq_grid_dep_wait();
    tpq_grid_dep_launch();
    if (row >= b.n_tokens) return;
    const int s = kv_find_seq(b, row, lane);
    if (s < 0) return;
    const kv_seq seq = kv_load_seq(b, s);
    if (seq.n < 0 || row >= seq.start + seq.n) return;
    const int pos = seq.len - seq.n + (int)(row - seq.start);
    float q[V], o[V], m = -INFINITY, l = 0.0f;
    for (int i = 0; i < V; ++i) {
        q[i] = __uint_as_float((uint32_t)c.q.p[row * c.q.stride + (int64_t)h * D + lane * V + i] << 16);
        o[i] = 0.0f;
    }
    const int blocks = b.page_size / KV_BLOCK;
    const int64_t from = c.window ? (int64_t)pos - c.window + 1 : 0;
    for (int t = 0; t <= pos; ++t) {
        if (t < from && t >= c.n_first) {
            t = (int)from - 1;
            continue;
        }
        const int page = b.table[s * b.table_stride + (t >> b.page_shift)];
        if (page < 0 || page >= b.n_pages) {
            if (lane == 0) kv_report(b);
            continue;
        }
        const uint8_t *p = b.cache + (((int64_t)page * b.n_kv_heads + kh) * blocks + (t & (b.page_size - 1)) / KV_BLOCK) * kv_block_bytes(D);
        const int r = t % KV_BLOCK;
        const uint32_t kw = *reinterpret_cast<const uint32_t *>(p + kv_k_words(D) + 4 * r), vw = *reinterpret_cast<const uint32_t *>(p + kv_v_words(D) + 4 * r);
        float dot = 0.0f, x[V];
        for (int i = 0; i < V; ++i) {
            const int d = lane * V + i;
            const int ck = (p[r * (D / 2) + d / 2] >> (4 * (d & 1))) & 15, cv = (p[kv_v_codes(D) + r * (D / 2) + d / 2] >> (4 * (d & 1))) & 15;
            dot += q[i] * (__uint_as_float(kw & 0xffff0000u) + __uint_as_float(kw << 16) * ck);
            x[i] = __uint_as_float(vw & 0xffff0000u) + __uint_as_float(vw << 16) * cv;
        }
        for (int k = 16; k > 0; k >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, k);
        dot *= c.scale;
        const float m2 = fmaxf(m, dot), a = m == m2 ? 1.0f : __expf(m - m2), w = dot == m2 ? 1.0f : __expf(dot - m2);
        l = l * a + w;
        for (int i = 0; i < V; ++i) o[i] = o[i] * a + w * x[i];
        m = m2;
    }
    for (int i = 0; i < V; ++i)
        reinterpret_cast<__nv_bfloat16 *>(c.out)[row * c.out_stride + (int64_t)h * D + lane * V + i] = __float2bfloat16_rn(l > 0.0f || l != l ? o[i] / l : 0.0f);
}

}  // namespace

size_t kv_attention_workspace(int, int, int, int, int64_t, int64_t, int64_t) { return 0; }

cudaError_t kv_launch_attention(const kv_batch &b, int D, const kv_attention_call &c, int, cudaStream_t st, int64_t *launches)
{
    const int64_t blocks = (b.n_tokens * b.n_heads + 3) / 4;
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    auto go = [&](auto kern) { return tpq_launch_pdl(kern, dim3((unsigned)blocks), dim3(128), 0, st, b, c); };
    const cudaError_t e = D == 128 ? go(attention_rows<128>) : go(attention_rows<64>);
    if (e == cudaSuccess) ++*launches;
    return e;
}
