// Declarations shared by the kernels of the feed-forward block, 4-bit weights and answers (not installed).
#pragma once

#include "tpq_internal.h"

struct tpq_block {
    int device, sm_count;
    int clusters[9], clusters_half[9];  // clusters of 2 .. 8 blocks of the product kernels that run side by side: one block an SM, two
    int *status;  // device status word (0 = ok)
    int64_t launches;
    char err[512];
};

// Weights in 4 bits (layout in tpq.h): blocks of 128 outputs x 128 inputs, the outputs' factors behind them.
#define W4_TILE 128
#define W4_CODE_BYTES 8192
#define W4_MOST_INPUTS (INT64_C(1) << 17)
static inline int64_t w4_tiles(int64_t n) { return (n + W4_TILE - 1) / W4_TILE; }
#ifdef __CUDACC__
__host__ __device__
#endif
static inline int w4_block_bytes(int group) { return W4_CODE_BYTES + W4_TILE * (W4_TILE / group); }
static inline int64_t w4_factors_at(int64_t n, int64_t K, int group) { return w4_tiles(n) * w4_tiles(K) * w4_block_bytes(group); }
static inline int64_t w4_bytes(int64_t n, int64_t K, int group) { return w4_factors_at(n, K, group) + w4_tiles(n) * W4_TILE * 4; }

cudaError_t w4_prepare();
cudaError_t w4_launch_quantize(const uint16_t *w, int64_t stride, int64_t n, int64_t K, int group, uint8_t *w4, cudaStream_t st, int64_t *launches);
cudaError_t w4_launch_read(const uint8_t *w4, int64_t n, int64_t K, int group, uint16_t *out, int64_t stride, cudaStream_t st, int64_t *launches);

// x W^T (one weight), or act(x Wg^T) * (x Wu^T) (two)
struct product_call {
    const void *w[2];        // BF16: [n][K] with w_stride; 4 bits: blocks
    int64_t w_stride[2];
    int n_weights, group;    // group 0: BF16
    int64_t T, n, K;
    const void *x;
    int64_t x_stride;
    void *out;
    int64_t out_stride;
    int out_fp32, act;
};
cudaError_t product_prepare(tpq_block *b);
cudaError_t product_launch(const product_call &c, const tpq_block *b, cudaStream_t st, int64_t *launches);

// Answers
struct stats_call {
    const void *logits;
    int64_t stride, T;
    int fp32, n_vocab, first, n_top;
    const int32_t *tokens;
    uint32_t *records;
};
struct join_call {
    const uint32_t *records[TPQ_MAX_SHARDS];
    int n, n_top;
    int64_t T;
    float *logprob, *entropy, *top_logprob;
    int32_t *top;
};
cudaError_t answers_launch_stats(const stats_call &c, const tpq_block *b, cudaStream_t st, int64_t *launches);
cudaError_t answers_launch_join(const join_call &c, const tpq_block *b, cudaStream_t st, int64_t *launches);
