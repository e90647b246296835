// Declarations shared by the kernels of the 4-bit key/value cache (not installed).
#pragma once

#include "tpq_internal.h"

#define KV_BLOCK 16  // positions of a block of the cache
#define KV_MOST (1 << 30)  // positions of a sequence
#define KV_MOST_UNITS (INT32_MAX - 1024)  // tiles that an attention call deals out (numbers of them are held in 32 bits; the sum is not)

struct tpq_kv {
    int n_heads, n_kv_heads, head_dim, page_size;
    int device, sm_count;
    int *status;  // device status word (0 = ok)
    int64_t launches;
    char err[512];
};

// A batch as the kernels see it.
struct kv_batch {
    uint8_t *cache;
    const int32_t *table, *start, *lengths;
    int64_t n_pages, table_stride, n_tokens;
    int n_seqs, max_new;
    int n_heads, n_kv_heads;
    int page_size, page_shift;  // page_size = 1 << page_shift
    int *status;
};

struct kv_rows {  // BF16 rows and their stride in elements
    const uint16_t *p;
    int64_t stride;
};

cudaError_t kv_launch_append(const kv_batch &b, int D, const tpq_kv_rotation *rot, kv_rows k, kv_rows v, kv_rows q, uint16_t *q_out,
                             int64_t q_out_stride, int sm_count, cudaStream_t st, int64_t *launches);
cudaError_t kv_launch_read(const kv_batch &b, int D, uint16_t *k_out, int64_t k_stride, uint16_t *v_out, int64_t v_stride,
                           int sm_count, cudaStream_t st, int64_t *launches);

struct kv_attention_call {
    kv_rows q;
    uint16_t *out;
    int64_t out_stride;
    float scale;
    int window, n_first;  // at most KV_MOST; window 0: none
    void *workspace;
};
size_t kv_attention_workspace(int D, int n_heads, int n_kv_heads, int sm_count, int64_t n_seqs, int64_t max_new, int64_t n_tokens);
cudaError_t kv_launch_attention(const kv_batch &b, int D, const kv_attention_call &c, int sm_count, cudaStream_t st, int64_t *launches);
// Sequences with more than `few` rows (new positions x query heads of a key head); kv_launch_attention calls it.
size_t kv_prompt_workspace(int D, int group, int sm_count, int64_t n_seqs, int64_t n_tokens);
cudaError_t kv_launch_prompt(const kv_batch &b, int D, const kv_attention_call &c, int few, void *workspace, int sm_count, cudaStream_t st,
                             int64_t *launches);

#ifdef __CUDACC__
__host__ __device__ constexpr int kv_block_bytes(int D) { return KV_BLOCK * (D + 8); }
// byte offsets inside a block
__host__ __device__ constexpr int kv_v_codes(int D) { return KV_BLOCK * D / 2; }
__host__ __device__ constexpr int kv_k_words(int D) { return KV_BLOCK * D; }
__host__ __device__ constexpr int kv_v_words(int D) { return KV_BLOCK * D + 4 * KV_BLOCK; }

__device__ __forceinline__ void kv_report(const kv_batch &b) { atomicExch(b.status, (int)TPQ_ERR_INVALID_ARG); }

// A sequence's first row, number of rows and length; n = -1 (and the status word set) if they contradict each other or the batch.
struct kv_seq {
    int start, n, len;
};
__device__ __forceinline__ kv_seq kv_load_seq(const kv_batch &b, int s)
{
    kv_seq q;
    q.start = b.start[s];
    q.n = b.start[s + 1];
    q.len = b.lengths[s];
    const bool ok = q.start >= 0 && q.start <= q.n && q.n <= b.n_tokens && q.n - q.start <= b.max_new && q.n - q.start <= q.len &&
                    q.len <= b.table_stride * (int64_t)b.page_size && q.len <= KV_MOST;
    q.n -= q.start;
    if (!ok) {
        kv_report(b);
        q.n = -1;
    }
    return q;
}

// The last sequence that starts at or before `row`, by a whole warp (-1 if there is none): 32 probes a round.
__device__ __forceinline__ int kv_find_seq(const kv_batch &b, int64_t row, int lane)
{
    int lo = 0, n = b.n_seqs;  // the answer is in [lo - 1, lo + n - 1]
    while (n > 0) {
        const int step = (n + 31) / 32;  // probes at lo + step - 1, lo + 2 step - 1, ..., the last one at lo + n - 1
        const int at = (lane + 1) * step - 1 < n ? (lane + 1) * step - 1 : n - 1;
        const unsigned below = __ballot_sync(0xffffffffu, b.start[lo + at] <= row);
        const int c = __popc(below);  // ascending starts: the probes at or before the row are the first c
        const int skip = c * step < n ? c * step : n;
        lo += skip;
        n = c == 32 ? 0 : (n - skip < step - 1 ? n - skip : step - 1);
    }
    return lo - 1;
}
// Whether the sequence that kv_find_seq gave for a row has it.  Where starts do not ascend, that may be one that begins behind it.
__device__ __forceinline__ bool kv_owns(const kv_batch &b, const kv_seq &q, int64_t row)
{
    if (row < q.start) kv_report(b);
    return row >= q.start && row < q.start + q.n;
}
#endif
