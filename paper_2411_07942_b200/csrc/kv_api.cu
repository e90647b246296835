// C entry points of the 4-bit key/value cache declared in tpq.h: handle, checks of arguments, launches.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>

#include "kv_internal.h"

namespace {

tpq_status fail(tpq_kv *kv, tpq_status st, const char *fmt, ...)
{
    if (kv) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(kv->err, sizeof kv->err, fmt, ap);
        va_end(ap);
    }
    return st;
}

// (the runtime's last error would otherwise be taken for the next launch's)
tpq_status cuda_fail(tpq_kv *kv, cudaError_t e, const char *what)
{
    (void)cudaGetLastError();
    return fail(kv, e == cudaErrorMemoryAllocation ? TPQ_ERR_NOMEM : TPQ_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// (a memset may still be under way when it returns, and a kernel on a stream that does not wait for it may have reported by then)
cudaError_t clear(int *word)
{
    const cudaError_t e = cudaMemset(word, 0, sizeof *word);
    return e == cudaSuccess ? cudaStreamSynchronize(nullptr) : e;
}

inline bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

tpq_status check_device(tpq_kv *kv)
{
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(kv, e, "cudaGetDevice");
    if (dev != kv->device) return fail(kv, TPQ_ERR_BAD_STATE, "the handle's device (%d) must be the current CUDA device (%d)", kv->device, dev);
    return TPQ_OK;
}

// Checks of a batch that need no device; nothing is left to do where *empty comes back true.
tpq_status check_batch(tpq_kv *kv, const tpq_kv_batch *a, kv_batch *b, bool *empty)
{
    kv->err[0] = 0;
    *empty = false;
    if (!a) return fail(kv, TPQ_ERR_INVALID_ARG, "batch is NULL");
    if (a->n_seqs < 0 || a->n_tokens < 0 || a->n_tokens > INT32_MAX || a->n_pages < 0 || a->page_table_stride < 0 || a->max_new < 0)
        return fail(kv, TPQ_ERR_INVALID_ARG, "negative or too large sizes: n_seqs %d, max_new %d, n_tokens %lld, n_pages %lld, page_table_stride %lld",
                    a->n_seqs, a->max_new, (long long)a->n_tokens, (long long)a->n_pages, (long long)a->page_table_stride);
    if (a->n_seqs == 0 || a->n_tokens == 0 || a->max_new == 0) {
        *empty = true;
        return TPQ_OK;
    }
    if (!a->cache_dev || !a->page_table_dev || !a->token_start_dev || !a->lengths_dev)
        return fail(kv, TPQ_ERR_INVALID_ARG, "NULL cache, page table, token starts or lengths");
    if (!aligned(a->cache_dev, 16)) return fail(kv, TPQ_ERR_ALIGN, "the cache must be 16-byte aligned");
    if (!aligned(a->page_table_dev, 4) || !aligned(a->token_start_dev, 4) || !aligned(a->lengths_dev, 4))
        return fail(kv, TPQ_ERR_ALIGN, "page table, token starts and lengths must be 4-byte aligned");
    if (a->n_pages > INT32_MAX || a->page_table_stride > INT32_MAX)
        return fail(kv, TPQ_ERR_INVALID_ARG, "n_pages or page_table_stride above 2^31 - 1");
    const tpq_status st = check_device(kv);
    if (st != TPQ_OK) return st;
    int shift = 0;
    while ((1 << shift) < kv->page_size) ++shift;
    *b = kv_batch{static_cast<uint8_t *>(a->cache_dev), a->page_table_dev, a->token_start_dev, a->lengths_dev, a->n_pages,
                  a->page_table_stride, a->n_tokens, a->n_seqs, a->max_new, kv->n_heads, kv->n_kv_heads, kv->page_size, shift, kv->status};
    return TPQ_OK;
}

tpq_status check_rows(tpq_kv *kv, const char *name, const void *p, int64_t stride, int heads)
{
    if (!p) return fail(kv, TPQ_ERR_INVALID_ARG, "%s is NULL", name);
    if (!aligned(p, 16)) return fail(kv, TPQ_ERR_ALIGN, "%s must be 16-byte aligned", name);
    if (stride < (int64_t)heads * kv->head_dim) return fail(kv, TPQ_ERR_INVALID_ARG, "row stride %lld of %s < %d", (long long)stride, name, heads * kv->head_dim);
    if (stride % 8 != 0) return fail(kv, TPQ_ERR_ALIGN, "row stride %lld of %s is not a multiple of 8 elements", (long long)stride, name);
    return TPQ_OK;
}

}  // namespace

extern "C" {

tpq_status tpq_kv_create(tpq_kv **out, int n_heads, int n_kv_heads, int head_dim, int page_size)
{
    if (!out) return TPQ_ERR_INVALID_ARG;
    *out = nullptr;
    if (n_kv_heads < 1 || n_heads < n_kv_heads || n_heads % n_kv_heads != 0 || n_heads / n_kv_heads > 256 || n_kv_heads > 4096)
        return TPQ_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return TPQ_ERR_INVALID_ARG;
    if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0) return TPQ_ERR_INVALID_ARG;
    tpq_kv *kv = new (std::nothrow) tpq_kv();
    if (!kv) return TPQ_ERR_NOMEM;
    kv->n_heads = n_heads;
    kv->n_kv_heads = n_kv_heads;
    kv->head_dim = head_dim;
    kv->page_size = page_size;
    cudaError_t e = cudaGetDevice(&kv->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kv->sm_count, cudaDevAttrMultiProcessorCount, kv->device);
    if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void **>(&kv->status), sizeof(int));
    if (e == cudaSuccess) {
        e = clear(kv->status);
        if (e != cudaSuccess) cudaFree(kv->status);
    }
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        delete kv;
        return e == cudaErrorMemoryAllocation ? TPQ_ERR_NOMEM : TPQ_ERR_CUDA;
    }
    *out = kv;
    return TPQ_OK;
}

tpq_status tpq_kv_destroy(tpq_kv *kv)
{
    if (!kv) return TPQ_OK;
    cudaFree(kv->status);
    delete kv;
    return TPQ_OK;
}

size_t tpq_kv_page_bytes(const tpq_kv *kv)
{
    return kv ? (size_t)kv->n_kv_heads * (kv->page_size / KV_BLOCK) * kv_block_bytes(kv->head_dim) : 0;
}

tpq_status tpq_kv_append(tpq_kv *kv, const tpq_kv_batch *batch, const tpq_kv_rotation *rot, const void *k, int64_t k_stride, const void *v,
                         int64_t v_stride, const void *q, int64_t q_stride, void *q_out, int64_t q_out_stride, void *stream)
{
    if (!kv) return TPQ_ERR_INVALID_ARG;
    kv_batch b;
    bool empty;
    tpq_status st = check_batch(kv, batch, &b, &empty);
    if (st != TPQ_OK || empty) return st;
    if ((st = check_rows(kv, "k", k, k_stride, kv->n_kv_heads)) != TPQ_OK) return st;
    if ((st = check_rows(kv, "v", v, v_stride, kv->n_kv_heads)) != TPQ_OK) return st;
    if (q) {
        if (!rot) return fail(kv, TPQ_ERR_INVALID_ARG, "q without a rotation");
        if ((st = check_rows(kv, "q", q, q_stride, kv->n_heads)) != TPQ_OK) return st;
        if ((st = check_rows(kv, "q_out", q_out, q_out_stride, kv->n_heads)) != TPQ_OK) return st;
        if (q == q_out && q_stride != q_out_stride) return fail(kv, TPQ_ERR_INVALID_ARG, "q_out is q with another row stride");
    } else if (q_out) {
        return fail(kv, TPQ_ERR_INVALID_ARG, "q_out without q");
    }
    if (rot) {
        if (!rot->table_dev) return fail(kv, TPQ_ERR_INVALID_ARG, "the rotation's table is NULL");
        if (rot->n_positions < 1) return fail(kv, TPQ_ERR_INVALID_ARG, "the rotation's table has %lld positions", (long long)rot->n_positions);
        if (rot->rot_dim < 16 || rot->rot_dim > kv->head_dim || rot->rot_dim % 16 != 0)
            return fail(kv, TPQ_ERR_INVALID_ARG, "rot_dim = %d is not a multiple of 16 in [16, %d]", rot->rot_dim, kv->head_dim);
        if (!aligned(rot->table_dev, 16)) return fail(kv, TPQ_ERR_ALIGN, "the rotation's table must be 16-byte aligned");
        if (!aligned(rot->positions_dev, 4)) return fail(kv, TPQ_ERR_ALIGN, "the rotation's positions must be 4-byte aligned");
    }
    cudaError_t e = kv_launch_append(b, kv->head_dim, rot, kv_rows{static_cast<const uint16_t *>(k), k_stride}, kv_rows{static_cast<const uint16_t *>(v), v_stride},
                                     kv_rows{static_cast<const uint16_t *>(q), q_stride}, static_cast<uint16_t *>(q_out), q_out_stride,
                                     kv->sm_count, static_cast<cudaStream_t>(stream), &kv->launches);
    if (e != cudaSuccess) return cuda_fail(kv, e, "kv_append kernel");
    return TPQ_OK;
}

tpq_status tpq_kv_read(tpq_kv *kv, const tpq_kv_batch *batch, void *k_out, int64_t k_stride, void *v_out, int64_t v_stride, void *stream)
{
    if (!kv) return TPQ_ERR_INVALID_ARG;
    kv_batch b;
    bool empty;
    tpq_status st = check_batch(kv, batch, &b, &empty);
    if (st != TPQ_OK || empty) return st;
    if (!k_out && !v_out) return fail(kv, TPQ_ERR_INVALID_ARG, "both outputs are NULL");
    if (k_out && (st = check_rows(kv, "k_out", k_out, k_stride, kv->n_kv_heads)) != TPQ_OK) return st;
    if (v_out && (st = check_rows(kv, "v_out", v_out, v_stride, kv->n_kv_heads)) != TPQ_OK) return st;
    if (k_out == v_out) return fail(kv, TPQ_ERR_INVALID_ARG, "k_out is v_out");
    cudaError_t e = kv_launch_read(b, kv->head_dim, static_cast<uint16_t *>(k_out), k_stride, static_cast<uint16_t *>(v_out), v_stride, kv->sm_count,
                                   static_cast<cudaStream_t>(stream), &kv->launches);
    if (e != cudaSuccess) return cuda_fail(kv, e, "kv_read kernel");
    return TPQ_OK;
}

size_t tpq_kv_attention_workspace(const tpq_kv *kv, int32_t n_seqs, int32_t max_new, int64_t n_tokens)
{
    if (!kv || n_seqs < 1 || max_new < 1 || n_tokens < 1) return 0;
    return kv_attention_workspace(kv->head_dim, kv->n_heads, kv->n_kv_heads, kv->sm_count, n_seqs, max_new, n_tokens);
}

tpq_status tpq_kv_attention(tpq_kv *kv, const tpq_kv_batch *batch, const void *q, int64_t q_stride, float scale, int64_t window, int64_t n_first,
                            void *out, int64_t out_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!kv) return TPQ_ERR_INVALID_ARG;
    kv_batch b;
    bool empty;
    tpq_status st = check_batch(kv, batch, &b, &empty);
    if (st != TPQ_OK) return st;
    if (!std::isfinite(scale)) return fail(kv, TPQ_ERR_INVALID_ARG, "scale is not finite");
    if (window < 0 || n_first < 0) return fail(kv, TPQ_ERR_INVALID_ARG, "negative window or n_first");
    if (empty) return TPQ_OK;
    if ((st = check_rows(kv, "q", q, q_stride, kv->n_heads)) != TPQ_OK) return st;
    if ((st = check_rows(kv, "out", out, out_stride, kv->n_heads)) != TPQ_OK) return st;
    if (q == out) return fail(kv, TPQ_ERR_INVALID_ARG, "out is q");
    if (batch->n_tokens * (kv->n_heads / kv->n_kv_heads) > KV_MOST)
        return fail(kv, TPQ_ERR_INVALID_ARG, "%lld rows of %d query heads per key head are more than 2^30", (long long)batch->n_tokens, kv->n_heads / kv->n_kv_heads);
    const size_t need = tpq_kv_attention_workspace(kv, batch->n_seqs, batch->max_new, batch->n_tokens);
    if (need && !workspace) return fail(kv, TPQ_ERR_INVALID_ARG, "workspace is NULL");
    if (!aligned(workspace, 16)) return fail(kv, TPQ_ERR_ALIGN, "the workspace must be 16-byte aligned");
    if (workspace_bytes < need) return fail(kv, TPQ_ERR_SIZE, "workspace of %zu bytes < %zu", workspace_bytes, need);
    const int64_t most = KV_MOST;  // (a window or prefix beyond any length is as good as this one)
    kv_attention_call c{kv_rows{static_cast<const uint16_t *>(q), q_stride}, static_cast<uint16_t *>(out), out_stride, scale,
                        (int)(window < most ? window : most), (int)(n_first < most ? n_first : most), workspace};
    cudaError_t e = kv_launch_attention(b, kv->head_dim, c, kv->sm_count, static_cast<cudaStream_t>(stream), &kv->launches);
    if (e != cudaSuccess) return cuda_fail(kv, e, "kv_attention kernel");
    return TPQ_OK;
}

tpq_status tpq_kv_device_status(tpq_kv *kv)
{
    if (!kv) return TPQ_ERR_INVALID_ARG;
    kv->err[0] = 0;
    const tpq_status st = check_device(kv);
    if (st != TPQ_OK) return st;
    int word = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(&word, kv->status, sizeof word, cudaMemcpyDeviceToHost);
    if (e == cudaSuccess && word != 0) e = clear(kv->status);
    if (e != cudaSuccess) return cuda_fail(kv, e, "device status");
    if (word != 0) return fail(kv, (tpq_status)word, "a kernel reported status %d", word);
    return TPQ_OK;
}

int64_t tpq_kv_launch_count(const tpq_kv *kv) { return kv ? kv->launches : 0; }

const char *tpq_kv_last_error(const tpq_kv *kv) { return kv ? kv->err : ""; }

}  // extern "C"
