// C entry points of the feed-forward block, 4-bit weights and answers declared in tpq.h: handle, checks of arguments, launches.
#include <cstdarg>
#include <cstdio>
#include <new>

#include "block_internal.h"

namespace {

tpq_status fail(tpq_block *b, tpq_status st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(b->err, sizeof b->err, fmt, ap);
    va_end(ap);
    return st;
}

// (the runtime's last error would otherwise be taken for the next launch's)
tpq_status cuda_fail(tpq_block *b, cudaError_t e, const char *what)
{
    (void)cudaGetLastError();
    return fail(b, e == cudaErrorMemoryAllocation ? TPQ_ERR_NOMEM : TPQ_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// (a memset may still be under way when it returns, and a kernel on a stream that does not wait for it may have reported by then)
cudaError_t clear(int *word)
{
    const cudaError_t e = cudaMemset(word, 0, sizeof *word);
    return e == cudaSuccess ? cudaStreamSynchronize(nullptr) : e;
}

inline bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

tpq_status check_device(tpq_block *b)
{
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(b, e, "cudaGetDevice");
    if (dev != b->device) return fail(b, TPQ_ERR_BAD_STATE, "the handle's device (%d) must be the current CUDA device (%d)", b->device, dev);
    return TPQ_OK;
}

constexpr int64_t MOST_OUTPUTS = INT64_C(1) << 30, MOST_INPUTS = W4_MOST_INPUTS, MOST_ROWS = INT64_C(1) << 30;

bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
bool shape_ok(int64_t n, int64_t K) { return n >= 1 && n <= MOST_OUTPUTS && K >= 1 && K <= MOST_INPUTS; }

tpq_status check_shape(tpq_block *b, int64_t n, int64_t K, int group)
{
    b->err[0] = 0;
    if (!shape_ok(n, K)) return fail(b, TPQ_ERR_INVALID_ARG, "%lld outputs of %lld inputs: 1 to 2^30 and 1 to 2^17 are possible", (long long)n, (long long)K);
    if (!group_ok(group)) return fail(b, TPQ_ERR_INVALID_ARG, "group = %d is not 32, 64 or 128", group);
    return TPQ_OK;
}

tpq_status check_weight(tpq_block *b, const char *name, const tpq_weight *w)
{
    if (!w) return fail(b, TPQ_ERR_INVALID_ARG, "%s is NULL", name);
    if (w->kind != TPQ_WEIGHT_BF16 && w->kind != TPQ_WEIGHT_INT4) return fail(b, TPQ_ERR_INVALID_ARG, "kind %d of %s", (int)w->kind, name);
    if (!shape_ok(w->n_out, w->n_in))
        return fail(b, TPQ_ERR_INVALID_ARG, "%s: %lld outputs of %lld inputs: 1 to 2^30 and 1 to 2^17 are possible", name, (long long)w->n_out, (long long)w->n_in);
    if (!w->data_dev) return fail(b, TPQ_ERR_INVALID_ARG, "%s has no data", name);
    if (!aligned(w->data_dev, 16)) return fail(b, TPQ_ERR_ALIGN, "%s must be 16-byte aligned", name);
    if (w->kind == TPQ_WEIGHT_INT4) {
        if (!group_ok(w->group)) return fail(b, TPQ_ERR_INVALID_ARG, "%s: group = %d is not 32, 64 or 128", name, w->group);
    } else {
        if (w->row_stride < w->n_in) return fail(b, TPQ_ERR_INVALID_ARG, "row stride %lld of %s < %lld", (long long)w->row_stride, name, (long long)w->n_in);
        if (w->row_stride > (INT64_C(1) << 38)) return fail(b, TPQ_ERR_INVALID_ARG, "row stride %lld of %s is above 2^38", (long long)w->row_stride, name);
        if (w->row_stride % 8) return fail(b, TPQ_ERR_ALIGN, "row stride %lld of %s is not a multiple of 8 elements", (long long)w->row_stride, name);
    }
    return TPQ_OK;
}

// Checks of the rows of a product, and the call's part of them.
tpq_status check_rows(tpq_block *b, product_call *c, int64_t n, int64_t K, const void *x, int64_t x_stride, int64_t T, void *out, int out_bytes, int64_t out_stride)
{
    if (T < 0 || T > MOST_ROWS) return fail(b, TPQ_ERR_INVALID_ARG, "T = %lld", (long long)T);
    if (((T + 15) / 16) * ((n + 127) / 128) > INT32_MAX / 2) return fail(b, TPQ_ERR_INVALID_ARG, "%lld rows of %lld outputs are too many", (long long)T, (long long)n);
    if (T == 0) return TPQ_OK;
    if (!x || !out) return fail(b, TPQ_ERR_INVALID_ARG, "x or out is NULL");
    if (x == out) return fail(b, TPQ_ERR_INVALID_ARG, "out is x");
    if (!aligned(x, 16)) return fail(b, TPQ_ERR_ALIGN, "x must be 16-byte aligned");
    if (!aligned(out, out_bytes)) return fail(b, TPQ_ERR_ALIGN, "out must be %d-byte aligned", out_bytes);
    if (x_stride < K) return fail(b, TPQ_ERR_INVALID_ARG, "row stride %lld of x < %lld", (long long)x_stride, (long long)K);
    if (x_stride % 8) return fail(b, TPQ_ERR_ALIGN, "row stride %lld of x is not a multiple of 8 elements", (long long)x_stride);
    if (out_stride < n) return fail(b, TPQ_ERR_INVALID_ARG, "row stride %lld of out < %lld", (long long)out_stride, (long long)n);
    if (x_stride > (INT64_C(1) << 38) || out_stride > (INT64_C(1) << 38)) return fail(b, TPQ_ERR_INVALID_ARG, "a row stride is above 2^38");
    c->T = T;
    c->n = n;
    c->K = K;
    c->x = x;
    c->x_stride = x_stride;
    c->out = out;
    c->out_stride = out_stride;
    return check_device(b);
}

tpq_status check_top(tpq_block *b, int64_t T, int n_top)
{
    b->err[0] = 0;
    if (T < 0 || T > (INT64_C(1) << 27)) return fail(b, TPQ_ERR_INVALID_ARG, "T = %lld is not in [0, 2^27]", (long long)T);
    if (n_top < 0 || n_top > 32) return fail(b, TPQ_ERR_INVALID_ARG, "n_top = %d is not in [0, 32]", n_top);
    return TPQ_OK;
}

}  // namespace

extern "C" {

tpq_status tpq_block_create(tpq_block **out)
{
    if (!out) return TPQ_ERR_INVALID_ARG;
    *out = nullptr;
    tpq_block *b = new (std::nothrow) tpq_block();
    if (!b) return TPQ_ERR_NOMEM;
    cudaError_t e = cudaGetDevice(&b->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&b->sm_count, cudaDevAttrMultiProcessorCount, b->device);
    if (e == cudaSuccess) e = product_prepare(b);
    if (e == cudaSuccess) e = w4_prepare();
    if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void **>(&b->status), sizeof(int));
    if (e == cudaSuccess) {
        e = clear(b->status);
        if (e != cudaSuccess) cudaFree(b->status);
    }
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        delete b;
        return e == cudaErrorMemoryAllocation ? TPQ_ERR_NOMEM : TPQ_ERR_CUDA;
    }
    *out = b;
    return TPQ_OK;
}

tpq_status tpq_block_destroy(tpq_block *b)
{
    if (!b) return TPQ_OK;
    cudaFree(b->status);
    delete b;
    return TPQ_OK;
}

size_t tpq_weight4_bytes(int64_t n_out, int64_t n_in, int group) { return shape_ok(n_out, n_in) && group_ok(group) ? (size_t)w4_bytes(n_out, n_in, group) : 0; }

tpq_status tpq_quantize_weight(tpq_block *b, const void *w, int64_t row_stride, int64_t n_out, int64_t n_in, int group, void *w4, size_t capacity, void *stream)
{
    if (!b) return TPQ_ERR_INVALID_ARG;
    tpq_status st = check_shape(b, n_out, n_in, group);
    if (st != TPQ_OK) return st;
    if (!w || !w4) return fail(b, TPQ_ERR_INVALID_ARG, "w or w4 is NULL");
    if (row_stride < n_in) return fail(b, TPQ_ERR_INVALID_ARG, "row stride %lld < %lld", (long long)row_stride, (long long)n_in);
    if (!aligned(w, 2)) return fail(b, TPQ_ERR_ALIGN, "w must be 2-byte aligned");
    if (!aligned(w4, 16)) return fail(b, TPQ_ERR_ALIGN, "w4 must be 16-byte aligned");
    if (capacity < tpq_weight4_bytes(n_out, n_in, group))
        return fail(b, TPQ_ERR_SIZE, "w4 of %zu bytes < %zu", capacity, tpq_weight4_bytes(n_out, n_in, group));
    if ((st = check_device(b)) != TPQ_OK) return st;
    const cudaError_t e = w4_launch_quantize(static_cast<const uint16_t *>(w), row_stride, n_out, n_in, group, static_cast<uint8_t *>(w4),
                                             static_cast<cudaStream_t>(stream), &b->launches);
    return e == cudaSuccess ? TPQ_OK : cuda_fail(b, e, "quantize_weight kernel");
}

tpq_status tpq_read_weight(tpq_block *b, const void *w4, int64_t n_out, int64_t n_in, int group, void *out, int64_t out_row_stride, void *stream)
{
    if (!b) return TPQ_ERR_INVALID_ARG;
    tpq_status st = check_shape(b, n_out, n_in, group);
    if (st != TPQ_OK) return st;
    if (!w4 || !out) return fail(b, TPQ_ERR_INVALID_ARG, "w4 or out is NULL");
    if (out_row_stride < n_in) return fail(b, TPQ_ERR_INVALID_ARG, "row stride %lld < %lld", (long long)out_row_stride, (long long)n_in);
    if (!aligned(out, 2)) return fail(b, TPQ_ERR_ALIGN, "out must be 2-byte aligned");
    if (!aligned(w4, 16)) return fail(b, TPQ_ERR_ALIGN, "w4 must be 16-byte aligned");
    if ((st = check_device(b)) != TPQ_OK) return st;
    const cudaError_t e = w4_launch_read(static_cast<const uint8_t *>(w4), n_out, n_in, group, static_cast<uint16_t *>(out), out_row_stride,
                                         static_cast<cudaStream_t>(stream), &b->launches);
    return e == cudaSuccess ? TPQ_OK : cuda_fail(b, e, "read_weight kernel");
}

tpq_status tpq_linear4(tpq_block *b, const tpq_weight *w, const void *x, int64_t x_stride, int64_t T, void *out, tpq_out_dtype dt, int64_t out_stride, void *stream)
{
    if (!b) return TPQ_ERR_INVALID_ARG;
    b->err[0] = 0;
    tpq_status st = check_weight(b, "w", w);
    if (st != TPQ_OK) return st;
    if (w->kind != TPQ_WEIGHT_INT4) return fail(b, TPQ_ERR_INVALID_ARG, "w is not in 4 bits");
    if (dt != TPQ_OUT_BF16 && dt != TPQ_OUT_FP32) return fail(b, TPQ_ERR_INVALID_ARG, "output type %d", (int)dt);
    product_call c = {};
    if ((st = check_rows(b, &c, w->n_out, w->n_in, x, x_stride, T, out, dt == TPQ_OUT_FP32 ? 4 : 2, out_stride)) != TPQ_OK || T == 0) return st;
    c.w[0] = w->data_dev;
    c.n_weights = 1;
    c.group = w->group;
    c.out_fp32 = dt == TPQ_OUT_FP32;
    const cudaError_t e = product_launch(c, b, static_cast<cudaStream_t>(stream), &b->launches);
    return e == cudaSuccess ? TPQ_OK : cuda_fail(b, e, "product kernel");
}

tpq_status tpq_gated(tpq_block *b, const tpq_weight *gate, const tpq_weight *up, tpq_activation act, const void *x, int64_t x_stride, int64_t T, void *out,
                     int64_t out_stride, void *stream)
{
    if (!b) return TPQ_ERR_INVALID_ARG;
    b->err[0] = 0;
    tpq_status st = check_weight(b, "gate", gate);
    if (st != TPQ_OK || (st = check_weight(b, "up", up)) != TPQ_OK) return st;
    if (gate->kind != up->kind || gate->n_out != up->n_out || gate->n_in != up->n_in || (gate->kind == TPQ_WEIGHT_INT4 && gate->group != up->group))
        return fail(b, TPQ_ERR_INVALID_ARG, "gate and up differ in kind, size or group");
    if (act != TPQ_ACT_SILU && act != TPQ_ACT_GELU_TANH && act != TPQ_ACT_GELU_ERF) return fail(b, TPQ_ERR_INVALID_ARG, "activation %d", (int)act);
    product_call c = {};
    if ((st = check_rows(b, &c, gate->n_out, gate->n_in, x, x_stride, T, out, 2, out_stride)) != TPQ_OK || T == 0) return st;
    c.w[0] = gate->data_dev;
    c.w[1] = up->data_dev;
    c.w_stride[0] = gate->row_stride;
    c.w_stride[1] = up->row_stride;
    c.n_weights = 2;
    c.group = gate->kind == TPQ_WEIGHT_INT4 ? gate->group : 0;
    c.act = act;
    const cudaError_t e = product_launch(c, b, static_cast<cudaStream_t>(stream), &b->launches);
    return e == cudaSuccess ? TPQ_OK : cuda_fail(b, e, "product kernel");
}

size_t tpq_token_record_bytes(int64_t T, int n_top) { return T < 0 || T > (INT64_C(1) << 27) || n_top < 0 || n_top > 32 ? 0 : (size_t)T * 4 * (5 + 2 * n_top); }

tpq_status tpq_token_stats(tpq_block *b, const void *logits, tpq_out_dtype dt, int64_t row_stride, int64_t T, int64_t n_vocab, int64_t first, const int32_t *tokens,
                           int n_top, void *records, size_t capacity, void *stream)
{
    if (!b) return TPQ_ERR_INVALID_ARG;
    tpq_status st = check_top(b, T, n_top);
    if (st != TPQ_OK) return st;
    if (dt != TPQ_OUT_BF16 && dt != TPQ_OUT_FP32) return fail(b, TPQ_ERR_INVALID_ARG, "logits of type %d", (int)dt);
    if (n_vocab < 1 || n_vocab > (INT64_C(1) << 30) || first < 0 || first > INT32_MAX - n_vocab)
        return fail(b, TPQ_ERR_INVALID_ARG, "columns %lld .. + %lld: 1 to 2^30 of them, numbers below 2^31", (long long)first, (long long)n_vocab);
    if (row_stride < n_vocab) return fail(b, TPQ_ERR_INVALID_ARG, "row stride %lld < %lld", (long long)row_stride, (long long)n_vocab);
    if (T == 0) return TPQ_OK;
    if (!logits || !records) return fail(b, TPQ_ERR_INVALID_ARG, "logits or records is NULL");
    if (!aligned(logits, dt == TPQ_OUT_FP32 ? 4 : 2)) return fail(b, TPQ_ERR_ALIGN, "logits must be aligned to their values");
    if (!aligned(records, 4) || !aligned(tokens, 4)) return fail(b, TPQ_ERR_ALIGN, "records and tokens must be 4-byte aligned");
    if (capacity < tpq_token_record_bytes(T, n_top)) return fail(b, TPQ_ERR_SIZE, "records of %zu bytes < %zu", capacity, tpq_token_record_bytes(T, n_top));
    if ((st = check_device(b)) != TPQ_OK) return st;
    const stats_call c = {logits, row_stride, T, dt == TPQ_OUT_FP32, (int)n_vocab, (int)first, n_top, tokens, static_cast<uint32_t *>(records)};
    const cudaError_t e = answers_launch_stats(c, b, static_cast<cudaStream_t>(stream), &b->launches);
    return e == cudaSuccess ? TPQ_OK : cuda_fail(b, e, "token_stats kernel");
}

tpq_status tpq_token_logprobs(tpq_block *b, const void *const *records, int n, int64_t T, float *logprob, float *entropy, int n_top, int32_t *top, float *top_logprob,
                              void *stream)
{
    if (!b) return TPQ_ERR_INVALID_ARG;
    tpq_status st = check_top(b, T, n_top);
    if (st != TPQ_OK) return st;
    if (n < 1 || n > TPQ_MAX_SHARDS) return fail(b, TPQ_ERR_INVALID_ARG, "%d records are not 1 to %d", n, TPQ_MAX_SHARDS);
    if (!records) return fail(b, TPQ_ERR_INVALID_ARG, "records is NULL");
    if ((top || top_logprob) && n_top == 0) return fail(b, TPQ_ERR_INVALID_ARG, "alternatives without n_top");
    if (!logprob && !entropy && !top && !top_logprob) return fail(b, TPQ_ERR_INVALID_ARG, "all outputs are NULL");
    if (T == 0) return TPQ_OK;
    join_call c = {};
    for (int i = 0; i < n; ++i) {
        if (!records[i]) return fail(b, TPQ_ERR_INVALID_ARG, "record %d is NULL", i);
        if (!aligned(records[i], 4)) return fail(b, TPQ_ERR_ALIGN, "records must be 4-byte aligned");
        c.records[i] = static_cast<const uint32_t *>(records[i]);
    }
    if (!aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(top, 4) || !aligned(top_logprob, 4)) return fail(b, TPQ_ERR_ALIGN, "outputs must be 4-byte aligned");
    if ((st = check_device(b)) != TPQ_OK) return st;
    c.n = n;
    c.n_top = n_top;
    c.T = T;
    c.logprob = logprob;
    c.entropy = entropy;
    c.top = top;
    c.top_logprob = top_logprob;
    const cudaError_t e = answers_launch_join(c, b, static_cast<cudaStream_t>(stream), &b->launches);
    return e == cudaSuccess ? TPQ_OK : cuda_fail(b, e, "token_logprobs kernel");
}

tpq_status tpq_block_device_status(tpq_block *b)
{
    if (!b) return TPQ_ERR_INVALID_ARG;
    b->err[0] = 0;
    const tpq_status st = check_device(b);
    if (st != TPQ_OK) return st;
    int word = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(&word, b->status, sizeof word, cudaMemcpyDeviceToHost);
    if (e == cudaSuccess && word != 0) e = clear(b->status);
    if (e != cudaSuccess) return cuda_fail(b, e, "device status");
    if (word != 0) return fail(b, (tpq_status)word, "a kernel reported status %d", word);
    return TPQ_OK;
}

int64_t tpq_block_launch_count(const tpq_block *b) { return b ? b->launches : 0; }

const char *tpq_block_last_error(const tpq_block *b) { return b ? b->err : ""; }

}  // extern "C"
