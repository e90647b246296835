/*
 * tpq.h -- C ABI of libtpq: low-bit synchronisation of tensor-parallel partial
 * sums on NVIDIA B200 (sm_100a), after "Towards Low-bit Communication for
 * Tensor Parallel LLM Inference" (arXiv 2411.07942).
 *
 * Setting (paper Section 2): N devices each hold a partial sum
 * f^(i)(x^(i)) in R^E per token; the synchronised value is their sum.  The
 * library provides the per-device compression C^(i) (tpq_quantize_pack), the
 * decompress-and-sum  sum_i D^(i)  (tpq_dequant_reduce), and the calibration
 * that fixes their static parameters (tpq_calibrate_ranges,
 * tpq_select_features), paper Section 3.
 *
 * Conventions for every entry point
 *   - "dev" pointers are CUDA device pointers, "host" pointers are host memory.
 *   - BF16 tensors are 16-bit patterns, row-major, row stride given in ELEMENTS
 *     (any stride >= E; the Int4 kernels need E, k and the strides to be
 *     multiples of 8, other shapes run on the bit-stream and group kernels,
 *     and very small ones on shape-generic kernels).
 *   - The caller owns every data buffer.  The library owns only the context
 *     and its small device tables (O(N*E) floats), released by tpq_destroy.
 *   - Calls that take a `cuda_stream` (a cudaStream_t passed as void*; NULL is
 *     the default stream) only ENQUEUE work on it and never synchronise.  Calls
 *     that return host data synchronise the device.
 *   - Arguments are validated before anything is launched; a non-zero status
 *     means nothing was enqueued.  No entry point throws, aborts or traps.
 *   - A context is bound to the CUDA device that was current at tpq_create and
 *     may be used from one host thread at a time.  Work enqueued through one
 *     context must not overlap on the GPU with itself: use one stream, or
 *     streams ordered by events (the kernels share the context's status word,
 *     the calibration scratch and the block counter of tpq_quantize_pack_push).
 *   - One context serves all N simulated devices: the static parameters and
 *     the selected feature set are identical on every device by construction
 *     (Section 3: the set is static and shared by every sequence and device).
 */
#ifndef TPQ_H
#define TPQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tpq_ctx tpq_ctx; /* opaque */

typedef enum {
    TPQ_OK = 0,
    TPQ_ERR_INVALID_ARG = 1, /* null pointer, negative size, shard out of range, unsorted index set ... */
    TPQ_ERR_BAD_STATE = 2,   /* e.g. quantize before a feature set exists, select before calibration */
    TPQ_ERR_SIZE = 3,        /* a caller buffer is too small */
    TPQ_ERR_ALIGN = 4,       /* a device pointer is not 16-byte aligned */
    TPQ_ERR_CUDA = 5,        /* a CUDA call failed; text in tpq_last_error */
    TPQ_ERR_NOMEM = 6,       /* host or device allocation failed */
    TPQ_ERR_TIMEOUT = 7      /* a bounded device-side wait gave up (see tpq_device_status) */
} tpq_status;

typedef enum { TPQ_OUT_BF16 = 0, TPQ_OUT_FP32 = 1 } tpq_out_dtype;

/* Options for tpq_set_option. */
typedef enum {
    /* 0 = automatic (default); 1 = always the shape-generic kernels; 2 = never those: the kernels
     * for E, k and strides that are multiples of 8, whatever the size (the Int4 kernels; at other
     * code widths the bit-stream or group kernels, chosen as by 0), TPQ_ERR_INVALID_ARG from the
     * call if the shape does not admit them. */
    TPQ_OPT_KERNEL_PATH = 0,
    /* Which tiled kernel tpq_dequant_reduce uses when the tiled path is taken: 0 = chosen from the
     * shape (default); 1 = row kernel (needs N <= 4 and (E-k)/8 <= 768, or N <= 8 and (E-k)/8 <= 640); 2 = tensor-map panel kernel
     * (needs N <= 16 and at least as many rows as it takes for the code stream to be 16-byte aligned again:
     * 1, 2 or 4); 3 = copy-ring panel kernel.  A kernel that the shape
     * does not admit makes the call return TPQ_ERR_INVALID_ARG.  For tests and measurements: all
     * kernels give identical results. */
    TPQ_OPT_DEQUANT_KERNEL = 1
} tpq_option;

/* Bytes a real exchange would move per synchronisation and per device
 * (paper Section 5: all-reduce executed as all-gather + local reduction). */
typedef struct tpq_comm_report {
    int64_t payload_bytes;             /* P: one device's payload for T tokens                         */
    int64_t quantized_allgather_send;  /* (N-1) * P, unicast all-gather of payloads (the method)        */
    int64_t bf16_allgather_send;       /* (N-1) * 2*T*E, all-gather of the raw BF16 partial sums         */
    int64_t bf16_ring_allreduce_send;  /* 2*(N-1)/N * 2*T*E, bandwidth-optimal BF16 all-reduce           */
    double bits_per_value;             /* 8*P / (T*E); equals b + (16-b)k/E up to the 16-byte pad (Sec. 4) */
    double bits_per_value_formula;     /* b + (16-b)k/E for b-bit codes: 4 + 12k/E for the paper's Int4   */
} tpq_comm_report;

/* ---------------------------------------------------------------- context */

/* Create a context for n_shards (N >= 1) devices and n_features (E >= 1)
 * features on the current CUDA device.  bits is the code width: 4 is the
 * paper's Int4 (Section 3) and the width the tiled kernels serve; 2..8 are
 * accepted (other code widths, as evaluated in Section 4 / Figure 3:
 * step R/(2^bits - 1), codes -2^(bits-1) .. 2^(bits-1)-1, one little-endian
 * stream of bits-wide codes) and run on the bit-stream or group kernels.  gamma is
 * the moving-average constant of Eq. (1)-(2) (the paper uses 0.01),
 * 0 <= gamma <= 1.  Errors: INVALID_ARG, NOMEM, CUDA. */
tpq_status tpq_create(tpq_ctx **ctx, int n_shards, int n_features, int bits, float gamma);
tpq_status tpq_destroy(tpq_ctx *ctx); /* NULL is accepted */
tpq_status tpq_set_option(tpq_ctx *ctx, tpq_option opt, int value);

/* ------------------------------------------------------------ calibration */

/* Section 3 "Calibration", Eq. (1)-(2): fold n_seq sequences of device `shard`
 * into its running (m_j, M_j), in index order.  For every sequence the
 * column-wise minimum and maximum over its S tokens are taken; the first
 * sequence a device ever sees initialises (m, M), later ones update
 *   m <- (1-gamma) m + gamma min,  M <- (1-gamma) M + gamma max
 * in binary32, evaluated left to right.
 *   y_bf16_dev : [n_seq][S][E] BF16, row stride row_stride_elems (>= E), the
 *                sequences back to back (sequence q starts at row q*S).
 * Enqueues on cuda_stream.  May grow a context-owned scratch buffer
 * (cudaMalloc) when n_seq*S exceeds every earlier call, or when there are more
 * sequences than it has room for (4 * n_seq * E bytes).
 * n_seq == 0 is a no-op.  Errors: INVALID_ARG, ALIGN, NOMEM, CUDA. */
tpq_status tpq_calibrate_ranges(tpq_ctx *ctx, int shard, const void *y_bf16_dev, int64_t n_seq, int64_t S,
                                int64_t row_stride_elems, void *cuda_stream);

/* The same fold as tpq_calibrate_ranges, for callers that must not allocate.  (The paper has no
 * counterpart: this is a deployment variant of the call above.)  tpq_calibrate_ranges may grow its
 * scratch buffer with cudaMalloc / cudaFree, which a caller cannot afford when it runs inside a
 * serving loop whose device memory is owned by a pool, under a framework that forbids allocation
 * outside start-up, or at a point where the implicit device synchronisation of cudaFree would stall
 * other streams.  This variant keeps the per-sequence column extremes in a fixed array that is part
 * of the library image: TPQ_NOALLOC_SCRATCH_MAX_BYTES (4 MiB) of global memory on every device that
 * loads the library, held until the process exits.  It calls no cudaMalloc, no cudaFree and no
 * allocating library routine.
 *   Limit: 4 * n_seq * E bytes must fit the array, i.e. n_seq * E <= 1 048 576 (e.g. 204 sequences at
 *   E = 5120) and n_seq <= 65535; larger calls return TPQ_ERR_SIZE and enqueue nothing: fold fewer
 *   sequences per call (the result does not depend on how the sequences are split over calls).
 *   The first call on a device looks up the array's device address (cudaGetSymbolAddress); make that
 *   first call before any stream capture begins.  The device the context was created on must be current.
 *   All calls, from every context, share the one array per device: two calls whose kernels can overlap
 *   on the GPU (different streams) race on it; serialise them on one stream or with events.  Nothing
 *   in the array has to be cleared between calls: every element a call reads it has written first.
 * Same arguments, results and errors as tpq_calibrate_ranges otherwise. */
#define TPQ_NOALLOC_SCRATCH_MAX_BYTES (4u << 20)
tpq_status tpq_calibrate_ranges_noalloc(tpq_ctx *ctx, int shard, const void *y_bf16_dev, int64_t n_seq, int64_t S,
                                        int64_t row_stride_elems, void *cuda_stream);

/* Section 3 "Selecting High Precision Features": R^(i)_j = 2 max(-m, M),
 * aggregated range Rbar_j = sum_i R^(i)_j (binary32, devices ascending), the
 * k features with the largest Rbar_j (ties: lower index; a NaN ranks above
 * every number) become the BF16 set;
 * every other feature gets its static Int4 step s = R/15 (floored at 2^-23)
 * and reciprocal.  k < 0 selects the paper's k = floor(E/64) (Section 4).
 * Every device must have been calibrated with at least one sequence
 * (else BAD_STATE).  Writes the k indices, ascending, to hp_idx_out_host
 * (capacity >= k int32; may be NULL) and k to k_out (may be NULL).
 * Synchronises the device. */
tpq_status tpq_select_features(tpq_ctx *ctx, int k, int32_t *hp_idx_out_host, int *k_out);

/* Install an arbitrary feature set (strictly ascending indices in [0, E),
 * 0 <= k <= E) instead of the top-k one: the paper's "Int4" (k = 0) and
 * "Int4 + Random BF16" baselines (Section 4), or a restored set.  Steps are
 * derived from the calibrated ranges as in tpq_select_features.  Synchronises. */
tpq_status tpq_set_features(tpq_ctx *ctx, const int32_t *hp_idx_host, int k);

/* Install calibration state directly: m and M are [N][E] binary32 (host),
 * counts[N] the number of sequences each device has folded.  Used to resume
 * calibration or to skip it.  Synchronises. */
tpq_status tpq_set_ranges(tpq_ctx *ctx, const float *m_host, const float *M_host, const int64_t *counts_host);

/* Read back state (host outputs, any may be NULL; synchronises):
 * m, M, R are [N][E]; Rbar is [E].  R and Rbar are valid after a feature set exists. */
tpq_status tpq_get_ranges(tpq_ctx *ctx, float *m_host, float *M_host, float *R_host, float *Rbar_host);
/* s and inv_s are [N][E] (entries at selected features are defined but unused). BAD_STATE before a feature set. */
tpq_status tpq_get_scales(tpq_ctx *ctx, float *s_host, float *inv_s_host);
/* Number of selected features, or -1 before a feature set exists. */
int tpq_num_selected(const tpq_ctx *ctx);
/* The selected indices, ascending (capacity >= k).  BAD_STATE before a feature set. */
tpq_status tpq_get_features(tpq_ctx *ctx, int32_t *hp_idx_out_host);
/* The slot order of the payload's code section (see "Wire format" below): slot_feature_out_host[c],
 * 0 <= c < E-k, is the feature whose code slot c of every token carries (capacity >= E-k int32).
 * The order is this library's choice (the paper gives only the bit count, Section 4).
 * BAD_STATE before a feature set; synchronises. */
tpq_status tpq_get_slot_order(tpq_ctx *ctx, int32_t *slot_feature_out_host);

/* ------------------------------------------------------------- the payload */

/* Payload size in bytes for T tokens with the current feature set:
 *   roundup16(ceil(T*(E-k)/2)) + 2*T*k
 * (Section 4 counts (E-k) 4-bit codes and k BF16 values per token; the byte
 * layout below is this library's: the paper fixes only the bit count).
 *
 * Wire format.  With L = E-k:
 *   bytes [0, roundup16(ceil(T*L/2)))  the code section: one flat stream of
 *       4-bit two's-complement codes; code p = t*L + c (token t, slot c) is
 *       the low nibble of byte p/2 if p is even, the high nibble if p is odd;
 *       unused nibbles and the padding up to a multiple of 16 bytes are 0;
 *   then T*k BF16 values, token-major: value t*k + h is the h-th selected
 *       feature (ascending feature index) of token t, its bits unchanged.
 * No header; the static steps are never transmitted.
 *
 * Slot order ("hole filling"): which feature slot c of a token carries.
 * Let S be the selected set.  The holes are the selected features below L,
 * ascending: h_0 < h_1 < ...; the fillers are the unselected features at or
 * above L, ascending: f_0 < f_1 < ... (there are equally many of both).
 *   slot c, 0 <= c < L, carries feature c        if c is not selected,
 *                               feature f_i      if c = h_i.
 * So every unselected feature below L keeps its own index as slot, and the
 * i-th filler takes the i-th hole.  Example: E = 8, S = {1, 6}, L = 6: the
 * hole is 1, the filler is 7, the slots carry features 0 7 2 3 4 5 and the
 * BF16 values are features 1 and 6.  tpq_get_slot_order returns the table.
 * For code widths other than 4 bits the stream is the same with bits-wide
 * codes: code p occupies bits [p*bits, (p+1)*bits) of the little-endian stream.
 * tpq_payload_bytes returns 0 before a feature set exists or for T <= 0. */
size_t tpq_payload_bytes(const tpq_ctx *ctx, int64_t T);
/* The same closed form without a context (Int4), and for a code width of
 * 2..8 bits: roundup16(ceil(T*(E-k)*bits / 8)) + 2*T*k. */
size_t tpq_payload_bytes_for(int64_t T, int64_t E, int64_t k);
size_t tpq_payload_bytes_for_bits(int64_t T, int64_t E, int64_t k, int bits);

/* Section 5 / Section 4: bytes per synchronisation and bits per value. */
tpq_status tpq_comm_bytes(const tpq_ctx *ctx, int64_t T, tpq_comm_report *out);

/* --------------------------------------------------------- the hot path */

/* C^(i) (Sections 2-3, Figure 2): one device's [T][E] BF16 partial sums ->
 * payload.  Low-precision feature: u = fl(x * inv_s); u clamped to [-8, 7];
 * code = round-half-to-even(u) (two binary32 roundings, never fused).
 * Selected feature: the BF16 pattern is copied unchanged.
 *   y_bf16_dev  : [T][E] BF16, row stride row_stride_elems (>= E)
 *   payload_dev : >= tpq_payload_bytes(ctx, T) bytes, 16-byte aligned; every
 *                 byte of the payload (padding included) is written.
 * Enqueues on cuda_stream; T == 0 is a no-op.
 * Errors: BAD_STATE (no feature set), INVALID_ARG, ALIGN, SIZE, CUDA. */
tpq_status tpq_quantize_pack(tpq_ctx *ctx, int shard, const void *y_bf16_dev, int64_t T, int64_t row_stride_elems,
                             void *payload_dev, size_t payload_capacity, void *cuda_stream);

/* The same C^(i) for n consecutive devices first_shard .. first_shard+n-1 in ONE launch, for a process
 * that holds several devices' partial sums on one GPU (the single-GPU simulation of N ranks; in a real
 * deployment every rank calls tpq_quantize_pack once).  The SMs are divided among the shards; every payload
 * is byte-identical to what tpq_quantize_pack writes for that shard.
 *   ys_dev_host / payloads_dev_host : HOST arrays of n DEVICE pointers (inputs [T][E] with the common row
 *   stride; payloads of payload_capacity bytes each), all 16-byte aligned.
 * Enqueues on cuda_stream; T == 0 or n == 0 is a no-op.  Errors as tpq_quantize_pack. */
tpq_status tpq_quantize_pack_batch(tpq_ctx *ctx, int first_shard, int n, const void *const *ys_dev_host, int64_t T,
                                   int64_t row_stride_elems, void *const *payloads_dev_host, size_t payload_capacity,
                                   void *cuda_stream);

/* sum_i D^(i) (Figure 2 caption; Section 5 "local reduction"): N payloads ->
 * the synchronised [T][E] output in the original feature order.
 * Low-precision feature: sum_i code_i * s^(i)_j; selected feature: sum_i of
 * the BF16 values.  Accumulation is binary32 in ascending device order with
 * one final rounding for BF16 output.
 *   payloads_dev_host : HOST array of n_payloads DEVICE pointers, device order;
 *                       n_payloads must equal N; each 16-byte aligned
 *   out_dev           : [T][E] of dt, row stride out_row_stride_elems (>= E)
 * Enqueues on cuda_stream; T == 0 is a no-op.
 * Errors: BAD_STATE, INVALID_ARG, ALIGN, CUDA. */
tpq_status tpq_dequant_reduce(tpq_ctx *ctx, const void *const *payloads_dev_host, int n_payloads, int64_t T,
                              void *out_dev, tpq_out_dtype dt, int64_t out_row_stride_elems, void *cuda_stream);

/* The same with the layer's bias added after the sum (Section 2: f(x) = sum_i f^(i)(x^(i)) + b):
 * out[t][j] = round(fl32(acc[t][j] + bias[j])), acc the binary32 sum of tpq_dequant_reduce before its
 * final rounding.  bias_dev: DEVICE pointer to E binary32 values, 16-byte aligned, read during the
 * call's kernels (the caller keeps it alive and unchanged until they have run).  Errors as
 * tpq_dequant_reduce, plus INVALID_ARG for a NULL bias and ALIGN for a misaligned one. */
tpq_status tpq_dequant_reduce_bias(tpq_ctx *ctx, const void *const *payloads_dev_host, int n_payloads, int64_t T,
                                   void *out_dev, tpq_out_dtype out_dtype, int64_t out_row_stride,
                                   const float *bias_dev, void *stream);

/* ------------------------------------------------- the layer ahead of the synchronisation point (Section 2) */

/* Section 2 defines what is synchronised: the output of the last linear layer of an attention or
 * feed-forward block, f^(i)(x^(i)) = x^(i) W^(i) on device i.  These two calls compute that product on the
 * tensor cores and compress it in the same kernel, so the [T][E] partial sums are never written:
 *   payload = C^(i)( bf16( x W^T ) ),  x: [T][K] BF16,  W: [E][K] BF16 (one row per output feature),
 * FP32 accumulation, one rounding to BF16 (the layer's output type), then exactly tpq_quantize_pack.
 *
 * tpq_permute_weight: once per weight matrix and feature set, gather the rows of w_bf16_dev ([E][K],
 * row-major, 16-byte aligned) into the payload's slot order ("Wire format" above; tpq_get_slot_order): row
 * c < E-k is the feature that code slot c carries, row E-k+h the h-th selected feature.  w_slots_dev: [E][K], 16-byte aligned, not aliasing w.
 * Errors: BAD_STATE (no feature set), INVALID_ARG, ALIGN, CUDA. */
tpq_status tpq_permute_weight(tpq_ctx *ctx, const void *w_bf16_dev, int64_t K, void *w_slots_dev, void *cuda_stream);

/* tpq_linear_quantize_pack: the fused layer for one device.
 *   x_bf16_dev  : [T][K] BF16, row-major, 16-byte aligned; K a multiple of 8
 *   w_slots_dev : output of tpq_permute_weight for the current feature set
 *   payload_dev : as tpq_quantize_pack; byte-identical to tpq_quantize_pack applied to bf16(x W^T)
 *   y_slots_dev : NULL, or [T][E] BF16 (16-byte aligned) that receives the rounded partial sums in slot
 *                 order (column c as the rows of w_slots_dev) -- for verification or a residual path
 * Needs 4-bit codes and E, k multiples of 8 (INVALID_ARG otherwise).  Enqueues on cuda_stream; T == 0 is a
 * no-op.  Errors: BAD_STATE, INVALID_ARG, ALIGN, SIZE, CUDA; TPQ_ERR_TIMEOUT through tpq_device_status. */
tpq_status tpq_linear_quantize_pack(tpq_ctx *ctx, int shard, const void *x_bf16_dev, const void *w_slots_dev, int64_t T,
                                    int64_t K, void *payload_dev, size_t payload_capacity, void *y_slots_dev,
                                    void *cuda_stream);

/* ------------------------------------------------- exchange (Section 5) */

/* Section 5 describes the system-level form of the method: the payloads are all-gathered and every
 * device then reduces locally.  These two calls are that exchange without a collective library: the
 * quantiser stores its payload straight into every destination (its own receive slot and, through
 * peer-mapped pointers over NVLink, the slot it owns in each peer's receive buffer), and the reducing
 * side waits, with a limit, for the N arrival words in its own memory.
 *
 * tpq_quantize_pack_push: C^(i) of tpq_quantize_pack for one shard, the payload written to n_dst
 * destinations (byte-identical in each), then `epoch` written to the n_dst arrival words with release
 * semantics at system scope once every byte of every destination has been stored.
 *   dst_dev_host     : HOST array of n_dst DEVICE pointers (local or peer-mapped), each of dst_capacity
 *                      >= tpq_payload_bytes(ctx, T) bytes, 16-byte aligned
 *   arrived_dev_host : HOST array of n_dst DEVICE pointers to 32-bit words, 4-byte aligned, one per
 *                      destination, in the same memory as the destination
 *   n_dst            : 1 .. 16
 *   epoch            : the step's tag; a receiver waits for exactly this value, so consecutive steps
 *                      on the same slot use different tags
 * T must be >= 1.  Enqueues on cuda_stream.  The caller owns the slot discipline (a slot is not
 * pushed again before its reader has finished: two alternating slot sets suffice when every step
 * waits for all N arrivals).  Errors: BAD_STATE, INVALID_ARG, ALIGN, SIZE, CUDA. */
tpq_status tpq_quantize_pack_push(tpq_ctx *ctx, int shard, const void *y_bf16_dev, int64_t T, int64_t row_stride_elems,
                                  void *const *dst_dev_host, uint32_t *const *arrived_dev_host, int n_dst,
                                  size_t dst_capacity, uint32_t epoch, void *cuda_stream);

/* Enqueue a wait, on cuda_stream, until the n arrival words at arrived_dev (DEVICE pointer, this GPU's
 * memory, 4-byte aligned) all equal `epoch`; work enqueued behind it on the stream (tpq_dequant_reduce)
 * then reads complete payloads.  The wait gives up after timeout_ns (0: one second; at most 5 s): the
 * context's device status becomes TPQ_ERR_TIMEOUT (tpq_device_status), the kernel returns, the stream
 * continues and whatever is reduced afterwards is unspecified.  n: 1 .. 1024.
 * Errors: INVALID_ARG, ALIGN, CUDA. */
tpq_status tpq_wait_arrivals(tpq_ctx *ctx, const uint32_t *arrived_dev, int n, uint32_t epoch, uint64_t timeout_ns,
                             void *cuda_stream);

/* tpq_dequant_reduce (with the bias of tpq_dequant_reduce_bias when bias_dev is not NULL) whose kernels wait
 * themselves, in their prologue and with the limit of tpq_wait_arrivals, for the N arrival words at
 * arrived_dev (word i beside payload i) before they read any payload: the wait costs no launch of its own.
 * Errors as tpq_dequant_reduce and tpq_wait_arrivals; expiry is reported through tpq_device_status. */
tpq_status tpq_dequant_reduce_arrivals(tpq_ctx *ctx, const void *const *payloads_dev_host, int n_payloads, int64_t T,
                                       void *out_dev, tpq_out_dtype out_dtype, int64_t out_row_stride,
                                       const float *bias_dev, const uint32_t *arrived_dev, uint32_t epoch,
                                       uint64_t timeout_ns, void *cuda_stream);

/* ------------------------------------------------- the attention block ahead of the layer: keys and values in 4 bits
 *
 * What a device of a tensor-parallel group computes ahead of the output projection (tpq_linear_quantize_pack):
 * attention of its own heads over keys and values that stay in memory in 4 bits.  The three calls below append a
 * step's keys and values to a paged cache, read them back, and attend to them.
 *
 * The cache of one layer is a pool of n_pages pages of tpq_kv_page_bytes bytes each, owned by the caller, which also
 * decides which page holds which positions of which sequence.  Format of a page: [n_kv_heads][page_size / 16] blocks
 * of 16 positions; a block of 16 * (head_dim + 8) bytes holds
 *   16 rows of head_dim/2 bytes, the keys' codes: code d of a row is the low nibble of byte d/2 if d is even, else
 *      the high nibble (unsigned, 0 .. 15);
 *   16 such rows of the values' codes;
 *   16 32-bit words of the keys, one per position, then 16 words of the values: BF16 `step` in the low half, BF16
 *      `low` in the high half.
 * Code c of a vector stands for  low + step * c.  A vector x (one position, one head, head_dim values in binary32)
 * becomes
 *   low  = bf16(min x),  step = bf16(max((max x - low) c15, 2^-16 max |x|, 2^-60)),  c15 = binary32(1/15) (0x3D888889; a
 *          product, rounded to binary32, and not a quotient: where a 15th of the range is a tie of BF16, the step goes up),
 *   code = clamp(round-half-to-even((x - low) / step), 0, 15),
 * one range per vector as it arrives: unlike the partial sums' ranges (Section 3) the keys' and values' are not
 * static.  A vector that holds a NaN or an infinity, or whose max - min exceeds binary32, becomes low = NaN,
 * step = 1, codes 0: every value of it reads as NaN.  4 + 32/head_dim bits per value (4.25 at head_dim = 128).
 * Pages that append has not written may hold anything, and are values by the same rule if a row sees them; attention
 * takes a vector whose low or step is infinite, or whose step is negative and a value's, for one that is NaN.
 *
 * Conventions beside those above: a handle holds no data of a caller's and serves any number of layers and caches
 * of its geometry; its device must be the current one in every call (BAD_STATE).  What a batch says on the DEVICE
 * is checked by the kernels.  A sequence whose description contradicts itself or the batch is left out, and so is a row whose
 * position is outside the rotation's table (outputs stay as they were, nothing is appended); keys and values of a
 * position whose page number is outside the pool are not appended, read or seen.  The handle's device status becomes TPQ_ERR_INVALID_ARG in
 * each case (tpq_kv_device_status). */

typedef struct tpq_kv tpq_kv; /* opaque */

/* n_heads query heads in n_kv_heads groups of consecutive heads (n_heads a multiple of n_kv_heads, at most 256 per
 * key head), head_dim 64 or 128, page_size (positions per page) 16, 32, 64, 128 or 256.  Errors: INVALID_ARG, NOMEM, CUDA. */
tpq_status tpq_kv_create(tpq_kv **kv, int n_heads, int n_kv_heads, int head_dim, int page_size);
tpq_status tpq_kv_destroy(tpq_kv *kv); /* NULL is accepted */
size_t tpq_kv_page_bytes(const tpq_kv *kv); /* 0 for NULL */

/* One step of a batch of sequences.  Sequence s brings rows token_start[s] .. token_start[s+1] - 1 of the step's
 * tensors (none is allowed); they are its LAST positions: with n rows and length lengths[s] >= n, row i of the
 * sequence is position lengths[s] - n + i.  Position t lies in page page_table[s][t / page_size], entry t % page_size.
 * Only entries of the page table that a call needs are read (attention: pages with a visible position), so entries
 * of pages that a window has left behind may hold anything.  Rows from token_start[n_seqs] on belong to nobody: what
 * they hold does not matter, nothing of theirs is written, and a captured call can be replayed with fewer rows, sequences (n = 0) or
 * other lengths. */
typedef struct tpq_kv_batch {
    void *cache_dev;               /* n_pages * tpq_kv_page_bytes bytes, 16-byte aligned */
    int64_t n_pages;
    const int32_t *page_table_dev; /* [n_seqs][page_table_stride], 4-byte aligned, as the next two */
    int64_t page_table_stride;     /* = most pages of a sequence */
    const int32_t *token_start_dev; /* [n_seqs + 1], ascending from 0 */
    const int32_t *lengths_dev;    /* [n_seqs] positions of a sequence, the new ones included; at most 2^30 */
    int32_t n_seqs;
    int32_t max_new;               /* no sequence brings more rows than this (it chooses kernels) */
    int64_t n_tokens;              /* rows of the step's tensors, >= token_start[n_seqs] */
} tpq_kv_batch;

/* Rotation of the first rot_dim values of a head by their position (rot_dim a multiple of 16, at most head_dim):
 * pair j, 0 <= j < rot_dim/2, becomes (a cos - b sin, b cos + a sin) in binary32, each product and sum rounded, with
 * cos = table[p][j], sin = table[p][rot_dim/2 + j].  Pair j is values j and rot_dim/2 + j, or, if interleaved is not 0, values
 * 2j and 2j + 1. */
typedef struct tpq_kv_rotation {
    const float *table_dev;       /* [n_positions][rot_dim], 16-byte aligned */
    int64_t n_positions;
    int32_t rot_dim;
    int32_t interleaved;
    const int32_t *positions_dev; /* [n_tokens] p of every row, or NULL: a row's position in its sequence */
} tpq_kv_rotation;

/* Append: the step's keys (rotated) and values (as they are) go to their entries of the cache, quantised as above from the rotated binary32
 * values; the queries, if given, are rotated and rounded to BF16.
 *   rotation          : NULL for none (then q must be NULL: there would be nothing to do)
 *   k, v              : [n_tokens][n_kv_heads * head_dim] BF16; q, q_out : [n_tokens][n_heads * head_dim] BF16; q may
 *                       be NULL, q_out may be q (same stride).  Rows 16-byte aligned: strides (in elements) multiples of 8.
 * Two sequences must not append to the same entry (which one it holds is then not specified, nor that it is one of
 * them).  Enqueues on cuda_stream; n_tokens == 0 or n_seqs == 0 is a no-op.  Errors: INVALID_ARG, ALIGN, BAD_STATE, CUDA. */
tpq_status tpq_kv_append(tpq_kv *kv, const tpq_kv_batch *batch, const tpq_kv_rotation *rotation, const void *k_bf16_dev,
                         int64_t k_stride, const void *v_bf16_dev, int64_t v_stride, const void *q_bf16_dev,
                         int64_t q_stride, void *q_out_dev, int64_t q_out_stride, void *cuda_stream);

/* Read back: the values that the cache holds for the batch's rows, bf16(low + step * code), the sum rounded to binary32 first.  A batch whose
 * sequences bring all their positions reads whole sequences.  Either output may be NULL.
 *   k_out, v_out : [n_tokens][n_kv_heads * head_dim] BF16, rows 16-byte aligned
 * Enqueues on cuda_stream.  Errors as tpq_kv_append. */
tpq_status tpq_kv_read(tpq_kv *kv, const tpq_kv_batch *batch, void *k_out_dev, int64_t k_out_stride, void *v_out_dev,
                       int64_t v_out_stride, void *cuda_stream);

/* Attention: row i of a sequence, at position p, and query head h:
 *   out = sum_t w_t v_t / sum_t w_t,  w_t = exp(scale q . k_t),  over the visible t:
 *   t <= p, and, if window > 0, t > p - window or t < n_first
 * (the sliding window of the last `window` positions, p's own among them, and the first n_first positions, which stay
 * visible).  k_t, v_t: the values low + step * code of key head h / (n_heads / n_kv_heads).  Zeros where nothing is
 * visible to a row of finite queries (all its pages were bad).  A position whose key or value is NaN makes the rows that see it NaN, and no
 * others.  A value's step below 2^-60 or below 2^-24 |low| (append writes none) counts as that.
 * Sums and softmax statistics are binary32.  Roundings on the way, for sequences of at most 32 rows (new positions times
 * query heads per key head): the weights times the values' steps, to 11 bits (those below 2^-21 of a row's largest: to
 * 2^-32 of it).  For sequences of more, and for any number in a batch of one sequence whose max_new allows more: the
 * weights times a power of two that 16 positions share, likewise; the keys' and values' values, to 11 bits (those below
 * 2^-28 of the 16 positions' largest magnitude M: to 2^-39 M).  That power of two is M's whether a row sees M's position
 * or not, so that each of the positions may cost a row 2^-31 M.  Where the steps, or M, of a sequence's values differ by more
 * than 2^100, weights of the smaller ones may be lost.  One rounding to BF16 at the end.
 *   q, out    : [n_tokens][n_heads * head_dim] BF16, rows 16-byte aligned; out must not overlap q; at most 2^30 rows times query
 *               heads per key head
 *   work      : the sum over each 256 rows of a sequence of more than 32, and that over each 16 rows of the others, of (positions that
 *               they see / 128 + 6) n_kv_heads must be below 2^31 - 1024 (as rows of a call: 1.4 million new tokens of 64 heads on 8);
 *               beyond it those sequences are left out as above
 *   scale     : finite (1/sqrt(head_dim) as a rule);  window : 0 for none;  n_first : >= 0, without effect if there is no window
 *   workspace : >= tpq_kv_attention_workspace(kv, n_seqs, max_new, n_tokens) bytes of device memory, 16-byte aligned, whose
 *               contents need no preparation and mean nothing afterwards.  Calls that may overlap on the GPU (other
 *               streams, two graphs) need workspaces of their own.
 * Enqueues on cuda_stream; n_tokens == 0 or n_seqs == 0 is a no-op.  Errors: INVALID_ARG, ALIGN, SIZE, BAD_STATE, CUDA;
 * TPQ_ERR_TIMEOUT through tpq_kv_device_status. */
size_t tpq_kv_attention_workspace(const tpq_kv *kv, int32_t n_seqs, int32_t max_new, int64_t n_tokens);
tpq_status tpq_kv_attention(tpq_kv *kv, const tpq_kv_batch *batch, const void *q_bf16_dev, int64_t q_stride, float scale,
                            int64_t window, int64_t n_first, void *out_dev, int64_t out_stride, void *workspace_dev,
                            size_t workspace_bytes, void *cuda_stream);

/* As tpq_device_status, tpq_launch_count and tpq_last_error, for this handle. */
tpq_status tpq_kv_device_status(tpq_kv *kv);
int64_t tpq_kv_launch_count(const tpq_kv *kv);
const char *tpq_kv_last_error(const tpq_kv *kv);

/* ------------------------------------------------- a device's own blocks: feed-forward, weights in 4 bits, answers
 *
 * What a device of a tensor-parallel group computes between the synchronisations: its columns of a gated feed-forward
 * block's first two projections (tpq_gated), whose result is the x of the row-parallel down projection
 * (tpq_linear_quantize_pack, or tpq_linear4 and tpq_quantize_pack where the weights are in 4 bits); and, behind the last
 * synchronisation, its slice of the vocabulary's logits (tpq_linear4), from which log probabilities come
 * (tpq_token_stats, tpq_token_logprobs).
 *
 * One handle serves any number of layers and keeps no data of a caller's; its device must be the current one in every call (BAD_STATE).
 * Unlike a context's, its calls may overlap on the GPU (other streams, captured graphs): they share nothing but the status
 * word.  From the host it is used by one thread at a time. */

typedef struct tpq_block tpq_block; /* opaque */

tpq_status tpq_block_create(tpq_block **block);   /* on the current CUDA device; errors: INVALID_ARG, NOMEM, CUDA */
tpq_status tpq_block_destroy(tpq_block *block);   /* NULL is accepted */

/* Weights in 4 bits.  W is [n_out][n_in], a row per output.  Every `group` (32, 64 or 128) adjacent values of a row share a step:
 *   w = step * code,  code in -8 .. 7,  step = F 2^(e - 8) (1 + m/16)  with e, m in 0 .. 15 (one byte, e the high half) and
 * one binary32 factor F per row.  step / F has 5 significant bits, so that code * step / F is a BF16 number exactly:
 * products with the weights round nothing before they are summed.  4 + 8/group bits per value, and 32 per row.
 *
 * Quantised from BF16, the symmetric grid of Section 3 with one range per group: a the group's largest magnitude,
 *   step = binary32(2a / 15) rounded up to 5 significant bits, but at least 2^(E - 15),
 *   code = clamp(round-half-to-even(w / step), -8, 7),
 * E the exponent of the row's largest step, or -87 if that is less; F = 2^(E - 7).  |w - step code| <= step / 2.  A row that holds a
 * NaN, an infinity or a magnitude of 2^120 and more gets F = NaN: its output is NaN, and no other.
 *
 * Layout: [ceil(n_out / 128)][ceil(n_in / 128)] blocks of 128 outputs x 128 inputs, then ceil(n_out / 128) * 128 factors F
 * (binary32).  A block is 8192 bytes of codes, then [128 / group][128] bytes of steps (the group's, of every output).  16 bytes at
 * p * 2048 + 16 r hold inputs 32p .. 32p + 31 of output r as four words of eight; with u = code + 8, a word is
 *   sum over i = 0 .. 3 of (u_2i 2^(4i) + u_2i+1 2^(16 + 4i)).
 * Inputs and outputs beyond n_in and n_out have code 0. */
typedef enum { TPQ_WEIGHT_BF16 = 0, TPQ_WEIGHT_INT4 = 1 } tpq_weight_kind;
typedef struct tpq_weight {
    const void *data_dev;   /* 16-byte aligned: BF16 [n_out][row_stride], or tpq_weight4_bytes bytes */
    int64_t n_out, n_in;    /* 1 .. 2^30, 1 .. 2^17 */
    int64_t row_stride;     /* BF16: elements, a multiple of 8, >= n_in; 4 bits: not read */
    int32_t kind;           /* tpq_weight_kind */
    int32_t group;          /* 4 bits: 32, 64 or 128; BF16: not read */
} tpq_weight;

size_t tpq_weight4_bytes(int64_t n_out, int64_t n_in, int group); /* 0 for what is not possible */

/* BF16 rows (2-byte aligned, any stride >= n_in) to 4 bits; every byte of w4 (16-byte aligned, capacity >= tpq_weight4_bytes) is written.
 * Enqueues on cuda_stream.  Errors: INVALID_ARG, ALIGN, SIZE, BAD_STATE, CUDA. */
tpq_status tpq_quantize_weight(tpq_block *block, const void *w_bf16_dev, int64_t row_stride, int64_t n_out, int64_t n_in, int group,
                               void *w4_dev, size_t capacity, void *cuda_stream);
/* And back: bf16(step * code) (exact for what tpq_quantize_weight writes, where it is no subnormal of BF16); out: [n_out][n_in] BF16, 2-byte aligned. */
tpq_status tpq_read_weight(tpq_block *block, const void *w4_dev, int64_t n_out, int64_t n_in, int group, void *out_bf16_dev,
                           int64_t out_row_stride, void *cuda_stream);

/* out = x W^T, W in 4 bits; binary32 sums, one rounding for BF16 output.  The tensor cores cut off what does not fit their sums (3 to 4e-9 of the
 * output's norm for every 16 inputs, which the rounding to BF16 hides); for FP32 output, whatever T is, they add up at most 512 inputs, and these sums are added
 * up in binary32, rounded: about 1e-7 of the norm, as a sum of binary32 products has.
 *   x   : [T][n_in] BF16, 16-byte aligned, row stride a multiple of 8 elements (what lies between the rows is not read)
 *   out : [T][n_out] of dt, aligned to its type, any stride >= n_out; it must not overlap x
 * A row of x that holds infinities or NaN makes its own row of out such (an infinite input times a code of 0 is NaN), and no other.
 * Enqueues on cuda_stream; T == 0 is a no-op.  Errors: INVALID_ARG, ALIGN, BAD_STATE, CUDA; TIMEOUT through the status. */
tpq_status tpq_linear4(tpq_block *block, const tpq_weight *w, const void *x_bf16_dev, int64_t x_row_stride, int64_t T, void *out_dev,
                       tpq_out_dtype dt, int64_t out_row_stride, void *cuda_stream);

/* The gated feed-forward block ahead of the down projection: out = bf16(act(x Wg^T) * (x Wu^T)), in one kernel; sums (the tensor cores' own), activation and
 * product in binary32.  gate and up: both BF16 or both in 4 bits (the same group), the same sizes.
 *   SILU g / (1 + e^-g);  GELU_ERF g (1 + erf(g / sqrt 2)) / 2;  GELU_TANH g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2
 * (an activation below 2^-100 may come out as 0).  x, out (BF16), T and errors as tpq_linear4. */
typedef enum { TPQ_ACT_SILU = 0, TPQ_ACT_GELU_TANH = 1, TPQ_ACT_GELU_ERF = 2 } tpq_activation;
tpq_status tpq_gated(tpq_block *block, const tpq_weight *gate, const tpq_weight *up, tpq_activation act, const void *x_bf16_dev,
                     int64_t x_row_stride, int64_t T, void *out_dev, int64_t out_row_stride, void *cuda_stream);

/* Answers.  The logits' columns are split over devices; a device reduces its own to a record of 5 + 2 n_top words per row, the records are
 * exchanged as payloads are (20 + 8 n_top bytes a row instead of the logits), and every device joins them.
 *
 * tpq_token_stats: the records of columns first .. first + n_vocab - 1.
 *   logits  : [T][n_vocab] of dt, aligned to its type, any stride
 *   tokens  : NULL, or [T] the token of each row whose log probability is wanted (a column's number over all devices; negative: none)
 *   n_top   : most likely tokens wanted, 0 .. 32
 *   records : capacity >= tpq_token_record_bytes(T, n_top), 4-byte aligned
 * tpq_token_logprobs: of n records (1 .. 64, HOST array of DEVICE pointers) of the same T and n_top, whose columns differ:
 *   logprob[t]     = x_token - ln sum e^x; 0 where no token is wanted; NaN, and INVALID_ARG through the status, where no record has it
 *   entropy[t]     = - sum p ln p
 *   top[t][i], top_logprob[t][i] : the n_top largest logits' columns, largest first, equal ones by column; -1 and -inf where there are no more
 * Any of the outputs may be NULL.  Logits are taken as they are: a cap or a temperature comes ahead.  A logit of -inf is a token that cannot be; in a row of nothing else every log probability is -inf and the
 * entropy 0.  A NaN or +inf makes its row's log probabilities and entropy NaN; a NaN is not among the most likely.  Sums are binary32.
 * Both enqueue on cuda_stream; T == 0 is a no-op.  Errors: INVALID_ARG, ALIGN, SIZE, BAD_STATE, CUDA. */
size_t tpq_token_record_bytes(int64_t T, int n_top);
tpq_status tpq_token_stats(tpq_block *block, const void *logits_dev, tpq_out_dtype dt, int64_t row_stride, int64_t T, int64_t n_vocab,
                           int64_t first, const int32_t *tokens_dev, int n_top, void *records_dev, size_t capacity, void *cuda_stream);
tpq_status tpq_token_logprobs(tpq_block *block, const void *const *records_dev_host, int n, int64_t T, float *logprob_dev,
                              float *entropy_dev, int n_top, int32_t *top_dev, float *top_logprob_dev, void *cuda_stream);

/* As tpq_device_status, tpq_launch_count and tpq_last_error, for this handle. */
tpq_status tpq_block_device_status(tpq_block *block);
int64_t tpq_block_launch_count(const tpq_block *block);
const char *tpq_block_last_error(const tpq_block *block);

/* ------------------------------------------------- checkpoint and status */

/* Serialise / restore the whole static state (N, E, bits, gamma, counts, m, M,
 * feature set) as a flat little-endian blob.  tpq_get_state with blob == NULL
 * writes the required size to *bytes; otherwise *bytes is the capacity on
 * entry and the size written on return.  tpq_set_state requires a context of
 * the same N, E and bits.  Both synchronise. */
tpq_status tpq_get_state(tpq_ctx *ctx, void *blob_host, size_t *bytes);
tpq_status tpq_set_state(tpq_ctx *ctx, const void *blob_host, size_t bytes);

/* Synchronise and read the device-side status word: TPQ_OK, or
 * TPQ_ERR_TIMEOUT if a kernel's bounded wait on an asynchronous copy gave up
 * (the kernel then returned early and its output is incomplete).  The word is
 * cleared by the call. */
tpq_status tpq_device_status(tpq_ctx *ctx);

/* Kernels launched by this context since creation (for launch accounting). */
int64_t tpq_launch_count(const tpq_ctx *ctx);

const char *tpq_status_string(tpq_status st);
const char *tpq_last_error(const tpq_ctx *ctx); /* "" if none; valid until the next call on ctx */
const char *tpq_version(void);

#ifdef __cplusplus
}
#endif
#endif /* TPQ_H */
