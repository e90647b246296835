// Answers: log probabilities of given tokens, entropies and the most likely tokens of rows of logits whose columns are split over devices
// (tpq_token_stats on every device's columns, tpq_token_logprobs over the records).
//
// One walk over the logits.  A thread keeps the running maximum m of its values, S = sum e^(x - m) and A = sum e^(x - m) (x - m); two such
// triples combine as S = S1 e^(m1 - m) + S2 e^(m2 - m), A likewise with e^(m1 - m) (A1 + (m1 - m) S1).  Then with all of a row's
//   log p(t) = x_t - m - ln S,      entropy = -sum p ln p = ln S - A / S.
// The most likely tokens: a thread's maximum is a by-product; the n-th largest of the maxima of 64 groups of threads is a bound that at least n
// values reach, and only threads whose maximum does read their values again (from L2): about n of 256.
#include <cuda_bf16.h>

#include <cmath>

#include "block_internal.h"

namespace {

constexpr int THREADS = 256, GROUPS = 64, MOST_TOP = 32, LIST = 1024, AHEAD = 4;
constexpr float LOG2E = 1.4426950408889634f;

struct triple {
    float m, S, A;
};
__device__ __forceinline__ float exp_of(float d)  // e^d, d <= 0 or NaN
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d * LOG2E));
    return r;
}
// A triple for the maximum to >= its own.  Differences of lowest numbers and infinities are kept finite where a sum of 0 meets them.
__device__ __forceinline__ void move_to(triple &t, float to)
{
    const float d = t.m - to, e = exp_of(d);
    t.A = e * fmaf(fmaxf(d, -1e30f), t.S, t.A);
    t.S *= e;
    t.m = to;
}
__device__ __forceinline__ float or_zero(float m) { return m == -INFINITY ? 0.0f : m; }  // (nothing so far: any number will do)
__device__ __forceinline__ triple join(triple a, triple b)
{
    const float m = fmaxf(a.m, b.m), ref = or_zero(m);
    move_to(a, ref);
    move_to(b, ref);
    return {m, a.S + b.S, a.A + b.A};
}

// Numbers as integers of the same order, -0 as 0; 0: no value, or one that is no number (never an alternative).
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return x != x ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k); }

template <bool FP32>
struct row_reader {  // the row as 16-byte pieces that start at 16-byte boundaries; piece v holds values v * VE - off ...
    static constexpr int VE = FP32 ? 4 : 8;
    const uint8_t *at;  // piece 0 (its first `off` values lie ahead of the row)
    int off, n;
    __device__ __forceinline__ row_reader(const void *row, int n_) : n(n_)
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(row);
        off = (int)(a & 15) / (FP32 ? 4 : 2);
        at = reinterpret_cast<const uint8_t *>(a & ~(uintptr_t)15);
    }
    __device__ __forceinline__ int pieces() const { return (off + n + VE - 1) / VE; }
    __device__ __forceinline__ bool whole(int v) const { return v * VE >= off && (v + 1) * VE <= off + n; }
    __device__ __forceinline__ uint4 raw(int v) const  // a piece; values outside the row are -inf
    {
        if (whole(v)) return __ldcs(reinterpret_cast<const uint4 *>(at) + v);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (FP32) {
                const int k = v * 4 + i - off;
                w[i] = k >= 0 && k < n ? reinterpret_cast<const uint32_t *>(at)[v * 4 + i] : 0xFF800000u;
            } else {
                const int k = v * 8 + 2 * i - off;
                const uint16_t *h = reinterpret_cast<const uint16_t *>(at) + v * 8 + 2 * i;
                w[i] = (k >= 0 && k < n ? h[0] : 0xFF80u) | (k + 1 >= 0 && k + 1 < n ? (uint32_t)h[1] : 0xFF80u) << 16;
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ static void values(const uint4 &q, float (&x)[VE])
    {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (FP32) x[i] = __uint_as_float(w[i]);
            else {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
    }
    __device__ __forceinline__ int index(int v, int i) const { return v * VE + i - off; }
};

struct shared {
    uint32_t group[GROUPS];
    uint32_t bound;
    int n_active, n_above, n_equal;
    uint16_t active[THREADS];
    uint32_t above_key[LIST];
    int32_t above_at[LIST], equal_at[LIST];
    triple warps[THREADS / 32];
    triple all;
    uint32_t top_key[MOST_TOP];
    int32_t top_at[MOST_TOP];
    unsigned long long best;
    int counts[THREADS / 32];
};

__device__ __forceinline__ unsigned long long order_of(uint32_t key, int at) { return (unsigned long long)key << 32 | (uint32_t)~at; }

// The n largest of a block's part of a row, largest first, equal ones by index: s.top_key (0 where there are no more) and s.top_at.
// mine: the largest key of this thread's pieces v0 + threadIdx.x, + THREADS, ... < v1.
template <bool FP32>
__device__ void most_likely(shared &s, const row_reader<FP32> &r, int v0, int v1, uint32_t mine, int n)
{
    constexpr int VE = row_reader<FP32>::VE;
    const int tid = threadIdx.x;
    uint32_t g = max(mine, __shfl_xor_sync(0xffffffffu, mine, 1));
    g = max(g, __shfl_xor_sync(0xffffffffu, g, 2));
    if (tid % 4 == 0) s.group[tid / 4] = g;
    if (tid == 0) s.n_active = s.n_above = s.n_equal = 0;
    if (tid < MOST_TOP) s.top_key[tid] = 0, s.top_at[tid] = -1;
    __syncthreads();
    {   // the place of each group's maximum among the 64: four threads a group
        int above = 0;
        for (int i = tid % 4; i < GROUPS; i += 4) above += s.group[i] > g || (s.group[i] == g && i < tid / 4);
        above += __shfl_xor_sync(0xffffffffu, above, 1);
        above += __shfl_xor_sync(0xffffffffu, above, 2);
        if (tid % 4 == 0 && above == n - 1) s.bound = g;
    }
    __syncthreads();
    const uint32_t bound = s.bound;
    if (mine >= bound && mine) s.active[atomicAdd(&s.n_active, 1)] = (uint16_t)tid;
    __syncthreads();
    const int each = (v1 - v0 + THREADS - 1) / THREADS, items = s.n_active * each;
    for (int i = tid; i < items; i += THREADS) {
        const int v = v0 + s.active[i / each] + i % each * THREADS;
        if (v >= v1) continue;
        float x[VE];
        r.values(r.raw(v), x);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const uint32_t k = key_of(x[j]);
            const int at = r.index(v, j);
            if (k == 0 || k < bound || at < 0 || at >= r.n) continue;
            if (k > bound) {
                const int to = atomicAdd(&s.n_above, 1);
                if (to < LIST) s.above_key[to] = k, s.above_at[to] = at;
            } else {
                const int to = atomicAdd(&s.n_equal, 1);
                if (to < LIST) s.equal_at[to] = at;
            }
        }
    }
    __syncthreads();
    const int above = s.n_above, equal = s.n_equal;
    if (above > LIST) {
        // values so arranged that a few threads have most of the large ones: n walks, each for the largest behind the one before
        unsigned long long last = ~0ull;
        for (int i = 0; i < n; ++i) {
            if (tid == 0) s.best = 0;
            __syncthreads();
            unsigned long long b = 0;
            for (int v = v0 + tid; v < v1; v += THREADS) {
                float x[VE];
                r.values(r.raw(v), x);
                for (int j = 0; j < VE; ++j) {
                    const int at = r.index(v, j);
                    const unsigned long long o = order_of(key_of(x[j]), at);
                    if (at >= 0 && at < r.n && o >> 32 && o < last && o > b) b = o;
                }
            }
            atomicMax(&s.best, b);
            __syncthreads();
            last = s.best;
            if (tid == 0 && last) s.top_key[i] = (uint32_t)(last >> 32), s.top_at[i] = (int)~(uint32_t)last;
            __syncthreads();
        }
        return;
    }
    for (int i = tid; i < above; i += THREADS) {
        const unsigned long long mine_ = order_of(s.above_key[i], s.above_at[i]);
        int place = 0;
        for (int j = 0; j < above; ++j) place += order_of(s.above_key[j], s.above_at[j]) > mine_;
        if (place < n) s.top_key[place] = s.above_key[i], s.top_at[place] = s.above_at[i];
    }
    const int left = n - above;  // the rest: those equal to the bound, the lowest indexes
    if (left > 0 && equal <= LIST) {
        for (int i = tid; i < equal; i += THREADS) {
            int place = 0;
            for (int j = 0; j < equal; ++j) place += s.equal_at[j] < s.equal_at[i];
            if (place < left) s.top_key[above + place] = bound, s.top_at[above + place] = s.equal_at[i];
        }
    } else if (left > 0) {  // very many of them (masked columns): in order from the front until there are enough
        int found = 0;
        for (int v = v0; v < v1 && found < left; v += THREADS) {
            int mine_ = 0;
            float x[VE];
            if (v + tid < v1) {
                r.values(r.raw(v + tid), x);
                for (int j = 0; j < VE; ++j) mine_ += key_of(x[j]) == bound && r.index(v + tid, j) >= 0 && r.index(v + tid, j) < r.n;
            }
            int before = mine_;
            for (int m = 1; m < 32; m <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, before, m);
                if (tid % 32 >= m) before += o;
            }
            if (tid % 32 == 31) s.counts[tid / 32] = before;
            __syncthreads();
            int all = 0, ahead = 0;
            for (int w = 0; w < THREADS / 32; ++w) {
                ahead += w < tid / 32 ? s.counts[w] : 0;
                all += s.counts[w];
            }
            int to = found + ahead + before - mine_;
            if (mine_)
                for (int j = 0; j < VE; ++j)
                    if (key_of(x[j]) == bound && r.index(v + tid, j) >= 0 && r.index(v + tid, j) < r.n) {
                        if (to < left) s.top_key[above + to] = bound, s.top_at[above + to] = r.index(v + tid, j);
                        ++to;
                    }
            found += all;
            __syncthreads();
        }
    }
    __syncthreads();
}

__device__ __forceinline__ uint32_t peer(const void *p, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ uint32_t ld_cluster(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The first n of `lists` sorted lists, by a warp: lane <-> lists lane and lane + 32, whose heads (order_of) `head` gives.
template <typename Head, typename Take>
__device__ __forceinline__ void merge(int lists, int n, Head head, Take take)
{
    const int lane = threadIdx.x & 31;
    int p0 = 0, p1 = 0;
    unsigned long long h0 = lane < lists ? head(lane, 0) : 0, h1 = lane + 32 < lists ? head(lane + 32, 0) : 0;
    for (int i = 0; i < n; ++i) {
        const unsigned long long mine = h0 > h1 ? h0 : h1;
        const uint32_t key = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32));
        const uint32_t at = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32) == key ? (uint32_t)mine : 0u);
        const unsigned long long best = (unsigned long long)key << 32 | at;
        take(i, key, (int)~at);
        if (!key) continue;
        if (h0 == best) h0 = ++p0 < n ? head(lane, p0) : 0;
        else if (h1 == best) h1 = ++p1 < n ? head(lane + 32, p1) : 0;
    }
}

constexpr int HEAD_WORDS = 5;  // of a record: m, S, A, the token's logit, 0: not here, 1: here, 2: none asked for; then n keys, n indexes

// A cluster of `split` blocks a row (gridDim.x = rows * split).
template <bool FP32>
__global__ void __launch_bounds__(THREADS) token_stats(const stats_call c, int split)
{
    __shared__ shared s;
    constexpr int VE = row_reader<FP32>::VE;
    const int tid = threadIdx.x, rank = split > 1 ? blockIdx.x % split : 0;
    const int64_t t = blockIdx.x / split;
    tpq_grid_dep_wait();
    tpq_grid_dep_launch();
    const uint8_t *const row = static_cast<const uint8_t *>(c.logits) + t * c.stride * (FP32 ? 4 : 2);
    const row_reader<FP32> r(row, c.n_vocab);
    const int v0 = (int)((int64_t)r.pieces() * rank / split), v1 = (int)((int64_t)r.pieces() * (rank + 1) / split);
    triple a = {-INFINITY, 0.0f, 0.0f};
    float most = -INFINITY;
    uint32_t any = 0;
    for (int v = v0 + tid; v < v1; v += AHEAD * THREADS) {
        uint4 q[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) q[i] = v + i * THREADS < v1 ? r.raw(v + i * THREADS) : (FP32 ? make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u) : make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u));
        any = 1;
        float m = a.m;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            float x[VE];
            r.values(q[i], x);
#pragma unroll
            for (int j = 0; j < VE; ++j) m = fmaxf(m, x[j]);
        }
        most = m;
        const float ref = or_zero(m);
        move_to(a, ref);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            float x[VE];
            r.values(q[i], x);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const float d = x[j] - ref, e = exp_of(d);
                a.S += e;
                a.A = fmaf(e, fmaxf(d, -1e4f), a.A);
            }
        }
        a.m = m;
    }
#pragma unroll
    for (int m = 16; m; m >>= 1) {
        const triple o = {__shfl_xor_sync(0xffffffffu, a.m, m), __shfl_xor_sync(0xffffffffu, a.S, m), __shfl_xor_sync(0xffffffffu, a.A, m)};
        a = (tid & m) ? join(o, a) : join(a, o);
    }
    if (tid % 32 == 0) s.warps[tid / 32] = a;
    if (c.n_top) most_likely<FP32>(s, r, v0, v1, any ? key_of(most) : 0u, c.n_top);
    else __syncthreads();
    uint32_t *const out = c.records + t * (HEAD_WORDS + 2 * c.n_top);
    if (split > 1) cluster_sync();
    if (rank == 0 && tid < 32) {
        triple all = s.warps[0];
        for (int k = 0; k < split; ++k)
            for (int w = k ? 0 : 1; w < THREADS / 32; ++w) {
                triple o;
                if (split > 1) {
                    const uint32_t at = peer(&s.warps[w], k);
                    o = {__uint_as_float(ld_cluster(at)), __uint_as_float(ld_cluster(at + 4)), __uint_as_float(ld_cluster(at + 8))};
                } else {
                    o = s.warps[w];
                }
                all = join(all, o);
            }
        if (tid == 0) {
            out[0] = __float_as_uint(all.m);
            out[1] = __float_as_uint(all.S);
            out[2] = __float_as_uint(all.A);
            const int64_t token = c.tokens ? c.tokens[t] : -1, at = token - c.first;
            const bool here = token >= 0 && at >= 0 && at < c.n_vocab;
            float x = 0.0f;
            if (here) x = FP32 ? reinterpret_cast<const float *>(row)[at] : __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(row)[at] << 16);
            out[3] = __float_as_uint(x);
            out[4] = here ? 1u : token < 0 ? 2u : 0u;
        }
        if (c.n_top)
            merge(split, c.n_top,
                  [&](int k, int p) { return split > 1 ? order_of(ld_cluster(peer(&s.top_key[p], k)), (int)ld_cluster(peer(&s.top_at[p], k))) : order_of(s.top_key[p], s.top_at[p]); },
                  [&](int i, uint32_t key, int at) {
                      if (tid == 0) {
                          out[HEAD_WORDS + i] = key;
                          out[HEAD_WORDS + c.n_top + i] = key ? (uint32_t)(at + c.first) : 0xFFFFFFFFu;
                      }
                  });
    }
    if (split > 1) cluster_sync();
}

// A warp a row.
__global__ void __launch_bounds__(128) token_logprobs(const join_call c, int *status)
{
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * 4 + threadIdx.x / 32;
    tpq_grid_dep_wait();
    tpq_grid_dep_launch();
    if (t >= c.T) return;
    const int64_t at = t * (HEAD_WORDS + 2 * c.n_top);
    triple a = {-INFINITY, 0.0f, 0.0f};
    float x = 0.0f;
    uint32_t state = 0;
    for (int i = 0; i < c.n; ++i) {
        const uint32_t *const r = c.records[i] + at;
        a = join(a, {__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[2])});
        if (r[4] == 1u && state != 1u) x = __uint_as_float(r[3]);
        if (state != 1u && r[4] != 0u) state = r[4];
    }
    // (S is 0 where every logit is -inf: nothing is likely, and nothing is unsure)
    const bool none = a.S == 0.0f;
    const float ln = logf(a.S);
    auto logp = [&](float v) { return none ? -INFINITY : (v - a.m) - ln; };
    if (lane == 0) {
        if (c.logprob) c.logprob[t] = state == 1u ? logp(x) : state == 2u ? 0.0f : NAN;
        if (c.entropy) c.entropy[t] = none ? 0.0f : ln - a.A / a.S;
        if (state == 0u) atomicExch(status, (int)TPQ_ERR_INVALID_ARG);
    }
    if (c.n_top)
        merge(c.n, c.n_top,
              [&](int k, int p) {
                  const uint32_t *const r = c.records[k] + at + HEAD_WORDS;
                  return r[p] ? order_of(r[p], (int)r[c.n_top + p]) : 0ull;
              },
              [&](int i, uint32_t key, int index) {
                  if (lane != 0) return;
                  if (c.top) c.top[t * c.n_top + i] = key ? index : -1;
                  if (c.top_logprob) c.top_logprob[t * c.n_top + i] = key ? logp(value_of(key)) : -INFINITY;
              });
}

template <bool FP32>
cudaError_t launch_stats(const stats_call &c, const tpq_block *b, cudaStream_t st)
{
    // Few rows: a cluster for each, as long as all blocks run at once and a block has 4096 values.
    int split = 1;
    while (split < 8 && c.T * split * 2 <= 2 * b->sm_count && c.n_vocab / (split * 2) >= 4096) split *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(c.T * split));
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = split;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, token_stats<FP32>, c, split);
}

}  // namespace

cudaError_t answers_launch_stats(const stats_call &c, const tpq_block *b, cudaStream_t st, int64_t *launches)
{
    const cudaError_t e = c.fp32 ? launch_stats<true>(c, b, st) : launch_stats<false>(c, b, st);
    if (e == cudaSuccess) ++*launches;
    return e;
}

cudaError_t answers_launch_join(const join_call &c, const tpq_block *b, cudaStream_t st, int64_t *launches)
{
    const cudaError_t e = tpq_launch_pdl(token_logprobs, dim3((unsigned)((c.T + 3) / 4)), dim3(128), 0, st, c, b->status);
    if (e == cudaSuccess) ++*launches;
    return e;
}
