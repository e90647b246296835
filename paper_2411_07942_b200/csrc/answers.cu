// Answers: log probabilities of given tokens, entropies and the most likely tokens of rows of logits whose columns are split over devices
// (tpq_token_stats on every device's columns, tpq_token_logprobs over the records).
//
// One walk over the logits.  A thread keeps the running maximum m of its values, S = sum e^(x - m) and A = sum e^(x - m) (x - m); two such
// triples combine as S = S1 e^(m1 - m) + S2 e^(m2 - m), A likewise with e^(m1 - m) (A1 + (m1 - m) S1).  Then with all of a row's
//   log p(t) = x_t - m - ln S,      entropy = -sum p ln p = ln S - A / S.
// 2048 rows of 32000 in BF16 take 30 us, where memory would take 20, the exponentials (16 a clock) 14.6 and the instructions (5 to 6 a value, with
// differences, sums and products of two values at a time) 62 % of the issue slots: nothing is full.  A thread's loads and arithmetic take turns, and
// 2048 blocks on 1184 places are two rounds.
// The most likely tokens: a thread's maximum is a by-product; the n-th largest of the maxima of 64 groups of threads is a bound that at least n
// values reach.  Of the values, whose maxima per 32 to 64 of a thread's are kept, only those chunks are read again (from L2) whose maximum
// reaches the bound: about n of them.
#include <cuda_bf16.h>

#include <cmath>

#include "block_internal.h"

namespace {

constexpr int GROUPS = 64, MOST_TOP = 32, LIST = 512, MOST_SPLIT = 8, CHUNKS = 4096;
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
    int off, n, whole0, whole1;  // pieces whole0 .. whole1 - 1 lie inside the row
    __device__ __forceinline__ row_reader(const void *row, int n_) : n(n_)
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(row);
        off = (int)(a & 15) / (FP32 ? 4 : 2);
        at = reinterpret_cast<const uint8_t *>(a & ~(uintptr_t)15);
        whole0 = off != 0;
        whole1 = (off + n) / VE;
    }
    __device__ __forceinline__ int pieces() const { return (off + n + VE - 1) / VE; }
    __device__ __forceinline__ bool whole(int v) const { return v >= whole0 && v < whole1; }
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

template <int THREADS>
struct shared {
    uint32_t group[GROUPS];
    uint32_t bound;
    int n_active, n_above, n_equal;
    uint16_t chunk[CHUNKS / THREADS][THREADS];  // high halves of the keys of chunks' maxima
    uint16_t active[LIST];                       // chunks to read again, numbered through that array
    uint32_t above_key[LIST];
    int32_t above_at[LIST], equal_at[LIST];
    triple warps[THREADS / 32];
    unsigned long long top[MOST_TOP];  // order_of, largest first, 0 where there are no more
    unsigned long long best;
    int counts[THREADS / 32];
    // of the cluster's first block: what the others found
    triple parts[MOST_SPLIT];
    unsigned long long lists[MOST_SPLIT][MOST_TOP], merged[MOST_TOP];
    int place[MOST_SPLIT * MOST_TOP];
};

__device__ __forceinline__ unsigned long long order_of(uint32_t key, int at) { return (unsigned long long)key << 32 | (uint32_t)~at; }

// The n largest of a block's part of a row, largest first, equal ones by index: s.top.
// mine: the largest key of this thread's pieces v0 + threadIdx.x, + THREADS, ... < v1; a chunk has `span` of them, the thread `chunks` chunks.
template <bool FP32, int THREADS>
__device__ void most_likely(shared<THREADS> &s, const row_reader<FP32> &r, int v0, int v1, uint32_t mine, int n, int span, int chunks)
{
    constexpr int VE = row_reader<FP32>::VE, EACH = THREADS / GROUPS;
    const int tid = threadIdx.x;
    uint32_t g = mine;
#pragma unroll
    for (int m = 1; m < EACH; m <<= 1) g = max(g, __shfl_xor_sync(0xffffffffu, g, m));
    if (tid % EACH == 0) s.group[tid / EACH] = g;
    if (tid == 0) s.n_active = s.n_above = s.n_equal = 0;
    if (tid < MOST_TOP) s.top[tid] = 0;
    __syncthreads();
    {   // the place of each group's maximum among the 64, by the group's threads
        int above = 0;
#pragma unroll 8
        for (int i = tid % EACH; i < GROUPS; i += EACH) above += s.group[i] > g || (s.group[i] == g && i < tid / EACH);
#pragma unroll
        for (int m = 1; m < EACH; m <<= 1) above += __shfl_xor_sync(0xffffffffu, above, m);
        if (tid % EACH == 0 && above == n - 1) s.bound = g;
    }
    __syncthreads();
    const uint32_t bound = s.bound;
    if (mine >= bound && mine)
        for (int i = 0; i < chunks; ++i)
            if (s.chunk[i][tid] >= bound >> 16) {
                const int to = atomicAdd(&s.n_active, 1);
                if (to < LIST) s.active[to] = (uint16_t)(i * THREADS + tid);
            }
    __syncthreads();
    // (very many chunks: equal values all over the row; then all of it)
    const bool listed = s.n_active <= LIST;
    const int items = listed ? s.n_active * span : v1 - v0;
    for (int i = tid; i < items; i += THREADS) {
        int v = v0 + i;
        if (listed) {
            const int k = s.active[i / span], chunk = k / THREADS;
            v = v0 + k % THREADS + (chunk * span + i % span) * THREADS;
        }
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
            if (tid == 0) s.top[i] = last;
            __syncthreads();
        }
        return;
    }
    for (int i = tid; i < above; i += THREADS) {
        const unsigned long long mine_ = order_of(s.above_key[i], s.above_at[i]);
        int place = 0;
        for (int j = 0; j < above; ++j) place += order_of(s.above_key[j], s.above_at[j]) > mine_;
        if (place < n) s.top[place] = mine_;
    }
    const int left = n - above;  // the rest: those equal to the bound, the lowest indexes
    if (left > 0 && equal <= LIST) {
        for (int i = tid; i < equal; i += THREADS) {
            int place = 0;
            for (int j = 0; j < equal; ++j) place += s.equal_at[j] < s.equal_at[i];
            if (place < left) s.top[above + place] = order_of(bound, s.equal_at[i]);
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
                        if (to < left) s.top[above + to] = order_of(bound, r.index(v + tid, j));
                        ++to;
                    }
            found += all;
            __syncthreads();
        }
    }
    __syncthreads();
}

// Puts `lists` sorted lists of n (order_of, 0: no more; list l at from + l * pitch) together: the n first to `out`.  By all threads of a block, one
// for each pair of an entry and another list; place: room for lists * n numbers.
template <int THREADS>
__device__ void merge(const unsigned long long *from, int pitch, int lists, int n, int *place, unsigned long long *out)
{
    const int entries = lists * n;
    for (int i = threadIdx.x; i < n; i += THREADS) out[i] = 0;
    for (int i = threadIdx.x; i < entries; i += THREADS) place[i] = i % n;  // and those of the other lists that come first:
    __syncthreads();
    for (int i = threadIdx.x; i < entries * lists; i += THREADS) {
        const int k = i / entries, e = i - k * entries, l = e / n;
        const unsigned long long o = from[l * pitch + e - l * n];
        if (!o || k == l) continue;
        int before = 0;
#pragma unroll
        for (int step = MOST_TOP; step; step >>= 1)
            if (before + step <= n && from[k * pitch + before + step - 1] > o) before += step;
        if (before) atomicAdd(&place[e], before);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < entries; i += THREADS) {
        const unsigned long long o = from[i / n * pitch + i % n];
        if (o && place[i] < n) out[place[i]] = o;
    }
    __syncthreads();
}

// Of a warp's triples: one (in a fixed order), for lane 0.
__device__ __forceinline__ triple join_warp(triple a)
{
#pragma unroll
    for (int m = 16; m; m >>= 1) {
        const triple o = {__shfl_down_sync(0xffffffffu, a.m, m), __shfl_down_sync(0xffffffffu, a.S, m), __shfl_down_sync(0xffffffffu, a.A, m)};
        a = join(a, o);
    }
    return a;
}

__device__ __forceinline__ uint32_t first_block(const void *p)  // the same place in the cluster's first block
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(p)));
    return a;
}
__device__ __forceinline__ void st_cluster(uint32_t a, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ void st_cluster(uint32_t a, unsigned long long v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// two values at a time
__device__ __forceinline__ uint64_t pack2(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// A piece with what is below -3e38 at -3e38 (of BF16: the number next to it), and its values' largest
template <bool FP32>
__device__ __forceinline__ uint4 clamped(uint4 q)
{
    uint32_t *const w = reinterpret_cast<uint32_t *>(&q);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (FP32) asm("max.NaN.f32 %0, %0, %1;" : "+f"(reinterpret_cast<float *>(w)[i]) : "f"(-3e38f));
        else asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(w[i]) : "r"(0xFF62FF62u));
    }
    return q;
}
template <bool FP32>
__device__ __forceinline__ float largest(const uint4 &q, float m)
{
    if (FP32) return fmaxf(fmaxf(m, fmaxf(__uint_as_float(q.x), __uint_as_float(q.y))), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
    uint32_t a, b;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(q.x), "r"(q.y));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(q.z), "r"(q.w));
    asm("max.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    return fmaxf(m, fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u)));
}

constexpr int HEAD_WORDS = 5;  // of a record: m, S, A, the token's logit, 0: not here, 1: here, 2: none asked for; then n keys, n indexes

// A cluster of `split` blocks a row (gridDim.x = rows * split).
template <bool FP32, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 128 ? 8 : 2) token_stats(const stats_call c, int split)
{
    __shared__ shared<THREADS> s;
    constexpr int VE = row_reader<FP32>::VE, AHEAD = THREADS == 128 ? 8 : 4;  // pieces on the way to a thread
    const int tid = threadIdx.x, rank = split > 1 ? blockIdx.x % split : 0;
    const int64_t t = blockIdx.x / split;
    if (split > 1) cluster_arrive();  // (the first block's memory is there: waited for ahead of the first store to it)
    tpq_grid_dep_wait();
    tpq_grid_dep_launch();
    const uint8_t *const row = static_cast<const uint8_t *>(c.logits) + t * c.stride * (FP32 ? 4 : 2);
    const row_reader<FP32> r(row, c.n_vocab);
    const int v0 = (int)((int64_t)r.pieces() * rank / split), v1 = (int)((int64_t)r.pieces() * (rank + 1) / split);
    // chunks of whole rounds of the walk, as few rounds each as there is room for
    const int rounds = (v1 - v0 + AHEAD * THREADS - 1) / (AHEAD * THREADS), each = (rounds + CHUNKS / THREADS - 1) / (CHUNKS / THREADS);
    triple a = {-INFINITY, 0.0f, 0.0f};
    bool any = false;
    float of_chunk = -INFINITY;
    int chunk = 0, in_chunk = 0;
    for (int v = v0 + tid; v < v1; v += AHEAD * THREADS) {
        uint4 q[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {  // (pieces beyond the block's are -inf)
            const uint32_t out = FP32 ? 0xFF800000u : 0xFF80FF80u;
            q[i] = v + i * THREADS < v1 ? r.raw(v + i * THREADS) : make_uint4(out, out, out, out);
        }
        any = true;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) of_chunk = largest<FP32>(q[i], of_chunk);
        const float m = fmaxf(a.m, of_chunk);
        if (c.n_top) {
            s.chunk[chunk][tid] = (uint16_t)(key_of(of_chunk) >> 16);
            if (++in_chunk == each) ++chunk, in_chunk = 0, of_chunk = -INFINITY;
        }
        const float ref = or_zero(m);
        move_to(a, ref);
        if (fabsf(ref) < 1e30f) {
            // What is below -3e38 counts as that, which is e^-inf = 0 for a maximum above -1e30, and stays finite.
            const uint64_t ref2 = pack2(-ref, -ref), log2 = pack2(LOG2E, LOG2E);
            uint64_t S = pack2(0.0f, 0.0f), A = S;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (v + i * THREADS >= v1) break;
                float x[VE];
                r.values(clamped<FP32>(q[i]), x);
#pragma unroll
                for (int j = 0; j < VE; j += 2) {
                    const uint64_t d = add2(pack2(x[j], x[j + 1]), ref2);
                    float y0, y1;
                    unpack2(mul2(d, log2), y0, y1);
                    const uint64_t e = pack2(ex2(y0), ex2(y1));
                    S = add2(S, e);
                    A = fma2(e, d, A);
                }
            }
            float s0, s1, a0, a1;
            unpack2(S, s0, s1);
            unpack2(A, a0, a1);
            a.S += s0 + s1;
            a.A += a0 + a1;
        } else {
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
        }
        a.m = m;
    }
    const float most = a.m;
    // of a warp: one reference for all, then sums
    {
        float m = a.m;
#pragma unroll
        for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
        move_to(a, or_zero(m));
#pragma unroll
        for (int k = 16; k; k >>= 1) {
            a.S += __shfl_xor_sync(0xffffffffu, a.S, k);
            a.A += __shfl_xor_sync(0xffffffffu, a.A, k);
        }
        a.m = m;
    }
    if (tid % 32 == 0) s.warps[tid / 32] = a;
    if (c.n_top) most_likely<FP32, THREADS>(s, r, v0, v1, any ? key_of(most) : 0u, c.n_top, AHEAD * each, chunk + (in_chunk != 0));
    else __syncthreads();
    uint32_t *const out = c.records + t * (HEAD_WORDS + 2 * c.n_top);
    triple all = {-INFINITY, 0.0f, 0.0f};
    if (tid < 32) {
        if (tid < THREADS / 32) all = s.warps[tid];
        all = join_warp(all);
    }
    const unsigned long long *top = s.top;
    if (split > 1) {
        cluster_wait();
        if (tid == 0) {
            const uint32_t to = first_block(&s.parts[rank]);
            st_cluster(to, __float_as_uint(all.m));
            st_cluster(to + 4, __float_as_uint(all.S));
            st_cluster(to + 8, __float_as_uint(all.A));
        }
        if (tid < c.n_top) st_cluster(first_block(&s.lists[rank][tid]), s.top[tid]);
        cluster_arrive();
        if (rank != 0) return;  // (nobody reads this block's memory)
        cluster_wait();
        if (tid < 32) {
            all = triple{-INFINITY, 0.0f, 0.0f};
            if (tid < split) all = s.parts[tid];
            all = join_warp(all);
        }
        if (c.n_top) merge<THREADS>(&s.lists[0][0], MOST_TOP, split, c.n_top, s.place, s.merged);
        top = s.merged;
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
    if (tid < c.n_top) {
        const unsigned long long o = top[tid];
        out[HEAD_WORDS + tid] = (uint32_t)(o >> 32);
        out[HEAD_WORDS + c.n_top + tid] = o ? (uint32_t)(~(uint32_t)o + (uint32_t)c.first) : 0xFFFFFFFFu;
    }
}

// A warp a row, or with alternatives a block of 4 warps.  Record i is lane i's, and i + 32.
__global__ void __launch_bounds__(128) token_logprobs(const join_call c, int *status)
{
    extern __shared__ unsigned long long lists[];  // [n + 1][n_top], and as many places
    const int lane = threadIdx.x & 31;
    const int64_t t = c.n_top ? blockIdx.x : (int64_t)blockIdx.x * 4 + threadIdx.x / 32;
    tpq_grid_dep_wait();
    tpq_grid_dep_launch();
    if (t >= c.T) return;  // (whole warps; with alternatives no thread)
    const int64_t at = t * (HEAD_WORDS + 2 * c.n_top);
    triple a = {-INFINITY, 0.0f, 0.0f};
    float x = 0.0f;
    uint32_t here = 0, none_asked = 0;
    for (int i = lane; i < c.n; i += 32) {
        const uint32_t *const r = c.records[i] + at;
        const uint32_t m = r[0], S = r[1], A = r[2], v = r[3], state = r[4];
        a = join(a, {__uint_as_float(m), __uint_as_float(S), __uint_as_float(A)});
        if (state == 1u && !here) x = __uint_as_float(v);
        here |= state == 1u;
        none_asked |= state == 2u;
    }
    a = join_warp(a);
    a.m = __shfl_sync(0xffffffffu, a.m, 0), a.S = __shfl_sync(0xffffffffu, a.S, 0), a.A = __shfl_sync(0xffffffffu, a.A, 0);
    const uint32_t has = __ballot_sync(0xffffffffu, here), without = __ballot_sync(0xffffffffu, none_asked);
    x = __shfl_sync(0xffffffffu, x, has ? __ffs(has) - 1 : 0);
    // (S is 0 where every logit is -inf: nothing is likely, and nothing is unsure)
    const bool none = a.S == 0.0f;
    const float ln = logf(a.S);
    auto logp = [&](float v) { return none ? -INFINITY : (v - a.m) - ln; };
    if (lane == 0 && (c.n_top == 0 || threadIdx.x == 0)) {
        if (c.logprob) c.logprob[t] = has ? logp(x) : without ? 0.0f : NAN;
        if (c.entropy) c.entropy[t] = none ? 0.0f : ln - a.A / a.S;
        if (!has && !without) atomicExch(status, (int)TPQ_ERR_INVALID_ARG);
    }
    if (c.n_top == 0) return;
    for (int i = threadIdx.x; i < c.n * c.n_top; i += 128) {
        const int k = i / c.n_top, p = i - k * c.n_top;
        const uint32_t *const r = c.records[k] + at + HEAD_WORDS;
        const uint32_t key = r[p], index = r[c.n_top + p];
        lists[i] = key ? order_of(key, (int)index) : 0ull;
    }
    __syncthreads();
    unsigned long long *const merged = lists + c.n * c.n_top;
    merge<128>(lists, c.n_top, c.n, c.n_top, reinterpret_cast<int *>(merged + c.n_top), merged);
    if (threadIdx.x < c.n_top) {
        const unsigned long long o = merged[threadIdx.x];
        if (c.top) c.top[t * c.n_top + threadIdx.x] = o ? (int)~(uint32_t)o : -1;
        if (c.top_logprob) c.top_logprob[t * c.n_top + threadIdx.x] = o ? logp(value_of((uint32_t)(o >> 32))) : -INFINITY;
    }
}

template <bool FP32, int THREADS>
cudaError_t launch_stats(const stats_call &c, int split, cudaStream_t st)
{
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
    return cudaLaunchKernelEx(&cfg, token_stats<FP32, THREADS>, c, split);
}

}  // namespace

cudaError_t answers_launch_stats(const stats_call &c, const tpq_block *b, cudaStream_t st, int64_t *launches)
{
    // Few rows: blocks of 512 threads, and a cluster of them for each row as long as all run at once and a block has 4096 values.  Many, or short
    // ones: blocks of 128.
    int split = 1;
    while (split < MOST_SPLIT && c.T * split * 2 <= 2 * b->sm_count && c.n_vocab / (split * 2) >= 4096) split *= 2;
    const bool few = c.T <= 2 * b->sm_count && c.n_vocab / split >= 4096;
    cudaError_t e;
    if (c.fp32) e = few ? launch_stats<true, 512>(c, split, st) : launch_stats<true, 128>(c, split, st);
    else e = few ? launch_stats<false, 512>(c, split, st) : launch_stats<false, 128>(c, split, st);
    if (e == cudaSuccess) ++*launches;
    return e;
}

cudaError_t answers_launch_join(const join_call &c, const tpq_block *b, cudaStream_t st, int64_t *launches)
{
    const int64_t blocks = c.n_top ? c.T : (c.T + 3) / 4;
    const cudaError_t e = tpq_launch_pdl(token_logprobs, dim3((unsigned)blocks), dim3(128), (size_t)(c.n + 1) * c.n_top * 12, st, c, b->status);
    if (e == cudaSuccess) ++*launches;
    return e;
}
