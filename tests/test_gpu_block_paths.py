"""Weights in 4 bits, products, the gated block and answers on the paths that large sizes, long rows and repeated calls take, against 64 bits.

Helpers and worst-case bounds per element are those of test_gpu_block.py."""
import ctypes
import math
import os
import subprocess
import threading

import numpy as np
import pytest
import torch

import block_ref
import gpu_util as gu
from paper_2411_07942_b200 import binding, build
from test_gpu_block import bf16, check_product, quantised, rows, up8, weights

pytestmark = pytest.mark.gpu
NAN = math.nan


@pytest.fixture(scope="module", autouse=True)
def _lib():
    gu.ensure_lib()


@pytest.fixture(scope="module")
def block():
    b = binding.TpqBlock()
    yield b
    assert b.device_status() == 0
    b.close()


def some_weights(n, K, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(n, K, generator=g, device="cuda") / math.sqrt(K)).to(torch.bfloat16)


def in_4_bits(block, n, K, group, seed=0):
    """(binding.Weight, its buffer) of some_weights."""
    w = some_weights(n, K, seed)
    w4 = torch.empty(binding.weight4_bytes(n, K, group), dtype=torch.uint8, device="cuda")
    block.quantize_weight(w.data_ptr(), n, K, group, w4.data_ptr(), w4.numel())
    torch.cuda.synchronize()
    return binding.Weight(w4.data_ptr(), n, K, 0, binding.TPQ_WEIGHT_INT4, group), w4


# ------------------------------------------------------------------------------------------------ products
@pytest.mark.parametrize("T", [1, 32])
def test_fp32_products_back_to_back_leave_each_other_alone(block, T):
    """Blocks of a stage or two, each followed on its SM by another call's, whose barriers lie where an arrival that came too late would land."""
    rng = np.random.default_rng(T)
    n, K = 20000, 256
    weight, keep, value = quantised(block, weights(rng, n, K), 64)
    x = bf16(rng.standard_normal((T, K)))
    xd = x.cuda()
    outs = [torch.full((T, n), 7.0, device="cuda") for _ in range(60)]
    small = [torch.zeros(T, n, dtype=torch.bfloat16, device="cuda") for _ in range(60)]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for o, s in zip(outs, small):
        block.linear4(weight, xd.data_ptr(), T, o.data_ptr(), binding.TPQ_OUT_FP32)
        block.linear4(weight, xd.data_ptr(), T, s.data_ptr(), stream=stream.cuda_stream)
    torch.cuda.synchronize()
    want, bound = x.double().cuda() @ value.T, K * 2.0 ** -24 * (x.double().cuda().abs() @ value.abs().T)
    check_product(outs[0], want, bound)
    check_product(small[0], want, bound)
    assert all(torch.equal(o, outs[0]) for o in outs) and all(torch.equal(s, small[0]) for s in small)
    assert block.device_status() == 0


def values_of(block, weight):
    """step * code in 64 bits on the device, read back (exactly)."""
    out = torch.empty(weight.n_out, weight.n_in, dtype=torch.bfloat16, device="cuda")
    block.read_weight(weight.data_ptr, weight.n_out, weight.n_in, weight.group, out.data_ptr())
    return out.double()


@pytest.mark.parametrize("T", [1, 31, 33, 64, 65, 100, 128, 300, 2048])
@pytest.mark.parametrize("n,K", [(1000, 5120), (700, 13825), (40000, 2000)])
def test_sums_are_near_in_norm_whatever_the_number_of_tokens(block, T, n, K):
    """FP32 outputs.  The tensor cores' own sums cut off what does not fit: 4e-9 of the norm for every 16 inputs, measured over 2000 (5e-7).  They add up at most 512 inputs:
    1.28e-7, 2.15 * 2^-24.  The sums of 256 or 512 are added with roundings of at most 2^-24, which have signs of their own, over partial sums that grow like sqrt(j):
    sqrt(K / 512) 2^-24.  One rounding of the product with the row's factor.  In all (3.2 + sqrt(K / 512)) 2^-24 of the norm, 3.8e-7 at 5120 inputs, for one
    token as for thousands (sums cut off over all of these: 1.3e-6).  BF16 outputs: 2^-9 of the norm for the rounding (log-uniform values:
    2^-7 / sqrt(12) / 1.47 = 1.5e-3), and sums that may be cut off over all inputs, twice 4e-9 for every 16."""
    if T * n > 40000 * 300:
        n = 5000
    weight, keep = in_4_bits(block, n, K, 64)
    value = values_of(block, weight)
    x = torch.randn(T, up8(K), generator=torch.Generator("cuda").manual_seed(T), device="cuda").to(torch.bfloat16)
    want = x[:, :K].double() @ value.T
    for kind, dtype, bound in ((torch.float32, binding.TPQ_OUT_FP32, (3.2 + math.sqrt(K / 512)) * 2.0 ** -24),
                               (torch.bfloat16, binding.TPQ_OUT_BF16, 2.0 ** -9 + K / 16 * 8e-9)):
        out = torch.zeros(T, n, dtype=kind, device="cuda")
        block.linear4(weight, x.data_ptr(), T, out.data_ptr(), dtype, x_stride=up8(K))
        err = (out.double() - want).norm() / want.norm()
        print(f"T {T} n {n} K {K} {dtype}: {err:.3g} of the norm, bound {bound:.3g}")
        assert err <= bound


# Sizes at which blocks walk more stages than their ring holds (up to 16), and more than one tile; what runs together on the GPU is at most 296 blocks.
LONG_WALKS = [
    (300, 2304, 3456, 128), (2048, 1280, 3456, 64), (700, 1500, 2000, 32),
    (1, 45000, 1500, 64), (20, 45000, 2500, 32), (40, 40000, 1300, 128), (60, 40000, 2300, 64), (100, 20000, 3000, 64), (200, 25000, 1100, 128),
    (128, 3840, 5120, 64),         # (partial sums of two weights in the place of the stages)
    (3, 700, 36864, 128), (40, 300, 36864, 32)]


def with_lone_terms(T, K, seed):
    """x [T][K]: in each row one input that outweighs all others, at the ends of pieces of 64, 128 and 256 and of shares of the inputs in turn, so that no tolerance hides its absence."""
    x = torch.randn(T, K, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")
    at = sorted({min(K - 1, max(0, p + d)) for p in [0, K, *(64 * round(K * i / 64 / s) for s in (1, 2, 3, 4, 5, 6, 7, 8) for i in range(s)), 64, 128, 256, 512, 1024] for d in (-1, 0)})
    x[torch.arange(T), torch.tensor(at, device="cuda")[torch.arange(T, device="cuda") % len(at)]] = 512.0
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("T,n,K,group", LONG_WALKS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lone", [False, True])
def test_products_of_long_walks(block, T, n, K, group, dtype, lone):
    weight, keep = in_4_bits(block, n, K, group)
    value = values_of(block, weight)
    x = with_lone_terms(T, K, T) if lone else torch.randn(T, K, generator=torch.Generator("cuda").manual_seed(T), device="cuda").to(torch.bfloat16)
    xd = torch.full((T, up8(K)), NAN, dtype=torch.bfloat16, device="cuda")
    xd[:, :K] = x
    out = torch.full((T, n), 7.0, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    again = out.clone()
    for o in (out, again):
        block.linear4(weight, xd.data_ptr(), T, o.data_ptr(), binding.TPQ_OUT_BF16 if dtype == "bf16" else binding.TPQ_OUT_FP32, x_stride=up8(K))
    xl = x.double()
    check_product(out, xl @ value.T, K * 2.0 ** -24 * (xl.abs() @ value.abs().T))
    assert torch.equal(out, again)


@pytest.mark.parametrize("T,n,K,group", LONG_WALKS)
@pytest.mark.parametrize("bf16_weights", [False, True])
@pytest.mark.parametrize("lone", [False, True])
def test_gated_blocks_of_long_walks(block, T, n, K, group, bf16_weights, lone):
    if bf16_weights:
        keep = [torch.nn.functional.pad(some_weights(n, K, seed), (0, up8(K) - K)) for seed in range(2)]
        made = [binding.Weight(w.data_ptr(), n, K, up8(K), binding.TPQ_WEIGHT_BF16, 0) for w in keep]
        value = [w[:, :K].double() for w in keep]
    else:
        made, keep = zip(*[in_4_bits(block, n, K, group, seed) for seed in range(2)])
        value = [values_of(block, w) for w in made]
    x = with_lone_terms(T, K, T) if lone else torch.randn(T, K, generator=torch.Generator("cuda").manual_seed(T), device="cuda").to(torch.bfloat16)
    xd = torch.full((T, up8(K)), NAN, dtype=torch.bfloat16, device="cuda")
    xd[:, :K] = x
    out = torch.full((T, n), 7.0, dtype=torch.bfloat16, device="cuda")
    again = out.clone()
    for o in (out, again):
        block.gated(*made, binding.TPQ_ACT_SILU, xd.data_ptr(), T, o.data_ptr(), x_stride=up8(K))
    want, bound = block_ref.gated(x.double(), *value, 0)
    check_product(out, want, bound)
    assert torch.equal(out, again)
    if not lone:
        # (of the norm: the rounding to BF16; the sums, cut off over all inputs, of gate and up)
        assert (out.double() - want).norm() <= (2.0 ** -9 + 3 * K / 16 * 8e-9) * want.norm()


# ------------------------------------------------------------------------------------------------ weights
LOOP = """
#include <stdint.h>
#include <stddef.h>
#include "tpq.h"
/* calls that follow one another without anything in between; how many failed */
int64_t loop(tpq_block *b, const void *w, int64_t n, int64_t k, void *w4, size_t capacity, void *stream, int64_t count)
{
    int64_t failed = 0;
    for (int64_t i = 0; i < count; ++i) failed += tpq_quantize_weight(b, w, k, n, k, 32, w4, capacity, stream) != TPQ_OK;
    return failed;
}
"""


def test_threads_with_a_handle_each_quantise_side_by_side(tmp_path):
    """Rows that need more shared memory than others, in the same kernel: no thread's calls take anything from another's."""
    src, so = tmp_path / "loop.c", tmp_path / "loop.so"
    src.write_text(LOOP)
    subprocess.run(["gcc", "-O2", "-shared", "-fPIC", f"-I{build.INCLUDE}", str(src), str(build.LIB), f"-Wl,-rpath,{build.LIB.parent}", "-o", str(so)], check=True)
    loop = ctypes.CDLL(str(so)).loop
    loop.restype = ctypes.c_int64
    loop.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int64] * 2 + [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int64]
    sizes = [(8, 2 ** 17), (8, 5248), (8, 6000), (8, 9000)]
    b = [binding.TpqBlock() for _ in sizes]
    w = [torch.ones(n, K, dtype=torch.bfloat16, device="cuda") for n, K in sizes]
    cap = [binding.weight4_bytes(n, K, 32) for n, K in sizes]
    w4 = [torch.zeros(c, dtype=torch.uint8, device="cuda") for c in cap]
    streams = [torch.cuda.Stream() for _ in sizes]
    torch.cuda.synchronize()
    failed = [None] * len(sizes)
    start = threading.Barrier(len(sizes))

    def run(i):
        start.wait()
        failed[i] = loop(b[i]._h, w[i].data_ptr(), *sizes[i], w4[i].data_ptr(), cap[i], streams[i].cuda_stream, 3000)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(sizes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert failed == [0] * len(sizes), [binding.lib().tpq_block_last_error(x._h) for x in b]
    for i, (n, K) in enumerate(sizes):
        codes, byte, factor = block_ref.quantise(np.ones((n, K)), 32)
        assert np.array_equal(w4[i].cpu().numpy(), block_ref.pack(codes, byte, factor, 32))
        b[i].close()


@pytest.mark.parametrize("n,K,group,pad,offset", [(5, 5121, 32, 0, 0), (3, 9216, 128, 0, 8), (130, 9216, 64, 8, 8), (7, 13824, 32, 0, 8), (4, 14337, 64, 3, 1), (2, 36864, 128, 0, 3), (3, 2 ** 17, 32, 0, 8),
                                                  (2, 2 ** 17 - 1, 64, 2, 2), (1, 98305, 32, 7, 0)])
def test_long_rows_in_4_bits_are_the_bytes_of_the_definition(block, n, K, group, pad, offset):
    """Rows that are read twice, aligned or not, above 48 KB of shared memory too (groups of 32 of more than 98304 inputs)."""
    rng = np.random.default_rng(K)
    w = weights(rng, n, K)
    if n > 2:
        w[1] = bf16(rng.standard_normal(K) * np.exp(8 * rng.standard_normal(K)))
        w[2, K - 1] = math.inf
    if n > 3:
        w[3, : K - 1] = 0
    buf, ptr = rows(w, K + pad, offset)
    size = binding.weight4_bytes(n, K, group)
    whole, w4 = gu.guarded(size)
    block.quantize_weight(ptr, n, K, group, w4.data_ptr(), size, row_stride=K + pad)
    out = torch.full((n * (K + pad) + 1,), 7.0, dtype=torch.bfloat16, device="cuda")
    block.read_weight(w4.data_ptr(), n, K, group, out.data_ptr() + 2 * (offset % 2), out_stride=K + pad)
    torch.cuda.synchronize()
    codes, byte, factor = block_ref.quantise(w.double().numpy(), group)
    assert np.array_equal(w4.cpu().numpy(), block_ref.pack(codes, byte, factor, group)) and gu.guards_intact(whole, size)
    got = out[offset % 2: offset % 2 + n * (K + pad)].view(n, K + pad)
    value = block_ref.values(codes, byte, factor, group)
    assert np.array_equal(got[:, :K].double().cpu().numpy(), value, equal_nan=True)
    assert (got[:, K:] == 7).all()


# ------------------------------------------------------------------------------------------------ answers
def exact_answers(x, n_top):
    """x [T][V] on the device -> log probabilities (64 bits), entropy, the n_top largest (lowest index first), and per row sum p |x - m| and sum p (x - m)^2."""
    got = [[], [], [], [], []]
    for part in x.split(max(1, (1 << 26) // x.shape[1])):
        p = part.double()
        d = p - p.amax(1, keepdim=True)
        logp = torch.log_softmax(p, 1)
        prob = logp.exp()
        d = torch.where(torch.isneginf(d), torch.zeros_like(d), d)
        got[0].append(logp), got[1].append(torch.special.entr(prob).sum(1)), got[3].append((prob * d.abs()).sum(1)), got[4].append((prob * d * d).sum(1))
        got[2].append(torch.argsort(p, dim=1, descending=True, stable=True)[:, :n_top])
    return [torch.cat(g) for g in got]


class Answers:
    """A row's logits on one device: the calls and where their results go."""

    def __init__(self, T, V, n_top):
        self.T, self.V, self.n_top = T, V, n_top
        self.record = torch.full((binding.token_record_bytes(T, n_top),), 0xA5, dtype=torch.uint8, device="cuda")
        self.logprob, self.entropy = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
        self.top, self.top_logprob = torch.full((T, n_top), 7, dtype=torch.int32, device="cuda"), torch.full((T, n_top), 7.0, device="cuda")

    def run(self, block, x, tokens, stream=0):
        dtype = binding.TPQ_OUT_BF16 if x.dtype == torch.bfloat16 else binding.TPQ_OUT_FP32
        block.token_stats(x.data_ptr(), self.T, self.V, self.record.data_ptr(), self.record.numel(), dtype=dtype, stride=x.stride(0), tokens_ptr=tokens.data_ptr(), n_top=self.n_top, stream=stream)
        block.token_logprobs([self.record.data_ptr()], self.T, self.logprob.data_ptr(), self.entropy.data_ptr(), self.n_top, self.top.data_ptr() if self.n_top else None,
                             self.top_logprob.data_ptr() if self.n_top else None, stream=stream)

    def results(self):
        return [t.clone() for t in (self.logprob, self.entropy, self.top, self.top_logprob)]


def check_in_norm(got, x, tokens, n_top):
    """With u = 2^-24: x - m is off by u of itself, the exponential's argument by as much again, the exponential by 4u; a thread's sums (of V / 256 terms at least two
    at a time) by roundings that have signs of their own, below 2u of the whole; a logarithm, a difference and their sum by 2u of their sizes.  So ln S is off by
    (2 sum p |x - m| + 6) u, log p by 2 |log p| u more, and the entropy, whose A / S = sum p (x - m) has terms |x - m| times as far off, by
    (2 sum p (x - m)^2 + 8 sum p |x - m| + 8) u beside ln S's.  Of the norm over the rows."""
    logp, entropy, top, first, second = exact_answers(x, n_top)
    u = 2.0 ** -24
    want = logp.gather(1, tokens.long()[:, None])[:, 0]
    lns = (2 * first + 6) * u

    def near(a, b, bound):
        assert (a.double() - b).norm() <= bound.norm(), ((a.double() - b).norm() / bound.norm()).item()

    near(got[0], want, lns + 2 * want.abs() * u)
    near(got[1], entropy, lns + (2 * second + 8 * first + 8) * u)
    assert torch.equal(got[2].long(), top)
    if n_top:
        best = logp.gather(1, top)
        near(got[3], best, lns[:, None] + 2 * best.abs() * u)


@pytest.mark.parametrize("T,V,n_top", [(2048, 32000, 0), (300, 32000, 20), (61, 64000, 20), (7, 128256, 32), (1000, 1003, 5), (100, 256000, 32), (299, 256000, 20), (400, 262144, 32), (2, 5000000, 32), (1, 2500001, 1)])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_answers_are_near_in_norm(block, T, V, n_top, kind):
    """From rows that a thread walks once to such as have more rounds of it than there is room for their maxima (100 and more of 256000 in FP32, millions of columns)."""
    g = torch.Generator("cuda").manual_seed(T + V)
    x = torch.empty(T, V, dtype=kind, device="cuda")
    for a in range(0, T, 64):
        part = torch.randn(min(64, T - a), V, generator=g, device="cuda")
        x[a: a + 64] = part * (1 + 2 * torch.rand(part.shape[0], 1, generator=g, device="cuda"))
    tokens = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    a = Answers(T, V, n_top)
    a.run(block, x, tokens)
    got = a.results()
    some = torch.arange(T, device="cuda") if T * V < 1 << 25 else torch.unique(torch.cat([torch.tensor([0, T - 1], device="cuda"), torch.randint(0, T, (40,), generator=g, device="cuda")]))
    check_in_norm([v[some] for v in got], x[some], tokens[some], n_top)


@pytest.mark.parametrize("T,V,n_top", [(1, 32000, 20), (61, 64000, 20), (500, 8000, 5), (2048, 2000, 0)])
def test_answers_on_two_streams_and_in_a_graph(block, T, V, n_top):
    """Calls side by side with buffers of their own, then captured and replayed over new logits: the bits of calls one by one."""
    g = torch.Generator("cuda").manual_seed(T)
    xs = [(torch.randn(T, V, generator=g, device="cuda") * 3).to(torch.bfloat16) for _ in range(3)]
    tokens = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    want = []
    for x in xs:
        a = Answers(T, V, n_top)
        a.run(block, x, tokens)
        want.append(a.results())
        check_in_norm(want[-1], x, tokens, n_top)
    streams, sets = [torch.cuda.Stream() for _ in range(2)], [Answers(T, V, n_top) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(30):
        for i in range(2):
            sets[i].run(block, xs[i], tokens, streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(sets[i].results(), want[i]))
    x, a, b = xs[2].clone(), Answers(T, V, n_top), Answers(T, V, n_top)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run(block, x, tokens, torch.cuda.current_stream().cuda_stream)
    for i in (0, 2, 1):
        x.copy_(xs[i])
        graph.replay()
        b.run(block, xs[i - 1], tokens)           # (an eager call with buffers of its own behind it)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a.results(), want[i])) and all(torch.equal(p, q) for p, q in zip(b.results(), want[i - 1]))


# ------------------------------------------------------------------------------------------------ waits that expire
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
@pytest.fixture(scope="module")
def expiring(tmp_path_factory):
    """The library, built so that waits for a parity expire that are not over at the first look (parities -> library)."""
    out = tmp_path_factory.mktemp("expiring")
    flags = [f for f in build.NVCC_FLAGS] + [f"-I{build.INCLUDE}", f"-I{build.CSRC}"]
    jobs = {f"products{m}": ["products.cu", f"-DTPQ_GIVE_UP={m}"] for m in (1, 2, 3)}
    jobs |= {f"{s.stem}": [s.name] for s in build.sources() if s.stem != "products" and not (build.OBJ / f"{s.stem}.o").exists()}
    running = [subprocess.Popen([NVCC, *flags, "-c", str(build.CSRC / f[0]), *f[1:], "-o", str(out / f"{name}.o")])
               for name, f in jobs.items()]
    assert [p.wait() for p in running] == [0] * len(running)
    rest = [str(o if (o := build.OBJ / f"{s.stem}.o").exists() else out / f"{s.stem}.o") for s in build.sources() if s.stem != "products"]
    libs = {}
    for m in (1, 2, 3):
        so = out / f"expiring{m}.so"
        subprocess.run([NVCC, *build.LINK_FLAGS, "-o", str(so), str(out / f"products{m}.o"), *rest], check=True)
        libs[m] = ctypes.CDLL(str(so))
        for name, (res, args) in binding.SIGNATURES.items():
            f = getattr(libs[m], name)
            f.restype, f.argtypes = res, args
    return libs


EXPIRING = [
    (1, 5120, 1728, 64, 0),          # a tile over a cluster, two blocks an SM
    (1, 45000, 700, 32, 0), (1, 45000, 700, 32, 1), (20, 40000, 1300, 128, 1),     # several tiles a block, two blocks an SM
    (60, 40000, 640, 64, 0), (60, 2000, 4096, 64, 1),
    (300, 2304, 3456, 128, 0), (300, 2304, 3456, 128, 1), (2048, 1280, 3456, 64, 0), (2048, 1280, 3456, 64, 1)]


@pytest.mark.parametrize("gated,T,n,K,group,out_fp32", [(None, *c) for c in EXPIRING] + [(g, *c) for g in (0, 64) for c in EXPIRING if not c[4]])
@pytest.mark.parametrize("parities", [1, 2, 3])
def test_waits_that_expire_leave_everything_in_order(block, expiring, parities, gated, T, n, K, group, out_fp32):
    """Every role of the kernels gives up where it does not find at once what it waits for, at the beginning (parity 0) or in the midst of its walk: the
    status says so, nothing wrong is stored, nothing is written beside the output, and calls that follow are as ever.  The limits by which copies and
    MMAs under way are waited for at the end are the shipped ones."""
    L, rng = expiring[parities], np.random.default_rng(T + n + K)
    handle = ctypes.c_void_p()
    assert L.tpq_block_create(ctypes.byref(handle)) == 0
    x = bf16(rng.standard_normal((T, K)))
    xbuf, xptr = rows(x, up8(K))
    n_weights = 1 if gated is None else 2
    if gated == 0:
        keep = [torch.nn.functional.pad(some_weights(n, K, seed), (0, up8(K) - K)) for seed in range(2)]
        made = [binding.Weight(w.data_ptr(), n, K, up8(K), binding.TPQ_WEIGHT_BF16, 0) for w in keep]
    else:
        made, keep = zip(*[in_4_bits(block, n, K, gated or group, seed) for seed in range(n_weights)])
    kind = torch.float32 if out_fp32 else torch.bfloat16

    def call(lib, h, out):
        if gated is None:
            return lib.tpq_linear4(h, made[0], xptr, up8(K), T, out.data_ptr(), out_fp32, n, None)
        return lib.tpq_gated(h, made[0], made[1], 0, xptr, up8(K), T, out.data_ptr(), n, None)

    want = torch.zeros(T, n, dtype=kind, device="cuda")
    assert call(binding.lib(), block._h, want) == 0 and block.device_status() == 0
    for _ in range(5):
        whole = torch.full((2 * 4096 + T * n,), 7.0, dtype=kind, device="cuda")
        got = whole[4096: 4096 + T * n].view(T, n)
        assert call(L, handle, got) == 0
        status = L.tpq_block_device_status(handle)
        assert status in ((binding.TPQ_ERR_TIMEOUT,) if parities & 1 else (0, binding.TPQ_ERR_TIMEOUT))
        assert ((got == want) | (got == 7.0)).all() and (status or torch.equal(got, want))
        assert (whole[:4096] == 7.0).all() and (whole[4096 + T * n:] == 7.0).all()
        again = torch.zeros(T, n, dtype=kind, device="cuda")
        assert call(binding.lib(), block._h, again) == 0 and block.device_status() == 0
        assert torch.equal(again, want)
    assert L.tpq_block_destroy(handle) == 0
