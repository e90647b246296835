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
