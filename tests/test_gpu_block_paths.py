"""Weights in 4 bits, products, the gated block and answers on the paths that large sizes, long rows and repeated calls take, against 64 bits.

Helpers and worst-case bounds per element are those of test_gpu_block.py."""
import ctypes
import math
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
