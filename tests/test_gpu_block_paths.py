"""Weights in 4 bits, products, the gated block and answers on the paths that large sizes, long rows and repeated calls take, against 64 bits.

Helpers and worst-case bounds per element are those of test_gpu_block.py."""
import math

import numpy as np
import pytest
import torch

import block_ref
import gpu_util as gu
from paper_2411_07942_b200 import binding
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
