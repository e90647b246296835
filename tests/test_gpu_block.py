"""Weights in 4 bits, products with them, the gated feed-forward block and answers, through the C ABI, against 64 bits.

Tolerances.  A product's sum of K terms in binary32: K 2^-24 sum |x w| (each partial sum rounded once); BF16 output: 2^-8 of the value more.  The gated
block: block_ref.gated carries the sums' bounds through the activation (|slope| <= 1.13).  Answers: see check_answers."""
import math

import numpy as np
import pytest
import torch

import block_ref
import gpu_util as gu
from paper_2411_07942_b200 import binding

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


def bf16(a) -> torch.Tensor:
    return torch.as_tensor(np.asarray(a, np.float32)).to(torch.bfloat16)


def weights(rng, n, K):
    w = rng.standard_normal((n, K)) * np.exp(0.5 * rng.standard_normal((n, 1))) / math.sqrt(K)
    w[rng.random((n, K)) < 0.003] *= 8
    return bf16(w)


def rows(t: torch.Tensor, stride: int, offset: int = 0):
    """t's rows `stride` apart on the device, NaN in the gaps; (buffer, pointer)."""
    buf = torch.full((offset + t.shape[0] * stride,), NAN, dtype=t.dtype, device="cuda")
    buf[offset:].view(t.shape[0], stride)[:, : t.shape[1]] = t.cuda()
    return buf, buf.data_ptr() + offset * t.element_size()


def up8(n):
    return (n + 7) // 8 * 8


def quantised(block, w: torch.Tensor, group: int):
    """(binding.Weight, its buffer, values in 64 bits on the device)."""
    n, K = w.shape
    size = binding.weight4_bytes(n, K, group)
    buf = torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")
    wd = w.cuda()
    block.quantize_weight(wd.data_ptr(), n, K, group, buf.data_ptr(), size)
    codes, byte, factor = block_ref.quantise(w.double().numpy(), group)
    return binding.Weight(buf.data_ptr(), n, K, 0, binding.TPQ_WEIGHT_INT4, group), buf, torch.from_numpy(block_ref.values(codes, byte, factor, group)).cuda()


# ------------------------------------------------------------------------------------------------ weights
@pytest.mark.parametrize("n,K,group,pad", [(1, 1, 32, 0), (128, 128, 32, 0), (130, 257, 64, 0), (5, 1000, 128, 3), (300, 96, 64, 8), (64, 2049, 32, 7), (257, 4608, 128, 0)])
def test_quantised_weights_are_the_bytes_of_the_definition(block, n, K, group, pad):
    rng = np.random.default_rng(n + K)
    w = weights(rng, n, K)
    if n > 4:
        w[1] = 0
        w[2, : K // 2] = 0
        w[3, :] = bf16(rng.standard_normal(K) * np.exp(8 * rng.standard_normal(K)))      # steps more than 2^15 apart
        w[4, :] = bf16(7.5 * 2.0 ** rng.integers(-3, 3, K))                               # ties, steps that need no rounding
    buf, ptr = rows(w, K + pad, 1)
    size = binding.weight4_bytes(n, K, group)
    whole, w4 = gu.guarded(size)
    block.quantize_weight(ptr, n, K, group, w4.data_ptr(), size, row_stride=K + pad)
    out = torch.full((n, K + pad), NAN, dtype=torch.bfloat16, device="cuda")
    block.read_weight(w4.data_ptr(), n, K, group, out.data_ptr(), out_stride=K + pad)
    torch.cuda.synchronize()
    codes, byte, factor = block_ref.quantise(w.double().numpy(), group)
    want = block_ref.pack(codes, byte, factor, group)
    assert want.size == size and gu.guards_intact(whole, size)
    assert np.array_equal(w4.cpu().numpy(), want)
    value = block_ref.values(codes, byte, factor, group)
    assert np.array_equal(out[:, :K].double().cpu().numpy(), value)
    assert out[:, K:].isnan().all()
    step = np.repeat(factor[:, None] * 2.0 ** ((byte >> 4) - 8.0) * (1 + (byte & 15) / 16), group, 1)[:, :K]
    assert (np.abs(value - w.double().numpy()) <= step / 2).all()


def test_rows_of_weights_that_are_no_numbers_or_tiny(block):
    w = np.ones((140, 70), np.float32)
    w[1, 3], w[2, 69], w[129, 0], w[130, 1] = NAN, math.inf, -math.inf, 2.0 ** 120
    w[3], w[4] = 2.0 ** -100, 2.0 ** -126
    w[5, 0] = 2.0 ** 119
    w = bf16(w)
    size = binding.weight4_bytes(140, 70, 32)
    w4 = torch.empty(size, dtype=torch.uint8, device="cuda")
    wd = w.cuda()
    block.quantize_weight(wd.data_ptr(), 140, 70, 32, w4.data_ptr(), size)
    codes, byte, factor = block_ref.quantise(w.double().numpy(), 32)
    assert np.array_equal(w4.cpu().numpy(), block_ref.pack(codes, byte, factor, 32))
    assert sorted(np.flatnonzero(np.isnan(factor))) == [1, 2, 129, 130]
    x = torch.ones(2, 72, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros(2, 140, device="cuda")
    weight = binding.Weight(w4.data_ptr(), 140, 70, 0, binding.TPQ_WEIGHT_INT4, 32)
    block.linear4(weight, x.data_ptr(), 2, out.data_ptr(), binding.TPQ_OUT_FP32, x_stride=72)
    bad = torch.zeros(140, dtype=torch.bool, device="cuda")
    bad[[1, 2, 129, 130]] = True
    assert torch.equal(out.isnan(), bad.expand(2, 140))
    want = torch.from_numpy(block_ref.values(codes, byte, factor, 32)).cuda().sum(1)
    assert ((out[0].double() - want).abs() <= 70 * 2.0 ** -24 * want.abs() + 2.0 ** -149)[~bad].all()


# ------------------------------------------------------------------------------------------------ products
def check_product(out, want, bound):
    err = (out.double() - want).abs()
    assert (err <= bound + want.abs() * (2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24)).all(), f"largest error {((err - bound) / want.abs()).max():.3g}"


@pytest.mark.parametrize("T,n,K,group", [
    (1, 1, 1, 32), (1, 128, 128, 32), (1, 5120, 1728, 64), (1, 200, 5000, 128), (2, 130, 100, 64), (16, 128, 640, 32), (17, 257, 300, 128), (33, 640, 1024, 64),
    (61, 1000, 2000, 32), (100, 129, 4096, 128), (160, 1280, 512, 64), (192, 300, 200, 32), (193, 512, 700, 64), (300, 2304, 384, 128), (700, 1111, 256, 32),
    (2050, 640, 333, 64), (5000, 130, 130, 32), (1, 20000, 129, 32), (31, 20000, 130, 128), (1200, 5120, 256, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_products_with_4_bit_weights(block, T, n, K, group, dtype):
    rng = np.random.default_rng(T + n + K)
    weight, keep, value = quantised(block, weights(rng, n, K), group)
    x = bf16(rng.standard_normal((T, K)))
    xbuf, xptr = rows(x, up8(K) + 8 * (T % 3), 8)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    stride = n + T % 5
    out = torch.full((T * stride + 2,), 7.0, dtype=kind, device="cuda")
    block.linear4(weight, xptr, T, out.data_ptr() + out.element_size(), binding.TPQ_OUT_BF16 if dtype == "bf16" else binding.TPQ_OUT_FP32,
                  x_stride=up8(K) + 8 * (T % 3), out_stride=stride)
    got = out[1: 1 + T * stride].view(T, stride)
    xd = x.double().cuda()
    check_product(got[:, :n], xd @ value.T, K * 2.0 ** -24 * (xd.abs() @ value.abs().T))
    assert (got[:, n:] == 7).all() and out[0] == 7 and out[-1] == 7


@pytest.mark.parametrize("T,n,K", [(1, 1, 1), (1, 128, 64), (1, 1728, 5120), (3, 130, 100), (16, 200, 1000), (33, 640, 777), (61, 1152, 2048), (128, 257, 300),
                                   (200, 1000, 520), (256, 128, 128), (257, 384, 640), (700, 300, 130), (2050, 700, 96), (40, 20000, 72), (1100, 2600, 200)])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("group", [0, 32, 128])
def test_gated_blocks(block, T, n, K, act, group):
    rng = np.random.default_rng(T + n + K + act)
    x = bf16(rng.standard_normal((T, K)) * 2)
    xbuf, xptr = rows(x, up8(K) + 8 * (T % 3))
    made, keep, value = [], [], []
    for i in range(2):
        w = weights(rng, n, K)
        if group:
            m, k, v = quantised(block, w, group)
        else:
            k, ptr = rows(w, up8(K) + 16 * i)
            m, v = binding.Weight(ptr, n, K, up8(K) + 16 * i, binding.TPQ_WEIGHT_BF16, 0), w.double().cuda()
        made.append(m), keep.append(k), value.append(v)
    stride = n + T % 3
    out = torch.full((T, stride), 7.0, dtype=torch.bfloat16, device="cuda")
    block.gated(*made, act, xptr, T, out.data_ptr(), x_stride=up8(K) + 8 * (T % 3), out_stride=stride)
    want, bound = block_ref.gated(x.double().cuda(), *value, act)
    check_product(out[:, :n], want, bound)
    assert (out[:, n:] == 7).all()


@pytest.mark.parametrize("act", [0, 1, 2])
def test_activations_over_their_range(block, act):
    """x = e_i times values from -100 to 100 as the gate, up = 1: the activation itself."""
    n, K = 300, 64
    g = bf16(np.concatenate([np.linspace(-100, 100, 200), np.linspace(-8, 8, 96), [0.0, -0.0, 1e-30, -3e38]]))
    wg = torch.zeros(n, K, dtype=torch.bfloat16)
    wg[:, 0] = g
    wu = torch.zeros(n, K, dtype=torch.bfloat16)
    wu[:, 1] = 1
    x = torch.zeros(1, K, dtype=torch.bfloat16)
    x[0, :2] = 1
    wg, wu, x = wg.cuda(), wu.cuda(), x.cuda()
    out = torch.zeros(1, n, dtype=torch.bfloat16, device="cuda")
    made = [binding.Weight(w.data_ptr(), n, K, K, binding.TPQ_WEIGHT_BF16, 0) for w in (wg, wu)]
    block.gated(*made, act, x.data_ptr(), 1, out.data_ptr())
    want = block_ref.act(g.double(), act)
    if act == 1:        # (the tail without the cancellation that tanh has)
        z = math.sqrt(2 / math.pi) * (g.double() + 0.044715 * g.double() ** 3)
        want = torch.where(g.double() < -60, torch.zeros(n, dtype=torch.float64), g.double() / (1 + torch.exp(-2 * z)))
    got = out[0].double().cpu()
    # the exponential's argument is rounded, which the result feels |argument| times; below 2^-100 it may be 0
    arg = {0: g.double().abs(), 1: (1.6 * g.double().abs() * (1 + 0.0448 * g.double() ** 2)).clamp(max=200), 2: (g.double() ** 2).clamp(max=200)}[act]
    assert ((got - want).abs() <= want.abs() * (2.0 ** -8 + (8 + 3 * arg) * 2.0 ** -23) + 2.0 ** -100 * 1.01).all()


def test_rows_that_are_no_numbers_stay_alone(block):
    rng = np.random.default_rng(5)
    T, n, K = 70, 200, 300
    x = bf16(rng.standard_normal((T, K)))
    x[3, 17], x[64, 299], x[69, 0] = NAN, math.inf, -math.inf
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[[3, 64, 69]] = True
    xbuf, xptr = rows(x, up8(K))
    w4, keep, value = quantised(block, weights(rng, n, K), 64)
    out = torch.zeros(T, n, device="cuda")
    block.linear4(w4, xptr, T, out.data_ptr(), binding.TPQ_OUT_FP32, x_stride=up8(K))
    assert torch.equal(~out.isfinite(), bad[:, None].expand(T, n))
    clean = torch.where(bad.cpu()[:, None], 0, x).double().cuda()
    check_product(out[~bad], (clean @ value.T)[~bad], (K * 2.0 ** -24 * (clean.abs() @ value.abs().T))[~bad])
    h = torch.zeros(T, n, dtype=torch.bfloat16, device="cuda")
    block.gated(w4, w4, 0, xptr, T, h.data_ptr(), x_stride=up8(K))
    assert h[~bad].isfinite().all() and (~h[bad].isfinite()).any(1).all()


def test_the_same_call_gives_the_same_bits_on_any_stream_and_in_a_graph(block):
    rng = np.random.default_rng(6)
    for T, n, K in ((1, 640, 4096), (40, 640, 4096), (1500, 640, 512)):
        gate, k0, _ = quantised(block, weights(rng, n, K), 64)
        down, k1, _ = quantised(block, weights(rng, 256, n), 32)
        x = bf16(rng.standard_normal((T, K))).cuda()
        def run(h, y, stream):
            block.gated(gate, gate, 0, x.data_ptr(), T, h.data_ptr(), stream=stream)
            block.linear4(down, h.data_ptr(), T, y.data_ptr(), binding.TPQ_OUT_FP32, stream=stream)
        outs = [(torch.zeros(T, n, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, 256, device="cuda")) for _ in range(4)]
        torch.cuda.synchronize()
        run(*outs[0], 0)
        s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
        for _ in range(20):   # two streams at once
            run(*outs[1], s1.cuda_stream)
            run(*outs[2], s2.cuda_stream)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(*outs[3], torch.cuda.current_stream().cuda_stream)
        for _ in range(3):
            outs[3][1].zero_()
            graph.replay()
        torch.cuda.synchronize()
        for h, y in outs[1:]:
            assert torch.equal(h, outs[0][0]) and torch.equal(y, outs[0][1])


# ------------------------------------------------------------------------------------------------ answers
def run_answers(block, parts, tokens, n_top, dtype, firsts=None, pad=0, offset=0):
    T = parts[0].shape[0]
    size = binding.token_record_bytes(T, n_top)
    tok = None if tokens is None else torch.as_tensor(tokens, dtype=torch.int32).cuda()
    keep, records, first = [], [], 0
    for i, p in enumerate(parts):
        buf, ptr = rows(p, p.shape[1] + pad, offset)
        r = torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")
        block.token_stats(ptr, T, p.shape[1], r.data_ptr(), size, dtype=dtype, stride=p.shape[1] + pad, first=first if firsts is None else firsts[i],
                          tokens_ptr=None if tok is None else tok.data_ptr(), n_top=n_top)
        first += p.shape[1]
        keep.append(buf), records.append(r)
    logprob, entropy = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
    top, top_logprob = torch.full((T, n_top), 7, dtype=torch.int32, device="cuda"), torch.full((T, n_top), 7.0, device="cuda")
    block.token_logprobs([r.data_ptr() for r in records], T, logprob.data_ptr(), entropy.data_ptr(), n_top, top.data_ptr() if n_top else None,
                         top_logprob.data_ptr() if n_top else None)
    torch.cuda.synchronize()
    return logprob.cpu().double(), entropy.cpu().double(), top.cpu(), top_logprob.cpu().double()


def check_answers(got, x, tokens, n_top):
    """A difference x - m is off by 2^-24 of itself and an exponential by that and 4 units more; the sum of V of them by V / 32 roundings at most of
    its own (a thread's share, then a tree): ln S by (V / 32 + 8) 2^-24, and log p by a rounding of x - m and of itself.
    The entropy: A / S = sum p (x - m) feels the same relative errors, its terms are at most |x - m|: sum p |x - m| (V / 32 + 8) 2^-24 beside ln S's."""
    T, V = x.shape
    want = block_ref.answers(x, [-1] * T if tokens is None else tokens, n_top)
    sums = (V / 32 + 16) * 2.0 ** -24
    m = x.amax(1)
    d = torch.where(torch.isneginf(m)[:, None], torch.zeros_like(x), (x - m[:, None]).clamp(min=-1e4))
    spread = (torch.softmax(torch.where(torch.isneginf(m)[:, None], torch.zeros_like(x), x), 1) * d.abs()).sum(1)

    def near(a, b, bound):
        return ((a == b) | ((a - b).abs() <= bound)).all()

    assert near(got[0], want[0], sums + want[0].abs() * 2.0 ** -22)
    assert near(got[1], want[1], sums * (2 + spread) + want[1].abs() * 2.0 ** -22)
    assert torch.equal(got[2], want[2])
    assert near(got[3], want[3], sums + want[3].abs() * 2.0 ** -22)


@pytest.mark.parametrize("T,V,n_top", [(1, 1, 0), (1, 1, 1), (1, 40, 32), (1, 32000, 20), (3, 300, 20), (5, 1023, 32), (1, 256000, 32), (17, 50257, 5), (61, 8000, 20),
                                       (300, 1000, 1), (1000, 130, 0), (2, 100000, 32), (148, 4100, 7), (700, 9000, 20)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_answers(block, T, V, n_top, dtype):
    rng = np.random.default_rng(T + V)
    x = torch.from_numpy(rng.standard_normal((T, V)) * rng.uniform(0.5, 6, (T, 1))).float()
    if V > 100:
        x[:, rng.random(V) < 0.2] = -math.inf
    kind, code = (torch.bfloat16, binding.TPQ_OUT_BF16) if dtype == "bf16" else (torch.float32, binding.TPQ_OUT_FP32)
    x = x.to(kind)
    tokens = rng.integers(0, V, T)
    tokens[::7] = -1
    got = run_answers(block, [x], tokens, n_top, code, pad=T % 3, offset=V % 5)
    check_answers(got, x.double(), tokens, n_top)


@pytest.mark.parametrize("shares,n_top", [((8, 8, 8, 9), 32), ((1, 1, 1), 5), ((4000, 1, 4000), 20), ((32000,) * 8, 20), ((64,) * 64, 32), ((100, 30), 32)])
def test_answers_over_devices(block, shares, n_top):
    rng = np.random.default_rng(len(shares))
    T, V = 9, sum(shares)
    x = torch.from_numpy(rng.standard_normal((T, V)) * 3).to(torch.bfloat16)        # (BF16: many equal ones, on different devices)
    x[2, : shares[0]] = -math.inf                                                     # a device with nothing
    tokens = rng.integers(0, V, T)
    got = run_answers(block, list(x.split(shares, 1)), tokens, min(n_top, V), binding.TPQ_OUT_BF16)
    check_answers(got, x.double(), tokens, min(n_top, V))


def arrangements():
    V = 20000
    asc = torch.linspace(-5, 5, V)
    late = torch.full((V,), -3.0)
    late[-1] = 4
    strided = torch.zeros(V)
    strided[::2048] = 5 + torch.arange(len(strided[::2048])) / 100
    one_thread = torch.randn(V, generator=torch.Generator().manual_seed(1))
    for v in range(0, V // 8, 256):
        one_thread[8 * v + 24: 8 * v + 32] += 20
    few = torch.full((V,), -math.inf)
    few[[5, 19990, 777]] = torch.tensor([1.0, 2.0, 1.0])
    lowest = torch.full((V,), torch.finfo(torch.bfloat16).min)
    some = lowest.clone()
    some[[3, 9000]] = 1.0
    mixed = lowest.clone()
    mixed[::2] = -math.inf
    return {"equal": torch.zeros(V), "ascending": asc, "descending": asc.flip(0), "last": late, "strided": strided, "one_thread": one_thread, "few": few,
            "none": torch.full((V,), -math.inf), "lowest": lowest, "some_lowest": some, "lowest_and_out": mixed, "zeros": torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0),
            "wide": torch.where(torch.arange(V) % 3 == 0, 3e38, -3e38)}


@pytest.mark.parametrize("name", sorted(arrangements()))
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n_top", [1, 32])
@pytest.mark.parametrize("T", [1, 400])
def test_answers_of_rows_arranged_against_the_search(block, name, dtype, n_top, T):
    kind, code = (torch.bfloat16, binding.TPQ_OUT_BF16) if dtype == "bf16" else (torch.float32, binding.TPQ_OUT_FP32)
    x = arrangements()[name].to(kind)[None].repeat(T, 1)
    tokens = [5] * T
    got = run_answers(block, [x], tokens, n_top, code)
    if T > 1:
        assert all(torch.equal(g[:1].expand_as(g), g) for g in got)
    check_answers([g[:1] for g in got], x[:1].double(), tokens[:1], n_top)


def test_more_large_values_in_a_threads_share_than_its_list_holds(block):
    """17 of 256 threads have nothing but large values (distinct ones): the walk for each of the n."""
    V = 256 * 8 * 40
    x = torch.randn(V, generator=torch.Generator().manual_seed(2)).reshape(40, 256, 8)
    x[:, :17] = 100 + torch.randperm(40 * 17 * 8, generator=torch.Generator().manual_seed(3)).float().reshape(40, 17, 8)
    x = x.reshape(1, V).expand(300, V).contiguous()
    got = run_answers(block, [x], [7] * 300, 32, binding.TPQ_OUT_FP32)
    check_answers([g[:1] for g in got], x[:1].double(), [7], 32)
    assert all(torch.equal(g[:1].expand_as(g), g) for g in got)


@pytest.mark.parametrize("bad", [NAN, math.inf])
def test_rows_with_logits_that_are_no_numbers(block, bad):
    x = torch.randn(4, 5000, generator=torch.Generator().manual_seed(4))
    x[1, 4321] = bad
    x[2, :] = NAN
    got = run_answers(block, list(x.split(2500, 1)), [1, 2, 3, 4], 5, binding.TPQ_OUT_FP32)
    keep = [0, 3]
    check_answers([g[keep] for g in got], x[keep].double(), [1, 4], 5)
    assert got[0][1:3].isnan().all() and got[1][1:3].isnan().all() and got[3][1].isnan().all()
    order = torch.argsort(torch.where(x[1].isnan(), -math.inf, x[1]), descending=True, stable=True)[:5]
    assert torch.equal(got[2][1].long(), order) and (got[2][2] == -1).all()


def test_tokens_that_nobody_has_are_reported():
    b = binding.TpqBlock()
    x = torch.randn(3, 100)
    got = run_answers(b, [x[:, :50], x[:, 50:]], [99, 100, -1], 0, binding.TPQ_OUT_FP32)
    assert got[0][0].isfinite() and got[0][1].isnan() and got[0][2] == 0
    assert b.device_status() == binding.TPQ_ERR_INVALID_ARG and b.device_status() == 0
    b.close()


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("T", [1, 45])
def test_a_feed_forward_block_and_the_answer_behind_it(T):
    """x -> gated -> the down projection's partial sums of two devices -> synchronised -> the head of each -> log probabilities."""
    rng = np.random.default_rng(T)
    N, E, F, V, group = 2, 512, 300, 1000, 64
    b, t = binding.TpqBlock(), binding.Tpq(N, E)
    x = bf16(rng.standard_normal((T, E)))
    xd = x.cuda()
    shards = []
    for i in range(N):
        shards.append([quantised(b, weights(rng, n, K), group) for n, K in ((F, E), (F, E), (E, F), (V // N, E))])
    hs = [torch.zeros(T, F + 4, dtype=torch.bfloat16, device="cuda") for _ in range(N)]
    ys = [torch.zeros(T, E, dtype=torch.bfloat16, device="cuda") for _ in range(N)]
    for i, (g, u, d, _) in enumerate(shards):
        b.gated(g[0], u[0], 0, xd.data_ptr(), T, hs[i].data_ptr(), out_stride=F + 4)
        b.linear4(d[0], hs[i].data_ptr(), T, ys[i].data_ptr(), x_stride=F + 4)
        h, bound = block_ref.gated(x.double().cuda(), g[2], u[2], 0)
        check_product(hs[i][:, :F], h, bound)
        hd = hs[i][:, :F].double()
        check_product(ys[i], hd @ d[2].T, F * 2.0 ** -24 * (hd.abs() @ d[2].abs().T))
    lim = np.stack([y.double().abs().amax(0).cpu().numpy() for y in ys]).astype(np.float32) + 1e-3
    t.set_ranges(-lim, lim, np.ones(N, np.int64))
    t.select_features(8)
    P = t.payload_bytes(T)
    payloads = [torch.zeros(P, dtype=torch.uint8, device="cuda") for _ in range(N)]
    for i in range(N):
        t.quantize_pack(i, ys[i].data_ptr(), T, payloads[i].data_ptr(), P)
    out = torch.zeros(T, E, dtype=torch.bfloat16, device="cuda")
    t.dequant_reduce([p.data_ptr() for p in payloads], T, out.data_ptr())
    logits = [torch.zeros(T, V // N, device="cuda") for _ in range(N)]
    for i in range(N):
        b.linear4(shards[i][3][0], out.data_ptr(), T, logits[i].data_ptr(), binding.TPQ_OUT_FP32)
    tokens = rng.integers(0, V, T)
    got = run_answers(b, [x.cpu() for x in logits], tokens, 10, binding.TPQ_OUT_FP32)
    check_answers(got, torch.cat(logits, 1).cpu().double(), tokens, 10)
    od = out.double()
    for i in range(N):
        check_product(logits[i], od @ shards[i][3][2].T, E * 2.0 ** -24 * (od.abs() @ shards[i][3][2].abs().T))
    assert b.device_status() == 0 and t.device_status() == 0
    b.close()
    t.close()


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals_launch_nothing():
    b = binding.TpqBlock()
    buf = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p = buf.data_ptr()
    B, I = binding.TPQ_WEIGHT_BF16, binding.TPQ_WEIGHT_INT4
    ok4, ok16 = (p, 64, 64, 0, I, 32), (p, 64, 64, 64, B, 0)
    INV, ALIGN, SIZE = binding.TPQ_ERR_INVALID_ARG, binding.TPQ_ERR_ALIGN, binding.TPQ_ERR_SIZE
    cap = binding.weight4_bytes(64, 64, 32)
    out = p + 32768

    def weight(base, **kw):
        f = dict(zip(("data_ptr", "n_out", "n_in", "row_stride", "kind", "group"), base))
        f.update(kw)
        return binding.Weight(*f.values())

    def refused(status, name, *args):
        assert b.raw(name, *args) == status, (name, args)
        assert binding.lib().tpq_block_last_error(b._h)

    for args, status in [((None, 64, 64, 64, 32, out, cap), INV), ((p, 64, 64, 64, 32, None, cap), INV), ((p, 63, 64, 64, 32, out, cap), INV), ((p, 64, 0, 64, 32, out, cap), INV),
                         ((p, 64, 64, 0, 32, out, cap), INV), ((p, 64, 64, 64, 48, out, cap), INV), ((p, 2 ** 18, 64, 2 ** 17 + 1, 32, out, cap), INV), ((p + 1, 64, 64, 64, 32, out, cap), ALIGN),
                         ((p, 64, 64, 64, 32, out + 8, cap), ALIGN), ((p, 64, 64, 64, 32, out, cap - 1), SIZE)]:
        refused(status, "tpq_quantize_weight", *args, None)
    for args, status in [((None, 64, 64, 32, out, 64), INV), ((p, 64, 64, 32, None, 64), INV), ((p, 64, 64, 32, out, 63), INV), ((p, 64, 64, 0, out, 64), INV),
                         ((p + 8, 64, 64, 32, out, 64), ALIGN), ((p, 64, 64, 32, out + 1, 64), ALIGN)]:
        refused(status, "tpq_read_weight", *args, None)
    for kw, status in [(dict(data_ptr=None), INV), (dict(n_out=0), INV), (dict(n_in=0), INV), (dict(n_in=2 ** 17 + 1), INV), (dict(n_out=2 ** 30 + 1), INV), (dict(group=16), INV), (dict(kind=2), INV),
                       (dict(data_ptr=p + 8), ALIGN), (dict(kind=B), INV)]:
        refused(status, "tpq_linear4", weight(ok4, **kw), p, 64, 2, out, 0, 64, None)
    refused(INV, "tpq_linear4", None, p, 64, 2, out, 0, 64, None)
    rows_ = [((None, 64, 2, out, 64), INV), ((p, 64, 2, None, 64), INV), ((p, 64, 2, p, 64), INV), ((p, 56, 2, out, 64), INV), ((p, 64, 2, out, 63), INV), ((p, 64, -1, out, 64), INV),
             ((p, 64, 2 ** 31, out, 64), INV), ((p + 8, 64, 2, out, 64), ALIGN), ((p, 68, 2, out, 64), ALIGN), ((p, 64, 2, out + 1, 64), ALIGN), ((p, 2 ** 39, 2, out, 64), INV)]
    for (x, xs, T, o, os), status in rows_:
        refused(status, "tpq_linear4", weight(ok4), x, xs, T, o, 0, os, None)
        refused(status, "tpq_gated", weight(ok16), weight(ok16), 0, x, xs, T, o, os, None)
    refused(ALIGN, "tpq_linear4", weight(ok4), p, 64, 2, out + 2, 1, 64, None)
    refused(INV, "tpq_linear4", weight(ok4), p, 64, 2, out, 2, 64, None)
    refused(INV, "tpq_linear4", weight(ok4, n_out=2 ** 30), p, 64, 2 ** 20, out, 0, 2 ** 30, None)
    for g, u, act, status in [(ok16, ok4, 0, INV), (ok16, (p, 65, 64, 64, B, 0), 0, INV), (ok16, (p, 64, 56, 64, B, 0), 0, INV), (ok4, (p, 64, 64, 0, I, 64), 0, INV), (ok16, ok16, 3, INV),
                              (ok16, ok16, -1, INV), ((p, 64, 64, 56, B, 0), ok16, 0, INV), (ok16, (p, 64, 64, 68, B, 0), 0, ALIGN), ((p + 2, 64, 64, 64, B, 0), ok16, 0, ALIGN)]:
        refused(status, "tpq_gated", weight(g), weight(u), act, p, 64, 2, out, 64, None)
    refused(INV, "tpq_gated", None, weight(ok16), 0, p, 64, 2, out, 64, None)
    size = binding.token_record_bytes(2, 4)
    for args, status in [((None, 0, 64, 2, 64, 0, None, 4, out, size), INV), ((p, 2, 64, 2, 64, 0, None, 4, out, size), INV), ((p, 0, 63, 2, 64, 0, None, 4, out, size), INV),
                         ((p, 0, 64, -1, 64, 0, None, 4, out, size), INV), ((p, 0, 64, 2, 0, 0, None, 4, out, size), INV), ((p, 0, 64, 2, 64, -1, None, 4, out, size), INV),
                         ((p, 0, 64, 2, 64, 2 ** 31 - 64, None, 4, out, size), INV), ((p, 0, 64, 2, 64, 0, None, 33, out, size), INV), ((p, 0, 64, 2, 64, 0, None, -1, out, size), INV),
                         ((p, 0, 64, 2, 64, 0, None, 4, None, size), INV), ((p, 0, 64, 2, 64, 0, None, 4, out, size - 1), SIZE), ((p + 1, 0, 64, 2, 64, 0, None, 4, out, size), ALIGN),
                         ((p + 2, 1, 64, 2, 64, 0, None, 4, out, size), ALIGN), ((p, 0, 64, 2, 64, 0, p + 2, 4, out, size), ALIGN), ((p, 0, 64, 2, 64, 0, None, 4, out + 2, size), ALIGN)]:
        refused(status, "tpq_token_stats", *args, None)
    import ctypes
    arr = lambda *v: (ctypes.c_void_p * len(v))(*v)  # noqa: E731
    for args, status in [((None, 1, 2, out, None, 0, None, None), INV), ((arr(p), 0, 2, out, None, 0, None, None), INV), ((arr(*[p] * 65), 65, 2, out, None, 0, None, None), INV),
                         ((arr(p, None), 2, 2, out, None, 0, None, None), INV), ((arr(p), 1, -1, out, None, 0, None, None), INV), ((arr(p), 1, 2, out, None, 33, None, None), INV),
                         ((arr(p), 1, 2, out, None, 0, out, None), INV), ((arr(p), 1, 2, None, None, 4, None, None), INV), ((arr(p + 2), 1, 2, out, None, 0, None, None), ALIGN),
                         ((arr(p), 1, 2, out + 2, None, 0, None, None), ALIGN), ((arr(p), 1, 2, out, out + 1, 0, None, None), ALIGN), ((arr(p), 1, 2, out, None, 4, out + 2, None), ALIGN),
                         ((arr(p), 1, 2, out, None, 4, None, out + 1), ALIGN)]:
        refused(status, "tpq_token_logprobs", *args, None)
    assert b.launch_count() == 0
    # nothing to do
    b.linear4(weight(ok4), None, 0, None)
    b.gated(weight(ok16), weight(ok16), 0, None, 0, None)
    b.token_stats(None, 0, 64, None, 0)
    b.token_logprobs([p], 0, out)
    assert b.launch_count() == 0 and b.device_status() == 0
    assert not buf.any()
    b.close()
