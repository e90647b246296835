"""The 4-bit key/value cache on the GPU against the plain implementation: bytes of the cache, values read back, attention, refusals."""
import math

import numpy as np
import pytest
import torch

import kv_ref
from gpu_util import ensure_lib, guarded, guards_intact
from paper_2411_07942_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()


def bits(t: torch.Tensor) -> np.ndarray:
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


def dev(a: np.ndarray) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def rows_of(rng, rows, width, pad=0, scale=1.0):
    """A BF16 device tensor of rows of `width` inside rows of width + pad, and the float32 values."""
    x = torch.from_numpy((rng.standard_normal((rows, width + pad)) * scale).astype(np.float32)).to(torch.bfloat16)
    return x.cuda(), x[:, :width].float().numpy()


class Setup:
    """A batch of sequences with new[s] rows and lengths[s] positions on pages dealt out at random."""

    def __init__(self, heads, kv_heads, dim, page, new, lengths, pad=0, seed=0, fill=None, max_new=None):
        self.rng = rng = np.random.default_rng(seed)
        self.heads, self.kv_heads, self.dim, self.page = heads, kv_heads, dim, page
        self.lengths, self.start = np.array(lengths, np.int32), np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        per = max(1, max(-(-ln // page) for ln in lengths))
        need = sum(-(-ln // page) for ln in lengths)
        self.n_pages = need + 2
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(lengths), per), -7, np.int32)
        at = 0
        for s, ln in enumerate(lengths):
            m = -(-ln // page)
            self.table[s, :m] = order[at:at + m]
            at += m
        self.T = int(self.start[-1]) + pad
        self.cache = kv_ref.Cache(self.n_pages, kv_heads, dim, page, fill=fill, rng=rng)
        self.kv = binding.TpqKv(heads, kv_heads, dim, page)
        assert self.kv.page_bytes() == self.cache.bytes[0].size
        self.d_cache, self.d_table, self.d_start, self.d_lengths = dev(self.cache.bytes), dev(self.table), dev(self.start), dev(self.lengths)
        self.batch = binding.KvBatch(self.d_cache.data_ptr(), self.n_pages, self.d_table.data_ptr(), per, self.d_start.data_ptr(), self.d_lengths.data_ptr(),
                                     len(lengths), max(new) if max_new is None else max_new, self.T)

    def fill_with_data(self, k_scale=1.0):
        """Every position of every sequence holds quantised normal data; everything else what it held."""
        rng = self.rng
        for s, ln in enumerate(self.lengths):
            for which, sc in ((0, k_scale), (1, 1.0)):
                x = (rng.standard_normal((ln, self.kv_heads, self.dim)) * sc + 0.3 * rng.standard_normal((1, self.kv_heads, self.dim))).astype(np.float32)
                codes, words = kv_ref.quantise(x)
                for t in range(ln):
                    for h in range(self.kv_heads):
                        self.cache.put(self.table[s, t // self.page], h, t % self.page, which, codes[t, h], words[t, h])
        self.d_cache.copy_(torch.from_numpy(self.cache.bytes))
        return self

    def attention(self, q, scale, window=0, first=0, q_stride=None, out_pad=0, stream=0, ws=None):
        width = self.heads * self.dim
        nbytes = self.T * (width + out_pad) * 2
        whole, view = guarded(nbytes)
        need = self.kv.attention_workspace_bytes(self.batch)
        if ws is None:
            ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")   # contents need no preparation
        self.kv.attention(self.batch, q.data_ptr(), view.data_ptr(), ws.data_ptr(), ws.numel(), scale, window, first, q_stride=q_stride,
                          out_stride=width + out_pad, stream=stream)
        torch.cuda.synchronize()
        assert guards_intact(whole, nbytes)
        out = view.view(torch.int16).view(self.T, width + out_pad)
        if out_pad:
            assert (out[:, width:] == out[0, -1]).all() and int(out[0, -1]) == int(np.uint16(0xA5A5).view(np.int16))
        return out[:, :width].contiguous().cpu().numpy().view(np.uint16)


def tolerance(out, bound):
    """Half a step of BF16 (2^-8 of the value), and of the bound B = sum of weight * largest value: the weights' rounding to 11 bits
    acts on numerator and normaliser (2 * 2^-11 B); exponents off by 2^-12 at most (products are exact; sums of at most
    dim terms of size 143 |q| step in binary32 stay below 2^-15 for the |scale q| step of these tests, the power itself is
    good to 2^-21) twice the same way (2 * 2^-12 B)."""
    return 2.0 ** -8 * np.abs(out) + (2 * 2.0 ** -11 + 2 * 2.0 ** -12) * bound


def check(setup, q32, got_bits, scale, window=0, first=0):
    rows, used = setup.T, int(setup.start[-1])
    want, bound = kv_ref.attention(setup.cache, setup.table, setup.start, setup.lengths, q32.reshape(rows, setup.heads, setup.dim), scale, window, first)
    got = kv_ref.wide(got_bits).reshape(rows, setup.heads, setup.dim).astype(np.float64)
    assert (got_bits[used:] == 0xA5A5).all()                       # rows behind the last sequence, as they were
    err = np.abs(got - want)[:used]
    ok = err <= tolerance(want, bound)[:used]
    assert ok.all(), f"{int((~ok).sum())} of {ok.size} off; worst {float(np.nanmax(err / tolerance(want, bound)[:used])):.3g} times the tolerance"


APPEND = [  # heads, kv_heads, dim, page, new, lengths, rot, interleaved, pad rows, pad elements
    (1, 1, 128, 16, [1], [1], 128, False, 0, 0),
    (10, 10, 128, 16, [1], [17], 128, False, 0, 0),
    (4, 2, 128, 32, [1, 1, 1, 0, 1], [1, 33, 32, 40, 500], 128, True, 3, 24),
    (8, 1, 64, 16, [5, 0, 17, 1], [5, 0, 17, 16], 64, False, 1, 8),
    (6, 3, 64, 64, [70, 1, 3], [100, 64, 65], 16, True, 0, 0),
    (5, 5, 128, 256, [300, 2], [300, 513], 96, False, 0, 40),
    (12, 4, 64, 128, [129], [129], 48, False, 2, 0),
    (16, 16, 128, 32, [600], [600], 64, True, 0, 0),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}p{c[3]}r{c[6]}{'i' if c[7] else ''}")
@pytest.mark.parametrize("with_q", [True, False])
def test_append_writes_the_bytes_of_the_definition(case, with_q):
    heads, kvh, dim, page, new, lengths, rot, inter, pad, pad_el = case
    s = Setup(heads, kvh, dim, page, new, lengths, pad=pad, seed=3)
    k, k32 = rows_of(s.rng, s.T, kvh * dim, pad_el, 2.0)
    v, v32 = rows_of(s.rng, s.T, kvh * dim, 2 * pad_el)
    q, q32 = rows_of(s.rng, s.T, heads * dim, pad_el)
    a = s.rng.uniform(0, 7, (max(lengths) + 3, rot // 2))
    table = np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)
    d_rot = dev(table)
    positions = s.rng.integers(0, len(table), s.T).astype(np.int32) if inter else None
    d_pos = None if positions is None else dev(positions)
    r = binding.KvRotation(d_rot.data_ptr(), len(table), rot, int(inter), None if d_pos is None else d_pos.data_ptr())
    out = torch.full((s.T, heads * dim + 8), 7, dtype=torch.int16, device="cuda")
    opts = dict(q_ptr=q.data_ptr(), q_stride=heads * dim + pad_el, q_out_ptr=out.data_ptr(), q_out_stride=heads * dim + 8) if with_q else {}
    s.kv.append(s.batch, k.data_ptr(), v.data_ptr(), k_stride=kvh * dim + pad_el, v_stride=kvh * dim + 2 * pad_el, rotation=r, **opts)
    assert s.kv.device_status() == binding.TPQ_OK
    shape = lambda x, h: x.reshape(s.T, h, dim)  # noqa: E731
    want_q = kv_ref.append(s.cache, s.table, s.start, s.lengths, shape(k32, kvh), shape(v32, kvh), shape(q32, heads) if with_q else None, table, rot, inter, positions)
    assert np.array_equal(s.d_cache.cpu().numpy(), s.cache.bytes)
    if with_q:
        used = int(s.start[-1])
        got = out.cpu().numpy().view(np.uint16)
        assert np.array_equal(got[:used, : heads * dim], want_q[:used].reshape(used, -1))
        assert (got[used:] == 7).all() and (got[:, heads * dim:] == 7).all()
    # and what the cache holds reads back as low + step * code
    ko, vo = (torch.full((s.T, kvh * dim + 8), 9, dtype=torch.int16, device="cuda") for _ in range(2))
    s.kv.read(s.batch, ko.data_ptr(), vo.data_ptr(), k_out_stride=kvh * dim + 8, v_out_stride=kvh * dim + 8)
    torch.cuda.synchronize()
    for which, o in ((0, ko), (1, vo)):
        got = o.cpu().numpy().view(np.uint16)
        assert (got[:, kvh * dim:] == 9).all() and (got[int(s.start[-1]):] == 9).all()
        for i in range(len(lengths)):
            n, ln = new[i], lengths[i]
            for h in range(kvh):
                if n:
                    st, lo, codes, _ = s.cache.sequence(s.table[i], ln, h, which)
                    want = kv_ref.bf16((lo[:, None] + st[:, None] * codes).astype(np.float32))[ln - n:]
                    assert np.array_equal(got[s.start[i]:s.start[i + 1], h * dim:(h + 1) * dim], want)


def test_append_without_rotation_in_place_queries_and_odd_numbers():
    """No rotation; vectors of one value, of zeros, with NaN, infinities, the type's ends; q rotated in place."""
    s = Setup(4, 2, 128, 16, [40], [45], seed=5)
    k, k32 = rows_of(s.rng, s.T, 256)
    for row, val in ((0, 0.0), (1, 5.0), (2, -3.3e38), (4, 1e-40)):
        k[row] = val
    k[5, 3], k[6, 200], k[7, 0] = math.nan, math.inf, -math.inf
    k[8, 10], k[8, 11] = 3.38e38, -3.38e38
    k[9, :128] = torch.arange(128).cuda() * 0.5          # many exact ties
    k32 = k.float().cpu().numpy()
    v = k.flip(0).contiguous()
    s.kv.append(s.batch, k.data_ptr(), v.data_ptr())
    kv_ref.append(s.cache, s.table, s.start, s.lengths, k32.reshape(-1, 2, 128), v.float().cpu().numpy().reshape(-1, 2, 128))
    torch.cuda.synchronize()
    assert np.array_equal(s.d_cache.cpu().numpy(), s.cache.bytes)
    q, q32 = rows_of(s.rng, s.T, 512)
    table = np.concatenate([np.full((64, 64), 0.6), np.full((64, 64), 0.8)], 1).astype(np.float32)
    d = dev(table)
    s.kv.append(s.batch, k.data_ptr(), v.data_ptr(), rotation=binding.KvRotation(d.data_ptr(), 64, 128, 0, None), q_ptr=q.data_ptr(), q_out_ptr=q.data_ptr())
    torch.cuda.synchronize()
    assert np.array_equal(bits(q).reshape(-1, 4, 128), kv_ref.bf16(kv_ref.rotate(q32.reshape(-1, 4, 128), table, np.zeros(s.T, int), 128, False)))


ATTENTION = [  # heads, kv_heads, dim, page, new, lengths, window, first, pad
    (1, 1, 128, 16, [1], [1], 0, 0, 0),
    (4, 4, 64, 16, [1, 1], [2, 31], 0, 0, 1),
    (10, 10, 128, 16, [1], [777], 0, 0, 0),
    (8, 1, 128, 32, [1, 1, 0, 1], [16, 129, 7, 1000], 0, 0, 2),
    (12, 1, 128, 64, [1, 1], [127, 300], 0, 0, 0),
    (32, 4, 64, 128, [4, 2, 1], [4, 500, 257], 0, 0, 0),
    (10, 2, 128, 16, [3, 5], [3, 200], 0, 0, 0),
    (6, 2, 64, 256, [40, 1, 7], [40, 600, 300], 0, 0, 5),
    (4, 2, 128, 32, [130], [130], 0, 0, 0),
    (20, 1, 128, 16, [33], [90], 0, 0, 0),
    (8, 2, 128, 32, [1, 1], [1000, 64], 100, 4, 0),
    (8, 2, 128, 16, [1, 3], [700, 900], 1, 0, 0),
    (4, 2, 64, 64, [1, 2], [900, 333], 200, 130, 0),
    (4, 1, 128, 32, [150, 1], [400, 400], 64, 3, 3),
    (2, 2, 64, 16, [260], [260], 17, 20, 0),
    (64, 1, 64, 16, [1], [200], 0, 0, 0),
    (100, 1, 128, 16, [2], [50], 5000, 1, 0),
]


@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}p{c[3]}n{max(c[4])}l{max(c[5])}w{c[6]}f{c[7]}")
def test_attention_against_64_bits(case):
    heads, kvh, dim, page, new, lengths, window, first, pad = case
    s = Setup(heads, kvh, dim, page, new, lengths, pad=pad, seed=11, fill=0xFF).fill_with_data()   # 0xFF: unused entries' words are NaN
    q, q32 = rows_of(s.rng, s.T, heads * dim, 16)
    scale = 1.5 / math.sqrt(dim)
    got = s.attention(q, scale, window, first, q_stride=heads * dim + 16, out_pad=8)
    assert s.kv.device_status() == binding.TPQ_OK
    check(s, q32, got, scale, window, first)
    assert np.array_equal(got, s.attention(q, scale, window, first, q_stride=heads * dim + 16, out_pad=8))   # and the same twice


@pytest.mark.parametrize("new", [3, 40])
@pytest.mark.parametrize("which", [0, 1])
def test_a_vector_that_is_no_number_reaches_the_rows_that_see_it_and_no_others(new, which):
    s = Setup(4, 2, 128, 16, [new, new], [200, 150], seed=21, fill=0xFF).fill_with_data()
    at = 200 - new + 2                              # position of the first sequence's row 2: rows 0 and 1 do not see it
    s.cache.put(s.table[0, at // 16], 1, at % 16, which, np.zeros(128, np.uint8), 0x7FC03F80)
    gone = 30                                       # and one that the window hides from everybody
    s.cache.put(s.table[0, gone // 16], 0, gone % 16, which, np.zeros(128, np.uint8), 0x7FC03F80)
    s.d_cache.copy_(torch.from_numpy(s.cache.bytes))
    q, q32 = rows_of(s.rng, s.T, 512)
    got = kv_ref.wide(s.attention(q, 0.08, window=100, first=5)).reshape(s.T, 4, 128)
    nan = np.isnan(got)
    assert nan[2:new, 2:].all() and not nan[:2].any() and not nan[:, :2].any() and not nan[new:].any()
    want, bound = kv_ref.attention(s.cache, s.table, s.start, s.lengths, q32.reshape(s.T, 4, 128), 0.08, 100, 5)
    assert (np.abs(got - want)[~nan] <= np.broadcast_to(tolerance(want, bound), got.shape)[~nan]).all()


def test_attention_reads_no_page_that_a_window_left_behind():
    s = Setup(4, 2, 128, 16, [1, 90], [500, 700], seed=12, fill=0xFF).fill_with_data()
    q, q32 = rows_of(s.rng, s.T, 512)
    window, first = 70, 20
    table = s.table.copy()
    for i, n in enumerate((1, 90)):
        seen = s.lengths[i] - n - window + 1
        for p in range(table.shape[1]):
            if p * 16 >= first and (p + 1) * 16 <= seen:
                table[i, p] = 2 ** 30 if p % 2 else -1
    s.d_table.copy_(torch.from_numpy(table))
    got = s.attention(q, 0.1, window, first)
    assert s.kv.device_status() == binding.TPQ_OK
    check(s, q32, got, 0.1, window, first)
