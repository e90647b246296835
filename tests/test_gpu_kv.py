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
    ok = (err <= tolerance(want, bound)[:used]) | (np.isnan(want) & np.isnan(got))[:used]   # (what was never appended may be NaN: then so is the answer)
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


MORE = [  # many sequences, several items and runs, odd scales: heads, kv_heads, dim, page, new, lengths, window, first, pad, scale
    (2, 1, 64, 16, [1] * 300, [1 + (7 * i) % 90 for i in range(300)], 0, 0, 1, 0.2),
    (3, 3, 128, 16, [i % 3 for i in range(1100)], [i % 3 + (5 * i) % 23 for i in range(1100)], 0, 0, 0, 0.1),
    (2, 1, 128, 64, [700], [1500], 0, 0, 0, 0.1),
    (1, 1, 128, 32, [1100], [1100], 300, 5, 0, 0.1),
    (5, 1, 64, 128, [200, 300, 1, 7, 90], [900, 300, 2000, 7, 450], 0, 0, 4, 0.15),
    (16, 2, 128, 32, [33, 64, 1], [640, 64, 3000], 128, 128, 0, 0.09),
    (4, 4, 128, 16, [1, 40], [300, 300], 0, 0, 0, -0.1),
    (4, 4, 128, 16, [1, 40], [300, 300], 0, 0, 0, 0.0),
    (4, 2, 128, 16, [2, 40], [500, 300], 0, 0, 0, 1.0),
    (4, 2, 64, 256, [1, 257], [4096, 257], 1, 0, 0, 0.1),
    (256, 1, 64, 16, [1], [70], 0, 0, 0, 0.1),
]


@pytest.mark.parametrize("case", MORE, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}s{len(c[4])}n{max(c[4])}l{max(c[5])}w{c[6]}x{c[9]}")
def test_attention_over_many_sequences_items_and_scales(case):
    heads, kvh, dim, page, new, lengths, window, first, pad, scale = case
    s = Setup(heads, kvh, dim, page, new, lengths, pad=pad, seed=31, fill=0xFF).fill_with_data()
    q, q32 = rows_of(s.rng, s.T, heads * dim)
    got = s.attention(q, scale, window, first)
    assert s.kv.device_status() == binding.TPQ_OK
    check(s, q32, got, scale, window, first)


@pytest.mark.parametrize("new", [1, 50])
def test_attention_over_vectors_of_very_different_sizes(new):
    """Keys' and values' magnitudes over 2^14, zero vectors and constant ones among them; queries over 2^20."""
    s = Setup(4, 2, 128, 16, [new], [260], seed=33, fill=0xFF)
    for t in range(260):
        for h in range(2):
            for which in (0, 1):
                x = s.rng.standard_normal(128) * 2.0 ** s.rng.integers(-10, 4)
                if t % 37 == 5:
                    x[:] = 0 if t % 2 else 0.75
                codes, words = kv_ref.quantise((x * (0.05 if which == 0 else 1)).astype(np.float32)[None])
                s.cache.put(s.table[0, t // 16], h, t % 16, which, codes[0], words[0])
    s.d_cache.copy_(torch.from_numpy(s.cache.bytes))
    q, q32 = rows_of(s.rng, s.T, 512)
    q[:, :128] *= 2.0 ** -20
    q32 = q.float().cpu().numpy()
    check(s, q32, s.attention(q, 0.1), 0.1)


def test_windows_beyond_every_length_are_none():
    s = Setup(8, 2, 128, 32, [1, 60], [700, 300], seed=35).fill_with_data()
    q, _ = rows_of(s.rng, s.T, 1024)
    plain = s.attention(q, 0.1)
    for window, first in ((700, 0), (2 ** 40, 3), (2 ** 62, 2 ** 62), (0, 5)):
        assert np.array_equal(plain, s.attention(q, 0.1, window, first))


def test_appending_in_pieces_gives_the_same_bytes():
    whole, parts = (Setup(4, 2, 64, 16, [90], [90], seed=41, fill=0) for _ in range(2))
    k, _ = rows_of(whole.rng, 90, 128)
    v, _ = rows_of(whole.rng, 90, 128)
    a = whole.rng.uniform(0, 7, (90, 32))
    d = dev(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32))
    rot = binding.KvRotation(d.data_ptr(), 90, 64, 0, None)
    whole.kv.append(whole.batch, k.data_ptr(), v.data_ptr(), rotation=rot)
    at = 0
    for n in (1, 15, 17, 40, 1, 16):
        start, lengths = dev(np.array([0, n], np.int32)), dev(np.array([at + n], np.int32))
        b = binding.KvBatch(parts.d_cache.data_ptr(), parts.n_pages, parts.d_table.data_ptr(), parts.table.shape[1], start.data_ptr(), lengths.data_ptr(), 1, n, n)
        parts.kv.append(b, k[at:].data_ptr(), v[at:].data_ptr(), rotation=rot)
        torch.cuda.synchronize()
        at += n
    assert at == 90 and torch.equal(whole.d_cache, parts.d_cache)


def test_captured_steps_replay_with_other_lengths_and_rows():
    """A step (append, attention) captured once for a padded batch, replayed with other rows, lengths, pages and fewer sequences; two graphs
    with workspaces of their own, replayed on two streams at a time."""
    new, lengths = [1, 40, 1, 1], [200, 90, 64, 33]
    s = Setup(8, 2, 128, 16, new, lengths, pad=5, seed=51, fill=0xFF).fill_with_data()
    width = 1024
    k, v, q = (torch.zeros(s.T, w, dtype=torch.bfloat16, device="cuda") for w in (256, 256, width))
    graphs, outs, caches = [], [], []
    for _ in range(2):
        cache = s.d_cache.clone()
        batch = binding.KvBatch(cache.data_ptr(), *[getattr(s.batch, f) for f, _ in s.batch._fields_[1:]])
        ws = torch.empty(s.kv.attention_workspace_bytes(batch), dtype=torch.uint8, device="cuda")
        out = torch.zeros(s.T, width, dtype=torch.bfloat16, device="cuda")
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            run = lambda: (s.kv.append(batch, k.data_ptr(), v.data_ptr(), stream=side.cuda_stream),  # noqa: E731
                           s.kv.attention(batch, q.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel(), 0.1, stream=side.cuda_stream))
            run()
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                run()
        graphs.append((graph, side, ws, batch))
        outs.append(out)
        caches.append(cache)
    for step, (new, lengths) in enumerate([([1, 40, 1, 1], [200, 90, 64, 33]), ([1, 3, 0, 1], [17, 90, 64, 40]), ([0, 0, 0, 0], [5, 90, 64, 40]), ([2, 40, 1, 0], [150, 95, 1, 0])]):
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        s.start, s.lengths = start, np.array(lengths, np.int32)
        s.d_start.copy_(torch.from_numpy(start))
        s.d_lengths.copy_(torch.from_numpy(s.lengths))
        for t in (k, v, q):
            t.copy_(torch.from_numpy(s.rng.standard_normal(tuple(t.shape)).astype(np.float32)).to(torch.bfloat16))
        for out in outs:
            out.view(torch.int16).fill_(np.int16(np.uint16(0xA5A5).view(np.int16)).item())
        torch.cuda.synchronize()
        for graph, side, _, _ in graphs:
            with torch.cuda.stream(side):
                graph.replay()
        torch.cuda.synchronize()
        assert s.kv.device_status() == binding.TPQ_OK
        kv_ref.append(s.cache, s.table, start, s.lengths, k.float().cpu().numpy().reshape(s.T, 2, 128), v.float().cpu().numpy().reshape(s.T, 2, 128))
        for out, cache in zip(outs, caches):
            assert np.array_equal(cache.cpu().numpy(), s.cache.bytes)
            check(s, q.float().cpu().numpy(), bits(out), 0.1)


def test_offsets_beyond_32_bits():
    """The last pages of a pool of more than 4 GiB, by append, read and both attention paths."""
    page, heads = 256, 16
    s = Setup(16, heads, 128, page, [40, 1], [300, 260], seed=61, fill=0)
    per_page = s.kv.page_bytes()
    n_pages = 2 ** 32 // per_page + 12
    pool = torch.empty(n_pages * per_page, dtype=torch.uint8, device="cuda")
    last = np.where(s.table >= 0, n_pages - 1 - s.table, s.table).astype(np.int32)
    d_last = dev(last)
    s.fill_with_data()
    for p in range(s.n_pages):
        pool[(n_pages - 1 - p) * per_page:][:per_page] = torch.from_numpy(s.cache.bytes[p].reshape(-1)).cuda()
    b = binding.KvBatch(pool.data_ptr(), n_pages, d_last.data_ptr(), last.shape[1], s.d_start.data_ptr(), s.d_lengths.data_ptr(), 2, 40, s.T)
    s.batch = b
    k, k32 = rows_of(s.rng, s.T, 16 * 128)
    s.kv.append(b, k.data_ptr(), k.data_ptr())
    kv_ref.append(s.cache, s.table, s.start, s.lengths, k32.reshape(s.T, 16, 128), k32.reshape(s.T, 16, 128))
    out = torch.zeros(s.T, 16 * 128, dtype=torch.bfloat16, device="cuda")
    s.kv.read(b, out.data_ptr(), None)
    torch.cuda.synchronize()
    for p in range(s.n_pages):
        assert np.array_equal(pool[(n_pages - 1 - p) * per_page:][:per_page].cpu().numpy(), s.cache.bytes[p].reshape(-1))
    assert (out.float().cpu().numpy() != 0).mean() > 0.9
    q, q32 = rows_of(s.rng, s.T, 2048)
    check(s, q32, s.attention(q, 0.1), 0.1)


def test_what_contradicts_itself_on_the_device_is_left_out_and_reported():
    """Bad sequences, pages and positions: nothing of theirs is written, the others are right, the status word says so once."""
    new, lengths = [1, 2, 1, 40, 1], [100, 64, 30, 80, 50]
    s = Setup(4, 2, 128, 16, new, lengths, seed=71, fill=0xFF).fill_with_data()
    q, q32 = rows_of(s.rng, s.T, 512)
    k, k32 = rows_of(s.rng, s.T, 256)
    good = s.attention(q, 0.1)
    for name, change in (("longer than the table", lambda ln, tb, st: ln.__setitem__(1, 7 * 16 + 1)), ("negative length", lambda ln, tb, st: ln.__setitem__(1, -5)),
                         ("more rows than positions", lambda ln, tb, st: ln.__setitem__(1, 1)), ("more rows than said", None)):
        ln, tb, st = s.lengths.copy(), s.table.copy(), s.start.copy()
        b = binding.KvBatch.from_buffer_copy(s.batch)
        skipped = 1
        if change is None:
            b.max_new, skipped = 39, 3
        else:
            change(ln, tb, st)
        d_ln = dev(ln)
        b.lengths_ptr = d_ln.data_ptr()
        keep, s.batch = s.batch, b
        got = s.attention(q, 0.1)
        assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG, name
        assert s.kv.device_status() == binding.TPQ_OK
        lo, hi = s.start[skipped], s.start[skipped + 1]
        assert (got[lo:hi] == 0xA5A5).all() and np.array_equal(np.delete(got, np.s_[lo:hi], 0), np.delete(good, np.s_[lo:hi], 0)), name
        before = s.d_cache.clone()
        s.kv.append(b, k.data_ptr(), k.data_ptr())
        assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG
        want = kv_ref.Cache(s.n_pages, 2, 128, 16, fill=0)
        want.bytes = before.cpu().numpy().copy()
        starts = s.start.copy()
        mask = [i for i in range(5) if i != skipped]
        for i in mask:
            r = slice(starts[i], starts[i + 1])
            kv_ref.append(want, s.table[i:i + 1], np.array([0, starts[i + 1] - starts[i]]), ln[i:i + 1], k32[r].reshape(-1, 2, 128), k32[r].reshape(-1, 2, 128))
        assert np.array_equal(s.d_cache.cpu().numpy(), want.bytes), name
        s.d_cache.copy_(before)
        s.batch = keep
    # starts that go down, or beyond the rows
    for bad in ([0, 3, 1, 44, 45], [-1, 1, 3, 4, 44], [0, 1, 3, 4, 1000]):
        d_st = dev(np.array(bad + [45], np.int32))
        b = binding.KvBatch.from_buffer_copy(s.batch)
        b.token_start_ptr = d_st.data_ptr()
        keep, s.batch = s.batch, b
        s.attention(q, 0.1)                                        # (guards intact)
        s.kv.append(b, k.data_ptr(), k.data_ptr())
        assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG
        s.batch = keep
    s.d_cache.copy_(torch.from_numpy(s.cache.bytes))
    # pages outside the pool: their positions are invisible, and a row that sees nothing else is zero
    for page_id in (-1, s.n_pages, 2 ** 31 - 1, -2 ** 31):
        table = s.table.copy()
        table[0, 2], table[3, 0], table[4, :] = page_id, page_id, page_id
        s.d_table.copy_(torch.from_numpy(table))
        got = s.attention(q, 0.1)
        assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG
        keep, s.table = s.table, table
        check(s, q32, got, 0.1)
        assert (got[s.start[4]:] == 0).all()
        before = s.d_cache.clone()
        s.kv.append(s.batch, k.data_ptr(), k.data_ptr())
        assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG
        s.d_cache.copy_(before)
        s.table = keep
        s.d_table.copy_(torch.from_numpy(s.table))
    # positions outside the rotation's table
    d_rot = torch.ones(90, 128, device="cuda")
    before, out = s.d_cache.clone(), torch.full((s.T, 512), 3, dtype=torch.int16, device="cuda")
    s.kv.append(s.batch, k.data_ptr(), k.data_ptr(), rotation=binding.KvRotation(d_rot.data_ptr(), 90, 128, 0, None), q_ptr=q.data_ptr(), q_out_ptr=out.data_ptr())
    assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG
    assert (out[0] == 3).all() and not (out[1:] == 3).all(1).any()           # (position 99 of the first sequence alone)
    s.d_cache.copy_(before)


def test_refusals_launch_nothing():
    s = Setup(8, 2, 128, 16, [1, 2], [40, 50], seed=81).fill_with_data()
    q, _ = rows_of(s.rng, s.T, 1024)
    k, _ = rows_of(s.rng, s.T, 256)
    out = torch.zeros(s.T, 1024, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(s.kv.attention_workspace_bytes(s.batch), dtype=torch.uint8, device="cuda")
    rot_table = torch.ones(64, 128, device="cuda")
    launches = s.kv.launch_count()

    def with_batch(**kw):
        b = binding.KvBatch.from_buffer_copy(s.batch)
        for name, value in kw.items():
            setattr(b, name, value)
        return b

    def attention(b=s.batch, q_ptr=q.data_ptr(), qs=1024, scale=0.1, window=0, first=0, o=out.data_ptr(), os=1024, w=ws.data_ptr(), n=ws.numel()):
        return s.kv.raw("tpq_kv_attention", b, q_ptr, qs, scale, window, first, o, os, w, n, None)

    def append(b=s.batch, rot=None, k_ptr=k.data_ptr(), ks=256, v_ptr=k.data_ptr(), vs=256, q_ptr=None, qs=1024, o=None, os=1024):
        return s.kv.raw("tpq_kv_append", b, rot, k_ptr, ks, v_ptr, vs, q_ptr, qs, o, os, None)

    def rot(**kw):
        r = binding.KvRotation(rot_table.data_ptr(), 64, 128, 0, None)
        for name, value in kw.items():
            setattr(r, name, value)
        return r

    A, I, S = binding.TPQ_ERR_ALIGN, binding.TPQ_ERR_INVALID_ARG, binding.TPQ_ERR_SIZE
    batches = [(I, None), (I, with_batch(n_seqs=-1)), (I, with_batch(max_new=-1)), (I, with_batch(n_tokens=-1)), (I, with_batch(n_tokens=2 ** 31)), (I, with_batch(n_pages=-1)),
               (I, with_batch(n_pages=2 ** 31)), (I, with_batch(page_table_stride=-1)), (I, with_batch(page_table_stride=2 ** 31)), (I, with_batch(cache_ptr=None)),
               (I, with_batch(page_table_ptr=None)), (I, with_batch(token_start_ptr=None)), (I, with_batch(lengths_ptr=None)), (A, with_batch(cache_ptr=s.batch.cache_ptr + 8)),
               (A, with_batch(page_table_ptr=s.batch.page_table_ptr + 2)), (A, with_batch(token_start_ptr=s.batch.token_start_ptr + 1)),
               (A, with_batch(lengths_ptr=s.batch.lengths_ptr + 2))]
    for want, b in batches:
        assert attention(b) == want and append(b) == want and s.kv.raw("tpq_kv_read", b, k.data_ptr(), 256, None, 256, None) == want
    for want, kw in [(I, dict(q_ptr=None)), (A, dict(q_ptr=q.data_ptr() + 2)), (I, dict(qs=1016)), (A, dict(qs=1028)), (I, dict(o=None)), (A, dict(o=out.data_ptr() + 8)), (I, dict(os=1000)),
                     (A, dict(os=1025)), (I, dict(o=q.data_ptr())), (I, dict(scale=float("inf"))), (I, dict(scale=float("nan"))), (I, dict(window=-1)), (I, dict(first=-1)),
                     (I, dict(w=None)), (A, dict(w=ws.data_ptr() + 4)), (S, dict(n=ws.numel() - 1)), (S, dict(n=0))]:
        assert attention(**kw) == want, kw
        assert binding.lib().tpq_kv_last_error(s.kv._h) != b""
    for want, kw in [(I, dict(k_ptr=None)), (I, dict(v_ptr=None)), (A, dict(k_ptr=k.data_ptr() + 8)), (I, dict(ks=248)), (A, dict(vs=260)), (I, dict(q_ptr=q.data_ptr(), o=out.data_ptr())),
                     (I, dict(o=out.data_ptr())), (I, dict(rot=rot(), q_ptr=q.data_ptr())), (I, dict(rot=rot(), q_ptr=q.data_ptr(), o=q.data_ptr(), os=1032)),
                     (I, dict(rot=rot(table_ptr=None))), (A, dict(rot=rot(table_ptr=rot_table.data_ptr() + 4))), (I, dict(rot=rot(n_positions=0))), (I, dict(rot=rot(rot_dim=0))),
                     (I, dict(rot=rot(rot_dim=24))), (I, dict(rot=rot(rot_dim=144))), (A, dict(rot=rot(positions_ptr=rot_table.data_ptr() + 2)))]:
        assert append(**kw) == want, kw
    assert s.kv.raw("tpq_kv_read", s.batch, None, 256, None, 256, None) == I and s.kv.raw("tpq_kv_read", s.batch, k.data_ptr(), 256, k.data_ptr(), 256, None) == I
    for b in (with_batch(n_seqs=0), with_batch(n_tokens=0), with_batch(max_new=0)):   # nothing to do, whatever else is given
        assert attention(b) == 0 and append(b) == 0 and s.kv.raw("tpq_kv_read", b, None, 0, None, 0, None) == 0
    assert s.kv.attention_workspace_bytes(with_batch(n_seqs=0)) == 0
    assert s.kv.launch_count() == launches and s.kv.device_status() == binding.TPQ_OK
    assert attention() == 0 and append(rot=rot(), q_ptr=q.data_ptr(), o=out.data_ptr()) == 0
    assert s.kv.launch_count() > launches


def test_an_attention_block_up_to_the_synchronised_sum():
    """Two devices of a tensor-parallel group: each appends its heads' keys and values, attends, multiplies by its part of the output
    projection and compresses the partial sums (tpq_linear_quantize_pack); the payloads are summed.  Against the same in 64 bits from the cache's
    values: off by half a step of each device's codes (the ranges cover the partial sums), and by what the partial sums themselves
    may be off: their rounding to BF16 and the attention's tolerance through the weights' magnitudes."""
    N, E, heads, kvh, dim, n = 2, 512, 4, 2, 128, 70
    rng = np.random.default_rng(91)
    K = heads * dim
    a = rng.uniform(0, 7, (120, dim // 2))
    table = np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)
    d_rot = dev(table)
    total, allowed, payloads, ys, ws_slots, xs = 0, 0, [], [], [], []
    t = binding.Tpq(N, E)
    for i in range(N):
        s = Setup(heads, kvh, dim, 16, [n, 1], [n + 13, 50], seed=100 + i, fill=0xFF).fill_with_data()
        k, k32 = rows_of(rng, s.T, kvh * dim)
        v, v32 = rows_of(rng, s.T, kvh * dim)
        q, q32 = rows_of(rng, s.T, K)
        s.kv.append(s.batch, k.data_ptr(), v.data_ptr(), rotation=binding.KvRotation(d_rot.data_ptr(), 120, dim, 0, None), q_ptr=q.data_ptr(), q_out_ptr=q.data_ptr())
        x = torch.empty(s.T, K, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(s.kv.attention_workspace_bytes(s.batch), dtype=torch.uint8, device="cuda")
        s.kv.attention(s.batch, q.data_ptr(), x.data_ptr(), ws.data_ptr(), ws.numel(), 1 / math.sqrt(dim))
        qr = kv_ref.wide(kv_ref.append(s.cache, s.table, s.start, s.lengths, k32.reshape(s.T, kvh, dim), v32.reshape(s.T, kvh, dim), q32.reshape(s.T, heads, dim), table, dim))
        torch.cuda.synchronize()
        assert np.array_equal(s.d_cache.cpu().numpy(), s.cache.bytes) and s.kv.device_status() == binding.TPQ_OK
        o, bound = kv_ref.attention(s.cache, s.table, s.start, s.lengths, qr, 1 / math.sqrt(dim))
        w = (rng.standard_normal((E, K)) / math.sqrt(K)).astype(np.float32)
        w_bf = torch.from_numpy(w).to(torch.bfloat16)
        w64 = w_bf.double().numpy()
        y = o.reshape(s.T, K) @ w64.T
        total = total + y
        allowed = allowed + np.broadcast_to(tolerance(o, bound), o.shape).reshape(s.T, K) @ np.abs(w64).T * (1 + 2.0 ** -7) + 2.0 ** -7 * np.abs(y)
        ys.append(y)
        xs.append((x, w_bf.cuda()))
    lim = np.stack([1.1 * np.abs(y).max(0) + 1e-3 for y in ys]).astype(np.float32)
    t.set_ranges(-lim, lim, [1] * N)
    t.select_features()
    for i, (x, w_bf) in enumerate(xs):
        slots = torch.empty_like(w_bf)
        t.permute_weight(w_bf.data_ptr(), K, slots.data_ptr())
        payload = torch.empty(t.payload_bytes(x.shape[0]), dtype=torch.uint8, device="cuda")
        t.linear_quantize_pack(i, x.data_ptr(), slots.data_ptr(), x.shape[0], K, payload.data_ptr(), payload.numel())
        payloads.append(payload)
        ws_slots.append(slots)
    out = torch.empty(xs[0][0].shape[0], E, dtype=torch.float32, device="cuda")
    t.dequant_reduce([p.data_ptr() for p in payloads], out.shape[0], out.data_ptr(), binding.TPQ_OUT_FP32)
    assert t.device_status() == binding.TPQ_OK
    step, _ = t.get_scales()
    # (codes reach from -8 to 7 steps of R/15: the upper end is half a step more than half a step away)
    allowed = allowed + step.astype(np.float64).sum(0)[None] + 1e-5
    err = np.abs(out.cpu().numpy() - total)
    assert (err <= allowed).all(), float((err / allowed).max())


def shared_scale(setup, window, first):
    """What a sequence of more than 32 rows (new positions x query heads per key head) may be off beside the tolerance, [rows, heads, 1]: 16
    positions share a power of two 2^F, the largest magnitude M of theirs is 2^14 .. 2^15 of it, and a weight is P = 2^(y + F - m) in FP16.  The
    row's largest P is 2^7 at least, and P is off by 2^-25 where it is subnormal: a value (below 2^15 2^F) by 2^-25 2^15 2^F0 / 2^7 =
    2^-17 2^F0 <= 2^-31 M0 of the block that the largest P is from, seen by this row or not except for one position.  Values themselves are
    off by half of FP16's smallest step, 2^-25 2^F <= 2^-39 M."""
    s, group = setup, setup.heads // setup.kv_heads
    extra = np.zeros((s.T, s.heads, 1))
    for i, ln in enumerate(s.lengths):
        n, t = s.start[i + 1] - s.start[i], np.arange(ln)
        for kh in range(s.kv_heads):
            if n * group <= 32:
                continue
            step, low, _, _ = s.cache.sequence(s.table[i], int(ln), kh, 1)
            big = np.zeros(-(-ln // 16) * 16)
            big[:ln] = np.nan_to_num(np.maximum(np.abs(low), np.abs(low + 15 * step)))
            big = np.repeat(big.reshape(-1, 16).max(1), 16)[:ln]
            for r in range(n):
                p = ln - n + r
                see = (t <= p) & ((window == 0) | (t > p - window) | (t < first))
                extra[s.start[i] + r, kh * group:(kh + 1) * group] = (see.sum() * 2.0 ** -31 + 2.0 ** -39) * big[see].max()
    return extra


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 3, 40])
def test_attention_over_steps_that_append_does_not_write(new, dim):
    """Pages are the caller's: words with a step of 0 (a pool of zeros), of -0, subnormal or far below `low` stand for low + step * code
    like any other.  Beyond the tolerance, 15 codes of the smallest step there is (2^-60, 2^-24 of `low`), and, as some values are 2^30,
    what sharing a power of two with one may cost."""
    s = Setup(4, 2, dim, 16, [new, new, 1], [200, 150, 40], seed=23, fill=0).fill_with_data()
    patterns = [0x0000, 0x8000, 0x0001, 0x0780, 0x2180]                     # 0, -0, the smallest subnormal, 2^-112, 2^-60
    lows = [0x0000, 0x3FA0, 0xBF80, 0x3100, 0x4E80]                         # 0, 1.25, -1, 2^-29, 2^30
    for i, (at, h) in enumerate([(t, h) for t in list(range(5, 140, 7)) + list(range(200 - new, 200)) for h in (0, 1)]):
        codes = s.rng.integers(0, 16, dim).astype(np.uint8)
        for which in (0, 1):
            low = lows[i % (5 if which else 4)]                             # (keys: none that outweighs all others)
            for q in (0, 1):
                if at < s.lengths[q] and (which or i % 3):
                    s.cache.put(s.table[q, at // 16], h, at % 16, which, codes, patterns[(i + which) % 5] | low << 16)
    for t in range(40):                                                     # a sequence whose pages hold nothing but zeros
        for h in (0, 1):
            for which in (0, 1):
                s.cache.put(s.table[2, t // 16], h, t % 16, which, np.zeros(dim, np.uint8), 0)
    s.d_cache.copy_(torch.from_numpy(s.cache.bytes))
    q, q32 = rows_of(s.rng, s.T, 4 * dim)
    for window, first in ((0, 0), (100, 5), (3, 0)):
        got = s.attention(q, 0.1, window, first)
        assert s.kv.device_status() == binding.TPQ_OK
        want, bound = kv_ref.attention(s.cache, s.table, s.start, s.lengths, q32.reshape(s.T, 4, dim), 0.1, window, first)
        err = np.abs(kv_ref.wide(got).reshape(s.T, 4, dim) - want)
        allowed = tolerance(want, bound) + 15 * (2.0 ** -60 + 2.0 ** -24 * bound) + shared_scale(s, window, first)
        assert (err <= allowed).all(), (window, float(np.nanmax(err)), int(np.isnan(err).sum()))
        assert (want[2 * new] == 0).all()


@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("which,word", [(0, 0x3F807F80), (0, 0x7F803F80), (0, 0xFF803F80), (1, 0x3F807F80), (1, 0x7F803F80), (1, 0x3F80BF80)])
def test_a_word_without_a_range_counts_as_no_number(new, which, word):
    """Steps and lows that are infinite, and negative steps of values: what a NaN is, in the kernels for few rows and in those for many."""
    s = Setup(4, 2, 128, 16, [new, new], [200, 150], seed=25, fill=0xFF).fill_with_data()
    at = 200 - new + (2 if new > 1 else 0)
    s.cache.put(s.table[0, at // 16], 1, at % 16, which, s.rng.integers(0, 16, 128).astype(np.uint8), word)
    s.d_cache.copy_(torch.from_numpy(s.cache.bytes))
    q, _ = rows_of(s.rng, s.T, 512)
    nan = np.isnan(kv_ref.wide(s.attention(q, 0.08, window=100, first=5)).reshape(s.T, 4, 128))
    seen = 2 if new > 1 else 0
    assert nan[seen:new, 2:].all() and not nan[:seen].any() and not nan[:, :2].any() and not nan[new:].any()


def test_append_multiplies_the_range_by_the_number_next_to_a_15th():
    """(22.5 - low) with low = -0.05859375 is 15 x 1.50390625, halfway between the BF16 numbers 1.5 and 1.5078125.  Times 0x3D888889, which is
    5.2e-8 of itself more than 1/15, it is above: 1.5078125 (0x3FC1).  And the word of a vector whose 15 steps are exact."""
    s = Setup(1, 1, 64, 16, [2], [2], seed=27, fill=0)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    x[0, 0], x[0, 1], x[1, 5] = -0.05859375, 22.5, 15.0
    s.kv.append(s.batch, x.data_ptr(), x.data_ptr())
    torch.cuda.synchronize()
    words = s.d_cache[int(s.table[0, 0]), 0, 0, 16 * 64:].cpu().numpy().view(np.uint32)
    for which in (0, 1):
        assert [hex(w) for w in words[16 * which: 16 * which + 2]] == ["0xbd703fc1", "0x3f80"]


@pytest.mark.parametrize("sign", [1, -1])
def test_append_at_ties_of_the_step(sign):
    """Pairs of BF16 ends whose difference (exact) times 0x3D888889 rounds to another step than its 15th, which is a tie of BF16, and as
    many others: words of the product, the low end's codes 0, the high end's 15."""
    f = np.float32
    c15 = np.array([0x3D888889], np.uint32).view(f)[0]
    hi = np.concatenate([np.arange(128, 256) * 2.0 ** (e - 7) for e in range(0, 6)])
    lo = np.concatenate([np.arange(128, 256) * 2.0 ** (e - 7) for e in range(-8, 6)])
    hi, lo = (x.ravel() for x in np.meshgrid(hi, -sign * lo, indexing="ij"))
    d = (hi - lo).astype(f)
    fits = (d == hi - lo) & (d > 0)
    differ = fits & (kv_ref.bf16(d * c15) != kv_ref.bf16(d / f(15)))
    assert differ.sum() > 2000
    rng = np.random.default_rng(5)
    pick = np.concatenate([np.flatnonzero(differ), rng.choice(np.flatnonzero(fits & ~differ), 2000, replace=False)])
    n = len(pick)
    s = Setup(1, 1, 64, 256, [n], [n], seed=29, fill=0)
    x = np.repeat(lo[pick, None], 64, 1)
    x[:, 7] = hi[pick]
    t = torch.from_numpy(x.astype(f)).to(torch.bfloat16).cuda()
    assert np.array_equal(t.double().cpu().numpy(), x)
    s.kv.append(s.batch, t.data_ptr(), t.data_ptr())
    torch.cuda.synchronize()
    s.cache.bytes[:] = s.d_cache.cpu().numpy()
    want = kv_ref.bf16(np.maximum(d[pick] * c15, np.maximum(np.abs(hi[pick]), np.abs(lo[pick])).astype(f) * f(2.0 ** -16)))
    for which in (0, 1):
        step, low, codes, _ = s.cache.sequence(s.table[0], n, 0, which)
        assert np.array_equal(step, kv_ref.wide(want)) and np.array_equal(low, lo[pick])
        assert (np.delete(codes, 7, 1) == 0).all() and (codes[:, 7] == 15).all()


class Alike:
    """One or two sequences over a pool of two pages, `alike` positions of which are one page again and again: attention over them is attention
    over that page (every weight as often).  The second sequence has 16 positions in the other page."""

    def __init__(self, heads, kv_heads, lengths, new, seed=1):
        self.page, self.dim, self.heads, self.kv_heads = 256, 64, heads, kv_heads
        self.kv = binding.TpqKv(heads, kv_heads, 64, 256)
        rng = self.rng = np.random.default_rng(seed)
        self.cache = kv_ref.Cache(2, kv_heads, 64, 256, rng=rng)
        word = rng.uniform(0.05, 0.3, (2, kv_heads, 16, 32)).astype(np.float32), rng.uniform(-2, -1, (2, kv_heads, 16, 32)).astype(np.float32)
        self.cache.bytes[..., 16 * 64:] = (kv_ref.bf16(word[0]).astype(np.uint32) | kv_ref.bf16(word[1]).astype(np.uint32) << 16).view(np.uint8)
        self.T = sum(new)
        self.table = torch.zeros(len(lengths), -(-max(lengths) // 256), dtype=torch.int32, device="cuda")
        self.table[1:] = 1
        self.d = [dev(self.cache.bytes), dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), dev(np.array(lengths, np.int32))]
        self.batch = binding.KvBatch(self.d[0].data_ptr(), 2, self.table.data_ptr(), self.table.shape[1], self.d[1].data_ptr(), self.d[2].data_ptr(), len(lengths), max(new), self.T)
        self.q, self.q32 = rows_of(rng, self.T, heads * 64)

    def run(self):
        whole, view = guarded(self.T * self.heads * 128)
        ws = torch.full((self.kv.attention_workspace_bytes(self.batch),), 0xFF, dtype=torch.uint8, device="cuda")
        self.kv.attention(self.batch, self.q.data_ptr(), view.data_ptr(), ws.data_ptr(), ws.numel(), 0.1)
        torch.cuda.synchronize()
        assert guards_intact(whole, self.T * self.heads * 128)
        return view.view(torch.int16).view(self.T, self.heads, 64).cpu().numpy().view(np.uint16)


def test_a_sequence_of_millions_of_tiles():
    """9.4 million tiles of 256 positions in one sequence (4096 key heads), beside a short one: both are answered.  A lane adds up 18
    thousand weights one after the other (590 000 positions over 4 warps and 8 lanes), each time within 2^-24 of the sum: 2^-10 of
    normaliser and offsets each (1.1 times that by the count, of which the tolerance's 2^-8 of the value has room for a tenth)."""
    s = Alike(4096, 4096, [2304 * 256, 16], [1, 1])
    got = kv_ref.wide(s.run()).astype(np.float64)
    assert s.kv.device_status() == binding.TPQ_OK
    want, bound = kv_ref.attention(s.cache, [[0], [1]], [0, 1, 2], [256, 16], s.q32.reshape(2, 4096, 64), 0.1)
    assert (np.abs(got - want) <= tolerance(want, bound) + np.array([2.0 ** -9, 0])[:, None, None] * bound).all()


@pytest.mark.parametrize("heads,kv_heads,new,length", [(4096, 4096, 1, 2 ** 27),      # few rows: 2^31 tiles and more
                                                       (8192, 4096, 4, 2 ** 27)])     # the same in tiles of 128
def test_more_work_than_can_be_numbered_is_left_out(heads, kv_heads, new, length):
    s = Alike(heads, kv_heads, [length, 16], [new, 1])
    assert (s.run() == 0xA5A5).all()
    assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG and s.kv.device_status() == binding.TPQ_OK
    s.d[2].copy_(torch.tensor([16, 16], dtype=torch.int32))                           # and the same call with less to do is answered
    got = kv_ref.wide(s.run()).astype(np.float64)
    assert s.kv.device_status() == binding.TPQ_OK
    want, bound = kv_ref.attention(s.cache, [[0], [1]], [0, new, new + 1], [16, 16], s.q32.reshape(new + 1, heads, 64), 0.1)
    assert (np.abs(got - want) <= tolerance(want, bound)).all()


@pytest.mark.parametrize("new", [256, 300, 1024])   # 2^31 tiles and more, the same with a block of rows that is not full, 2^33 (0 in 32 bits)
def test_more_tiles_of_many_rows_than_can_be_numbered_are_left_out(new):
    s = Alike(256, 1, [2 ** 30, 16], [new, 1])
    assert (s.run() == 0xA5A5).all()
    assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG and s.kv.device_status() == binding.TPQ_OK
    s.d[1].copy_(torch.tensor([0, 40, 41], dtype=torch.int32))
    s.d[2].copy_(torch.tensor([300, 16], dtype=torch.int32))
    got = s.run()
    assert s.kv.device_status() == binding.TPQ_OK and (got[41:] == 0xA5A5).all()
    want, bound = kv_ref.attention(s.cache, [[0, 0], [1, 1]], [0, 40, 41], [300, 16], s.q32[:41].reshape(41, 256, 64), 0.1)
    assert (np.abs(kv_ref.wide(got[:41]) - want) <= tolerance(want, bound)).all()


@pytest.mark.parametrize("new", [1, 5, 40])
def test_values_of_sizes_far_apart(new):
    """Zero vectors and blocks of them (steps of 2^-60) beside values of 2^37: their weights count all the same.  Beside the tolerance, what a
    power of two for 16 positions may cost (the definition's 2^-31 of the largest a position)."""
    s = Setup(4, 2, 128, 16, [new, new], [230, 90], seed=37, fill=0xFF).fill_with_data()
    for i, ln in enumerate(s.lengths):
        for t in range(ln):
            for h in range(2):
                x = np.zeros(128) if t // 16 % 3 == 1 or t % 5 == h else s.rng.standard_normal(128) * 2.0 ** 37
                codes, words = kv_ref.quantise(x.astype(np.float32)[None])
                s.cache.put(s.table[i, t // 16], h, t % 16, 1, codes[0], words[0])
    s.d_cache.copy_(torch.from_numpy(s.cache.bytes))
    q, q32 = rows_of(s.rng, s.T, 512)
    for window in (0, 40):
        got = kv_ref.wide(s.attention(q, 0.1, window)).reshape(s.T, 4, 128)
        want, bound = kv_ref.attention(s.cache, s.table, s.start, s.lengths, q32.reshape(s.T, 4, 128), 0.1, window)
        assert (np.abs(got - want) <= tolerance(want, bound) + shared_scale(s, window, 0)).all()


def test_reports_right_after_the_status_was_read_are_kept():
    """The status word is cleared before the call that reads it returns: what a kernel on a stream of its own reports next is still there."""
    s = Setup(4, 2, 128, 16, [1], [20], seed=39).fill_with_data()
    q, _ = rows_of(s.rng, s.T, 512)
    s.d_table.fill_(-1)
    side = torch.cuda.Stream()
    for _ in range(50):
        s.attention(q, 0.1, stream=side.cuda_stream)
        assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG
    assert s.kv.device_status() == binding.TPQ_OK


@pytest.mark.parametrize("start", [[9, 10, 0, 20, 50], [12, 40, 41, 3, 45, 50], [30, 31, 30, 31, 30, 31, 0, 31, 31, 31, 50]], ids=lambda s: f"{len(s) - 1}")
def test_rows_before_the_start_that_a_search_ends_at_are_nobodys(start):
    """Starts that go down lead the search for a row's sequence to one that begins behind the row, whose positions would lie ahead of the
    page table's row: nothing is read or written there.  Entries may be written for (row, sequence) pairs where the row is the sequence's."""
    n, page = len(start) - 1, 16
    s = Setup(4, 2, 128, page, [1] * n, [1] * n, pad=50 - n, seed=43, fill=0, max_new=50)
    table = torch.full((n + 2, 1), 2 ** 30, dtype=torch.int32, device="cuda")          # ahead of the table and behind it: no page
    table[1:-1] = dev(s.table)
    s.batch.page_table_ptr = table[1].data_ptr()
    d_start = dev(np.array(start, np.int32))
    s.batch.token_start_ptr = d_start.data_ptr()
    k, _ = rows_of(s.rng, 50, 256)
    s.kv.append(s.batch, k.data_ptr(), k.data_ptr())
    assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG
    want = kv_ref.Cache(s.n_pages, 2, 128, page, fill=0)
    for i in range(n):
        if start[i + 1] - start[i] == 1:                                               # (one row, one position: consistent by itself)
            x = k[start[i]].float().cpu().numpy().reshape(1, 2, 128)
            codes, words = kv_ref.quantise(x)
            for h in range(2):
                for which in (0, 1):
                    want.put(s.table[i, 0], h, 0, which, codes[0, h], words[0, h])
    got = s.d_cache.cpu().numpy()
    assert ((got == want.bytes) | (got == 0)).all()                                    # (or left out, where the search does not find it)
    out = torch.full((50, 256), 7, dtype=torch.int16, device="cuda")
    s.kv.read(s.batch, out.data_ptr(), None)
    assert s.kv.device_status() == binding.TPQ_ERR_INVALID_ARG
    mine = {start[i] for i in range(n) if start[i + 1] - start[i] == 1}
    assert all((out[r] == 7).all() for r in range(50) if r not in mine)


FULL = [  # calls of so many vectors that a lane takes four at a time (12 warps for every SM), their last job filled in part
    (10, 10, 128, 64, [720], [720], 128, False, 0, 0),
    (10, 10, 128, 16, [1, 719], [40, 900], 48, False, 3, 8),
    (18, 18, 64, 32, [800], [830], 64, False, 3, 8),
    (17, 17, 64, 16, [400, 0, 500], [400, 3, 512], 16, True, 0, 0),
    (20, 5, 128, 16, [300, 0, 1150], [320, 0, 1150], 64, True, 2, 8),
]


@pytest.mark.parametrize("case", FULL, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}p{c[3]}r{c[6]}{'i' if c[7] else ''}")
def test_append_and_read_of_many_vectors(case):
    heads, kvh, dim = case[:3]
    warps = lambda vectors: (sum(case[4]) + case[8]) * vectors // (256 // dim) // 4  # noqa: E731
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert warps(2 * kvh) >= 12 * sms and warps(2 * kvh + heads) >= 12 * sms and (kvh % (4 * 256 // dim) or heads % (4 * 256 // dim))
    test_append_writes_the_bytes_of_the_definition(case, True)


def tolerance_many(setup, q32, out, bound, scale, window, first):
    """Of sequences of more than 32 rows: keys are FP16 (2^-11 of a value, or 2^-25 2^Fk <= 2^-39 of its block's largest magnitude, the larger of
    which counts), which moves an exponent by scale sum |q_d| dk_d, E at most over what a row sees; a weight by exp(E) - 1 of itself, and
    numerator and normaliser by that of B.  The same for the weights' rounding (2^-11) and 2^-12 for the binary32 of the exponents: a sum of
    dim products whose magnitudes add up to at most 30 128 / dim (held to) is off by dim 2^-24 of that, 0.94 2^-12.
    Values 2^-11 of B, and what their shared power of two costs.  Half a step of BF16 of the answer."""
    s, group, allowed = setup, setup.heads // setup.kv_heads, np.zeros_like(out)
    q = np.abs(q32.reshape(s.T, s.heads, s.dim).astype(np.float64))
    for i, ln in enumerate(s.lengths):
        n, t = int(s.start[i + 1] - s.start[i]), np.arange(ln)
        for kh in range(s.kv_heads):
            step, low, codes, _ = s.cache.sequence(s.table[i], int(ln), kh, 0)
            k = np.abs(low[:, None] + step[:, None] * codes)
            big = np.zeros(-(-int(ln) // 16) * 16)
            big[:ln] = np.maximum(np.abs(low), np.abs(low + 15 * step))
            big = np.repeat(big.reshape(-1, 16).max(1), 16)[:ln, None]
            dk = np.maximum(2.0 ** -11 * k, 2.0 ** -39 * big)
            for r in range(n):
                p = int(ln) - n + r
                see = (t <= p) & ((window == 0) | (t > p - window) | (t < first))
                rows = np.s_[s.start[i] + r, kh * group:(kh + 1) * group]
                assert (abs(scale) * (q[rows] @ k[see].T)).max() < 30 * (128 / s.dim)
                E = abs(scale) * (q[rows] @ dk[see].T).max(1)[:, None]
                allowed[rows] = 2.0 ** -8 * np.abs(out[rows]) + (2 * np.expm1(E) + 2 * 2.0 ** -11 + 2 * 2.0 ** -12 + 2.0 ** -11) * bound[rows]
    return allowed + shared_scale(s, window, first)


@pytest.mark.parametrize("case", [(4, 2, 128, 32, [130], [130], 0, 0, 0.1), (6, 2, 64, 256, [40, 61], [40, 600], 0, 0, 0.15), (16, 2, 128, 32, [33, 64], [640, 64], 128, 128, 0.02),
                                  (2, 2, 64, 16, [260], [300], 17, 20, -0.2), (40, 1, 128, 16, [1, 2], [500, 33], 0, 0, 0.1)],
                         ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}n{max(c[4])}l{max(c[5])}w{c[6]}")
def test_attention_of_many_rows_within_what_its_roundings_allow(case):
    heads, kvh, dim, page, new, lengths, window, first, scale = case
    s = Setup(heads, kvh, dim, page, new, lengths, seed=45, fill=0xFF).fill_with_data()
    q, q32 = rows_of(s.rng, s.T, heads * dim)
    got = kv_ref.wide(s.attention(q, scale, window, first)).reshape(s.T, heads, dim)
    assert s.kv.device_status() == binding.TPQ_OK
    want, bound = kv_ref.attention(s.cache, s.table, s.start, s.lengths, q32.reshape(s.T, heads, dim), scale, window, first)
    assert (np.abs(got - want) <= tolerance_many(s, q32, want, bound, scale, window, first)).all()


@pytest.mark.parametrize("case", [(8, 1, 128, 64, [1, 4, 1, 0], [30000, 200, 9001, 50], 0, 0), (8, 1, 128, 256, [1, 40, 1], [30000, 300, 513], 0, 0), (4, 2, 64, 64, [1, 5, 2], [20000, 900, 7777], 0, 0),
                                  (2, 1, 64, 256, [1, 9, 3], [40000, 9, 12000], 0, 0), (8, 1, 128, 64, [1, 2], [30000, 16000], 5000, 70)],
                         ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}n{max(c[4])}l{max(c[5])}w{c[6]}")
def test_few_rows_beside_more_over_long_contexts(case):
    """Sequences of at most 8 rows at long contexts, in batches whose other sequences have them taken 16 rows at a time."""
    heads, kvh, dim, page, new, lengths, window, first = case
    s = Setup(heads, kvh, dim, page, new, lengths, seed=47, fill=0xFF).fill_with_data()
    q, q32 = rows_of(s.rng, s.T, heads * dim)
    got = s.attention(q, 0.1, window, first)
    assert s.kv.device_status() == binding.TPQ_OK
    check(s, q32, got, 0.1, window, first)
