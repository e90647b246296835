"""The 4-bit key/value cache without a GPU: the plain implementation, structure layouts, refusals that need no handle."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import kv_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2411_07942_b200 import binding, build

    build.build()
    binding.lib()
    return binding


def _value(codes, words):
    return kv_ref.wide((words >> 16).astype(np.uint16)).astype(float)[..., None] + kv_ref.wide((words & 0xFFFF).astype(np.uint16)).astype(float)[..., None] * codes


@pytest.mark.parametrize("dim", [64, 128])
def test_values_are_within_half_a_step(dim):
    """|x - value| <= step/2 + the excess of the ends: low is off by half a BF16 step of itself (2^-8 |low|), the rounded step's
    15 multiples by 15 step 2^-8."""
    rng = np.random.default_rng(1)
    x = kv_ref.wide(kv_ref.bf16((rng.standard_normal((200, dim)) * np.exp(3 * rng.standard_normal((200, 1))) + 2 * rng.standard_normal((200, 1))).astype(np.float32)))
    codes, words = kv_ref.quantise(x)
    step = kv_ref.wide((words & 0xFFFF).astype(np.uint16)).astype(float)
    low = kv_ref.wide((words >> 16).astype(np.uint16)).astype(float)
    err = np.abs(_value(codes, words) - x)
    assert (err <= (0.5 + 15 * 2.0 ** -8) * step[:, None] + 2.0 ** -8 * np.abs(low)[:, None] * 1e-6 + 1e-6 * np.abs(x)).all()
    assert codes.max() == 15 and codes.min() == 0


def test_constant_zero_and_tiny_vectors_read_back():
    x = np.stack([np.zeros(64), np.full(64, 3.0), np.full(64, -2.0 ** -100), np.full(64, 2.0 ** -70)]).astype(np.float32)
    codes, words = kv_ref.quantise(x)
    assert (codes == 0).all() and np.array_equal(_value(codes, words), x.astype(float))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_vectors_that_are_no_numbers_read_as_nan(bad):
    x = np.ones((3, 64), np.float32)
    x[1, 5] = bad
    codes, words = kv_ref.quantise(x)
    assert list(words) == [words[0], 0x7FC03F80, words[0]] and (codes == 0).all()
    assert np.isnan(_value(codes, words)[1]).all() and (_value(codes, words)[[0, 2]] == 1).all()
    x[1] = np.linspace(-3.3e38, 3.3e38, 64)   # finite, but its range is not
    assert kv_ref.quantise(x)[1][1] == 0x7FC03F80


def test_rotation_keeps_lengths_and_turns_pairs():
    rng = np.random.default_rng(2)
    a = rng.uniform(0, 6, (9, 8))
    table = np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)
    x = rng.standard_normal((9, 2, 64)).astype(np.float32)
    for inter in (False, True):
        y = kv_ref.rotate(x, table, np.arange(9), 16, inter)
        assert np.array_equal(y[..., 16:], x[..., 16:])
        z = (x[..., 0:16:2] + 1j * x[..., 1:16:2]) if inter else (x[..., :8] + 1j * x[..., 8:16])
        w = z * np.exp(1j * a)[:, None]
        got = (y[..., 0:16:2] + 1j * y[..., 1:16:2]) if inter else (y[..., :8] + 1j * y[..., 8:16])
        assert np.allclose(got, w, atol=1e-5)


def test_structures_have_the_layout_of_the_header(binding, tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "tpq.h"\n#define P(s, f) printf("%s %zu\\n", #f, offsetof(s, f))\nint main(void) {\n'
                   'printf("%zu %zu\\n", sizeof(tpq_kv_batch), sizeof(tpq_kv_rotation));\n'
                   + "".join(f"P(tpq_kv_batch, {f});\n" for f in ("cache_dev", "n_pages", "page_table_dev", "page_table_stride", "token_start_dev",
                                                                    "lengths_dev", "n_seqs", "max_new", "n_tokens"))
                   + "".join(f"P(tpq_kv_rotation, {f});\n" for f in ("table_dev", "n_positions", "rot_dim", "interleaved", "positions_dev")) + "return 0; }\n")
    exe = tmp_path / "s"
    subprocess.run(["gcc", f"-I{ROOT}/include", "-o", str(exe), str(src)], check=True)
    lines = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split("\n")
    assert lines[0] == f"{ctypes.sizeof(binding.KvBatch)} {ctypes.sizeof(binding.KvRotation)}"
    got = [int(x.split()[1]) for x in lines[1:] if x]
    assert got == [getattr(S, f).offset for S in (binding.KvBatch, binding.KvRotation) for f, _ in S._fields_]


@pytest.mark.parametrize("args", [(0, 1, 128, 16), (1, 0, 128, 16), (6, 4, 128, 16), (4, 8, 128, 16), (257, 1, 128, 16), (8, 8, 96, 16), (8, 8, 256, 16), (8, 8, 0, 16),
                                  (8, 8, 128, 0), (8, 8, 128, 8), (8, 8, 128, 48), (8, 8, 128, 512), (-8, -8, 128, 16)])
def test_create_refuses_geometries_before_touching_cuda(binding, args):
    h = ctypes.c_void_p()
    assert binding.lib().tpq_kv_create(ctypes.byref(h), *args) == binding.TPQ_ERR_INVALID_ARG and not h.value
    assert binding.lib().tpq_kv_create(None, 8, 8, 128, 16) == binding.TPQ_ERR_INVALID_ARG


def test_null_handles_are_rejected_not_crashed(binding):
    L = binding.lib()
    assert L.tpq_kv_destroy(None) == 0 and L.tpq_kv_page_bytes(None) == 0 and L.tpq_kv_last_error(None) == b"" and L.tpq_kv_launch_count(None) == 0
    assert L.tpq_kv_append(None, None, None, None, 0, None, 0, None, 0, None, 0, None) == 1
    assert L.tpq_kv_read(None, None, None, 0, None, 0, None) == 1
    assert L.tpq_kv_attention(None, None, None, 0, 1.0, 0, 0, None, 0, None, 0, None) == 1
    assert L.tpq_kv_attention_workspace(None, 1, 1, 1) == 0 and L.tpq_kv_device_status(None) == 1


def test_extension_calls_pass_on_what_ctypes_would(binding):
    """kv_append and kv_attention of the extension module, bound to recorders: structures arrive by value's address, plain arguments as the C
    signature types them; any other form is left to ctypes without a call."""
    seen, keep, addresses = [], [], []
    for name in binding._CALLS:
        res, types = binding.SIGNATURES[name]
        plain = [ctypes.c_void_p if isinstance(a, type) and issubclass(a, ctypes._Pointer) else a for a in types]

        def record(*args, _name=name):
            kinds = {1: binding.KvBatch, 2: binding.KvRotation} if _name == "tpq_kv_append" else {1: binding.KvBatch}
            seen.append((_name, [bytes(kinds[i].from_address(x)) if i in kinds and x else x for i, x in enumerate(args)]))
            return 5

        fn = ctypes.CFUNCTYPE(res, *plain)(record)
        keep.append(fn)
        addresses.append(ctypes.cast(fn, ctypes.c_void_p).value)
    c, ctx, big = binding._calls, 2 ** 47 + 8, 2 ** 64 - 16
    batch = binding.KvBatch(2 ** 47, 2 ** 33, 16, 7, 32, 48, 3, 4, 2 ** 20)
    rot = binding.KvRotation(64, 2 ** 21, 128, 1, None)
    try:
        c.bind(addresses)
        args = (ctx, batch, rot, 16, 24, 32, 40, 48, 56, 64, 72, big)
        assert c.kv_append(*args) == 5
        assert seen.pop() == ("tpq_kv_append", [ctx, bytes(batch), bytes(rot), 16, 24, 32, 40, 48, 56, 64, 72, big])
        assert c.kv_append(ctx, batch, None, 16, 24, 32, 40, None, 56, None, 72, 0) == 5
        assert seen.pop() == ("tpq_kv_append", [ctx, bytes(batch), None, 16, 24, 32, 40, None, 56, None, 72, None])
        for i, bad in ((1, rot), (1, bytes(batch)), (1, None), (2, batch), (3, 1.0), (4, None), (11, "0")):
            assert c.kv_append(*args[:i], bad, *args[i + 1:]) is None
        args = (ctx, batch, 16, 24, 0.125, 2 ** 40, -1, 32, 40, 48, 2 ** 63, big)
        assert c.kv_attention(*args) == 5
        assert seen.pop() == ("tpq_kv_attention", [ctx, bytes(batch), 16, 24, 0.125, 2 ** 40, -1, 32, 40, 48, 2 ** 63, big])
        for i, bad in ((1, rot), (1, ctypes.pointer(batch)), (4, 1), (4, np.float64(1)), (5, 1.5), (9, None), (10, -1)):
            assert c.kv_attention(*args[:i], bad, *args[i + 1:]) is None
        assert not seen
    finally:
        c.bind([ctypes.cast(getattr(binding.lib(), n), ctypes.c_void_p).value for n in binding._CALLS])
    kv = binding.TpqKv.__new__(binding.TpqKv)   # a closed handle: refused by the library either way
    kv._h, kv._p, kv.n_heads, kv.n_kv_heads, kv.head_dim, kv.page_size = ctypes.c_void_p(), None, 2, 2, 64, 16
    for call in (lambda: kv.append(batch, 16, 16), lambda: kv.attention(batch, 16, 32, 48, 64, scale=0.5), lambda: kv.attention(batch, 16, 32, 48, 64, scale=1),
                 lambda: kv.read(batch, 16, 32)):
        with pytest.raises(binding.TpqError) as e:
            call()
        assert e.value.status == binding.TPQ_ERR_INVALID_ARG
