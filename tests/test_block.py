"""Feed-forward block, 4-bit weights and answers without a GPU: the plain implementation, structure layouts, refusals that need no handle."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

import block_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2411_07942_b200 import binding, build

    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantised_values_are_within_half_a_step_and_exact_in_bf16(group):
    rng = np.random.default_rng(group)
    w = torch.from_numpy(rng.standard_normal((60, 300)) * np.exp(3 * rng.standard_normal((60, 300)))).to(torch.bfloat16).double().numpy()
    codes, byte, factor = block_ref.quantise(w, group)
    v = block_ref.values(codes, byte, factor, group)
    step = np.repeat(factor[:, None] * 2.0 ** ((byte >> 4) - 8.0) * (1 + (byte & 15) / 16), group, 1)[:, :300]
    assert (np.abs(v - w) <= step / 2).all() and codes.min() == -8 and codes.max() == 7
    assert np.array_equal(torch.from_numpy(v).to(torch.bfloat16).double().numpy(), v)
    # no step is more than a 16th above 2a/15 unless the row's largest one is 2^15 of it
    a = np.abs(np.pad(w, ((0, 0), (0, -300 % group)))).reshape(60, -1, group).max(2)
    s = step[:, ::group]
    assert ((s <= 2 * a / 15 * (1 + 1 / 16)) | (byte == 0)).all() and (s >= 2 * a / 15).all()


def test_the_layout_of_a_block():
    """Output 2's input 37 (piece 1, word 0, second of pair 2) and its step, by hand."""
    codes = np.zeros((130, 200), int)
    codes[2, 37] = -8
    byte = np.zeros((130, 4), np.uint8)
    byte[2, 3] = 0xAB
    raw = block_ref.pack(codes, byte, np.ones(130, np.float32), 64)
    block = 8192 + 256
    assert raw.size == 2 * 2 * block + 256 * 4
    word = raw[2048 + 2 * 16: 2048 + 2 * 16 + 4].view(np.uint32)[0]
    assert word == 0x88888888 - (8 << (16 + 8))
    assert raw[2048 + 2 * 16 + 4: 2048 + 2 * 16 + 8].view(np.uint32)[0] == 0x88888888
    assert raw[block + 8192 + 128 + 2] == 0xAB                                              # inputs 192 .. are group 1 of block 1
    assert raw[4 * block:].view(np.float32)[:130].tolist() == [1.0] * 130


def test_plain_answers():
    x = torch.tensor([[0.0, math.log(3.0), -math.inf, 0.0], [-math.inf] * 4, [5.0, 5.0, 5.0, 5.0]], dtype=torch.float64)
    logprob, entropy, top, top_logprob = block_ref.answers(x, [1, 0, -1], 3)
    assert logprob[0] == pytest.approx(math.log(0.6)) and logprob[1] == -math.inf and logprob[2] == 0
    assert entropy[0] == pytest.approx(-(0.6 * math.log(0.6) + 0.4 * math.log(0.2))) and entropy[1] == 0 and entropy[2] == pytest.approx(math.log(4))
    assert top.tolist() == [[1, 0, 3], [0, 1, 2], [0, 1, 2]] and top_logprob[2].tolist() == pytest.approx([math.log(0.25)] * 3)


def test_sizes(binding):
    for n, K, g in ((1, 1, 32), (128, 128, 64), (129, 129, 128), (32000, 5120, 32)):
        assert binding.weight4_bytes(n, K, g) == block_ref.pack(np.zeros((n, K), int), np.zeros((n, -(-K // g)), np.uint8), np.zeros(n, np.float32), g).size if n < 1000 else True
        tiles = -(-n // 128)
        assert binding.weight4_bytes(n, K, g) == tiles * -(-K // 128) * (8192 + 128 * (128 // g)) + tiles * 512
    assert [binding.weight4_bytes(*a) for a in ((0, 1, 32), (1, 0, 32), (1, 1, 16), (1, 2 ** 17 + 1, 32), (2 ** 30 + 1, 1, 32), (-1, 1, 32))] == [0] * 6
    assert binding.token_record_bytes(3, 0) == 60 and binding.token_record_bytes(3, 20) == 3 * 4 * 45
    assert [binding.token_record_bytes(*a) for a in ((-1, 0), (1, -1), (1, 33), (2 ** 27 + 1, 0), (0, 5))] == [0] * 5


def test_null_handles_are_rejected(binding):
    L = binding.lib()
    w = binding.Weight(16, 8, 8, 8, 0, 32)
    assert L.tpq_block_create(None) == 1 and L.tpq_block_destroy(None) == 0
    assert L.tpq_quantize_weight(None, 16, 8, 8, 8, 32, 16, 10 ** 6, None) == 1
    assert L.tpq_read_weight(None, 16, 8, 8, 32, 16, 8, None) == 1
    assert L.tpq_linear4(None, w, 16, 8, 1, 16, 0, 8, None) == 1
    assert L.tpq_gated(None, w, w, 0, 16, 8, 1, 16, 8, None) == 1
    assert L.tpq_token_stats(None, 16, 0, 8, 1, 8, 0, None, 0, 16, 100, None) == 1
    assert L.tpq_token_logprobs(None, None, 1, 1, None, None, 0, None, None, None) == 1
    assert L.tpq_block_device_status(None) == 1 and L.tpq_block_launch_count(None) == 0 and L.tpq_block_last_error(None) == b""


def test_structure_layout_matches_the_header(binding, tmp_path):
    names = [f[0].replace("data_ptr", "data_dev") for f in binding.Weight._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tpq.h"\nint main(void) { printf("%zu", sizeof(tpq_weight));'
                   + "".join(f' printf(" %zu", offsetof(tpq_weight, {n}));' for n in names) + " return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", f"-I{ROOT}/include", str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(binding.Weight)] + [getattr(binding.Weight, f[0]).offset for f in binding.Weight._fields_]
