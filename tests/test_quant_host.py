"""The 8-bit cache and the dealing of pages without a GPU: the reference the kernels' tests compare with is pinned against torch's e4m3 and
worked examples, and calls that the entry points refuse."""
from __future__ import annotations

import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
import quant_reference as ref


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pk.library_path()):
        from paper_2602_20732_amd.build import build
        build()
    return pk.load_library()


def test_e4m3_of_the_reference_is_the_one_torch_has():
    every = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(every.view(torch.float8_e4m3fn).double().numpy(), ref.TABLE, equal_nan=True)
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.normal(0, s, 4000) for s in (0.001, 0.02, 1, 100)] + [ref.TABLE[:127], (ref.TABLE[:126] + ref.TABLE[1:127]) / 2, [0.0, -0.0, 448, -448]])
    x = np.clip(x, -448, 448).astype(np.float32)
    got = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(got, ref.encode(x))


def test_scales_of_the_reference():
    for a, e in ((0.0, -64), (448.0, 0), (448.5, 1), (224.0, -1), (1.75, -8), (1.7578125, -7), (2.0 ** -60, -64), (float(torch.finfo(torch.bfloat16).max), 119)):
        assert ref.exponent(a) == e, a


def test_worked_example_of_the_dealing():
    """Two sequences, pages of 16: 15 held and 2 wanted (one joins a page, one opens one), 0 held and 17 wanted."""
    got = ref.map_tokens([15, 0], [2, 17], [[7, -1], [-1, -1]], [1, 2, 3, 4], 4, 100, 2, 16)
    assert got["table"] == [[7, 4], [3, 2]] and got["lens_after"] == [17, 17] and got["n_left"] == 1 and got["starts"] == [0, 2, 19]
    assert got["slots"][:3] == [7 * 16 + 15, 4 * 16, 3 * 16] and got["slots"][-1] == 2 * 16
    assert got["writes"] == [[7, 0, 15, 1], [4, 1, 0, 1], [3, 2, 0, 16], [2, 18, 0, 1]] and got["counts"] == [19, 4, 3, 0]
    # one page short: the second sequence waits; a third would have to wait behind it
    got = ref.map_tokens([15, 0, 0], [2, 17, 1], [[7, -1], [-1, -1], [-1, -1]], [1, 2], 2, 100, 2, 16)
    assert got["lens_after"] == [17, 0, 0] and got["counts"] == [2, 2, 1, 2]
    assert ref.release([17, 5, 3], [1, 0, 1], got["table"][:1] + [[9, -1], [8, -1]], [1, 2, -1, -1, -1], 1, 5, 16) == ([0, 5, 0], [1, 7, 2, 8, -1], 4)


def test_split_rule_of_8_bit_pages(tmp_path):
    """Over device sizes, heads, groups, batches and lengths the partials fit the workspace and one sequence's workgroups the compute units."""
    exe, root = str(tmp_path / "rule"), os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                          os.path.join(root, "paper_2602_20732_amd", "csrc"), os.path.join(root, "tests", "quant_split_rule_driver.cpp"), "-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr


def test_without_a_context_every_call_is_refused(lib):
    n = ctypes.c_size_t()
    assert lib.chess_write_rows(None, 1, 1, ctypes.byref(n)) == -1
    assert lib.chess_release_pages(None, None, None, 1, None, None, 1, None, None, None, None, None) == -1
    assert lib.chess_map_tokens(None, None, None, 1, 1, *[None] * 11) == -1
    assert lib.chess_quant_store(None, None, 1024, None, 1024, None, None, 1, None, None, None, None) == -1
    assert lib.chess_quant_summarize(None, None, None, None, None, 1, None, 0, None, None) == -1
    assert lib.chess_quant_sparse_decode(None, None, None, None, None, None, None, None, None, 1, None, None, None) == -1
    assert lib.chess_quant_dense_decode(None, None, None, None, None, None, None, 1, None, None, None) == -1


def test_the_binding_refuses_tensors_that_a_pointer_would_misread():
    """Types, sizes and strides are looked at before the device is."""
    c = pk.Chess.__new__(pk.Chess)
    c.cfg = pk.Config(8, 2, 16, 2, 4, 4)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(pk.ChessError, match="seq_lens"):
        c.map_tokens(torch.zeros(2, dtype=torch.int64), i32(2), i32(2, 4), i32(4), i32(1), i32(2), i32(1), i32(3), None, i32(8, 4), i32(4), None, max_tokens=8)
    with pytest.raises(pk.ChessError, match="slots or max_tokens"):
        c.map_tokens(i32(2), i32(2), i32(2, 4), i32(4), i32(1), i32(2), i32(1), i32(3), None, i32(8, 4), i32(4), None)
    with pytest.raises(pk.ChessError, match="seq_lens"):
        c.release_pages(i32(4)[::2], i32(2), i32(2, 4), i32(4), i32(1), i32(2), i32(1), None)
    with pytest.raises(pk.ChessError, match="k_new"):
        c.quant_store(torch.zeros(3, 2, 128), torch.zeros(3, 2, 128), i32(3, 4), i32(4), None, None, None)
    with pytest.raises(pk.ChessError, match="k_new"):
        c.quant_store(torch.zeros(3, 128, 2, dtype=torch.bfloat16).transpose(1, 2), None, i32(3, 4), i32(4), None, None, None)
    with pytest.raises(pk.ChessError, match="q: "):
        c.quant_dense_decode(torch.zeros(2, 8, 128), None, None, None, i32(2, 4), i32(2), None, None)
    with pytest.raises(pk.ChessError, match="scales"):
        c.quant_summarize(None, torch.zeros(4, 2, 2, dtype=torch.float16), i32(2, 4), i32(2), None)
