"""What the binding passes to the calls of the 8-bit cache, without a GPU: the library is a stand-in that keeps the arguments."""
from __future__ import annotations

import pytest
import torch

import paper_2602_20732_amd as pk


class Kept:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def chess(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    c = pk.Chess.__new__(pk.Chess)
    c.cfg, c.lib, c._h, c.device = pk.Config(8, 2, 16, 2, 4, 4), Kept(), None, -1      # (-1: where CPU tensors say they are)
    monkeypatch.setattr(pk.Chess, "__del__", lambda self: None, raising=False)
    return c


def store(chess, k_new, v_new, n_pages=7):
    writes, counts = torch.zeros((3, 4), dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    k, v = torch.zeros((n_pages, 2, 16, 128), dtype=torch.uint8), torch.zeros((n_pages, 2, 128, 16), dtype=torch.uint8)
    chess.quant_store(k_new, v_new, writes, counts, k, v, torch.zeros((n_pages, 2, 2)))
    (name, a), = chess.lib.calls
    return name, dict(zip(("ctx", "k", "k_stride", "v", "v_stride", "n_rows", "writes", "counts", "max_writes", "k_pool", "v_pool", "scales", "n_pages"), a))


def test_the_store_is_told_how_many_rows_and_pages_there_are(chess):
    wide = torch.zeros((9, 12, 128), dtype=torch.bfloat16)
    name, a = store(chess, wide[:5, 8:10], wide[:5, 10:])
    assert name == "chess_quant_store_bounded"
    assert (a["n_rows"], a["n_pages"], a["max_writes"], a["k_stride"], a["v_stride"]) == (5, 7, 3, 12 * 128, 12 * 128)


def test_without_a_context_the_bounded_store_is_refused():
    import os
    if not os.path.exists(pk.library_path()):
        from paper_2602_20732_amd.build import build
        build()
    lib = pk.load_library()
    assert lib.chess_quant_store_bounded(None, None, 1024, None, 1024, 5, None, None, 1, None, None, None, 7, None) == -1


def test_the_stride_of_one_token_is_not_passed_on(chess):
    """A dimension of size one may have any stride; the library wants one that a row fits in."""
    one = torch.zeros((2, 1, 128), dtype=torch.bfloat16).transpose(0, 1)
    assert one.stride(0) == 128
    _, a = store(chess, one, torch.zeros(256, dtype=torch.bfloat16).as_strided((1, 2, 128), (1, 128, 1)))
    assert (a["n_rows"], a["k_stride"], a["v_stride"]) == (1, 256, 256)
