"""The quantising store given entries that name tokens or pages which the tensors do not have."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
import quant_reference as ref
from test_gpu_quant import Cache, bf16, ints

pytestmark = pytest.mark.gpu
SUMMARY_DTYPE_SWEEP = False
D, H = 128, 3
TOP = 2 ** 31 - 1


@pytest.mark.parametrize("B", [16, 32])
def test_entries_beyond_the_tensors_store_nothing(B):
    """Rows and pages of a larger allocation lie on both sides of the tensors that are passed."""
    rng = np.random.default_rng(B)
    n, n_pages, margin = 40, 12, 3
    cache = Cache(rng, n_pages + 2 * margin, H, B)
    k, v, scales = cache.cuda()
    rows = bf16(rng.normal(0, 30, (2, n + 2 * B, H, D)))
    inside = [[0, 0, 0, B], [1, n - 1, 3, 1], [2, n - 5, B - 5, 5], [n_pages - 1, n - B, 0, B]]
    outside = [[3, n, 0, 1], [4, n - 1, 2, 2], [5, n - B + 1, 0, B], [6, -1, 0, 4], [7, -TOP - 1, 0, 4], [8, TOP, 0, 4], [9, TOP - 3, 0, B],
               [n_pages, 0, 0, 4], [-1, 0, 0, 4], [TOP, 0, 0, 4], [-TOP - 1, 0, 0, 4]]
    entries = [e for pair in zip(outside, inside + [[10, 1, 0, 0]] * 7) for e in pair]
    lib = pk.Chess(pk.Config(2 * H, H, B, 1, 4, 4))
    mid = slice(margin, margin + n_pages)
    x = [r[B:B + n] for r in rows.cuda()]
    lib.quant_store(*x, ints(entries), ints([0, len(entries), 0, 0]), k[mid], v[mid], scales[mid])
    torch.cuda.synchronize()
    host = [r[B:B + n].double().numpy() for r in rows]
    ref.store(cache.k[mid], cache.v[mid], cache.scales[mid], *host, inside)
    assert np.array_equal(scales.cpu().double().numpy(), cache.scales)
    assert ref.same_bytes(k.cpu().numpy(), cache.k) and ref.same_bytes(v.cpu().numpy(), cache.v)


def test_the_call_without_bounds_stores_the_same():
    """The entry point that takes no bounds, on entries that need none; and the bounded one's refusals."""
    rng = np.random.default_rng(1)
    cache = Cache(rng, 5, H, 16)
    k, v, scales = cache.cuda()
    rows = bf16(rng.normal(0, 1, (2, 30, H, D)))
    entries = [[4, 0, 0, 16], [1, 16, 2, 14], [0, 0, 15, 1]]
    lib = pk.Chess(pk.Config(2 * H, H, 16, 1, 4, 4))
    x, writes, counts = rows.cuda(), ints(entries), ints([30, 3, 0, 0])
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert lib.lib.chess_quant_store(lib._h, x[0].data_ptr(), H * D, x[1].data_ptr(), H * D, writes.data_ptr(), counts.data_ptr(), 3, k.data_ptr(),
                                     v.data_ptr(), scales.data_ptr(), stream) == 0
    torch.cuda.synchronize()
    ref.store(cache.k, cache.v, cache.scales, rows[0].double().numpy(), rows[1].double().numpy(), entries)
    assert ref.same_bytes(k.cpu().numpy(), cache.k) and ref.same_bytes(v.cpu().numpy(), cache.v)
    for n_rows, n_pages in ((0, 5), (30, 0), (-1, 5)):
        assert lib.lib.chess_quant_store_bounded(lib._h, x[0].data_ptr(), H * D, x[1].data_ptr(), H * D, n_rows, writes.data_ptr(), counts.data_ptr(), 3,
                                                 k.data_ptr(), v.data_ptr(), scales.data_ptr(), n_pages, stream) == -1


@pytest.mark.parametrize("B", [16, 32])
def test_one_token_of_heads_laid_out_first(B):
    """Keys [H, 1, 128] transposed: the token's stride is smaller than its row, and leads nowhere."""
    rng = np.random.default_rng(B)
    cache = Cache(rng, 2, H, B)
    k, v, scales = cache.cuda()
    rows = bf16(rng.normal(0, 1, (2, H, 1, D)))
    x = [r.transpose(0, 1) for r in rows.cuda()]
    assert x[0].stride(0) == D
    pk.Chess(pk.Config(2 * H, H, B, 1, 4, 4)).quant_store(*x, ints([[1, 0, 5, 1]]), ints([1, 1, 0, 0]), k, v, scales)
    torch.cuda.synchronize()
    ref.store(cache.k, cache.v, cache.scales, *[r.transpose(0, 1).double().numpy() for r in rows], [[1, 0, 5, 1]])
    assert np.array_equal(scales.cpu().double().numpy(), cache.scales)
    assert ref.same_bytes(k.cpu().numpy(), cache.k) and ref.same_bytes(v.cpu().numpy(), cache.v)


def test_more_entries_than_a_launch_has_threads_for():
    """128 threads an entry and KV head, fewer than 2^32: the largest list is launched (and has no entry here), one more is refused."""
    lib = pk.Chess(pk.Config(2, 2, 16, 1, 4, 4))
    x, pool, scales, counts = bf16(np.zeros((1, 2, D))).cuda(), torch.zeros((1, 2, 16, D), dtype=torch.uint8, device="cuda"), torch.ones((1, 2, 2), device="cuda"), ints([0] * 4)
    most = 2 ** 24 - 1
    writes = torch.zeros((most + 1, 4), dtype=torch.int32, device="cuda")
    call = lambda n: lib.lib.chess_quant_store_bounded(lib._h, x.data_ptr(), 2 * D, x.data_ptr(), 2 * D, 1, writes.data_ptr(), counts.data_ptr(), n,  # noqa: E731
                                                       pool.data_ptr(), pool.data_ptr(), scales.data_ptr(), 1, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert call(most) == 0
    assert call(most + 1) == call(2 ** 27) == call(2 ** 31 - 1) == -2                # CHESS_ENOTSUP
    torch.cuda.synchronize()
    assert not pool.any()
