"""Several tokens of a sequence in a step, without a GPU: the reference that the kernels' tests compare with is pinned against torch and worked examples, and
the entry points refuse calls without a context."""
from __future__ import annotations

import ctypes
import os

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
import step_reference as ref


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pk.library_path()):
        from paper_2602_20732_amd.build import build
        build()
    return pk.load_library()


def test_without_a_context(lib):
    n = ctypes.c_size_t()
    assert lib.chess_rotate(None, None, None, 0, None, 0, None, 1, None, None, None, None) == -1
    assert lib.chess_rotate_store(None, None, None, 0, None, 0, None, 0, None, 1, None, None, 1, None, None, None, 1, None) == -1
    assert lib.chess_attend_scratch_bytes(None, 1, 1, 1, ctypes.byref(n)) == -1
    assert lib.chess_dense_attend(None, None, None, 1, None, 1, None, None, None, None, 1, None, None, None, 0, None) == -1
    assert lib.chess_sparse_attend(None, None, None, 1, None, 1, None, None, None, None, None, None, 1, None, None, None, 0, None) == -1
    assert lib.chess_verify(None, None, 1, None, 0, 0, 1, None, 1, None, None, 0, None, 1, None, None, None, None, None) == -1
    assert lib.chess_trim_pages(None, None, None, 1, None, None, 1, None, None, None, None) == -1


def test_rotation_of_the_reference():
    """A quarter of a turn, by hand; norms against torch; a rotation keeps lengths."""
    x = np.zeros((1, 1, 128))
    x[0, 0, 0], x[0, 0, 64] = 3, 4
    y, _ = ref.rotated(x, np.array([[1]]), np.array([np.pi / 2] + [0.0] * 63), [0] * 64)
    assert np.allclose(y[0, 0, [0, 64]], [-4, 3])
    y, _ = ref.rotated(x, np.array([[1]]), np.array([np.pi / 2] + [0.0] * 63), [0] * 64, interleaved=True)
    assert np.allclose(y[0, 0, [0, 1, 64]], [0, 3, 4])
    rng = np.random.default_rng(0)
    x, w = rng.normal(0, 2, (5, 3, 128)), rng.normal(1, 0.1, 128)
    y, normed = ref.rotated(x, rng.integers(0, 9999, (2, 5)), rng.random(32), [0, 1] * 16, norm=w, eps=0.1)
    assert np.allclose(normed, torch.nn.functional.rms_norm(torch.from_numpy(x), (128,), torch.from_numpy(w), 0.1).numpy())
    assert np.allclose((y ** 2).sum(-1), (normed ** 2).sum(-1)) and np.allclose(y[..., 64:], normed[..., 64:])


def test_attention_of_the_reference():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(0, 1, (4, 2, 128)), rng.normal(0, 1, (9, 128)), rng.normal(0, 1, (9, 128))
    see = [ref.interval(p, 9) for p in range(5, 9)]
    assert see == [(0, 5), (0, 6), (0, 7), (0, 8)]
    out, size, off = ref.attend(q, k, v, np.arange(5, 9), see, 0.1)
    t = lambda x: torch.from_numpy(x)  # noqa: E731
    mask = torch.arange(9)[None] <= torch.arange(5, 9)[:, None]
    want = torch.nn.functional.scaled_dot_product_attention(t(q).transpose(0, 1), t(k)[None], t(v)[None], attn_mask=mask, scale=0.1).transpose(0, 1)
    assert np.allclose(out, want.numpy()) and (off > 0).all() and (size >= np.abs(out)).all()
    # windows, prefixes, documents
    assert ref.interval(5, 9, window=2) == (4, 5) and ref.interval(5, 9, prefix=20) == (0, 8) and ref.interval(5, 9, first=6) == (6, 5) and ref.interval(1, 9, window=7) == (0, 1)
    assert (ref.attend(q[:1], k, v, [5], [(6, 5)], 0.1)[0] == 0).all()
    # a steep slope leaves the key at the token itself, a small cap makes all keys alike
    out = ref.attend(q[:1], k, v, [5], [(0, 5)], 0.1, slopes=[1e4, 1e4])[0]
    assert np.allclose(out[0, 0], v[5])
    out = ref.attend(q[:1], k, v, [5], [(0, 5)], 0.1, cap=1e-9)[0]
    assert np.allclose(out[0, 1], v[:6].mean(0))


def test_verification_of_the_reference():
    """Worked example, and that the tokens it gives are the target's, whatever the draft's distribution is."""
    target = np.array([[0.5, 0.5, 0.0], [0.1, 0.2, 0.7]])
    draft = np.array([[[0.25, 0.25, 0.5]]])
    args = dict(target=target, draft=draft, starts=[0, 2], lens=[7])
    got = ref.verify(tokens=[9, 1], uniforms=np.array([[0.99, 0.25]]), **args)
    assert [x.tolist() for x in got] == [[1], [[1, 1]], [7]]                             # 0.99 x 0.25 < 0.5; then 0.1 <= 0.25 < 0.3
    got = ref.verify(tokens=[9, 2], uniforms=np.array([[0.0, 0.6]]), **args)
    assert [x.tolist() for x in got] == [[0], [[1, -1]], [6]]                            # 0 < 0 does not hold; left over: 0.25, 0.25, 0
    rng = np.random.default_rng(2)
    p, q, counts = np.array([0.5, 0.3, 0.15, 0.05]), np.array([0.1, 0.2, 0.3, 0.4]), np.zeros(4)
    n = 4000
    for _ in range(n):
        x = rng.choice(4, p=q)
        counts[ref.verify(np.array([p, p]), q[None, None], [0, x], [0, 2], rng.random((1, 2)), [5])[1][0, 0]] += 1
    assert (np.abs(counts / n - p) < 5 * np.sqrt(p * (1 - p) / n)).all()


def test_trimming_of_the_reference():
    assert ref.trim([33, 16, 40], [17, 16, 2], [[1, 2, 3], [4, 5, 6], [7, 8, 9]], [50, 0, 0, 0, 0], 1, 5, 16) == ([50, 3, 8, 9, 0], 4)
    assert ref.trim([33, 16, 40], [17, 16, 2], [[1, 2, 3], [4, 5, 6], [7, 8, 9]], [50, 0, 0], 1, 3, 16) == ([50, 3, 0], 2)
