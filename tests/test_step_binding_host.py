"""What the binding passes to the calls for several tokens of a sequence, and what it refuses, without a GPU: the library is a stand-in that keeps the
arguments."""
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
    c.cfg, c.lib, c._h, c.device, c.workspace_bytes = pk.Config(8, 2, 16, 2, 4, 4), Kept(), None, -1, 64      # (-1: where CPU tensors say they are)
    monkeypatch.setattr(pk.Chess, "__del__", lambda self: None, raising=False)
    return c


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def rotate_args(n=5):
    wide = bf16(n, 12, 128)
    return dict(rotary=pk.Rotary(torch.ones(64)), q=wide[:, :8], k_new=wide[:, 8:10], v_new=wide[:, 10:], positions=i32(1, n), writes=i32(3, 4), counts=i32(4), q_out=bf16(n, 8, 128),
                k_pool=bf16(7, 2, 16, 128), v_pool=bf16(7, 2, 128, 16))


def test_the_rotation_is_told_strides_rows_entries_and_pages(chess):
    chess.rotate_store(**rotate_args())
    (name, a), = chess.lib.calls
    assert name == "chess_rotate_store"
    assert (a[3], a[5], a[7], a[9], a[12], a[16]) == (12 * 128, 12 * 128, 12 * 128, 5, 3, 7)


def test_one_token_may_have_any_stride(chess):
    args = rotate_args(1)
    args["k_new"] = bf16(2, 1, 128).transpose(0, 1)
    chess.rotate_store(**args)
    a = chess.lib.calls[0][1]
    assert (a[3], a[5], a[7]) == (8 * 128, 2 * 128, 2 * 128)


def test_without_queries_and_without_rows(chess):
    args = rotate_args()
    args.update(q=None, q_out=None)
    chess.rotate_store(**args)
    assert chess.lib.calls[0][1][2] is None and chess.lib.calls[0][1][13] is None
    chess.rotate_store(**rotate_args(0))
    chess.rotate(pk.Rotary(torch.ones(64)), bf16(0, 8, 128), None, i32(1, 0), bf16(0, 8, 128))
    assert len(chess.lib.calls) == 1


@pytest.mark.parametrize("name,bad", [
    ("q", bf16(4, 8, 128)), ("q", bf16(5, 7, 128)), ("q", torch.zeros(5, 8, 128)), ("q", bf16(5, 8, 256)[:, :, ::2]), ("q_out", bf16(5, 8, 127)),
    ("k_new", bf16(2, 5, 128).transpose(0, 1)), ("positions", i32(4)), ("positions", i32(2, 5)), ("positions", i32(1, 5).long()), ("writes", i32(3)),
    ("counts", i32(1)), ("k_pool", bf16(6, 2, 16, 128)), ("v_pool", torch.zeros((7, 2, 128, 16)))])
def test_the_rotation_refuses(chess, name, bad):
    with pytest.raises(pk.ChessError):
        chess.rotate_store(**{**rotate_args(), name: bad})
    assert not chess.lib.calls


def test_how_to_rotate_is_checked():
    ones = torch.ones(64)
    for bad in (dict(inv_freq=ones.double()), dict(inv_freq=torch.ones(128)[::2]), dict(inv_freq=torch.ones(65)), dict(axis=[0]), dict(axis=[4] * 64), dict(axis=[-1] * 64),
                dict(q_norm=torch.ones(64)), dict(q_norm=torch.ones(128).half()), dict(q_norm=torch.ones(128), k_norm=torch.ones(2, 128)), dict(scale=0)):
        with pytest.raises(pk.ChessError):
            pk.Rotary(**{"inv_freq": ones, **bad})
    r = pk.Rotary(torch.ones(24), axis=[0, 2] * 12, q_norm=torch.ones(8, 128))
    assert (r.n_axes, r._c.rotary_dim, r._c.norm_per_head, r._c.n_axes, r._c.axis[1], r._c.k_norm) == (3, 48, 1, 3, 2, None)


def test_weights_of_other_heads_are_refused(chess):
    args = rotate_args()
    for bad in (dict(q_norm=torch.ones(7, 128)), dict(k_norm=torch.ones(8, 128))):
        with pytest.raises(pk.ChessError):
            chess.rotate_store(**{**args, "rotary": pk.Rotary(torch.ones(64), **bad)})
    chess.rotate_store(**{**args, "rotary": pk.Rotary(torch.ones(64), q_norm=torch.ones(8, 128), k_norm=torch.ones(2, 128))})


def attend_args(n=5):
    return dict(q=bf16(n, 8, 128), token_start=i32(3), max_new=3, k_pool=bf16(7, 2, 16, 128), v_pool=bf16(7, 2, 128, 16), block_table=i32(2, 4), seq_lens=i32(2), out=bf16(n, 8, 128),
                workspace=torch.zeros(64, dtype=torch.uint8), scratch=torch.zeros(128, dtype=torch.uint8), scores=pk.Scores(slopes=torch.ones(8), first_keys=i32(n)))


def test_attention_is_told_rows_and_scratch(chess):
    chess.dense_attend(**attend_args())
    chess.sparse_attend(**attend_args(), page_ids=i32(2, 2, 4), n_selected=i32(2, 2))
    chess.dense_attend(**attend_args(0))
    (dense, a), (sparse, b) = chess.lib.calls
    assert (dense, sparse) == ("chess_dense_attend", "chess_sparse_attend")
    assert (a[3], a[5], a[10], a[14]) == (5, 3, 2, 128) and (b[3], b[5], b[12], b[16]) == (5, 3, 2, 128)


@pytest.mark.parametrize("name,bad", [
    ("q", bf16(5, 7, 128)), ("q", bf16(5, 1024)), ("q", bf16(5, 16, 128)[:, ::2]), ("out", bf16(4, 8, 128)), ("out", torch.zeros(5, 8, 128)), ("token_start", i32(2)),
    ("block_table", i32(2, 3)), ("workspace", torch.zeros(63, dtype=torch.uint8)), ("scratch", torch.zeros(128)), ("scores", pk.Scores(slopes=torch.ones(7))),
    ("scores", pk.Scores(prefix_lens=i32(1))), ("scores", pk.Scores(first_keys=i32(4)))])
def test_attention_refuses(chess, name, bad):
    with pytest.raises(pk.ChessError):
        chess.dense_attend(**{**attend_args(), name: bad})
    assert not chess.lib.calls


def test_scores_are_checked():
    for bad in (dict(slopes=torch.ones(8).double()), dict(prefix_lens=torch.ones(2)), dict(first_keys=i32(10)[::2])):
        with pytest.raises(pk.ChessError):
            pk.Scores(**bad)


def verify_args():
    return dict(target=torch.zeros(5, 64), draft=torch.zeros(2, 3, 64), tokens=i32(5), token_start=i32(3), uniforms=torch.zeros(2, 3), seq_lens=i32(2), n_accepted=i32(2),
                out_tokens=i32(2, 3), lens_after=i32(2), workspace=torch.zeros(64, dtype=torch.uint8))


def test_verification_is_told_strides(chess):
    chess.verify(**{**verify_args(), "target": torch.zeros(5, 70)[:, 3:67], "draft": torch.zeros(3, 2, 64).transpose(0, 1)})
    chess.verify(**{**verify_args(), "draft": None})
    (name, a), (_, b) = chess.lib.calls
    assert name == "chess_verify"
    assert (a[2], a[4], a[5], a[6], a[8], a[11], a[13]) == (70, 64, 128, 64, 5, 2, 2)
    assert b[3] is None


@pytest.mark.parametrize("name,bad", [
    ("target", torch.zeros(5, 64).double()), ("target", torch.zeros(64, 5).t()), ("target", torch.zeros(5)), ("target", torch.zeros(0, 64)), ("draft", torch.zeros(2, 1, 64)),
    ("draft", torch.zeros(2, 3, 63)), ("draft", torch.zeros(1, 3, 64)), ("draft", torch.zeros(2, 64, 3).transpose(1, 2)), ("tokens", i32(4)), ("token_start", i32(2)),
    ("uniforms", torch.zeros(3)), ("uniforms", torch.zeros(2, 0)), ("uniforms", torch.zeros(1, 3)), ("n_accepted", i32(1)), ("out_tokens", i32(2, 2)),
    ("workspace", torch.zeros(60, dtype=torch.uint8))])
def test_verification_refuses(chess, name, bad):
    with pytest.raises(pk.ChessError):
        chess.verify(**{**verify_args(), name: bad})
    assert not chess.lib.calls


def test_positions_by_rows_are_refused(chess):
    """[rows, axes] has as many numbers as [axes, rows], in another order."""
    args = {**rotate_args(), "rotary": pk.Rotary(torch.ones(64), axis=[0, 1, 2, 1] * 16)}
    for bad in (i32(5, 3), i32(1, 5, 3), i32(15, 1)):
        with pytest.raises(pk.ChessError):
            chess.rotate_store(**{**args, "positions": bad})
        with pytest.raises(pk.ChessError):
            chess.rotate(args["rotary"], args["q"], None, bad, args["q_out"])
    assert not chess.lib.calls
    for good in (i32(3, 5), i32(15)):
        chess.rotate_store(**{**args, "positions": good})
    for one in (i32(5), i32(1, 5), i32(5, 1)):
        chess.rotate_store(**{**rotate_args(), "positions": one})
    assert len(chess.lib.calls) == 5
