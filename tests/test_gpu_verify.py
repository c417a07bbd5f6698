"""Drafted tokens verified, and the pages of refused ones taken back, against plain 64-bit forms."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
import step_reference as ref

pytestmark = pytest.mark.gpu
SUMMARY_DTYPE_SWEEP = False


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def distributions(rng, n, V, spread=3.0):
    z = rng.normal(0, spread, (n, V))
    p = np.exp(z - z.max(1, keepdims=True))
    return (p / p.sum(1, keepdims=True)).astype(np.float32)


class Case:
    def __init__(self, seed, new, V, given=True, most=None):
        rng = np.random.default_rng(seed)
        self.rng, self.new, self.V = rng, new, V
        rows, batch = sum(new), len(new)
        self.most = max(max(new) - 1, 0) if most is None else most
        self.starts = np.concatenate([[0], np.cumsum(new)])
        self.target = distributions(rng, max(rows, 1), V)
        self.tokens = rng.integers(0, V, max(rows, 1))
        self.draft = np.zeros((batch, max(self.most, 1), V), np.float32) if given else None
        for b, n in enumerate(new):
            for j in range(min(n - 1, self.most)):
                row = self.starts[b] + j
                q = self.target[row].astype(np.float64) * np.exp(rng.normal(0, 0.5, V))
                q /= q.sum()
                if given:
                    self.draft[b, j] = q
                self.tokens[row + 1] = rng.choice(V, p=q) if given or rng.random() < 0.5 else self.target[row].argmax()
        self.uniforms = rng.random((batch, self.most + 1), dtype=np.float32)
        self.lens = rng.integers(max(new), 300, batch)

    def run(self, lib, ws, target=None, draft=None):
        batch = len(self.new)
        out = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((batch,), (batch, self.most + 1), (batch,))]
        target = torch.from_numpy(self.target).cuda() if target is None else target
        if draft is None and self.draft is not None:
            draft = torch.from_numpy(self.draft).cuda()
        lib.verify(target, draft, ints(self.tokens), ints(self.starts), torch.from_numpy(self.uniforms).cuda(), ints(self.lens), *out, ws)
        torch.cuda.synchronize()
        return [x.cpu().numpy() for x in out]

    def want(self):
        f = lambda x: None if x is None else x.astype(np.float64)  # noqa: E731
        return ref.verify(f(self.target), f(self.draft), self.tokens, self.starts, f(self.uniforms), self.lens)

    def check(self, lib, ws, **kw):
        for got, want in zip(self.run(lib, ws, **kw), self.want()):
            assert np.array_equal(got, want), (got, want)


def library(batch=64):
    lib = pk.Chess(pk.Config(4, 2, 16, batch, 32, 32))
    return lib, lib.new_workspace()


@pytest.mark.parametrize("given", [True, False], ids=["probabilities", "certain"])
@pytest.mark.parametrize("V", [1, 2, 5, 1023, 1024, 1025, 4099, 50257])
@pytest.mark.parametrize("new", [[1], [5], [1, 2, 3, 4], [0, 3, 0, 7], [9] * 20], ids=str)
def test_verify(new, V, given):
    lib, ws = library()
    for seed in range(3):
        Case(seed * 1000 + V, new, V, given).check(lib, ws)


def test_many_drafts_and_a_large_vocabulary():
    lib, ws = library()
    Case(1, [200, 70, 1], 301).check(lib, ws)
    Case(2, [3, 2], 300007).check(lib, ws)                       # beyond 256 pieces of 1024 words


def test_more_drafts_than_are_looked_at():
    lib, ws = library()
    c = Case(5, [9, 2, 5], 64, most=3)
    c.uniforms[:, :3] = 0
    c.check(lib, ws)
    n_accepted, out, lens = c.run(lib, ws)
    assert n_accepted[0] == 3 and lens[0] == c.lens[0] - 5


def test_rows_of_wider_tensors():
    lib, ws = library()
    c = Case(7, [4, 1, 3], 1001)
    wide = torch.full((8, 1009), float("nan"), device="cuda")
    wide[:, 3:1004] = torch.from_numpy(c.target).cuda()
    d = torch.full((3, 5, 1010), float("nan"), device="cuda")
    d[:, 1:4, 4:1005] = torch.from_numpy(c.draft).cuda()
    c.check(lib, ws, target=wide[:, 3:1004], draft=d[:, 1:4, 4:1005])
    # drafts step by step: [step, batch, vocab]
    c.check(lib, ws, draft=torch.from_numpy(c.draft).cuda().transpose(0, 1).contiguous().transpose(0, 1))


def test_borders():
    """u q = p does not stand; u = 0; tokens that are no words; weights that are none."""
    lib, ws = library()
    c = Case(11, [3, 3, 3, 3, 3], 8)
    c.target[:] = 0.125
    c.draft[:] = 0.25
    c.tokens[:] = 3
    c.uniforms[:] = [[0.5, 0.5, 0.0], [np.float32(0.5) - np.float32(2) ** -25, 0.6, 0.99999994], [0.0, 0.0, 0.5], [0.1, 0.9, 0.3], [0.1, 0.1, 0.7]]
    c.target[c.starts[3] + 1] = [0, 0.5, np.nan, -1, 0.25, 0.25, 0, 0]
    c.draft[3, 1] = [0.1, 0.5, 0.1, 0.1, 0.05, 0.25, 0, 0]
    c.tokens[c.starts[4] + 1] = -1
    c.check(lib, ws)
    n_accepted, out, _ = c.run(lib, ws)
    assert list(n_accepted) == [0, 1, 2, 1, 0]
    assert out[0, 0] == 0 and out[3, 1] == 4                      # nothing left over: the target's own; one word left over
    c.tokens[c.starts[4] + 1] = 8
    c.check(lib, ws)


@pytest.mark.parametrize("bad", [0.0, np.inf, np.nan])
def test_rows_without_a_sum(bad):
    lib, ws = library()
    c = Case(12, [1, 2], 2000)
    c.target[0] = bad
    c.target[1:] = 0
    c.check(lib, ws)
    assert c.run(lib, ws)[1][0, 0] == -1


def test_starts_that_name_rows_that_are_not_there():
    lib, ws = library()
    c = Case(13, [2, 3, 4], 100)
    for starts in ([0, 2, 5, 10], [-1, 2, 5, 9], [5, 2, 2 ** 31 - 1, 9], [0, 2 ** 31 - 1, -2 ** 31, 3]):
        c.starts = np.array(starts)
        c.check(lib, ws)


def test_the_same_row_in_any_batch():
    """Cut into few or many workgroups, a row gives the same token."""
    lib, ws = library(300)
    one = Case(21, [3], 70001)
    alone = one.run(lib, ws)
    many = Case(22, [3] * 300, 70001, given=False)
    target = torch.from_numpy(one.target).cuda().repeat(300, 1)
    draft = torch.from_numpy(one.draft).cuda().expand(300, -1, -1).contiguous()
    many.tokens, many.uniforms, many.lens = np.tile(one.tokens, 300), np.tile(one.uniforms, (300, 1)), np.tile(one.lens, 300)
    got = many.run(lib, ws, target=target, draft=draft)
    for a, b in zip(alone, got):
        assert (b == a).all()


def test_lengths_in_place_on_a_stream_replayed():
    lib, ws = library()
    c = Case(31, [4, 6, 1, 2], 5000)
    want = c.want()
    dev = [torch.from_numpy(c.target).cuda(), torch.from_numpy(c.draft).cuda(), ints(c.tokens), ints(c.starts), torch.from_numpy(c.uniforms).cuda()]
    lens, n, out = ints(c.lens), ints([0] * 4), torch.zeros((4, c.most + 1), dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        lib.verify(*dev, lens, n, out, lens, ws)
    for _ in range(3):
        lens.copy_(ints(c.lens))
        g.replay()
        torch.cuda.synchronize()
        for got, x in zip((n, out, lens), want):
            assert np.array_equal(got.cpu().numpy(), x)


def test_verify_refusals():
    lib, ws = library(4)
    c = Case(1, [2, 2], 64)
    out = [ints([0, 0]), torch.zeros((2, 2), dtype=torch.int32, device="cuda"), ints([0, 0])]
    good = dict(target=torch.from_numpy(c.target).cuda(), draft=torch.from_numpy(c.draft).cuda(), tokens=ints(c.tokens), token_start=ints(c.starts),
                uniforms=torch.from_numpy(c.uniforms).cuda(), seq_lens=ints(c.lens), n_accepted=out[0], out_tokens=out[1], lens_after=out[2], workspace=ws)
    lib.verify(**good)
    for name, bad in (("target", good["target"].double()), ("target", good["target"].t()), ("draft", good["draft"][:, :, :60]), ("draft", good["draft"][:1]),
                      ("tokens", good["tokens"].long()), ("token_start", good["token_start"][:2]), ("uniforms", good["uniforms"][:1]), ("uniforms", good["uniforms"][:, :0]),
                      ("out_tokens", out[1][:1]), ("seq_lens", ints([1] * 5)), ("workspace", ws[:100])):
        with pytest.raises(pk.ChessError):
            lib.verify(**{**good, name: bad})
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    raw = lambda vocab, stride, most, batch: lib.lib.chess_verify(  # noqa: E731
        lib._h, good["target"].data_ptr(), stride, None, 0, 0, vocab, good["tokens"].data_ptr(), 4, good["token_start"].data_ptr(), good["uniforms"].data_ptr(), most,
        good["seq_lens"].data_ptr(), batch, out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), ws.data_ptr(), stream)
    assert raw(64, 64, 1, 2) == 0
    assert raw(64, 63, 1, 2) == raw(0, 64, 1, 2) == raw(64, 64, -1, 2) == raw(64, 64, 1, 0) == raw(64, 64, 1, 5) == -1
    torch.cuda.synchronize()


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("batch", [1, 5, 300, 1000])
def test_trim(batch, B):
    rng = np.random.default_rng(batch + B)
    width = 40
    lens = rng.integers(-1, width * B + 1, batch)
    keep = np.where(rng.random(batch) < 0.3, lens + rng.integers(-3, 50, batch), np.maximum(lens - rng.integers(0, 3 * B, batch), -2))
    table = rng.permutation(batch * width).reshape(batch, width)
    lib = pk.Chess(pk.Config(4, 2, B, batch, width, width))
    ws = lib.new_workspace()
    for capacity, n_free in ((batch * width + 9, 4), (batch + 4, 4), (4, 4), (3, 9)):
        free = rng.integers(0, 10 ** 6, capacity + 3)
        dev, count, left = ints(free), ints([n_free]), ints([-5])
        lib.trim_pages(ints(lens), ints(keep), ints(table), dev[:capacity], count, left, ws)
        torch.cuda.synchronize()
        want, n = ref.trim(lens, keep, table, free, n_free, capacity, B)
        assert np.array_equal(dev.cpu().numpy(), want) and left.item() == n and count.item() == n_free
        dev = ints(free)
        lib.trim_pages(ints(lens), ints(keep), ints(table), dev[:capacity], count, count, ws)     # in place
        torch.cuda.synchronize()
        assert np.array_equal(dev.cpu().numpy(), want) and count.item() == n


def test_trim_refusals():
    lib, ws = library(4)
    good = dict(seq_lens=ints([1, 2]), keep_lens=ints([1, 1]), block_table=torch.zeros((2, 32), dtype=torch.int32, device="cuda"), free_pages=ints([0] * 9), n_free=ints([0]),
                n_left=ints([0]), workspace=ws)
    lib.trim_pages(**good)
    for name, bad in (("seq_lens", ints([1] * 5)), ("keep_lens", ints([1])), ("block_table", good["block_table"][:1]), ("n_left", torch.zeros(1, device="cuda")),
                      ("workspace", ws[:16])):
        with pytest.raises(pk.ChessError):
            lib.trim_pages(**{**good, name: bad})
    torch.cuda.synchronize()
