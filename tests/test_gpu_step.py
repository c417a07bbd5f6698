"""The calls of a step of several tokens a sequence one after the other, as a decode loop makes them: chess_map_tokens, chess_rotate_store, chess_extend_window,
chess_sparse_attend or chess_dense_attend, chess_verify, chess_trim_pages.  Every result against its plain 64-bit form, eager and replayed."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
import step_reference as ref

pytestmark = pytest.mark.gpu
SUMMARY_DTYPE_SWEEP = False
D, V, Hq, H = 128, 71, 8, 2
G = Hq // H


def near(got, want, off):
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= off)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], off[bad][:5])


class Loop:
    """Sequences, their pages and everything that a step reads or writes, in tensors that stay where they are."""

    def __init__(self, B, batch, room, pages, width, drafts, shared=None, **rule):
        zeros = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
        self.B, self.batch, self.room, self.pages, self.drafts, self.rule = B, batch, room, pages, drafts, rule
        self.lib = shared.lib if shared else pk.Chess(pk.Config(Hq, H, B, batch, width, width))
        self.ws = shared.ws if shared else self.lib.new_workspace()
        self.scratch = shared.scratch if shared else self.lib.new_attend_scratch(room, room, batch)
        self.k, self.v = zeros(pages, H, B, D, t=torch.bfloat16), zeros(pages, H, D, B, t=torch.bfloat16)
        self.table, self.free, self.n_free = zeros(batch, width) - 1, torch.arange(pages, dtype=torch.int32, device="cuda").flip(0).contiguous(), zeros(1) + pages
        self.lens, self.kept, self.new = zeros(batch), zeros(batch), zeros(batch)
        self.starts, self.counts, self.writes = zeros(batch + 1), zeros(4), zeros(min(room, room // B + 2 * batch), 4)
        self.wide, self.positions = zeros(room, Hq + 2 * H, D, t=torch.bfloat16), zeros(1, room)
        self.q, self.out = zeros(room, Hq, D, t=torch.bfloat16), zeros(room, Hq, D, t=torch.bfloat16)
        self.ids, self.n = zeros(batch, H, width) - 1, zeros(batch, H)
        self.target, self.tokens, self.uniforms = zeros(room, V, t=torch.float32), zeros(room), zeros(batch, drafts + 1, t=torch.float32)
        self.accepted, self.out_tokens = zeros(batch), zeros(batch, drafts + 1)
        self.inv_freq = (1e4 ** (-np.arange(D // 2) / (D // 2))).astype(np.float32)
        self.norm = (1 + 0.1 * np.random.default_rng(0).normal(0, 1, D)).astype(np.float32)
        self.rotary = pk.Rotary(torch.from_numpy(self.inv_freq).cuda(), None, False, torch.from_numpy(self.norm).cuda(), torch.from_numpy(self.norm).cuda(), 1e-6)
        self.scores = pk.Scores(rule.get("cap", 0.0), None, rule.get("window", 0))

    def feed(self, rng, new):
        """A step's inputs, for `new` tokens of each sequence."""
        kept = self.kept.cpu().numpy()
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        self.wide.copy_(torch.from_numpy(rng.normal(0, 1, self.wide.shape).astype(np.float32)))
        at = np.zeros(self.room, np.int32)
        at[: sum(new)] = np.concatenate([np.arange(k, k + n) for k, n in zip(kept, new)])
        self.positions.copy_(torch.from_numpy(at[None]))
        z = rng.normal(0, 3, (self.room, V))
        p = np.exp(z - z.max(1, keepdims=True))
        p = (p / p.sum(1, keepdims=True)).astype(np.float32)
        tokens = np.where(rng.random(self.room) < 0.8, np.roll(p.argmax(1), 1), rng.integers(0, V, self.room))
        self.target.copy_(torch.from_numpy(p))
        self.tokens.copy_(torch.from_numpy(tokens.astype(np.int32)))
        self.uniforms.copy_(torch.from_numpy(rng.random(self.uniforms.shape, dtype=np.float32)))

    def step(self, most, listed, drafts=True):
        """drafts: the new tokens but the first are; else they are there to stay."""
        lib = self.lib
        lib.map_tokens(self.kept, self.new, self.table, self.free, self.n_free, self.lens, self.n_free, self.starts, None, self.writes, self.counts, self.ws,
                       max_tokens=self.room)
        lib.rotate_store(self.rotary, self.wide[:, :Hq], self.wide[:, Hq:Hq + H], self.wide[:, Hq + H:], self.positions, self.writes, self.counts, self.q,
                         self.k, self.v)
        attend = (self.q, self.starts, most, self.k, self.v, self.table, self.lens)
        if listed:
            lib.extend_window(self.lens, self.ids, self.n)
            lib.sparse_attend(*attend, self.ids, self.n, self.out, self.ws, self.scratch, self.scores)
        else:
            lib.dense_attend(*attend, self.out, self.ws, self.scratch, self.scores)
        if not drafts:
            self.kept.copy_(self.lens)
            return
        lib.verify(self.target, None, self.tokens, self.starts, self.uniforms, self.lens, self.accepted, self.out_tokens, self.kept, self.ws)
        lib.trim_pages(self.lens, self.kept, self.table, self.free, self.n_free, self.n_free, self.ws)

    STATE = ("k", "v", "table", "free", "n_free", "lens", "kept", "starts", "counts", "q", "out", "ids", "n", "accepted", "out_tokens")

    def state(self):
        torch.cuda.synchronize()
        return {x: getattr(self, x).clone() for x in self.STATE}

    def check(self, before, new, most, listed, drafts=True):
        """The step's results, from the state before it."""
        s, B = {x: y.cpu() for x, y in self.state().items()}, self.B
        kept0, lens = before["kept"].cpu().numpy(), s["lens"].numpy()
        assert (lens == kept0 + new).all() and s["starts"].tolist() == [0, *np.cumsum(new)] and s["counts"][0] == sum(new) and s["counts"][3] == 0
        rows, starts = sum(new), s["starts"].numpy()
        # pages: a sequence's are nobody else's, and none is lost
        table, kept, n_free = s["table"].numpy(), s["kept"].numpy(), int(s["n_free"])
        of_seqs = [p for b in range(self.batch) for p in table[b, : -(-kept[b] // B)]]
        assert sorted([*of_seqs, *s["free"][:n_free].tolist()]) == list(range(self.pages))
        # queries and the cache
        wide, at = self.wide[:rows].double().cpu().numpy(), self.positions[:, :rows].cpu().numpy()
        y, x = ref.rotated(wide[:, : Hq + H], at, self.inv_freq, [0] * (D // 2), False, self.norm, 1e-6)
        off = ref.rotation_error(y, x, self.inv_freq, False)
        near(s["q"][:rows], y[:, :Hq], off[:, :Hq])
        assert torch.equal(s["q"][rows:], before["q"][rows:].cpu())
        k_of = lambda page, slot: s["k"][torch.as_tensor(page).long(), :, torch.as_tensor(slot).long()]  # noqa: E731
        v_of = lambda page, slot: s["v"][torch.as_tensor(page).long(), :, :, torch.as_tensor(slot).long()]  # noqa: E731
        page = table[np.repeat(np.arange(self.batch), new), at[0] // B]
        near(k_of(page, at[0] % B), y[:, Hq:], off[:, Hq:])
        assert torch.equal(v_of(page, at[0] % B), self.wide[:rows, Hq + H:].cpu())
        # attention over what the pages hold
        q, want, off = s["q"].double().numpy(), np.zeros((rows, Hq, D)), np.zeros((rows, Hq, D))
        step = ref.HALF_STEP if most * G > 64 else ref.HALF_STEP ** 2
        for b in range(self.batch):
            logical = np.arange(lens[b])
            k, v = (of(table[b, logical // B], logical % B).double().numpy() for of in (k_of, v_of))
            see = [ref.interval(p, lens[b], self.rule.get("window", 0)) for p in range(kept0[b], lens[b])]
            some = slice(starts[b], starts[b + 1])
            for h in range(H):
                keys, heads = None, slice(h * G, h * G + G)
                if listed:
                    n = int(s["n"][b, h])
                    keys = (s["ids"][b, h, :n, None].numpy() * B + np.arange(B)).reshape(-1)
                    keys = keys[keys < lens[b]]
                    assert lens[b] == 0 or n > 0 and int(s["ids"][b, h, n - 1]) >= (lens[b] - 1) // B
                want[some, heads], size, e = ref.attend(q[some, heads], k[:, h], v[:, h], np.arange(kept0[b], lens[b]), see, 1 / math.sqrt(D), self.rule.get("cap", 0.0),
                                                        None, keys)
                off[some, heads] = ref.attention_error(want[some, heads], size, e, max(lens[b], 1), step)
        near(s["out"][:rows], want, off)
        assert torch.equal(s["out"][rows:], before["out"][rows:].cpu())
        if not drafts:
            assert (kept == lens).all()
            return
        f = lambda t: t.double().cpu().numpy()  # noqa: E731
        accepted, out_tokens, after = ref.verify(f(self.target), None, self.tokens.cpu().numpy(), starts, f(self.uniforms), lens)
        assert (s["accepted"].numpy() == accepted).all() and (s["out_tokens"].numpy() == out_tokens).all() and (kept == after).all()


def lists_of_prompts(loops):
    """Lists with a gap, for what the sequences hold so far: the first page and the last."""
    for x in loops:
        pages = -(-x.kept // x.B)
        x.ids[:, :, 0], x.ids[:, :, 1] = 0, (pages - 1).clamp(min=0)[:, None]
        x.n.copy_(pages.clamp(max=2)[:, None].expand(-1, H))


@pytest.mark.parametrize("rule", [dict(), dict(cap=15.0, window=40)], ids=["causal", "cap-window"])
@pytest.mark.parametrize("B", [16, 32])
def test_steps_of_a_loop(B, rule):
    rng = np.random.default_rng(B)
    loop = Loop(B, 4, 140, 40, 12, 5, **rule)
    steps = [([70, 3, 0, 45], False)] + [([int(n) for n in rng.integers(0, 7, 4)], i % 3 > 0) for i in range(6)] + [([1, 1, 1, 1], True), ([6, 0, 0, 1], False)]
    for i, (new, listed) in enumerate(steps):
        if i == 1:
            lists_of_prompts([loop])
        loop.feed(rng, new)
        before = loop.state()
        loop.step(max(new), listed, drafts=i > 0)
        loop.check(before, new, max(new), listed, drafts=i > 0)


def test_two_graphs_share_a_workspace_and_scratch():
    """Steps of two groups of sequences, captured and replayed in turn, beside eager steps of the same with a workspace of their own: the same bits."""
    B, seeds = 16, (1, 2)
    eager = [Loop(B, 3, 60, 30, 8, 4) for _ in seeds]
    first = Loop(B, 3, 60, 30, 8, 4)
    captured = [first, Loop(B, 3, 60, 30, 8, 4, shared=first)]
    rngs = [[np.random.default_rng(s) for s in seeds] for _ in range(2)]
    for pair, r in zip((eager, captured), rngs):
        for loop, rng in zip(pair, r):
            loop.feed(rng, [20, 9, 31])
            before = loop.state()
            loop.step(31, False, drafts=False)
            loop.check(before, [20, 9, 31], 31, False, drafts=False)
        lists_of_prompts(pair)
    graphs = []
    for loop in captured:
        saved = loop.state()
        side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            loop.step(5, True)
        graphs.append(g)
        assert all(torch.equal(x, saved[name]) for name, x in loop.state().items())      # (recorded, not run)
    for turn in range(4):
        for i in range(2):
            new = [int(n) for n in np.random.default_rng(10 * turn + i).integers(0, 6, 3)]
            eager[i].feed(rngs[0][i], new)
            captured[i].feed(rngs[1][i], new)
            before = eager[i].state()
            eager[i].step(5, True)
            eager[i].check(before, new, 5, True)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        for i in range(2):
            want, got = eager[i].state(), captured[i].state()
            for name in Loop.STATE:
                assert torch.equal(got[name], want[name]), (turn, i, name)


def test_on_streams_of_their_own():
    """Two loops on two streams at once, each with its own workspace and scratch, against the same alone."""
    results = []
    for at_once in (False, True):
        loops = [Loop(32, 2, 80, 12, 6, 3) for _ in range(2)]
        streams = [torch.cuda.Stream() for _ in loops] if at_once else [torch.cuda.current_stream()] * 2
        rngs = [np.random.default_rng(5 + i) for i in range(2)]
        for new in ([40, 33], [4, 2], [1, 4]):
            for loop, rng in zip(loops, rngs):
                loop.feed(rng, new)
            torch.cuda.synchronize()
            for loop, stream in zip(loops, streams):
                with torch.cuda.stream(stream):
                    loop.step(max(new), False, drafts=max(new) < 9)
            torch.cuda.synchronize()
        results.append([loop.state() for loop in loops])
    for a, b in zip(*results):
        for name in Loop.STATE:
            assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("listed", [False, True])
def test_one_token_is_what_the_decode_calls_compute(B, listed):
    """One new token a sequence: chess_dense_decode / chess_sparse_decode (fp32 out) to half a step of bf16 and what either loses (weights to 2^-16 at most here)."""
    from attend_common import Batch, ints
    x = Batch(B, [70, 300, 5, 33], [1] * 4, 8, 2, B=B, listed=4 if listed else None)
    got = x.run().double().cpu().numpy()
    a = x.cuda()
    out = torch.zeros((4, 8, D), dtype=torch.float32, device="cuda")
    rest = (x.ws,)
    if listed:
        x.lib.sparse_decode(a["q"], a["k_pool"].nan_to_num(0.0), a["v_pool"].nan_to_num(0.0), a["block_table"], a["seq_lens"], ints(x.ids), ints(x.n), out, *rest)
    else:
        x.lib.dense_decode(a["q"], a["k_pool"].nan_to_num(0.0), a["v_pool"].nan_to_num(0.0), a["block_table"], a["seq_lens"], out, *rest)
    torch.cuda.synchronize()
    want, off = x.want()
    other = out.double().cpu().numpy()
    # each is within its own error of the exact value; the decode calls round the weights to bf16 or less, so half a step of the sum of weights times |v| for theirs
    assert (np.abs(got - want) <= off).all()
    size = np.abs(a["v_pool"].nan_to_num(0.0).double().cpu().numpy()).max()
    assert (np.abs(got - other) <= off + ref.HALF_STEP * size + 2.0 ** -8 * np.abs(want)).all()
