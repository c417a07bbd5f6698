"""Attention of several new tokens of a sequence over the bf16 pages, against 64 bits: few rows (the keys are split) and many."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
import step_reference as ref
from attend_common import Batch, bf16, ints

pytestmark = pytest.mark.gpu
SUMMARY_DTYPE_SWEEP = False

HEADS = [(8, 2), (4, 4), (7, 1), (32, 2)]
RULES = [dict(), dict(cap=5.0), dict(window=37), dict(slopes=8.0), dict(cap=30.0, slopes=4.0, window=100)]
rule_name = lambda r: "-".join(r) or "causal"  # noqa: E731


@pytest.mark.parametrize("rule", RULES, ids=rule_name)
@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("new", [1, 2, 5, 8, 19])
def test_one_sequence(new, heads, B, rule):
    for held in (0, 1, 30, 15 + new, 700):
        Batch(new + held, [held], [new], *heads, B=B, **rule).check()


@pytest.mark.parametrize("rule", RULES[:3], ids=rule_name)
@pytest.mark.parametrize("B", [16, 32])
def test_ragged_batch_dealt_by_length(B, rule):
    Batch(3, [1500, 0, 3, 900, 64, 31, 2000], [5, 1, 0, 8, 2, 3, 4], 8, 2, B=B, **rule).check()
    Batch(4, [0] * 70 + [600], [2] * 70 + [3], 4, 1, B=B, **rule).check()


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("new", [3, 8, 40])
def test_lists(new, B):
    Batch(new, [777, 40, 0, 333], [new, new - 1, 1, 2], 8, 2, B=B, listed=9).check()
    Batch(new, [777, 40, 0, 333], [new, new - 1, 1, 2], 8, 2, B=B, listed=9, cap=7.0, window=200, slopes=3.0).check()


def test_lists_with_entries_that_are_no_pages():
    b = Batch(1, [200, 90], [3, 2], 8, 2, listed=8)
    want = b.want()
    pages = [[int(b.ids[s, h, b.n[s, h] - 1]) for h in range(2)] for s in range(2)]
    b.n -= 1
    for s in range(2):
        for h in range(2):
            assert pages[s][h] >= 0
    want = b.want()
    # entries behind the last page of the sequence, negative ones, and a count above the row
    for s in range(2):
        for h in range(2):
            b.ids[s, h, b.n[s, h]:] = [b.pages[s], -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6, -7, b.pages[s] + 1, -1][: 8 - b.n[s, h]]
    b.n[:] = 1000
    got = b.run().double().cpu().numpy()
    assert (np.abs(got - want[0]) <= want[1]).all()


@pytest.mark.parametrize("new", [6, 200])
@pytest.mark.parametrize("rule", [dict(), dict(cap=20.0)], ids=rule_name)
def test_prefixes(new, rule):
    Batch(2, [0, 50, 300, 0], [new, new, 5, new - 1], 8, 2, prefix=[4, 500, 302, 0], **rule).check()


@pytest.mark.parametrize("listed", [None, 6])
@pytest.mark.parametrize("new", [8, 150])
def test_documents_and_rows_that_see_nothing(new, listed):
    """Starts of documents, some behind the token itself: those rows are 0; a negative one is the beginning."""
    held = [90, 0, 400]
    first = np.concatenate([[(h + i) // 33 * 33 for i in range(new)] for h in held])
    first[::5] = [(h + i) + 1 for h in held for i in range(new)][::5]
    first[1] = -5
    b = Batch(5, held, [new] * 3, 8, 2, first=first, slopes=2.0, listed=listed)
    got = b.run()
    b.check(got)
    assert (got[::5] == 0).all()


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("rule", RULES, ids=rule_name)
def test_prompts(rule, B, heads):
    Batch(6, [0, 100, 7, 0], [129, 70, 1, 333], *heads, B=B, **rule).check()


@pytest.mark.parametrize("new", [4, 130])
def test_a_longer_context_with_peaks(new):
    Batch(7, [3000, 5], [new, new], 4, 2, sharp=3.0).check()


def poisoned(new, value, listed=None, **rule):
    """Sequences whose last tokens' keys and values are not finite: the rows before do not see them."""
    b = Batch(8, [60, 210], [new, new], 8, 2, listed=listed, **rule)
    for s in range(2):
        k, v = b.seqs[s]
        v[-1, 0, 3], v[-1, 1, 64:], v[-2, 1, 127] = value, value, -value
        k[-1, 0, 5] = value
        v[11, 0, 40] = value
        for p in range(b.pages[s]):
            b.put(s, p)
    return b


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("new", [5, 150])
@pytest.mark.parametrize("rule", [dict(), dict(window=20), dict(first=True)], ids=["causal", "window", "documents"])
def test_what_a_row_does_not_see_does_not_touch_it(rule, new, value):
    if "first" in rule:
        rule = dict(first=np.concatenate([np.arange(h, h + new) - 15 for h in (60, 210)]))
    b = poisoned(new, value, **rule)
    got = b.run()
    y, off = b.want()
    got = got.double().cpu().numpy()
    fine = np.isfinite(y)
    assert fine[:-1].any() and not fine.all()
    assert np.isfinite(got[fine]).all() and (np.abs(got - y) <= off)[fine].all()
    assert (np.isnan(got) == np.isnan(y)).all()
    assert (got[np.isinf(y)] == y[np.isinf(y)]).all()


def test_scores_of_any_size():
    """Keys so large that scores reach 1e30: the largest weighs 1."""
    for new in (3, 140):
        for size in (1e4, 1e12, 1e28):
            b = Batch(9, [40], [new], 4, 2)
            k, _ = b.seqs[0]
            k *= np.float32(size)
            k[:] = bf16(k).float().numpy()
            for p in range(b.pages[0]):
                b.put(0, p)
            got = b.run().double().cpu().numpy()
            # (one key outweighs all others unless two are within rounding: those rows say nothing)
            for r in range(new):
                for h in range(4):
                    s = b.sm * (k[: 41 + r, h // 2].astype(np.float64) @ b.q[r, h].double().numpy())
                    order = np.argsort(s)
                    if s[order[-1]] - s[order[-2]] > 1e-4 * abs(s[order[-1]]) + 40:
                        v = b.seqs[0][1][order[-1], h // 2]
                        assert (np.abs(got[r, h] - v) <= 2.0 ** -8 * np.abs(v) + 1e-6).all(), (size, r, h)
            assert np.isfinite(got).all()


def test_sequences_without_tokens_and_rows_behind():
    b = Batch(10, [0, 40, 0], [0, 3, 0], 8, 2)
    b.check()
    args = b.cuda()
    args["token_start"] = ints([0, 0, 2, 2])                      # the last row is nobody's
    out = b.launch(args)
    torch.cuda.synchronize()
    assert (out[2:] == 5).all() and (out[:2] != 5).any()
    args = b.cuda()
    args["token_start"] = ints([0, 0, 4, 4])                      # rows that are not there
    assert (b.launch(args) == 5).all()
    args = b.cuda()
    args["max_new"] = 2                                           # rows beyond max_new are left
    out = b.launch(args)
    torch.cuda.synchronize()
    assert (out[2:] == 5).all()


def test_lengths_shorter_than_the_new_tokens_say():
    """A row whose position would be negative sees nothing."""
    b = Batch(11, [0], [6], 4, 2)
    args = b.cuda()
    args["seq_lens"] = ints([2])
    out = b.launch(args)
    torch.cuda.synchronize()
    assert (out[:4] == 0).all() and (out[4:6] != 0).any()


@pytest.mark.parametrize("new", [5, 90])
def test_replayed_with_other_lengths_between_eager_work(new):
    """The launch reads lengths and starts on the device: a captured one follows them."""
    full = Batch(12, [500, 33, 250], [new, new, new - 2], 8, 2)
    args = full.cuda()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        full.launch(args)
    want = full.run()
    for step in range(3):
        args["out"].fill_(5.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(args["out"][: full.rows], want)
    shorter = ints([full.lens[0] - 3, full.lens[1] - 1, full.lens[2] - 7])
    args["seq_lens"].copy_(shorter)
    eager = {**full.cuda(), "seq_lens": shorter}
    out = full.launch(eager)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(args["out"], out)


@pytest.mark.parametrize("new", [2, 60])
def test_many_sequences(new):
    rng = np.random.default_rng(0)
    Batch(13, rng.integers(0, 90, 150), rng.integers(0, new + 1, 150), 4, 1).check()


def test_far_pages_of_a_large_pool():
    """Offsets beyond 2^32 bytes into the pools."""
    H, B = 8, 32
    page = H * B * 128
    n_phys = (1 << 32) // (2 * page) + 3
    b = Batch(14, [70], [3], 16, H, B=B)
    args = b.cuda()
    k, v = (torch.empty((n_phys, *x.shape[1:]), dtype=torch.bfloat16, device="cuda") for x in (args["k_pool"], args["v_pool"]))
    far = [n_phys - 1, 0, n_phys - 2]
    for p in range(b.pages[0]):
        k[far[p]], v[far[p]] = args["k_pool"][b.table[0, p]], args["v_pool"][b.table[0, p]]
    table = args["block_table"].clone()
    table[0, : b.pages[0]] = ints(far[: b.pages[0]])
    out = b.launch({**args, "k_pool": k, "v_pool": v, "block_table": table})
    torch.cuda.synchronize()
    b.check(out[: b.rows])


def test_refusals():
    b = Batch(15, [30], [4], 8, 2, listed=2)
    args = b.cuda()
    args["out"] = args["out"][:4]
    dense = b.lib.dense_attend
    dense(**args)
    s = pk.Scores
    for name, bad in (("q", args["q"].float()), ("q", args["q"][:, :4]), ("q", args["q"].reshape(4, -1)), ("out", args["out"].float()), ("out", args["out"][:3]),
                      ("token_start", args["token_start"][:1]), ("block_table", args["block_table"][:, :1]), ("workspace", args["workspace"][:64]),
                      ("scratch", args["scratch"][1:]), ("scratch", args["scratch"][:0]), ("max_new", 0), ("scores", s(cap=-1.0)), ("scores", s(cap=float("nan"))),
                      ("scores", s(cap=float("inf"))), ("scores", s(cap=1e-42)), ("scores", s(window=-1)),
                      ("scores", s(slopes=torch.ones(7, device="cuda"))), ("scores", s(slopes=torch.ones(8))), ("scores", s(first_keys=ints([0] * 3)))):
        with pytest.raises(pk.ChessError):
            dense(**{**args, name: bad})
    with pytest.raises(pk.ChessError):
        s(prefix_lens=torch.zeros(1, device="cuda"))
    with pytest.raises(pk.ChessError):
        b.lib.sparse_attend(**args, page_ids=ints([0]), n_selected=ints([1]))
    n = ctypes.c_size_t()
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, 2)):
        assert b.lib.lib.chess_attend_scratch_bytes(b.lib._h, *bad, ctypes.byref(n)) == -1
    torch.cuda.synchronize()


@pytest.mark.parametrize("new", [3, 40])
def test_lists_of_many_sequences(new):
    rng = np.random.default_rng(1)
    Batch(16, rng.integers(0, 200, 90), rng.integers(0, new + 1, 90), 4, 1, listed=5).check()


@pytest.mark.parametrize("new", [7, 160])
def test_lists_with_prefixes_and_windows(new):
    Batch(17, [150, 0, 61], [new, new, 2], 8, 2, listed=7, prefix=[100, new, 0], window=90, cap=25.0).check()


@pytest.mark.parametrize("new", [5, 90])
def test_prefixes_that_are_no_number_of_tokens(new):
    """A negative one is none, however low."""
    Batch(18, [30, 0, 77], [new] * 3, 8, 2, prefix=[-(2 ** 31), -1, -(2 ** 31) + 1]).check()


@pytest.mark.parametrize("new", [5, 90])
def test_starts_out_of_order(new):
    """Sequences whose starts fall, or name rows that are not there, have no new tokens; two may share rows' queries (of outputs, either's)."""
    b = Batch(19, [30, 50, 20], [new] * 3, 8, 2)
    args = b.cuda()
    for starts in ([0, new, 0, new], [-1, new, 2 * new, 3 * new + 1], [2 ** 31 - 1, -(2 ** 31), 2 ** 31 - 1, 5], [0, 3 * new + 1, 0, 0]):
        args["out"].fill_(5.0)
        out = b.launch({**args, "token_start": ints(starts)})
        torch.cuda.synchronize()
        rows = torch.zeros(len(out), dtype=torch.bool, device="cuda")
        for i in range(3):
            if 0 <= starts[i] <= starts[i + 1] <= b.rows:
                rows[starts[i]:starts[i + 1]] = True
        assert ((out != 5).flatten(1).any(1) == rows).all(), starts


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("H,length,new", [(32, 40000, 3), (2, 40000, 80)])
def test_long_contexts_of_few_pages(H, length, new, B):
    """More pages a workgroup than it looks up at a time; the physical ones are few and repeat, the reference is formed in 64 bits on the device."""
    G, n_phys, width = 2, 60, -(-length // B)
    gen = torch.Generator("cuda")
    gen.manual_seed(B)
    normal = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)  # noqa: E731
    k, v, q = normal(n_phys, H, B, 128), normal(n_phys, H, 128, B), normal(new, H * G, 128)
    table = torch.randint(0, n_phys, (1, width), dtype=torch.int32, device="cuda", generator=gen)
    lib = pk.Chess(pk.Config(H * G, H, B, 1, width, width))
    out = torch.zeros_like(q)
    lib.dense_attend(q, ints([0, new]), new, k, v, table, ints([length]), out, lib.new_workspace(), lib.new_attend_scratch(new, new, 1))
    at, t = table[0].long(), torch.arange(length, device="cuda")
    p = torch.arange(length - new, length, device="cuda").repeat_interleave(G)
    for h in range(H):
        keys, values = k[at, h].reshape(-1, 128)[:length].double(), v[at, h].transpose(1, 2).reshape(-1, 128)[:length].double()
        rows = q[:, h * G:h * G + G].reshape(-1, 128).double()
        s = rows @ keys.T / 128 ** 0.5
        e = 2.0 ** -24 * (130 / 128 ** 0.5 * (rows.abs() @ keys.abs().T).amax(1) + 3 * s.abs().amax(1))
        w = s.masked_fill(t[None] > p[:, None], -float("inf")).softmax(1)
        want, size = w @ values, w @ values.abs()
        step = ref.HALF_STEP if new * G > 64 else ref.HALF_STEP ** 2
        want, size, e, got = (x.double().cpu().numpy() for x in (want, size, e[:, None], out[:, h * G:h * G + G].reshape(-1, 128)))
        assert (np.abs(got - want) <= ref.attention_error(want, size, e, length, step)).all(), h


def test_more_sequences_than_there_may_be():
    n = 4097
    lib = pk.Chess(pk.Config(2, 1, 16, n, 1, 1))
    lens, out = ints([1] * n), torch.full((n, 2, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    pool = torch.ones((1, 1, 16, 128), dtype=torch.bfloat16, device="cuda")
    args = dict(q=out.clone(), max_new=1, k_pool=pool, v_pool=pool.view(1, 1, 128, 16), out=out, workspace=lib.new_workspace(), scratch=lib.new_attend_scratch(n, n, n))
    with pytest.raises(pk.ChessError):
        lib.dense_attend(**args, token_start=ints(range(n + 1)), block_table=ints([[0]] * n), seq_lens=lens)
    assert (out == 5).all()
    lib.dense_attend(**{**args, "max_new": 2 ** 32}, token_start=ints(range(n)), block_table=ints([[0]] * (n - 1)), seq_lens=lens[:-1])
    torch.cuda.synchronize()
    assert (out[:-1] == 1).all() and (out[-1] == 5).all()


@pytest.mark.parametrize("B", [16, 32])
def test_long_lists_of_many_rows(B):
    """Lists longer than a unit, of other lengths a head, one empty, for one sequence and for several."""
    for held in ([6400], [6000, 700, 0]):
        x = Batch(20, held, [45, 20, 3][: len(held)], 8, 2, B=B, listed=4800 // B)
        x.n[0, 1] = 37
        if len(held) > 1:
            x.n[1, 0] = 0
        x.check()


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("new", [1, 2, 5, 13])
def test_few_rows_deep_in_documents(new, B):
    """Documents that begin far behind the sequence's start, at a token of the step, behind all of them, and at numbers that are no key."""
    held = [900, 333, 64, 500]
    first = np.concatenate([[870 + (i > 2) * 15] * 1 for i in range(new)] + [[333 + i // 2 for i in range(new)], [2 ** 31 - 1] * new, [-(2 ** 31)] * new])
    Batch(21, held, [new] * 4, 8, 2, B=B, first=first).check()


RULES_OF_PLACES = [dict(), dict(window=20), dict(slopes=4.0, cap=10.0), dict(prefix=[45, 0, 1]), dict(first=True)]


@pytest.mark.parametrize("rule", RULES_OF_PLACES, ids=rule_name)
@pytest.mark.parametrize("listed", [None, 7])
@pytest.mark.parametrize("new,most", [(3, 2), (16, 5), (60, 9), (60, 17), (300, 150)])
def test_rows_before_max_new_keep_their_places(new, most, listed, rule):
    """Fewer of a sequence's new tokens than it has: the first ones, at the positions that they have; the others' rows are left."""
    held = [40, 333, 0]
    if "first" in rule:
        rule = dict(first=np.concatenate([(h + np.arange(new)) // 9 * 9 for h in held]))
    b = Batch(22, held, [new] * 3, 8, 2, listed=listed, **rule)
    b.most = most
    out = b.launch(b.cuda())
    torch.cuda.synchronize()
    y, off = b.want()
    rows = np.arange(b.rows) % new < most
    got = out[: b.rows].double().cpu().numpy()
    assert (np.abs(got - y) <= off)[rows].all() and (got[~rows] == 5).all() and (out[b.rows:] == 5).all()


def test_few_rows_whose_tiles_could_be_more_than_32_bits_count():
    """33 sequences with room for 2^31 tokens each: not a line of tiles.  Over lists, which are short, one all the same."""
    new, room = np.arange(33) % 4, (1 << 26) - 1
    b = Batch(25, np.arange(33) * 37, new, 4, 1, B=32)
    lib = pk.Chess(pk.Config(4, 1, 32, 33, room, b.width))
    args = b.cuda()
    table = torch.zeros((33, room), dtype=torch.int32, device="cuda")
    table[:, : b.width] = args["block_table"]
    args.update(block_table=table, workspace=torch.zeros(lib.workspace_bytes, dtype=torch.uint8, device="cuda"), scratch=lib.new_attend_scratch(b.rows, b.most, 33))
    b.lib = lib
    dense = b.launch(args).clone()
    torch.cuda.synchronize()
    assert (dense[b.rows:] == 5).all()
    b.ids = np.broadcast_to(np.arange(b.width), (33, 1, b.width)).copy()
    b.n = np.array(b.pages)[:, None]
    args["out"].fill_(5.0)
    b.check(b.launch(args)[: b.rows])
    b.most = 17                                                   # (weights of many rows)
    b.check(dense[: b.rows])


# single keys, a tile, several shares of a line, the last tile
LOW = [(300, 301), (320, 352), (0, 512), (1024, 2048), (2995, 2996)]


@pytest.mark.parametrize("rule", [dict(), dict(slopes=40.0), dict(listed=200, width=210)], ids=rule_name)
@pytest.mark.parametrize("value", [np.inf, np.nan])
@pytest.mark.parametrize("low", LOW, ids=str)
@pytest.mark.parametrize("new", [5, 16, 40])
def test_infinite_values_of_keys_that_weigh_next_to_nothing(new, low, value, rule):
    """Weights of e^-250 to e^-700 are not 0: their sum with an infinity is one, in whatever tile, share or unit the keys lie, and it stays in its dims."""
    b = Batch(23, [3000, 2300], [new, new], 8, 2, **rule)
    b.q = bf16(b.q.float().numpy() + 2)
    for s, (k, v) in enumerate(b.seqs):
        if low[1] <= len(k):
            k[low[0]:low[1]] = -15
            v[low[0], 0, 3], v[low[1] - 1, 1, 64:] = value, -value
            for p in range(b.pages[s]):
                b.put(s, p)
    y, _ = b.want()
    assert not np.isfinite(y).all() and np.isfinite(y).any()
    b.check()


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("value", [np.inf, -np.inf])
@pytest.mark.parametrize("new", [5, 150])
def test_infinite_keys_whose_values_are_infinite(new, value, cap):
    """A score of -infinity weighs nothing, and nothing times an infinity is NaN, in that value's dims; with a cap the key weighs something."""
    b = Batch(26, [1000], [new], 8, 2, cap=cap)
    b.q = bf16(b.q.float().numpy() + 2)
    k, v = b.seqs[0]
    key = np.array(k[300])
    # (an odd dim of the first KV head's key; all but the negative ones of the queries see -infinity)
    k[300, 0, 7], v[300, 0, 3], v[300, 1, 9], v[301, 0, 11] = -np.inf, value, value, value
    b.put(0, 300 // 16)
    got = b.run().double().cpu().numpy()
    y, _ = b.want()
    k[300, 0, 7], v[300, 0, 3] = key[0, 7], 0
    if not cap:
        k[300, 0] = -15                                           # (what weighs nothing, for the bounds)
    _, off = b.want()
    assert (np.isnan(got) == np.isnan(y)).all() and (got[np.isinf(y)] == y[np.isinf(y)]).all()
    fine = np.isfinite(y)
    assert np.isnan(y[:, :4, 3]).all() == (cap == 0) and np.isinf(y).any() and fine.any()
    # (with a cap the score of the key is the cap, off by no more than the others')
    assert (np.abs(got - y) <= off)[fine].all()


@pytest.mark.parametrize("new,heads,lengths", [(6, (4, 2), (46, 2, 1)), (60, (4, 2), (100, 2, 1)), (200, (2, 2), (240, 150, 100))], ids=str)
def test_windows_as_large_as_there_are(new, heads, lengths):
    """A window that no sequence reaches is none, also where a row's position would be negative."""
    b = Batch(24, [40], [new], *heads)
    for length in lengths:
        out = []
        for window in (0, 2 ** 31 - 1):
            b.window = window
            args = b.cuda()
            args["seq_lens"] = ints([length])
            out.append(b.launch(args))
        torch.cuda.synchronize()
        assert torch.equal(*out) and (out[0][new - min(new, length):new] != 0).any()
