"""Pages handed out on the device: chess_map_tokens and chess_release_pages against their definition sequence by sequence."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
import quant_reference as ref

pytestmark = pytest.mark.gpu
SUMMARY_DTYPE_SWEEP = False


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def library(batch, pages, B):
    return pk.Chess(pk.Config(8, 2, B, batch, pages, pages))


class Pool:
    """Rows of random lengths whose pages are dealt at random, the rest in the free list (which has room for an entry more at least)."""

    def __init__(self, rng, lens, pages, B, n_free, room=0):
        held = [-(-max(n, 0) // B) for n in lens]
        order = rng.permutation(sum(held) + n_free).astype(np.int32)
        self.table = np.full((len(lens), pages), -1, np.int32)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.free = np.concatenate([order[at:], np.full(max(room, 1), -5, np.int32)])
        self.lens, self.n_free, self.B, self.pages = list(lens), n_free, B, pages


def check_map(pool, new, max_tokens, in_place=False, with_slots=True):
    batch, B = len(pool.lens), pool.B
    want = ref.map_tokens(pool.lens, new, pool.table, pool.free, pool.n_free, max_tokens, pool.pages, B)
    lib = library(batch, pool.pages, B)
    ws = lib.new_workspace()
    lens, table, free, n_free = ints(pool.lens), torch.from_numpy(pool.table).cuda(), torch.from_numpy(pool.free).cuda(), ints([pool.n_free])
    after, left = (lens, n_free) if in_place else (ints([-9] * batch), ints([-9]))
    starts, counts = ints([-9] * (batch + 1)), ints([-9] * 4)
    rows = lib.write_rows(max_tokens, batch)
    assert rows == min(max_tokens, max_tokens // B + 2 * batch)
    writes = torch.full((rows + 3, 4), -9, dtype=torch.int32, device="cuda")
    slots = torch.full((max_tokens + 3,), -9, dtype=torch.int64, device="cuda") if with_slots else None
    lib.map_tokens(lens, ints(new), table, free, n_free, after, left, starts, slots, writes, counts, ws, max_tokens=max_tokens)
    torch.cuda.synchronize()
    assert counts.tolist() == want["counts"]
    assert after.tolist() == want["lens_after"] and left.item() == want["n_left"] and starts.tolist() == want["starts"]
    assert np.array_equal(table.cpu().numpy(), np.array(want["table"]))
    n, w = want["counts"][:2]
    assert np.array_equal(writes[:w].cpu().numpy(), np.array(want["writes"], np.int32).reshape(-1, 4)) and bool((writes[w:] == -9).all())
    if with_slots:
        assert np.array_equal(slots[:n].cpu().numpy(), np.array(want["slots"], np.int64)) and bool((slots[n:] == -9).all())
    assert np.array_equal(free.cpu().numpy(), pool.free)
    if not in_place:
        assert lens.tolist() == pool.lens and n_free.item() == pool.n_free
    return want


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("batch,most_new", [(1, 1), (1, 200), (3, 40), (64, 1), (65, 70), (257, 33), (1000, 3), (4096, 2)])
def test_dealing_follows_the_definition(B, batch, most_new):
    rng = np.random.default_rng(batch * 100 + B)
    pages = 20
    lens = rng.integers(0, pages * B - most_new + 1, batch)
    edge = rng.random(batch) < 0.5                            # half the lengths next to a page's end
    lens = np.where(edge, np.clip(lens // B * B + rng.integers(-1, 2, batch), 0, pages * B - most_new), lens).tolist()
    new = rng.integers(0, most_new + 1, batch).tolist()
    pool = Pool(rng, lens, pages, B, sum(-(-n // B) + 1 for n in new))
    check_map(pool, new, max(1, sum(new)), in_place=batch % 2 == 1)


@pytest.mark.parametrize("B", [16, 32])
def test_a_sequence_that_does_not_fit_ends_the_dealing(B):
    rng = np.random.default_rng(3 + B)
    lens, new = [5, 0, B, 2 * B - 1, 7], [B, 3 * B, 1, 1, 0]
    need = [1, 3, 1, 0, 0]
    for n_free in range(sum(need) + 1):                       # pages
        pool = Pool(rng, lens, 8, B, n_free)
        check_map(pool, new, sum(new) + 5)
    pool = Pool(rng, lens, 8, B, 20)
    for most in (1, B - 1, B, B + 1, 4 * B - 1, 4 * B, 4 * B + 1, 4 * B + 2, 4 * B + 3):      # tokens
        check_map(pool, new, most)


def test_rows_without_room_and_without_tokens():
    rng = np.random.default_rng(5)
    pool = Pool(rng, [64, 63, 64, -1, 10, 0, 3], 4, 16, 9)    # four pages a row
    want = check_map(pool, [0, 1, 1, 5, -3, 65, 0], 100)
    assert want["counts"][3] == 3 and want["lens_after"] == [64, 64, 64, -1, 10, 0, 3]
    want = check_map(pool, [0] * 7, 1, with_slots=False)      # nothing at all
    assert want["counts"] == [0, 0, 0, 0]
    want = check_map(Pool(rng, [0, 0], 4, 16, 0), [2 ** 31 - 1, 1], 100)
    assert want["counts"] == [0, 0, 0, 2]


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("batch", [1, 7, 300, 4096])
def test_released_pages_go_behind_the_free_ones(B, batch):
    rng = np.random.default_rng(batch + B)
    pages = 12
    lens = rng.integers(0, pages * B + 1, batch).tolist()
    done = (rng.random(batch) < 0.4).astype(int).tolist()
    done[0] = 1
    for room in (pages * batch, 5 * batch // 2, 1):           # room for all, for some, for hardly any
        pool = Pool(rng, lens, pages, B, 6, room)
        want_lens, want_free, want_n = ref.release(lens, done, pool.table, pool.free, 6, len(pool.free), B)
        for in_place in (False, True):
            lib = library(batch, pages, B)
            ws = lib.new_workspace()
            lens_d, table, free, n_free = ints(lens), torch.from_numpy(pool.table).cuda(), torch.from_numpy(pool.free).cuda(), ints([6])
            after, left = (lens_d, n_free) if in_place else (ints([-9] * batch), ints([-9]))
            lib.release_pages(lens_d, ints(done), table, free, n_free, after, left, ws)
            torch.cuda.synchronize()
            assert after.tolist() == want_lens and left.item() == want_n and free.tolist() == want_free
            assert np.array_equal(table.cpu().numpy(), pool.table)


def test_a_captured_server_step_follows_its_inputs():
    """Release and dealing in one graph, in place: replayed while requests come and go, every replay as the definition says, and no page in two
    places."""
    rng = np.random.default_rng(9)
    B, batch, pages, n_phys, most = 16, 40, 16, 400, 160
    lib = library(batch, pages, B)
    ws = lib.new_workspace()
    lens, done, new = ints([0] * batch), ints([0] * batch), ints([0] * batch)
    table = torch.full((batch, pages), -1, dtype=torch.int32, device="cuda")
    free, n_free = torch.from_numpy(rng.permutation(n_phys).astype(np.int32)).cuda(), ints([n_phys])
    starts, counts = ints([0] * (batch + 1)), ints([0] * 4)
    slots = torch.full((most,), -1, dtype=torch.int64, device="cuda")
    writes = torch.full((lib.write_rows(most, batch), 4), -1, dtype=torch.int32, device="cuda")

    def step():
        lib.release_pages(lens, done, table, free, n_free, lens, n_free, ws)
        lib.map_tokens(lens, new, table, free, n_free, lens, n_free, starts, slots, writes, counts, ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()                                                # (nothing ended, nothing wanted)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    h_lens, h_table, h_free, h_n = [0] * batch, table.cpu().numpy(), free.cpu().numpy(), n_free.item()
    for _ in range(30):
        h_done = (rng.random(batch) < 0.15).astype(int).tolist()
        h_new = np.where(np.array(h_done) | (np.array(h_lens) == 0), rng.integers(0, 60, batch), 1).tolist()
        done.copy_(ints(h_done))
        new.copy_(ints(h_new))
        graph.replay()
        torch.cuda.synchronize()
        h_lens, h_free, h_n = ref.release(h_lens, h_done, h_table, h_free, h_n, n_phys, B)
        want = ref.map_tokens(h_lens, h_new, h_table, h_free, h_n, most, pages, B)
        h_lens, h_table, h_n = want["lens_after"], np.array(want["table"]), want["n_left"]
        assert counts.tolist() == want["counts"] and lens.tolist() == h_lens and n_free.item() == h_n
        assert np.array_equal(table.cpu().numpy(), h_table) and slots[:want["counts"][0]].tolist() == want["slots"]
        held = [p for b, n in enumerate(h_lens) for p in h_table[b][: -(-n // B)].tolist()] + list(h_free[:h_n])
        assert sorted(held) == list(range(n_phys))


def test_refusals():
    lib = library(5000, 4, 16)
    ws = lib.new_workspace()
    t = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    call = lambda batch=2, most=8, writes=None: lib.map_tokens(t(batch), t(batch), t(batch, 4), t(4), t(1), t(batch), t(1), t(batch + 1), None,  # noqa: E731
                                                               t(8 * batch, 4) if writes is None else writes, t(4), ws, max_tokens=most)
    call()
    for bad in (dict(batch=5001), dict(most=0), dict(most=(1 << 29) + 1), dict(batch=4097), dict(writes=t(3, 4)), dict(writes=t(17, 4).view(-1)[1:-3])):
        with pytest.raises(pk.ChessError):
            call(**bad)
    with pytest.raises(pk.ChessError, match="lens_after"):
        lib.release_pages(t(3), t(3), t(3, 4), t(4), t(1), t(2), t(1), ws)
    with pytest.raises(pk.ChessError):
        lib.release_pages(t(4097), t(4097), t(4097, 4), t(4), t(1), t(4097), t(1), ws)
    torch.cuda.synchronize()
