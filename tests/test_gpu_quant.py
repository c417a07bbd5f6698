"""The cache in 8 bits: the store bit for bit against its definition, attention over 8-bit pages against fp64 within what fp32 sums may be off."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
import quant_reference as ref

pytestmark = pytest.mark.gpu
SUMMARY_DTYPE_SWEEP = False
D = 128


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)


class Cache:
    """Pools of random bytes (NaN among them) and of random scales, on both sides."""

    def __init__(self, rng, n_phys, H, B):
        self.k = rng.integers(0, 256, (n_phys, H, B, D), dtype=np.uint8)
        self.v = rng.integers(0, 256, (n_phys, H, D, B), dtype=np.uint8)
        self.scales = 2.0 ** rng.integers(-12, 4, (n_phys, H, 2)).astype(np.float64)

    def cuda(self):
        return torch.from_numpy(self.k).cuda(), torch.from_numpy(self.v).cuda(), torch.from_numpy(self.scales.astype(np.float32)).cuda()

    def clean(self):
        """No NaN bytes."""
        for pool in (self.k, self.v):
            pool[pool & 127 == 127] = 0x3a
        return self


def check_store(rng, writes, k_new, v_new, H, B, n_phys, extra=0, max_writes=None):
    """writes: entries; k_new / v_new fp32 [tokens, H, d]."""
    cache = Cache(rng, n_phys, H, B)
    lib = pk.Chess(pk.Config(2 * H, H, B, 1, 4, 4))
    k, v, scales = cache.cuda()
    kn, vn = bf16(k_new), bf16(v_new)
    # rows of a wider projection
    wide = torch.full((kn.shape[0], (2 * H + extra) * D), float("nan"), dtype=torch.bfloat16)
    wide[:, : H * D], wide[:, (H + extra) * D:] = kn.flatten(1), vn.flatten(1)
    wide = wide.cuda()
    held = np.full((max_writes or len(writes), 4), 7, np.int32)
    held[: len(writes)] = writes
    lib.quant_store(wide[:, : H * D].unflatten(1, (H, D)), wide[:, (H + extra) * D:].unflatten(1, (H, D)), ints(held), ints([0, len(writes), 0, 0]), k, v, scales)
    torch.cuda.synchronize()
    ref.store(cache.k, cache.v, cache.scales, kn.double().numpy(), vn.double().numpy(), writes)
    assert np.array_equal(scales.cpu().double().numpy(), cache.scales)
    assert ref.same_bytes(k.cpu().numpy(), cache.k), "keys"
    assert ref.same_bytes(v.cpu().numpy(), cache.v), "values"


@pytest.mark.parametrize("H", [1, 3, 8])
@pytest.mark.parametrize("B", [16, 32])
def test_every_offset_and_count(B, H):
    rng = np.random.default_rng(B + H)
    pairs = [(f, c) for f in range(B) for c in (1, 2, 3, B // 2, B - f) if f + c <= B]
    order, writes, row = rng.permutation(len(pairs) + 3), [], 0
    for (f, c), p in zip(pairs, order):
        writes.append([int(p), row, f, c])
        row += c
    size = 2.0 ** rng.integers(-14, 8, (row, 1, 1))              # pages whose scale grows, and pages whose scale does not
    check_store(rng, writes, rng.normal(0, 1, (row, H, D)) * size, rng.normal(0, 1, (row, H, D)) * size, H, B, len(pairs) + 3, extra=2, max_writes=len(writes) + 9)


@pytest.mark.parametrize("B", [16, 32])
def test_values_at_the_borders(B):
    """Zeros, halfway cases, subnormals, the largest and the smallest values, infinities and NaN: alone on a page and behind others."""
    rng = np.random.default_rng(8)
    big = float(torch.finfo(torch.bfloat16).max)
    kinds = [np.zeros(D), np.full(D, -0.0), np.full(D, big), np.linspace(-448, 448, D), np.linspace(-0.02, 0.02, D), np.full(D, 1.75), np.full(D, 1.7578125),
             np.full(D, 2.0 ** -133), np.full(D, 2.0 ** -74), np.r_[np.inf, np.full(D - 1, 3.0)], np.r_[-np.inf, np.nan, np.full(D - 2, -3.0)], np.full(D, np.nan),
             np.r_[big, np.full(D - 1, 1e-30)], rng.normal(0, 1e-20, D), np.repeat(ref.TABLE[64:127][:32] * 1.03125, 4)]
    rows, writes, p = [], [], 0
    for first in (0, 5):
        for a in kinds:
            writes.append([p, len(rows), first, 1])
            rows.append(a)
            p += 1
        for a in kinds:                                          # with an ordinary row in the page
            writes.append([p, len(rows), first, 2])
            rows += [a, rng.normal(0, 1, D)]
            p += 1
    x = np.stack(rows)[:, None, :].repeat(2, 1).astype(np.float32)
    check_store(rng, writes, x, x[::-1].copy(), 2, B, p)


def test_a_page_filled_token_by_token_has_the_scale_of_one_filled_at_once():
    rng = np.random.default_rng(12)
    H, B = 2, 16
    x = (rng.normal(0, 1, (B, H, D)) * 2.0 ** rng.integers(-4, 5, (B, 1, 1))).astype(np.float32)
    lib = pk.Chess(pk.Config(4, H, B, 1, 4, 4))
    pools = []
    for at_once in (True, False):
        k, v = torch.full((1, H, B, D), 255, dtype=torch.uint8, device="cuda"), torch.full((1, H, D, B), 255, dtype=torch.uint8, device="cuda")
        scales = torch.full((1, H, 2), 2.0 ** 60, device="cuda")
        rows = bf16(x).cuda()
        for t in [None] if at_once else range(B):
            entry = [0, 0, 0, B] if at_once else [0, t, t, 1]
            lib.quant_store(rows, rows, ints([entry]), ints([0, 1, 0, 0]), k, v, scales)
        torch.cuda.synchronize()
        pools.append((scales.cpu().numpy(), *(p.cpu().view(torch.float8_e4m3fn).double().numpy() for p in (k, v))))
    (s0, k0, v0), (s1, k1, v1) = pools
    assert np.array_equal(s0, s1) and s0.max() < 2.0 ** 10
    # rounded twice only where a value becomes subnormal: half a step of 2^-9 from each rounding
    for a, b in ((k0, k1), (v0, v1)):
        assert np.array_equal(a[np.abs(a) >= 2.0 ** -5], b[np.abs(a) >= 2.0 ** -5]) and np.abs(a - b).max() <= 2.0 ** -9


def test_nothing_to_store_and_refusals():
    lib = pk.Chess(pk.Config(4, 2, 16, 2, 4, 4))
    k, v, scales = Cache(np.random.default_rng(0), 3, 2, 16).cuda()
    before = k.clone(), v.clone(), scales.clone()
    rows = torch.zeros((4, 2, D), dtype=torch.bfloat16, device="cuda")
    lib.quant_store(rows[:0], rows[:0], ints([[0, 0, 0, 16]]), ints([0, 1, 0, 0]), k, v, scales)
    lib.quant_store(rows, rows, ints([[0, 0, 0, 16]]), ints([0, 0, 0, 0]), k, v, scales)       # no entries
    lib.quant_store(rows, rows, ints([[0, 0, 0, 0], [1, 0, 3, -2]]), ints([0, 2, 0, 0]), k, v, scales)   # entries without tokens
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, (k, v, scales)))
    out, ws = torch.empty((2, 4, D), device="cuda"), lib.new_workspace()
    q, table, lens = torch.zeros((2, 4, D), dtype=torch.bfloat16, device="cuda"), ints(np.zeros((2, 4))), ints([3, 4])
    lib.quant_dense_decode(q, k, v, scales, table, lens, out, ws)
    for bad in (dict(q=q.float()), dict(q=q[:1]), dict(k=k[:2]), dict(v=v.transpose(2, 3)), dict(scales=scales[:, :1]), dict(scales=scales.half()),
                dict(table=table[:, :3]), dict(lens=ints([1, 2, 3])), dict(out=out[:, ::2]), dict(ws=ws[:-256])):
        a = dict(q=q, k=k, v=v, scales=scales, table=table, lens=lens, out=out, ws=ws) | bad
        with pytest.raises(pk.ChessError):
            lib.quant_dense_decode(a["q"], a["k"], a["v"], a["scales"], a["table"], a["lens"], a["out"], a["ws"])
    with pytest.raises(pk.ChessError, match="page_ids"):
        lib.quant_sparse_decode(q, k, v, scales, table, lens, ints(np.zeros((2, 2, 3))), ints(np.zeros((2, 2))), out, ws)
    with pytest.raises(pk.ChessError):                           # both kinds of catch-up at once
        lib.quant_summarize(k, scales, table, lens, lib.new_summaries(), from_page=lens, recent_pages=2)
    with pytest.raises(pk.ChessError):
        lib.quant_summarize(k, scales, table, lens, lib.new_summaries(), recent_pages=-1)
    odd = torch.zeros(4 * 2 * D + 4, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(pk.ChessError):                           # rows not on 16 bytes
        lib.quant_store(odd[4:].view(4, 2, D), rows, ints([[0, 0, 0, 1]]), ints([0, 1, 0, 0]), k, v, scales)
    with pytest.raises(pk.ChessError):                           # tokens 260 elements apart
        lib.quant_store(odd.as_strided((3, 2, D), (260, D, 1)), rows[:3], ints([[0, 0, 0, 1]]), ints([0, 1, 0, 0]), k, v, scales)
    torch.cuda.synchronize()


# ---- attention
def dealt(rng, lens, pages, B):
    """A block table for these lengths, and the physical pages it needs; entries without a page are bad numbers."""
    held = [-(-n // B) for n in lens]
    order = rng.permutation(sum(held) + 2)
    table, at = np.full((len(lens), pages), -1, np.int32), 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(held) + 2


def check_attention(rng, lens, Hq, H, B, lists=None, pages=None, splits=(0, 4), scale_spread=True, sm_scale=0.0, q_size=1.0, room=None, scales_of=None):
    """Against fp64 over the listed pages (lists[b][h]) or every page; the bytes behind the last token stay as they fell, NaN among them."""
    G, batch = Hq // H, len(lens)
    pages = pages or max(1, max(-(-n // B) for n in lens))
    table, n_phys = dealt(rng, lens, pages, B)
    cache = Cache(rng, n_phys, H, B)
    if not scale_spread:
        cache.scales[:] = 2.0 ** -6
    if scales_of is not None:
        scales_of(cache.scales)
    for b, n in enumerate(lens):                                 # the tokens that exist are finite
        for p in range(-(-n // B)):
            m = min(B, n - p * B)
            for page in (cache.k[table[b, p]][:, :m], cache.v[table[b, p]][:, :, :m]):
                page[page & 127 == 127] = 0x31
    room = room or (pages if lists is None else max(1, max(len(x) for row in lists for x in row)))
    lib = pk.Chess(pk.Config(Hq, H, B, batch, pages, min(pages, room), sm_scale=sm_scale))
    ws = lib.new_workspace()
    if splits[0]:
        lib.debug_force_splits(*splits)
    q = bf16(rng.normal(0, q_size, (batch, Hq, D)) / 40)
    k, v, scales = cache.cuda()
    out = torch.full((batch, Hq, D), float("nan"), device="cuda")
    if lists is None:
        lib.quant_dense_decode(q.cuda(), k, v, scales, torch.from_numpy(table).cuda(), ints(lens), out, ws)
    else:
        ids, n_sel = np.full((batch, H, lib.cfg.max_selected_pages), -1, np.int32), np.zeros((batch, H), np.int32)
        for b in range(batch):
            for h in range(H):
                ids[b, h, : len(lists[b][h])] = lists[b][h]
                n_sel[b, h] = len(lists[b][h])
        lib.quant_sparse_decode(q.cuda(), k, v, scales, torch.from_numpy(table).cuda(), ints(lens), ints(ids), ints(n_sel), out, ws)
    torch.cuda.synchronize()
    got, qn = out.cpu().double().numpy(), q.double().numpy()
    for b, n in enumerate(lens):
        for h in range(H):
            kl, vl = (ref.rows_of(pool, cache.scales, w, table[b], h, n) for w, pool in ((0, cache.k), (1, cache.v)))
            if lists is not None:
                at = np.array([t for p in lists[b][h] for t in range(p * B, min(n, p * B + B))], int)
                kl, vl = kl[at], vl[at]
            mine = got[b, h * G:(h + 1) * G]
            if kl.shape[0] == 0:
                assert np.array_equal(mine, np.zeros((G, D))), (b, h)
                continue
            want, off = ref.attention(qn[b, h * G:(h + 1) * G], kl, vl, sm_scale or 1 / math.sqrt(D))
            assert (np.abs(mine - want) <= off).all(), (b, h, float((np.abs(mine - want) / off).max()))
    return out


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 79, 80, 127, 128, 129, 400, 1000]


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("Hq,H", [(1, 1), (8, 2), (14, 2), (16, 1)])
def test_every_page_of_short_and_odd_lengths(B, Hq, H):
    check_attention(np.random.default_rng(B + Hq), LENGTHS, Hq, H, B)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("Hq,H", [(1, 1), (8, 2), (14, 2), (16, 1)])
def test_short_and_odd_lengths_where_long_ones_could_be(B, Hq, H):
    """The same and fewer of them in rows of a configuration for longer ones: in a line, and dealt by length."""
    check_attention(np.random.default_rng(B + Hq), LENGTHS, Hq, H, B, pages=6000 // B)
    check_attention(np.random.default_rng(B + Hq), LENGTHS[::2], Hq, H, B, pages=6000 // B)
    check_attention(np.random.default_rng(B + Hq), [700, 700, 700], Hq, H, B, pages=6000 // B)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("n", [1, 40, 64, 700, 3001])
def test_one_sequence(B, n):
    check_attention(np.random.default_rng(n), [n], 8, 2, B)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("Hq,H", [(1, 1), (7, 1), (10, 2), (16, 1), (32, 2)])
def test_one_sequence_of_any_group(B, Hq, H):
    """Eight waves a workgroup; with sixteen heads their exchange takes more than 64 KB."""
    rng = np.random.default_rng(Hq)
    check_attention(rng, [1500], Hq, H, B)
    check_attention(rng, [1500], Hq, H, B, pages=330000 // B)
    check_attention(rng, [1500], Hq, H, B, lists=[[list(range(0, -(-1500 // B), 2)) for _ in range(H)]], splits=(2, 8))


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("Hq,H", [(1, 1), (14, 2), (16, 1)])
def test_batches_dealt_to_four_and_to_eight_waves(B, Hq, H):
    """Few sequences (eight waves a workgroup) and many (four), of equal and of very different lengths."""
    rng = np.random.default_rng(Hq + 50)
    for lens in ([3000, 5], [700, 700, 700], [0, 1, 2222], rng.integers(0, 400, 40).tolist(), [130] * 60):
        check_attention(rng, lens, Hq, H, B)
    check_attention(rng, [2000, 0, 65], Hq, H, B, pages=330000 // B)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("Hq,H", [(2, 1), (14, 2), (32, 8)])
def test_shares_that_hold_ends_whole_sequences_and_beginnings(B, Hq, H):
    """Many sequences in a line: empty ones, ones of a tile, and long ones that many workgroups share."""
    rng = np.random.default_rng(Hq + 60)
    for lens in ([0] * 30 + [5000] + [0, 1] * 20 + [900] * 10, [64] * 130, rng.integers(1, 3000, 70).tolist(), [3000] + [1] * 200 + [3000]):
        check_attention(rng, lens if H < 8 else lens[25:60], Hq, H, B, pages=6000 // B)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("e", [-64, 119])
def test_scales_at_either_end(B, e):
    """Values of the largest and the smallest scale; keys of the smallest."""
    rng = np.random.default_rng(33)
    check_attention(rng, [200, 65, 3], 8, 2, B, scales_of=lambda s: s.__setitem__((slice(None), slice(None), 1), 2.0 ** e))
    if e < 0:
        check_attention(rng, [200, 65, 3], 8, 2, B, q_size=2.0 ** 60, scales_of=lambda s: s.__setitem__((slice(None), slice(None), 0), 2.0 ** e))


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("splits", [(1, 1), (1, 4), (3, 4), (7, 1), (16, 4), (40, 4)])
def test_any_split(B, splits):
    check_attention(np.random.default_rng(4), [1000, 65, 1, 0, 513], 8, 2, B, splits=splits)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("splits", [(0, 4), (1, 4), (5, 4), (2, 8), (3, 1)])
@pytest.mark.parametrize("Hq,H", [(8, 2), (28, 4)])
def test_lists_of_any_length(B, splits, Hq, H):
    rng = np.random.default_rng(6)
    lens = [1000, 1, 70, 333, 0, 640]
    lists = []
    for b, n in enumerate(lens):
        P = -(-n // B)
        lists.append([sorted(rng.choice(P, rng.integers(0, P + 1), replace=False).tolist()) for _ in range(H)])
    lists[0][0], lists[0][1] = [], list(range(-(-1000 // B)))    # nothing listed, everything listed
    lists[3][0] = [-(-333 // B) - 1]                             # the tail page alone
    check_attention(rng, lens, Hq, H, B, lists=lists, splits=splits)


@pytest.mark.parametrize("B", [16, 32])
def test_more_rows_than_workgroups(B):
    rng = np.random.default_rng(21)
    lens = rng.integers(0, 150, 600).tolist()
    check_attention(rng, lens, 4, 1, B)
    check_attention(rng, lens, 4, 1, B, pages=9000 // B)                                  # (pools sized for more than stays in the caches)


@pytest.mark.parametrize("B", [16, 32])
def test_caches_sized_for_long_contexts(B):
    """Rows of a configuration whose pools are a stream: one sequence, several, lists."""
    rng = np.random.default_rng(22)
    check_attention(rng, [2500], 8, 2, B, pages=330000 // B)
    check_attention(rng, [0, 700, 1, 64, 2100], 8, 2, B, pages=80000 // B)
    lens = rng.integers(1, 200, 300).tolist()
    lists = [[sorted(rng.choice(-(-n // B), rng.integers(0, -(-n // B) + 1), replace=False).tolist())] for n in lens]
    check_attention(rng, lens, 4, 1, B, lists=lists, pages=2000 // B + 1, room=2000 // B)


@pytest.mark.parametrize("B", [16, 32])
def test_sharp_and_flat_softmax(B):
    rng = np.random.default_rng(7)
    check_attention(rng, [300, 64, 5], 8, 2, B, q_size=60.0, scale_spread=False)          # hundreds between scores
    check_attention(rng, [300, 64, 5], 8, 2, B, q_size=1e-30)
    check_attention(rng, [300, 64, 5], 8, 2, B, sm_scale=1.0)


def test_pools_beyond_4_gb():
    """Pages whose byte offset passes 32 bits, in the store, the summaries and attention."""
    H, B, n_phys = 8, 16, 300000                                 # 4.9 GB a pool
    rng = np.random.default_rng(2)
    lib = pk.Chess(pk.Config(16, H, B, 1, 4, 4))
    k = torch.empty((n_phys, H, B, D), dtype=torch.uint8, device="cuda")
    v = torch.empty((n_phys, H, D, B), dtype=torch.uint8, device="cuda")
    scales = torch.ones((n_phys, H, 2), device="cuda")
    at = [n_phys - 1, 280001, 262145]
    small = Cache(rng, 3, H, B)
    x, y = rng.normal(0, 1, (40, H, D)).astype(np.float32), rng.normal(0, 1, (40, H, D)).astype(np.float32)
    entries = [[0, 0, 0, 16], [1, 16, 0, 16], [2, 32, 0, 8]]
    lib.quant_store(bf16(x).cuda(), bf16(y).cuda(), ints([[at[p], *r] for p, *r in entries]), ints([40, 3, 0, 0]), k, v, scales)
    ref.store(small.k, small.v, small.scales, bf16(x).double().numpy(), bf16(y).double().numpy(), entries)
    table, lens = ints([at + [-1]]), ints([40])
    q, out, summ = bf16(rng.normal(0, 1, (1, 16, D))), torch.empty((1, 16, D), device="cuda"), lib.new_summaries()
    lib.quant_dense_decode(q.cuda(), k, v, scales, table, lens, out, lib.new_workspace())
    lib.quant_summarize(k, scales, table, lens, summ)
    torch.cuda.synchronize()
    got_k = k[at].cpu().numpy()
    assert np.array_equal(got_k[:2], small.k[:2]) and np.array_equal(got_k[2, :, :8], small.k[2, :, :8]) and np.array_equal(v[at[:2]].cpu().numpy(), small.v[:2])
    pages = lib.summary_views(summ)[0].cpu().double().numpy()
    for h in range(H):
        kl, vl = (ref.rows_of(p, small.scales, w, [0, 1, 2], h, 40) for w, p in ((0, small.k), (1, small.v)))
        want, off = ref.attention(q.double().numpy()[0, 2 * h:2 * h + 2], kl, vl, 1 / math.sqrt(D))
        assert (np.abs(out.cpu().double().numpy()[0, 2 * h:2 * h + 2] - want) <= off).all()
        for p in range(3):
            assert np.array_equal(pages[0, h, p], kl[16 * p:16 * p + 16].mean(0).astype(np.float32)), (h, p)


def test_the_same_bits_on_every_call_and_from_a_graph():
    """Eager calls, a captured graph replayed between other work, another stream: one result each."""
    rng = np.random.default_rng(11)
    H, B, lens = 2, 16, [900, 333, 64, 1]
    table, n_phys = dealt(rng, lens, 60, B)
    cache = Cache(rng, n_phys, H, B).clean()
    k, v, scales = cache.cuda()
    lib = pk.Chess(pk.Config(8, H, B, 4, 60, 60))
    ws, q = lib.new_workspace(), bf16(rng.normal(0, 0.05, (4, 8, D))).cuda()
    bt, sl = torch.from_numpy(table).cuda(), ints(lens)
    ids, n = ints(np.tile(np.arange(60), (4, H, 1))), ints(np.tile(-(-np.array(lens) // B)[:, None], (1, H)))
    outs = [torch.full((4, 8, D), float("nan"), device="cuda") for _ in range(2)]

    def both():
        lib.quant_sparse_decode(q, k, v, scales, bt, sl, ids, n, outs[0], ws)
        lib.quant_dense_decode(q, k, v, scales, bt, sl, outs[1], ws)

    both()
    torch.cuda.synchronize()
    first = [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    side = torch.cuda.Stream()
    for i in range(6):
        for o in outs:
            o.fill_(float("nan"))
        if i % 3 == 0:
            graph.replay()
        elif i % 3 == 1:
            both()
        else:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                both()
            torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outs)), i


@pytest.mark.parametrize("B", [16, 32])
def test_a_value_that_was_not_finite_stays_where_it_belongs(B):
    """Stored as NaN: in a value it spoils one output of its head group, in a key its sequence and KV head, and nothing else."""
    rng = np.random.default_rng(3)
    H, Hq, lens = 2, 8, [200, 90, 300]
    table, n_phys = dealt(rng, lens, 20, B)
    lib = pk.Chess(pk.Config(Hq, H, B, 3, 20, 20))
    ws, bt, sl = lib.new_workspace(), torch.from_numpy(table).cuda(), ints(lens)
    q = bf16(rng.normal(0, 1, (3, Hq, D))).cuda()
    k, v, scales = Cache(rng, n_phys, H, B).clean().cuda()
    ids, n = ints(np.tile(np.arange(20), (3, H, 1))), ints(np.tile(-(-np.array(lens) // B)[:, None], (1, H)))
    rows = [bf16(rng.normal(0, 1, (1, H, D))) for _ in range(2)]
    rows[0][0, 1, 5], rows[1][0, 0, 77] = float("inf"), float("nan")             # a key of head 1, a value of head 0

    def attend():
        outs = [torch.empty((3, Hq, D), device="cuda") for _ in range(2)]
        lib.quant_sparse_decode(q, k, v, scales, bt, sl, ids, n, outs[0], ws)
        lib.quant_dense_decode(q, k, v, scales, bt, sl, outs[1], ws)
        torch.cuda.synchronize()
        return [o.cpu() for o in outs]

    before = attend()
    lib.quant_store(rows[0].cuda(), rows[1].cuda(), ints([[int(table[0, 50 // B]), 0, 50 % B, 1]]), ints([1, 1, 0, 0]), k, v, scales)
    for old, new in zip(before, attend()):
        assert torch.equal(old[1:], new[1:]) and bool(new[0, 4:].isnan().all())
        assert bool(new[0, :4, 77].isnan().all()) and not new[0, :4, :77].isnan().any() and not new[0, :4, 78:].isnan().any()


def test_kernels_with_much_lds_can_be_captured():
    """Sixteen heads by eight waves, and the sums of 4096 sequences: more than 64 KB, asked for at the launch."""
    rng = np.random.default_rng(14)
    table, n_phys = dealt(rng, [700], 50, 16)
    k, v, scales = Cache(rng, n_phys, 1, 16).clean().cuda()
    lib = pk.Chess(pk.Config(16, 1, 16, 4096, 50, 50))
    ws, q, out = lib.new_workspace(), bf16(rng.normal(0, 0.05, (1, 16, D))).cuda(), torch.zeros((1, 16, D), device="cuda")
    bt, sl = torch.from_numpy(table).cuda(), ints([700])
    n = 4096
    big, free, left, counts = ints(np.full((n, 50), -1)), ints(np.arange(n)), ints([0]), ints([0] * 4)
    after, starts, writes = ints([0] * n), ints([0] * (n + 1)), ints(np.zeros((n, 4)))
    zero, one, n_free = ints([0] * n), ints([1] * n), ints([n])

    def both():
        lib.quant_dense_decode(q, k, v, scales, bt, sl, out, ws)
        lib.map_tokens(zero, one, big, free, n_free, after, left, starts, None, writes, counts, ws, max_tokens=n)

    both()
    torch.cuda.synchronize()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        out.zero_()
        counts.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first) and counts.tolist() == [n, n, n, 0] and left.item() == 0
        assert torch.equal(big[:, 0], torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda"))
