"""Attention over 8-bit pages with scores of any size that fp32 holds.

Every key row is one e4m3 value in all dims and every query +1 or -1 in all, so that a score is 128 times that value, exact, times a power of two:
tokens tie exactly or lie so far apart that only the largest weigh.  The output is the mean of their values.  Their weights are 1 and exact in every
part, so what may be off is the sum of n terms, merged over waves and splits: (n + 200) 2^-24 of the mean of the absolute values, as elsewhere."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
import quant_reference as ref
from test_gpu_quant import Cache, dealt, ints

pytestmark = pytest.mark.gpu
SUMMARY_DTYPE_SWEEP = False
D = 128


def check(seed, lens, Hq, H, B, e, sign, lists=None, pages=None, splits=(0, 4)):
    """Key scales 2^e and 2^(e - 1); lists[b]: the pages of every KV head, or None for every page."""
    rng = np.random.default_rng(seed)
    G, batch = Hq // H, len(lens)
    pages = pages or max(1, max(-(-n // B) for n in lens))
    table, n_phys = dealt(rng, lens, pages, B)
    cache = Cache(rng, n_phys, H, B).clean()
    # values 1 to 1.875 on pages of the larger scale, 2 to 3.75 on the others: rows tie within and between pages
    small = rng.integers(0, 2, (n_phys, H))
    cache.k[:] = (rng.integers(0x38, 0x40, (n_phys, H, B)) + 8 * small[..., None]).astype(np.uint8)[..., None]
    cache.scales[:, :, 0] = 2.0 ** (e - small)
    lib = pk.Chess(pk.Config(Hq, H, B, batch, pages, pages))
    ws = lib.new_workspace()
    if splits[0]:
        lib.debug_force_splits(*splits)
    k, v, scales = cache.cuda()
    q = torch.full((batch, Hq, D), float(sign), dtype=torch.bfloat16, device="cuda")
    out = torch.full((batch, Hq, D), float("nan"), device="cuda")
    if lists is None:
        lib.quant_dense_decode(q, k, v, scales, torch.from_numpy(table).cuda(), ints(lens), out, ws)
    else:
        ids, n_sel = np.full((batch, H, pages), -1, np.int32), np.zeros((batch, H), np.int32)
        for b in range(batch):
            ids[b, :, : len(lists[b])] = lists[b]
            n_sel[b] = len(lists[b])
        lib.quant_sparse_decode(q, k, v, scales, torch.from_numpy(table).cuda(), ints(lens), ints(ids), ints(n_sel), out, ws)
    torch.cuda.synchronize()
    got = out.cpu().double().numpy()
    for b, n in enumerate(lens):
        for h in range(H):
            kl, vl = (ref.rows_of(pool, cache.scales, w, table[b], h, n) for w, pool in ((0, cache.k), (1, cache.v)))
            if lists is not None:
                at = np.array([t for p in lists[b] for t in range(p * B, min(n, p * B + B))], int)
                kl, vl = kl[at], vl[at]
            mine = got[b, h * G:(h + 1) * G]
            if kl.shape[0] == 0:
                assert np.array_equal(mine, np.zeros((G, D))), (b, h)
                continue
            z = sign * kl[:, 0]
            vl = vl[z == z.max()]
            off = (n + 200) * 2.0 ** -24 * np.abs(vl).mean(0)
            assert (np.abs(mine - vl.mean(0)) <= off).all(), (b, h, n, mine[0, :3], vl.mean(0)[:3])


EVERY_WAY = [("one sequence", dict(lens=[1500], pages=330000)), ("one token", dict(lens=[1])), ("short rows", dict(lens=[1, 40, 0, 129, 2])),
             ("dealt by length", dict(lens=[3000, 1, 700], pages=6000)), ("in a line", dict(lens=[1, 900, 0, 2, 64, 3000, 33] * 10, pages=6000)),
             ("lists", dict(lens=[1000, 1, 333], lists=(2, 0, 4))), ("lists of eight waves", dict(lens=[1000, 1, 333], lists=(2, 0, 4), splits=(3, 8)))]


def call(seed, way, Hq, H, B, e, sign):
    way = dict(way)
    if "pages" in way:
        way["pages"] //= B
    if "lists" in way:                                # every second page but the first, the only one, every fifth
        way["lists"] = [list(range(1 if step else 0, -(-n // B), step or 1)) for n, step in zip(way["lens"], way["lists"])]
    check(seed, way.pop("lens"), Hq, H, B, e, sign, **way)


@pytest.mark.parametrize("way", [w for _, w in EVERY_WAY], ids=[n.replace(" ", "_") for n, _ in EVERY_WAY])
@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("e,sign", [(24, 1), (28, 1), (28, -1), (30, 1), (60, 1), (60, -1), (100, 1), (119, 1)])
def test_the_largest_score_weighs_one(way, B, e, sign):
    call(e + B, way, 8, 2, B, e, sign)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("Hq,H", [(1, 1), (16, 1)])
def test_the_largest_score_weighs_one_in_other_groups(B, Hq, H):
    for e, sign in ((30, 1), (60, -1)):
        for _, way in EVERY_WAY:
            call(Hq + B, way, Hq, H, B, e, sign)


@pytest.mark.parametrize("way", [w for _, w in EVERY_WAY], ids=[n.replace(" ", "_") for n, _ in EVERY_WAY])
@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("e", [94, 96, 100, 119])
def test_rows_whose_every_score_is_far_below_zero(way, B, e):
    """Scores from -1e30 down to -2e37 (the largest key scale) are scores all the same: the least of them in size weighs one."""
    call(e + B, way, 8, 2, B, e, -1)
