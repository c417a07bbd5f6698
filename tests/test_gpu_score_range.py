"""bf16 attention over rows whose every score is far below zero, through each call that attends.

Every key row is one bf16 value in all dims and every query -1 in all, so that a score is -128 times that value, exact, times the softmax scale: tokens
tie exactly or lie so far apart that only the largest weigh.  The output is the mean of their values; their weights are 1 and exact in both parts, so
what may be off is the sum of n terms, merged over waves and splits: (n + 200) 2^-24 of the mean of the absolute values."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
from test_gpu_quant import dealt, ints

pytestmark = pytest.mark.gpu
SUMMARY_DTYPE_SWEEP = False
D, H, HQ = 128, 2, 8
G = HQ // H


class Rows:
    def __init__(self, seed, lens, B, e, pages=None):
        rng = np.random.default_rng(seed)
        self.lens, self.B, self.pages = lens, B, pages or max(1, max(-(-n // B) for n in lens))
        # (room for a token more, and its page)
        self.table, n_phys = dealt(rng, [n + 1 for n in lens], self.pages + 1, B)
        self.k = (rng.integers(8, 16, (n_phys, H, B)) / 8 * 2.0 ** e)[..., None].repeat(D, 3)
        self.v = torch.from_numpy(rng.normal(0, 1, (n_phys, H, D, B)).astype(np.float32)).to(torch.bfloat16)
        self.kd, self.vd = torch.from_numpy(self.k.astype(np.float32)).to(torch.bfloat16).cuda(), self.v.cuda()
        self.q = torch.full((len(lens), HQ, D), -1.0, dtype=torch.bfloat16, device="cuda")
        self.out = torch.full((len(lens), HQ, D), float("nan"), device="cuda")
        self.bt, self.sl = torch.from_numpy(self.table).cuda(), ints(lens)
        room = self.pages + 1
        self.lib = pk.Chess(pk.Config(HQ, H, B, len(lens), room, room))
        self.ws = self.lib.new_workspace()
        held = -(-np.array(lens) // B)
        ids = np.full((len(lens), H, room), -1, np.int32)
        for b, n in enumerate(held):
            ids[b, :, :n] = np.arange(n)
        self.ids, self.n = ints(ids), ints(np.tile(held[:, None], (1, H)))

    def check(self, grown=None):
        """grown: fp64 key and value rows [batch, H, D] of one more token a row."""
        torch.cuda.synchronize()
        got = self.out.cpu().double().numpy()
        for b, n in enumerate(self.lens):
            for h in range(H):
                phys = self.table[b, : -(-n // self.B)]
                z = -self.k[phys, h, :, 0].reshape(-1)[:n]
                vl = self.v[phys, h].double().numpy().transpose(0, 2, 1).reshape(-1, D)[:n]
                if grown is not None:
                    z, vl = np.append(z, -grown[0][b, h, 0]), np.concatenate([vl, grown[1][b, h][None]])
                mine = got[b, h * G:(h + 1) * G]
                if len(z) == 0:
                    assert np.array_equal(mine, np.zeros((G, D)))
                    continue
                vl = vl[z == z.max()]
                off = (n + 200) * 2.0 ** -24 * np.abs(vl).mean(0)
                assert (np.abs(mine - vl.mean(0)) <= off).all(), (b, h, n)
        self.out.fill_(float("nan"))


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("e", [94, 100, 120])
def test_every_call(B, e):
    r = Rows(B + e, [1000, 1, 0, 333, 2], B, e)
    r.lib.dense_decode(r.q, r.kd, r.vd, r.bt, r.sl, r.out, r.ws)
    r.check()
    for splits in ((0, 4), (1, 4), (5, 4), (3, 8)):
        r.lib.debug_force_splits(*splits)
        r.lib.sparse_decode(r.q, r.kd, r.vd, r.bt, r.sl, r.ids, r.n, r.out, r.ws)
        r.check()
    r.lib.debug_force_splits(0, 4)
    r.lib.sparse_decode_static(r.q, r.kd, r.vd, r.bt, r.sl, r.ids, r.n, r.out)
    r.check()
    # one token more, whose score is the largest of some rows and ties with others
    grown = np.array([0.5, 1, 1, 2, 1])[:, None, None] * 2.0 ** e * np.ones((5, H, D)), np.random.default_rng(e).integers(-8, 9, (5, H, D)).astype(np.float64)
    new = [torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda() for x in grown]
    r.lib.reuse_step(r.q, *new, r.kd, r.vd, r.bt, r.sl, r.ids, r.n, r.out, r.ws)
    r.check(grown)


@pytest.mark.parametrize("B", [16, 32])
def test_long_and_many_rows(B):
    for lens, pages in (([3000], 90000 // B), ([2500], None), ([0, 700, 1, 64, 2100], 60000 // B), ([1, 0, 90, 500, 33] * 20, 4000 // B)):
        r = Rows(len(lens), lens, B, 105, pages)
        r.lib.dense_decode(r.q, r.kd, r.vd, r.bt, r.sl, r.out, r.ws)
        r.check()


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("lens", [[600], [900, 40, 1] * 3])
def test_the_step_in_one_launch(B, lens):
    """Selection of every page and attention over them; the longest row alone is spread over cooperating workgroups."""
    r = Rows(7, lens, B, 100)
    summ = r.lib.new_summaries()
    r.lib.summarize(r.kd, r.bt, r.sl, summ)
    plan = pk.SelectPlan(plan=pk.PLAN_FLAT, sink_pages=1, window_pages=2, budget_pages=r.pages + 1 - 3)
    r.lib.decode_step(r.q, r.kd, r.vd, r.bt, r.sl, summ, plan, r.ids, r.n, r.out, r.ws)
    torch.cuda.synchronize()
    assert r.n[:, 0].tolist() == [-(-n // B) for n in lens]
    r.check()
    assert r.lib.workspace_error(r.ws) == 0
