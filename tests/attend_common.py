"""Inputs for the tests of attention over the new tokens of a step, and the comparison with 64 bits."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2602_20732_amd as pk
import step_reference as ref

D = 128


def bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16)


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class Batch:
    """Sequences of `held` tokens and `new` ones behind them, pages in random order, everything that is no token of a sequence NaN."""

    def __init__(self, seed, held, new, Hq=8, H=2, B=16, sharp=1.0, width=None, cap=0.0, window=0, slopes=None, prefix=None, first=None, listed=None,
                 max_batch=None, sm_scale=0.0):
        rng = np.random.default_rng(seed)
        self.rng, self.held, self.new, self.Hq, self.H, self.B = rng, list(held), list(new), Hq, H, B
        self.lens = [h + n for h, n in zip(held, new)]
        self.pages = [-(-n // B) for n in self.lens]
        batch, self.width = len(self.lens), width or max(max(self.pages), 1) + 1
        n_phys = sum(self.pages) + 2
        order = list(rng.permutation(n_phys))
        self.table = rng.integers(0, n_phys, (batch, self.width))
        self.k = np.full((n_phys, H, B, D), np.nan, np.float32)
        self.v = np.full((n_phys, H, D, B), np.nan, np.float32)
        self.seqs = []
        for b, n in enumerate(self.lens):
            k, v = (bf16(rng.normal(0, s, (n, H, D))).float().numpy() for s in (sharp, 1.0))
            self.seqs.append((k, v))
            for p in range(self.pages[b]):
                self.table[b, p] = order.pop()
                self.put(b, p)
        self.starts = np.concatenate([[0], np.cumsum(self.new)])
        self.rows = int(self.starts[-1])
        self.q = bf16(rng.normal(0, 1, (max(self.rows, 1), Hq, D)))
        self.cap, self.window = cap, window
        self.slopes = None if slopes is None else (2.0 ** (-slopes * np.arange(1, Hq + 1) / Hq)).astype(np.float32)
        self.prefix = None if prefix is None else np.asarray(prefix)
        self.first = None if first is None else np.asarray(first)
        self.ids = self.n = None
        if listed:
            self.ids, self.n = np.full((batch, H, listed), -1), np.zeros((batch, H), int)
            for b in range(batch):
                for h in range(H):
                    n = min(listed, self.pages[b])
                    some = sorted(rng.choice(self.pages[b], n, replace=False)) if n else []
                    self.ids[b, h, :n], self.n[b, h] = some, n
        self.sm = sm_scale or 1 / math.sqrt(D)
        self.lib = pk.Chess(pk.Config(Hq, H, B, max_batch or batch, self.width, listed or self.width, sm_scale=sm_scale))
        self.ws = self.lib.new_workspace()
        self.most = max(max(self.new), 1)

    def put(self, b, p):
        """Page p of sequence b into the pools."""
        k, v = self.seqs[b]
        n = min(self.B, self.lens[b] - p * self.B)
        at = slice(p * self.B, p * self.B + n)
        self.k[self.table[b, p], :, :n] = k[at].transpose(1, 0, 2)
        self.v[self.table[b, p], :, :, :n] = v[at].transpose(1, 2, 0)

    def cuda(self):
        f = lambda x, t: None if x is None else torch.from_numpy(np.asarray(x)).to("cuda", t)  # noqa: E731
        scores = pk.Scores(self.cap, f(self.slopes, torch.float32), self.window, f(self.prefix, torch.int32), f(self.first, torch.int32))
        out = torch.full((max(self.rows, 1) + 1, self.Hq, D), 5.0, dtype=torch.bfloat16, device="cuda")
        scratch = self.lib.new_attend_scratch(max(self.rows, 1), self.most, len(self.lens))
        scratch.fill_(255)
        return dict(q=self.q.cuda(), token_start=ints(self.starts), max_new=self.most, k_pool=f(self.k, torch.bfloat16), v_pool=f(self.v, torch.bfloat16),
                    block_table=ints(self.table), seq_lens=ints(self.lens), out=out, workspace=self.ws, scratch=scratch, scores=scores)

    def launch(self, args):
        out = args["out"]
        args = {**args, "out": out[: max(self.rows, 1)]}
        if self.ids is None:
            self.lib.dense_attend(**args)
        else:
            self.lib.sparse_attend(**args, page_ids=ints(self.ids), n_selected=ints(self.n))
        return out

    def run(self):
        out = self.launch(self.cuda())
        torch.cuda.synchronize()
        assert (out[max(self.rows, 1):] == 5).all()
        return out[: self.rows]

    def want(self):
        # a weight is a bf16 number and a bf16 remainder, or, where a sequence and KV head may have more than 64 rows, one bf16 number: off by half a step of these
        weight_step = ref.HALF_STEP if self.most * (self.Hq // self.H) > 64 else ref.HALF_STEP ** 2
        G = self.Hq // self.H
        y, off = np.zeros((self.rows, self.Hq, D)), np.zeros((self.rows, self.Hq, D))
        for b, (held, new) in enumerate(zip(self.held, self.new)):
            at = slice(self.starts[b], self.starts[b] + new)
            p = np.arange(held, held + new)
            see = [ref.interval(x, self.lens[b], self.window, 0 if self.prefix is None else self.prefix[b], 0 if self.first is None else self.first[self.starts[b] + i])
                   for i, x in enumerate(p)]
            for h in range(self.H):
                keys = None
                if self.ids is not None:
                    keys = (self.ids[b, h, : self.n[b, h], None] * self.B + np.arange(self.B)).reshape(-1)
                    keys = keys[keys < self.lens[b]]
                heads = slice(h * G, h * G + G)
                k, v = (x[:, h].astype(np.float64) for x in self.seqs[b])
                with np.errstate(invalid="ignore", over="ignore"):
                    o, size, e = ref.attend(self.q[at, heads].double().numpy(), k, v, p, see, self.sm, self.cap, None if self.slopes is None else self.slopes[heads].astype(np.float64), keys)
                    y[at, heads], off[at, heads] = o, ref.attention_error(o, size, e, self.lens[b], weight_step)
        return y, off

    def check(self, got=None):
        got = (self.run() if got is None else got).double().cpu().numpy()
        y, off = self.want()
        odd = ~np.isfinite(y)
        assert (np.isnan(got) == np.isnan(y)).all() and (got[odd & ~np.isnan(y)] == y[odd & ~np.isnan(y)]).all()
        bad = ~odd & ~(np.abs(got - y) <= off)
        assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], y[bad][:5], off[bad][:5])
