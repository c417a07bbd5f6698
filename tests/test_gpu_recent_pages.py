"""A catch-up of more pages than there are, up to the largest number an argument can hold, is the summaries of everything."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import helpers
import paper_2602_20732_amd as pk
from test_gpu_quant_loop import cache_of, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("n_c,n_g", [(8, 8), (1, 1), (16, 16)])
def test_any_number_of_recent_pages(B, n_c, n_g):
    rng = np.random.default_rng(B + n_c)
    H, lens, pages = 2, [0, 1, 5 * B + 3, 70 * B - 1], 75
    table, k, scales = cache_of(rng, lens, pages, H, B)
    lib = pk.Chess(pk.Config(4, H, B, len(lens), pages, pages, n_c, n_g, summary_dtype=helpers.SUMMARY_DTYPE))
    bt, sl = torch.from_numpy(table).cuda(), ints(lens)
    k8, sd = torch.from_numpy(k).cuda(), torch.from_numpy(scales.astype(np.float32)).cuda()
    k16 = torch.from_numpy(rng.normal(0, 1, k.shape).astype(np.float32)).to(torch.bfloat16).cuda()
    calls = {"8 bits": (lambda s: lib.quant_summarize(k8, sd, bt, sl, s), lambda s, n: lib.quant_summarize(k8, sd, bt, sl, s, recent_pages=n)),
             "bf16": (lambda s: lib.summarize(k16, bt, sl, s), lambda s, n: lib.summarize_recent(k16, bt, sl, n, s))}
    for name, (whole, recent) in calls.items():
        want = lib.new_summaries()
        whole(want)
        for n in (pages, pages + 1, 2 ** 31 - 256, 2 ** 31 - 64, 2 ** 31 - 2, 2 ** 31 - 1):
            got = lib.new_summaries()
            recent(got, n)
            torch.cuda.synchronize()
            assert torch.equal(got, want), (name, n)
