"""The longest row a configuration may have: lengths are 32-bit numbers, and so is what they are capped by."""
from __future__ import annotations

import pytest

import paper_2602_20732_amd as pk

pytestmark = pytest.mark.gpu
SUMMARY_DTYPE_SWEEP = False


@pytest.mark.parametrize("B", [16, 32])
def test_rows_of_two_to_the_31_tokens_are_refused(B):
    pk.Chess(pk.Config(1, 1, B, 1, 2 ** 31 // B - 1, 4)).close()
    for pages in (2 ** 31 // B, 2 ** 31 // B + 1, 2 ** 31 - 1):
        with pytest.raises(pk.ChessError, match="-1"):
            pk.Chess(pk.Config(1, 1, B, 1, pages, 4))
