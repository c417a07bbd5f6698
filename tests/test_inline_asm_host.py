"""Inline assembly tells the compiler which special registers it writes, read from the sources: what the compiler keeps there would be lost without a word."""
from __future__ import annotations

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_20732_amd", "csrc")


def statements(text):
    """The asm statements of a source, from the word to the closing bracket."""
    for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        yield text[m.start():at]


def test_m0_is_named_where_it_is_written():
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        for s in statements(open(path).read()):
            if re.search(r"\bs_\w+ m0\b", s):
                found += 1
                clobbers = s.rsplit(":", 1)[1]
                assert '"m0"' in clobbers and '"memory"' in clobbers, (os.path.basename(path), s)
    assert found > 0
