"""Where the tiles of a step's sequences can be more than 32 bits count, without a GPU: they are not put in a line."""
from __future__ import annotations

import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_line_of_more_tiles_than_32_bits_count(tmp_path):
    exe = str(tmp_path / "line")
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2602_20732_amd", "csrc"),
                          os.path.join(ROOT, "tests", "attend_line_limit_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr
