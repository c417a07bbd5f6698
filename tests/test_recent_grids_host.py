"""The launch of a catch-up of the last pages, without a GPU: enough grids for any number of pages, up to the largest an argument can hold."""
from __future__ import annotations

import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_grids_of_the_last_pages(tmp_path):
    exe = str(tmp_path / "grids")
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2602_20732_amd", "csrc"),
                          os.path.join(ROOT, "tests", "recent_grids_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr
