"""Which positions a rotation reads, compiled for the host from the header that the kernels include: with one, two and three axes and any part of a
head rotated, no entry behind the positions that the caller has to give; and no other way to them in the append's kernels."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2604_20470_amd import build as b

HERE = os.path.dirname(os.path.abspath(__file__))


def test_positions_of_units(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    exe = str(tmp_path / "pairs")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall",
                        os.path.join(HERE, "stream_pair_check.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout, r.stderr[-2000:])


def test_the_append_reads_positions_through_the_checked_function_or_behind_a_comparison():
    """Two places index the positions: inside unit_positions' reader, and the one-channel path, which has left for channels from dim on."""
    with open(os.path.join(b.CSRC, "k_cache.hip")) as f:
        text = f.read()
    reads = [m.start() for m in re.finditer(r"a\.pos\[", text)]
    assert len(reads) == 2
    single, unit = (text[text.rindex("\n__device__", 0, at):at] for at in reads)
    assert "if (c >= a.r.dim) return" in single and "unit_positions<W>" in unit
