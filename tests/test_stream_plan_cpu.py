"""How the device cuts keys into pieces: the kernel that writes partial sums and the one that joins them work it out apart, so it is whole numbers, compiled here for the
host from the header that the kernels include."""
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2604_20470_amd", "csrc")


def test_plans_against_arithmetic_without_bounds(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    exe = str(tmp_path / "plan")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall",
                        os.path.join(HERE, "stream_plan_check.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout, r.stderr[-2000:])


@pytest.mark.parametrize("name", ["SequenceLanes", "Shares", "Tiles"])
def test_no_plan_is_made_in_floating_point(name):
    """A sum of products in fp32 may be contracted in one kernel and not in the other."""
    with open(os.path.join(CSRC, "stream_attn.h")) as f:
        body = re.search(r"^struct %s\b.*?^};" % name, f.read(), re.S | re.M).group(0)
    assert not re.search(r"\b(float|double)\b", re.sub(r"//[^\n]*", "", body))
