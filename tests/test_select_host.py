"""The selection that eviction and lists of blocks share (csrc/pkv_topk.h), by a workgroup that is emulated on the CPU: waves run from
barrier to barrier one after the other, in several orders, so that a wave that is late by all of the others' work is among them."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2406_02069_amd", "csrc")


@pytest.fixture(scope="module")
def select(tmp_path_factory):
    folder = tmp_path_factory.mktemp("select")
    shutil.copy(os.path.join(CSRC, "pkv_topk.h"), folder)        # (alone: what it includes is the emulation's)
    out = str(folder / "select")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", str(folder), "-I", os.path.join(HERE, "emulated"), "-o", out,
                           os.path.join(HERE, "emulated", "select.cpp")])
    return out


@pytest.mark.parametrize("n,k,tops,levels", [
    (1, 1, 0, 0), (64, 5, 0, 0), (300, 50, 0, 0), (300, 50, 50, 0), (300, 250, 20, 3), (300, 50, 0, 1), (9000, 700, 36, 0), (9000, 700, 0, 40),
    (20000, 2048, 36, 0)])
def test_the_largest_are_taken(select, n, k, tops, levels):
    assert subprocess.run([select, str(n), str(k), str(tops), str(levels), "7"], timeout=60).returncode == 0


@pytest.mark.parametrize("n,k,tops", [(300, 50, 51), (300, 50, 200), (300, 299, 300), (1500, 3, 1400), (20000, 700, 701), (20000, 700, 15000),
                                      (70000, 3001, 3002)])
def test_more_protected_keys_than_are_taken(select, n, k, tops):
    assert subprocess.run([select, str(n), str(k), str(tops), "0", "7"], timeout=60).returncode == 0
