"""The chunk attention's index arithmetic on the host: the kernel's own header, a warp's lanes as fibers (native/warp.h)."""
import os
import subprocess

import pytest

from paper_2602_08329_b200 import build as B

NATIVE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native")


def compiled(tmp_path_factory, name):
    out = str(tmp_path_factory.mktemp("native") / name)
    cuda = os.path.join(os.path.dirname(os.path.dirname(B.NVCC)), "include")
    res = subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", f"-I{cuda}", f"-I{B.CSRC}", f"-I{NATIVE}", os.path.join(NATIVE, name + ".cpp"),
                          "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    return out


def run(*cmd):
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-2000:]
    return res.stdout


@pytest.fixture(scope="module")
def chunk_walk(tmp_path_factory):
    return compiled(tmp_path_factory, "chunk_walk")


def test_every_tile_is_taken_once_in_one_round_and_in_several(chunk_walk):
    """Over random batches and masks: all tiles that a token sees, once; no workspace slot or ticket of two items in a launch; of every item as
    many pieces as are waited for; up to four rounds."""
    assert run(chunk_walk, "whole").split() == ["52", "runs"]          # 13 CTAs, four rounds


def test_lengths_that_change_under_way_end_the_walk(chunk_walk):
    """Lengths and starts change at a random read: the walk ends, stays in range, and reports it."""
    run(chunk_walk, "changed")
