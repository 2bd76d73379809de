"""The index arithmetic of block attention's walk over the cache, up to sequences of 2^31 - 1 tokens (CPU)."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


def test_the_walk_stays_in_the_cache_and_ends(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "attention_walk")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(os.path.dirname(HERE), "paper_2608_03447_amd", "csrc"),
                    os.path.join(HERE, "attention_walk.cpp"), "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-2000:]
