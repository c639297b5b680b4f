"""The walk of df_paged_attn over spans, units and tiles, on the host and against a walk key by key (paged_walk.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    exe = str(tmp_path_factory.mktemp("walk") / "walk")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2601_20499_amd", "csrc"), os.path.join(ROOT, "tests", "paged_walk.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("part", range(4))
def test_walks(program, part):
    r = subprocess.run([program, str(100 * part), str(100 * (part + 1))], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
