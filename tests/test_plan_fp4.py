"""The sizes of tests/test_gpu_fp4.py reach every tile that the planner of the 4-bit products
chooses, with a remainder of rows, columns and K among them (CPU;
tests/host/plan_fp4_check.cpp compiles the library's own planner header)."""
import math
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_fp4 as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = shutil.which("g++") or shutil.which("clang++")


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if CXX is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "plan_fp4_check")
    subprocess.run([CXX, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2609_34608_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "plan_fp4_check.cpp"), "-o", exe], check=True, timeout=120)

    def answers(lines):
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=120)
        assert r.returncode == 0
        return r.stdout.split()

    return answers


def _sweep(ask, blocks):
    rng = random.Random(4)
    size = lambda lo, hi: round(math.exp(rng.uniform(math.log(lo), math.log(hi))))  # noqa: E731
    return set(ask([f"{blocks} {size(1, 12000)} {size(16, 6200)} {size(16, 6200)}" for _ in range(4000)]))


def test_every_tile_is_tested(ask):
    tables = set(ask(["tables"]))
    got = ask([f"0 {m} {n} {k}" for m, n, k in ops.TILES])
    assert set(got) == tables
    for tile in tables:
        bm, bn = map(int, tile.split("x"))
        sizes = [s for s, t in zip(ops.TILES, got) if t == tile]
        assert any(m % bm for m, _, _ in sizes) and any(n % bn for _, n, _ in sizes)
        assert any(k % 256 for *_, k in sizes)


def test_every_tile_of_blocks_is_tested(ask):
    got = ask([f"1 {m} {n} {k}" for m, n, k in ops.BLOCK_TILES])
    assert set(got) == _sweep(ask, 1)


def test_every_tile_is_chosen(ask):
    """No entry of the table that no size takes."""
    assert _sweep(ask, 0) == set(ask(["tables"]))
