"""The sizes of tests/test_gpu_layer_ops.py reach every tile that the planner of the
e4m3 products chooses, with a remainder of rows, columns and K among them (CPU;
tests/host/plan_fp8_check.cpp compiles the library's own planner header)."""
import math
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_layer_ops as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = shutil.which("g++") or shutil.which("clang++")


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if CXX is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "plan_fp8_check")
    subprocess.run([CXX, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2609_34608_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "plan_fp8_check.cpp"), "-o", exe], check=True, timeout=120)

    def answers(lines):
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=120)
        assert r.returncode == 0
        return r.stdout.split()

    return answers


def test_every_tile_is_tested(ask):
    tables = set(ask(["tables"]))
    got = ask([f"{e} {m} {n} {k}" for e, m, n, k in ops.TILES])
    assert set(got) == tables
    for tile in tables:
        bm, bn = map(int, tile.split(":")[1].split("x"))
        sizes = [s for s, t in zip(ops.TILES, got) if t == tile]
        assert any(m % bm for _, m, _, _ in sizes) and any(n % bn for _, _, n, _ in sizes)
        assert any(k % 128 for _, _, _, k in sizes) and len({k for *_, k in sizes}) >= 2


def test_every_tile_is_chosen(ask):
    """No entry of a table that no size takes."""
    rng = random.Random(3)
    size = lambda lo, hi: round(math.exp(rng.uniform(math.log(lo), math.log(hi))))  # noqa: E731
    lines = [f"{rng.randint(0, 1)} {size(1, 12000)} {size(16, 6200)} {size(16, 6200)}" for _ in range(4000)]
    assert set(ask(lines)) == set(ask(["tables"]))


def _sweep(ask, form):
    rng = random.Random(4)
    size = lambda lo, hi: round(math.exp(rng.uniform(math.log(lo), math.log(hi))))  # noqa: E731
    return set(ask([f"{form} {size(1, 12000)} {size(16, 6200)} {size(16, 6200)}" for _ in range(4000)]))


def test_every_tile_of_blocks_is_tested(ask):
    got = ask([f"3 {m} {n} {k}" for m, n, k in ops.BLOCK_TILES])
    assert set(got) == _sweep(ask, 3)


def test_qkv_tiles_hold_whole_heads(ask):
    tiles = _sweep(ask, 2)
    assert tiles <= {"2:256x256", "2:192x256", "2:128x256", "2:160x128", "2:64x128", "2:32x64"} and "2:32x64" in tiles
