"""The sizes of tests/test_gpu_layer_variant_forms.py reach every tile that the planners
give the projections of the layer variants, with rows left over and, of 256 columns,
columns too (CPU; the host programs compile the library's own planner header)."""
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_layer_variant_forms as forms

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = shutil.which("g++") or shutil.which("clang++")


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if CXX is None:
        pytest.skip("no host C++ compiler")
    exe = {}
    for name in ("plan_check", "plan_fp8_check"):
        exe[name] = str(tmp_path_factory.mktemp("plan") / name)
        subprocess.run([CXX, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2609_34608_amd", "csrc"),
                        os.path.join(ROOT, "tests", "host", name + ".cpp"), "-o", exe[name]], check=True, timeout=120)

    def answers(name, lines):
        r = subprocess.run([exe[name]], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=120)
        assert r.returncode == 0
        out = [x.split()[0] for x in r.stdout.splitlines()]
        assert len(out) == len(lines)
        return out

    return answers


def _lines(mode, M, D, F):
    """(epilogue, N, question) of a layer's projections."""
    if mode == "fp8":
        return [("qkv", 3 * D, f"2 {M} {3 * D} {D}"), ("residual", D, f"0 {M} {D} {D}"),
                ("residual", D, f"0 {M} {D} {F}"), ("up", F, f"3 {M} {F} {D}")]
    return [("residual", D, f"{mode} {M} {D} {K} 0") for K in (D, F)]


def _found(ask, mode, sizes, remainders):
    asked = [(epi, B * T, N, line) for B, T, D, F in sizes for epi, N, line in _lines(mode, B * T, D, F)]
    got = ask("plan_fp8_check" if mode == "fp8" else "plan_check", [line for *_, line in asked])
    found = set()
    for (epi, M, N, _), tile in zip(asked, got):
        bm, bn = map(int, tile.split(":")[-1].split("x")[:2])
        # a batch's rows of MLP-up tiles: tests/test_plan_fp8.py has their remainders
        if remainders and epi != "up" and (M % bm == 0 or (bn == 256 and N % bn == 0)):
            continue
        found.add((epi, tile))
    return found


@pytest.mark.parametrize("mode,sizes", [("fp8", forms.FP8_TILES), ("bf16", forms.BF16_TILES), ("fp32", forms.FP32_TILES)])
def test_every_tile_of_the_layers_is_tested(ask, mode, sizes):
    rng = random.Random(17)
    sweep = []
    while len(sweep) < 12000:
        B, D = rng.choice([1, 1, 2, 3, 4, 8, 16]), 64 * rng.randint(1, 16 if mode == "fp32" else 32)
        T, F = int(3 * 1000 ** rng.random()), 128 * rng.randint(1, max(1, 4 * D // 128))
        if B * T <= 12000:
            sweep.append((B, T, D, F))
    missing = _found(ask, mode, sweep, False) - _found(ask, mode, sizes, True)
    assert not missing, missing
