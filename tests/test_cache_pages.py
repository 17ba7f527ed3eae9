"""Where the tokens of a paged cache lie and what a row sees (CPU): the library's header
against plain rules, with entries that are no page, lengths past the table and the ends of
32 bits; built with the address and undefined-behaviour sanitizers where they are there."""
import os
import random
import shutil
import subprocess

import pytest

import fp4_ref as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = shutil.which("g++") or shutil.which("clang++")
BIG = 2**31 - 1


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if CXX is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("cache") / "cache_check")
    cmd = [CXX, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2609_34608_amd", "csrc"),
           os.path.join(ROOT, "tests", "host", "cache_check.cpp"), "-o", exe]
    if subprocess.run([*cmd, "-fsanitize=address,undefined", "-fno-sanitize-recover=all"], capture_output=True,
                      timeout=120).returncode:
        subprocess.run(cmd, check=True, timeout=120)

    def answers(lines):
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr[-2000:]
        return [int(x) for x in r.stdout.split()]

    return answers


def test_pages(ask):
    rng = random.Random(1)
    lines, want = [], []
    for _ in range(2000):
        width, shift, pages = rng.randint(0, 6), rng.choice([4, 5, 7, 12]), rng.choice([0, 1, 5, BIG])
        row = [rng.choice([-1, 0, 1, 4, 5, BIG, -BIG - 1]) for _ in range(width)]
        t = rng.choice([rng.randint(-3, (width + 1) << shift), -BIG - 1, BIG, (width << shift) - 1, width << shift])
        lines.append(" ".join(map(str, ("page", width, shift, pages, t, *row))))
        held = 0 <= t < width << shift and 0 <= row[t >> shift] < pages
        want.append(row[t >> shift] if held else -1)
    assert ask(lines) == want


def test_tokens_held_and_seen(ask):
    rng = random.Random(2)
    ends = [-BIG - 1, -5, 0, 1, 17, 300, BIG]
    lines, want = [], []
    for _ in range(3000):
        width, shift, length = rng.choice([0, 1, 9, 1000]), rng.choice([4, 7, 12]), rng.choice(ends + [rng.randint(0, 400)])
        rows, t, causal = rng.choice([0, 1, 20, 16777215]), rng.choice([0, 1, 19, 20, 16777214]), rng.random() < 0.5
        room = width << shift
        lines.append(f"held {length} {width} {shift}")
        want.append(max(0, min(length, room)))
        lines.append(f"seen {want[-1]} {length} {int(causal)} {rows} {t}")
        want.append(F.seen(length, room, causal, rows, t))
    assert ask(lines) == want
