"""The tiles that the 8-bit products take, asked of the library's own rules on the CPU (i8_rules.h, the header that the launches
use, in a host program): the GPU tests' sizes get the tiles that these tests name, with K past the slices that a tile keeps."""
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_experts_tall_tiles as tall
import test_gpu_wb_i8_long_k as long_k
import test_gpu_wb_i8_tiles as tiles

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    cc = next((c for c in (shutil.which("g++"), "/opt/rocm/bin/amdclang++", shutil.which("c++")) if c and os.path.exists(c)), None)
    if cc is None:
        pytest.skip("no C++ compiler")
    exe = tmp_path_factory.mktemp("rules") / "i8_rules"
    subprocess.run([cc, "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2609_07008_amd", "csrc"), "-o", str(exe),
                    os.path.join(ROOT, "tests", "host", "i8_rules.cpp")], check=True, capture_output=True)

    def answers(lines):
        r = subprocess.run([str(exe)], input="".join("%s %d %d\n" % q for q in lines), capture_output=True, text=True, check=True, timeout=120)
        got = [tuple(map(int, a.split())) for a in r.stdout.splitlines()]
        assert len(got) == len(lines)
        return got
    return answers


def test_wb_tiles_have_their_cases(ask):
    cases = [(shape, n, d_out, d_in) for shape, c in tiles.CASES.items() for n, d_out, d_in in c]
    assert [a[:2] for a in ask([("wb", n, d_out) for _, n, d_out, _ in cases])] == [c[0] for c in cases]


def test_wb_tiles_have_long_cases(ask):
    assert set(long_k.CASES) == set(tiles.CASES)
    got = ask([("wb", n, d_out) for n, d_out, _ in long_k.CASES.values()])
    for (shape, (_, _, d_ins)), (rows, channels, slices) in zip(long_k.CASES.items(), got):
        assert (rows, channels) == shape
        k = 1024 if channels == 16 else 128   # of a slice
        whole, half = d_ins
        assert whole // k >= 2 * slices + 1 and whole % k == 0 and half == whole + 64


def test_the_tests_copy_of_the_rule(ask):
    """test_gpu_wb_i8_tiles.py has the rule a second time, in Python."""
    rng = random.Random(5)
    sizes = [(1 + int(2 ** rng.uniform(0, 18)), 1 + int(2 ** rng.uniform(0, 15))) for _ in range(4000)] + [(n, d) for n in range(1, 70) for d in (1, 16, 4080, 4096, 4097, 16384)]
    assert [a[:2] for a in ask([("wb", n, d) for n, d in sizes])] == [tiles.tile(n, d) for n, d in sizes]
    assert {a[:2] for a in ask([("wb", n, d) for n, d in sizes])} == set(tiles.CASES)


def test_experts_heights(ask):
    heights = list(tall.SIZES)
    assert heights == [64, 128, 256]
    assert [a[0] for a in ask([("experts", sum(tall.SIZES[h]), len(tall.SIZES[h])) for h in heights])] == heights
    for h in heights:
        assert max(tall.SIZES[h]) > 8 * h   # more than a group of row tiles
        assert {0, 1} <= set(tall.SIZES[h])
    assert ask([("experts", 150, 10)]) == [(64,)]
    for d, f in tall.WIDTHS:
        assert min(d, f) / 128 >= 2 * tall.SLICES and d > 3 * 256 and f > 3 * 128
    # the borders of the rule
    assert [a[0] for a in ask([("experts", n, 10) for n in (1, 1289, 1290, 3849, 3850, 10 ** 6)])] == [64, 64, 128, 128, 256, 256]
