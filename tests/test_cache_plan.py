"""The sharing-out of kvp_cache_attend (csrc/cache_attend_plan.h, host arithmetic): a C++ program walks it over its range, and each
shape has to run the kernel that was measured to be the faster one there."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cache_plan") / "cache_plan")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2512_14946_amd", "csrc"), "-o", exe,
                    os.path.join(ROOT, "tests", "cache_plan.cpp")], check=True)
    return exe


def test_every_plan_covers_the_tokens_and_fits_its_scratch(plan):
    out = subprocess.run([plan], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
    assert int(out.stdout) > 200_000


def _plan(exe, B, H, G, W, T):
    return tuple(map(int, subprocess.run([exe, *map(str, (B, H, G, W, T))], check=True, capture_output=True, text=True).stdout.split()))


def test_tiles_follow_the_rows_and_the_work(plan):
    for G, W in [(1, 1), (8, 1), (16, 1)]:
        assert _plan(plan, 1, 8, G, W, 8192)[0] == _plan(plan, 64, 8, G, W, 65536)[0] == 16
    for G, W in [(20, 1), (4, 8), (8, 12)]:
        assert _plan(plan, 1, 8, G, W, 8192)[0] == 16 and _plan(plan, 64, 8, G, W, 512)[0] == 16
        assert _plan(plan, 16, 8, G, W, 8192)[0] == 32
    assert _plan(plan, 1, 1, 97, 1, 64)[0] == _plan(plan, 16, 8, 8, 16, 8192)[0] == 32
    for G, W in [(1, 129), (4, 512), (7, 203)]:
        assert _plan(plan, 1, 8, G, W, 8192)[0] == 256


def test_few_cells_split_the_tokens(plan):
    assert _plan(plan, 1, 1, 4, 1, 131072)[1] == 256          # a block per compute unit
    assert _plan(plan, 1, 8, 4, 1, 4096)[1] == 16             # 256 tokens a block at least
    assert _plan(plan, 1, 8, 4, 1, 256)[1] == 1
    assert _plan(plan, 4, 4, 24, 24, 30000)[1] == 5           # 96 cells: 192 blocks would leave a quarter of them idle
    assert _plan(plan, 64, 8, 8, 1, 12288)[1] == 1
