"""The sizes of kvp_rotary (csrc/rotary_plan.h): a C++ program walks them over the limits of the header, and what lies behind them is refused
before any launch."""
import os
import subprocess

import pytest

from test_cache_abi import SHAPE, rotary, view

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_size_within_the_limits_fits_its_launch(tmp_path):
    exe = str(tmp_path / "rotary_plan")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2512_14946_amd", "csrc"), "-o", exe,
                    os.path.join(ROOT, "tests", "rotary_plan.cpp")], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
    assert int(out.stdout) > 1_000_000


@pytest.mark.parametrize("T,H,strides,rd", [((1 << 30) - 63, 1, (0, 1, 0), 128), ((1 << 31) - 127, 1, (0, 1, 1), 128), ((1 << 30) - 63, 1, (0, 1, 1), 34),
                                            ((1 << 30) - 63, 1, (0, 1, 0), 34), (1 << 28, 8, (0, 1, 0), 64)])
def test_launches_that_no_grid_takes_are_refused(T, H, strides, rd):
    assert rotary(x=view(L=1, T=T, H=H), strides=strides, rd=rd) == SHAPE
