"""What kvp_cache_attend accepts and refuses by size: its launches (csrc/cache_attend_plan.h) walked over the limits of the header, and shapes on
either side through the C ABI (whose pointers are never followed: what is accepted ends at the missing workspace)."""
import os
import subprocess

import pytest

import paper_2512_14946_amd as kvp
from test_cache_abi import SHAPE, WORKSPACE, attend, cache, evict, view

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def limits(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cache_limits") / "cache_limits")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2512_14946_amd", "csrc"), "-o", exe,
                    os.path.join(ROOT, "tests", "cache_limits.cpp")], check=True)
    return exe


def test_every_size_within_the_limits_fits_its_launches(limits):
    out = subprocess.run([limits], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
    assert int(out.stdout) > 100_000


@pytest.mark.parametrize("B,W,T", [(8, 32768, 32768), (32, 8192, 8192), (2, 131072, 131072), (16, 16384, 16384)])
def test_large_prompts_take_one_launch(limits, B, W, T):
    H, G = 8, 8
    n = list(map(int, subprocess.run([limits, *map(str, (B, H, G, W, T, 0))], check=True, capture_output=True, text=True).stdout.split()))
    assert n == [B * H * -(-W * G // 256), 0, 0, 0, 1]
    assert kvp.kvp_cache_attend_workspace_bytes(B, H, G * H, W, T, False) == 0


def _sized(B, H, G, W, T, **kw):
    c = cache(B=B, H=H, bs=16, max_blocks=-(-T // 16), table_stride=-(-T // 16), num_blocks=1)
    q = view(L=B, T=W, H=G * H)
    return attend(q=q, out=view(L=B, T=W, H=G * H, ptr=1 << 50), c=c, acc_out=4096, stride=T + 16, ws=None, **kw)


@pytest.mark.parametrize("B,H,G,W,T,code", [(8, 8, 8, 32768, 32768, WORKSPACE), (1, 8, 16, 131072, 131072, WORKSPACE), (16, 8, 8, 16384, 16384, WORKSPACE),
                                            (1 << 20, 7, 1, 200, 128, WORKSPACE), (1 << 20, 8, 1, 200, 128, SHAPE), ((1 << 20) - 1, 8, 1, 200, 128, WORKSPACE),
                                            (1 << 19, 15, 1, 16, 16, WORKSPACE), (1 << 19, 16, 1, 16, 16, SHAPE), (1 << 19, 8, 1, 17, 16, SHAPE),
                                            (1 << 13, 8, 1, 130, 32768 - 128, WORKSPACE), (1 << 13, 8, 1, 130, 32768, SHAPE)])
def test_shapes_on_either_side_of_the_limits(B, H, G, W, T, code):
    assert _sized(B, H, G, W, T) == code


@pytest.mark.parametrize("B,H,code", [((1 << 23) - 1, 1, WORKSPACE), (1 << 21, 4, SHAPE)])
def test_evict_refuses_more_rows_than_its_selection_takes(B, H, code):
    # nothing may be enqueued: the pages would move by a list that no selection wrote
    c = dict(B=B, H=H, max_blocks=1, table_stride=1, num_blocks=1)
    assert evict(src=cache(**c), dst=cache(block_table=1 << 21, **c), budget=8, stride=16, ws=None) == code


def test_selection_refuses_more_rows_than_a_grid_takes():
    call = kvp.kvp._lib.kvp_select_topk
    assert call(4096, 1 << 23, 16, 16, 4, 8192, None, 0, None) == SHAPE
    need = kvp.kvp_select_workspace_bytes(1 << 22, 16400, 4)
    assert call(4096, 1 << 22, 16400, 16400, 4, 8192, 4096, need, None) == SHAPE
    assert call(4096, (1 << 22) - 1, 16400, 16400, 4, 8192, None, 0, None) == WORKSPACE


@pytest.mark.parametrize("rows,budget", [(1, 16), (3, 100000), (64, 4096)])
def test_an_eviction_workspace_serves_every_smaller_bound(rows, budget):
    # rows of 2^14 + 1 to 2^18 weights need scratch for their selection, longer ones none
    before = 0
    for T in [1, 100, 16384, 16385, 20000, 250000, (1 << 18) - 1, 1 << 18, (1 << 18) + 1, 270000, 278000, 290000, 1 << 20]:
        need = kvp.kvp_cache_evict_workspace_bytes(rows, 1, T, budget)
        assert need >= before, T
        before = need


def test_sizes_behind_the_limits_have_no_workspace():
    m = (1 << 31) - 1
    assert kvp.kvp_cache_attend_workspace_bytes(m, 1, 1, 1, m, True) == 0            # logits of 2^62 tokens: a product that wraps
    assert kvp.kvp_cache_attend_workspace_bytes(1 << 19, 16, 16, 16, 16, True) == 0 < kvp.kvp_cache_attend_workspace_bytes(1 << 19, 15, 15, 16, 16, True)
    assert kvp.kvp_cache_evict_workspace_bytes(1 << 21, 4, 16, 8) == 0 < kvp.kvp_cache_evict_workspace_bytes(1 << 21, 3, 16, 8)
    assert kvp.kvp_cache_evict_workspace_bytes(1 << 13, 1 << 9, 1 << 20, 8) == 0
