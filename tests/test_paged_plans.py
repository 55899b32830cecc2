"""Workspaces of the attention over pages (no GPU): one for a program's largest step serves every smaller one."""
from __future__ import annotations

import itertools
import os
import subprocess

import pytest

import paper_2505_06901_amd as E

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(not os.path.exists("/opt/rocm/llvm/bin/clang++"), reason="needs ROCm's clang++")
def test_plans_fit_workspaces(tmp_path):
    """tests/plans/paged_plans_main.cpp, with undefined arithmetic trapped."""
    exe = str(tmp_path / "paged_plans")
    cmd = ["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-O2", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I" + os.path.join(ROOT, "include"),
           "-I" + os.path.join(ROOT, "paper_2505_06901_amd", "csrc"), os.path.join(ROOT, "tests", "plans", "paged_plans_main.cpp"), "-o", exe]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "conditions hold" in run.stdout, (run.stdout[-2000:], run.stderr[-2000:])


def test_workspaces_grow_with_the_sizes():
    """Every pair of neighbouring sizes, each of them by itself: no slack."""
    grid = dict(n_tokens=(1, 8, 31, 32, 95, 256, 512, 1024, 4096), B=(1, 8, 31, 32, 64, 300), max_new=(1, 2, 5, 9, 64, 512, 1024, 4096), max_kv=(1, 256, 257, 4096, 16384, 32768),
                total_kv=(1, 4096, 1 << 20))
    for Hq, Hkv in ((32, 8), (32, 32), (16, 1)):
        size = {}
        for key in itertools.product(*(range(len(v)) for v in grid.values())):
            n, B, max_new, max_kv, total = (v[i] for v, i in zip(grid.values(), key))
            size[key] = E.ecco_kv_attend_paged_workspace(n, B, Hq, Hkv, max_new, max_kv, total, device=-1)
        for key, s in size.items():
            for d in range(len(key)):
                less = key[:d] + (key[d] - 1,) + key[d + 1:]
                assert key[d] == 0 or size[less] <= s, (Hq, Hkv, less, key, size[less], s)


def test_workspace_sizes_by_hand():
    """256 compute units: ranges of 520 bytes per row, two for each unit and one per sequence and head; 16 KB per head and unit of 32 tokens; up to 256
    tiles of 128 rows in ranges."""
    size = lambda *a: E.ecco_kv_attend_paged_workspace(*a, device=-1)  # noqa: E731
    ranges = lambda B, rows: 256 * -(-B * 8 // 256) + (B * 8 + 512) * rows * 520  # noqa: E731
    assert size(31, 31, 32, 8, 1, 4096, 31 * 4096) == size(500, 500, 32, 8, 1, 4096, 500 * 4096) == ranges(31, 8)
    assert size(8, 8, 32, 8, 1, 256, 2048) == 0  # not cut
    # a chunk of 64 tokens alone: 129 units, their bits; beside ranges for up to 32 rows, and its two tiles and eight heads in eight splits
    assert size(64, 1, 32, 8, 64, 4096, 4096) == ranges(1, 32) + 512 + 768 + 129 * 8 * 16384 + 2 * 8 * 8 * 128 * 520
