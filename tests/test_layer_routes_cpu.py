"""The sizes that products with 4-bit weights and orthogonal updates are tested with reach each way of cutting them up; on the host, with the library's own rule."""
import math
import os
import subprocess

import pytest

import layer_routes as lr
from test_kernel_isa import CSRC

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = tmp_path_factory.mktemp("plan") / "plan"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, os.path.join(ROOT, "tests", "host_layer_plan.cpp"), "-o", str(exe)], check=True)
    return lambda *a: tuple(map(int, subprocess.run([str(exe), *map(str, a)], capture_output=True, text=True, check=True).stdout.split()))


def test_packed_products(plan):
    for route, sizes in lr.PACKED.items():
        for counts, behind, n, k, group, kinds in sizes:
            for size in kinds:
                got = plan("packed", sum(counts) + behind, n, k, len(counts), size, int(math.log2(group)))
                assert got[:3] == route, (route, counts, behind, n, k, group, size, got)


def test_packed_plans_hold_everywhere(plan):
    # what the kernels are built for: strips only as far as registers reach, a power of two of waves, no more than k has blocks for
    for m in (1, 16, 17, 64, 1000, 100000):
        for n in (1, 1000, 70000):
            for k in (8, 200, 5000):
                for groups in (0, 1, 60):
                    for size in (2, 4):
                        for shift in (5, 6, 7):
                            staged, rows, strips, waves = plan("packed", m, n, k, groups, size, shift)
                            assert waves in (1, 2, 4, 8, 16) and waves < 2 * max(1, -(-k // 128))
                            if staged:
                                assert (rows, strips) in ((1, 2), (2, 2), (2, 4) if shift == 7 else (2, 2), (1, 1) if size == 2 else (1, 2)) and waves <= 8
                            else:
                                assert rows == 1 and strips in (1, 2, 4 if shift > 5 else 2) and waves <= (16 if strips == 1 or strips * size <= 4 else 8)


def test_tiles_of_orthogonal_updates(plan):
    for parts, sizes in lr.ORTHO.items():
        for want, (batch, m, n) in sizes.items():
            got = plan("ortho", batch, m, n, parts)
            assert all(w in (g, None) for w, g in zip(want, got)), (parts, want, got)
        for at in (0, 1):
            assert {want[at] for want in sizes} >= {64, 128, 192, 256}, (parts, at)
