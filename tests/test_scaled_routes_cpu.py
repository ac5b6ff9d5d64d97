"""The sizes that the 8-bit products are tested with reach the kernels that they are meant for; on the host, with the library's own choice of routes."""
import os
import subprocess

import pytest

import scaled_routes as sr
from test_kernel_isa import CSRC

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = tmp_path_factory.mktemp("plan") / "plan"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, os.path.join(ROOT, "tests", "host_scaled_plan.cpp"), "-o", str(exe)], check=True)

    def run(kind, m, n, k, groups=0, by_rows=0, by_k=0):
        out = subprocess.run([str(exe), *map(str, (kind, m, n, k, groups, by_rows, by_k))], capture_output=True, text=True, check=True).stdout.split()
        return int(out[0]), int(out[1])
    return run


def check(label, kind, route, parts, size):
    want = sr.ROUTE[label]
    if kind not in sr.HAS.get(want, sr.KINDS):
        return
    assert route == want and (parts > 1) == ("cut" in label), (label, kind, size, route, parts)


def test_dense_sizes(plan):
    assert set(sr.DENSE) == set(sr.ROUTE)
    for label, sizes in sr.DENSE.items():
        for m, n, k in sizes:
            for kind in sr.KINDS:
                check(label, kind, *plan(kind, m, n, k), (m, n, k))
    for label, most in (("few rows, 16", 16), ("few rows, 32", 32), ("few rows, 64", 64)):
        assert all(most // 2 < m <= most or most == 16 for m, _, _ in sr.DENSE[label]) and max(m for m, _, _ in sr.DENSE[label]) == most
    assert [sorted((m > 16) + (m > 32) for m, _, _ in sr.DENSE["few rows, cut"])] == [[0, 1, 2]]       # each instance


def test_sizes_in_groups(plan):
    for label, sizes in sr.ROWS.items():
        for counts, behind, n, k in sizes:
            rows = sum(counts) + behind
            for kind in sr.KINDS:
                check(label, kind, *plan(kind, rows, n, k, len(counts), 1, 0), (counts, n, k))
            if label.startswith("few"):
                most = int(label.split()[-1])
                assert most // 2 < -(-rows // len(counts)) <= most, (label, rows, len(counts))
                assert max(counts) > 4 * most                    # a load that the average does not show
    for label, sizes in sr.CONTRACTION.items():
        for counts, behind, m, n in sizes:
            for kind in sr.KINDS:
                check(label, kind, *plan(kind, m, n, sr.columns(counts, behind), len(counts), 0, 1), (counts, m, n))
    # all routes that groups can take; the few rows' and the cut ones are not among the contraction's
    assert set(sr.ROWS) == set(sr.ROUTE) - {"few rows, cut", "64 x 64, cut"}
    assert set(sr.CONTRACTION) == {x for x in sr.ROWS if not x.startswith("few")}


def test_large_tiles_see_odd_and_even_steps_and_ragged_ends():
    for label in ("256 x 128", "256 x 256"):
        blocks = [(-(-k // 128) % 2, k % 128 == 0) for _, _, k in sr.DENSE[label]]
        assert {b for b, _ in blocks} == {0, 1} and {w for _, w in blocks} == {True, False}, label
        steps = {-(-c // 128) for counts, *_ in sr.CONTRACTION[label] for c in counts}
        assert {0, 1} <= steps and any(s > 2 and s % 2 for s in steps)


def test_registers_leave_room_for_the_workgroups_that_a_cu_holds(tmp_path):
    # a SIMD has 512: two workgroups of 128 x 128 tiles, four of 64 x 64 in two stages, sixteen waves of one few-row workgroup; nothing in memory
    from test_streaming_isa import resources
    most = {"scaled_gemm_kernelILi128E": 256, "scaled_gemm_kernelILi64ELi64ELi32ELi32ELi2E": 128, "scaled_gemm_kernelILi64ELi64ELi32ELi32ELi4E": 256,
            "scaled_gemm_few_kernelILi1E": 128, "scaled_gemm_few_kernelILi2E": 256, "scaled_gemm_few_kernelILi4E": 256}
    seen = set()
    for source in ("oz_scaled_gemm", "oz_scaled_gemm_few"):
        for name, (registers, scratch) in resources(source, tmp_path).items():
            for part, limit in most.items():
                if part in name:
                    seen.add(part)
                    assert registers <= limit and scratch == 0, (name, registers, scratch)
    assert seen == set(most)
