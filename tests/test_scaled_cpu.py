"""Host side of the 8-bit block-scaled operators, without a GPU: structs as the C compiler lays them out, refusals before a device is
touched, the choice of route against measured times, and registers of the large kernels."""
import ctypes as C
import os
import subprocess

import pytest

from test_kernel_isa import CSRC
from test_streaming_isa import resources

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2511_13778_amd import ozdgemm as g
    if not os.path.exists(g.LIB_PATH):
        from paper_2511_13778_amd.build import build_library
        build_library(verbose=False)
    return g, g.load_library()


def test_struct_layout(lib, tmp_path):
    g, _ = lib
    fields = [f for f, _ in g.oz_scaled_t._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ozdgemm.h"\nint main(void) { printf("%zu", sizeof(oz_scaled_t));\n'
                   + "".join('printf(" %%zu", offsetof(oz_scaled_t, %s));\n' % f for f in fields)
                   + 'printf(" %d %d %d %d %d %d", OZ_F32, OZ_BF16, OZ_F16, OZ_E4M3, OZ_E5M2, OZ_E8M0); return 0; }\n')
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert out == [C.sizeof(g.oz_scaled_t)] + [getattr(g.oz_scaled_t, f).offset for f in fields] + [0, 1, 2, 3, 4, 5]
    assert (g.OZ_F32, g.OZ_BF16, g.OZ_F16, g.OZ_E4M3, g.OZ_E5M2, g.OZ_E8M0) == tuple(range(6))


def test_refusals_without_a_handle(lib):
    g, dll = lib
    m = g.oz_scaled_t()
    assert dll.oz_quantize(None, None, 1, 1, None, 1, 0, 1, 0, None, 1, 1, None, 0, C.byref(m), None) == 1
    assert dll.oz_scaled_gemm(None, None, 1, 1, 1, C.byref(m), C.byref(m), None, 1, 0, 0, None, 0) == 1
    assert dll.oz_scaled_gemm_grouped(None, None, 1, None, 1, 1, 1, C.byref(m), C.byref(m), None, 1, 0) == 1
    assert dll.oz_scaled_gemm_grouped_k(None, None, 1, None, 1, 1, 128, C.byref(m), C.byref(m), None, 1, 1, 0, 0) == 1
    assert dll.oz_sort_tokens(None, None, 1, 1, 1, None, 8, None, None, None, None, 0) == 1
    assert dll.oz_gather_rows(None, None, 1, 1, 1, 0, None, 1, None, None, None, 1) == 1
    assert dll.oz_combine_rows(None, None, 1, 1, 1, 0, None, 1, 1, None, None, None, 1) == 1
    assert dll.oz_combine_rows_grad(None, None, 1, 1, 1, 0, None, 1, None, 1, 1, None, None, None, None, 1, None) == 1
    assert dll.oz_scaled_gemm_workspace_bytes(None, 8, 8, 8) == 0 and dll.oz_sort_tokens_workspace_bytes(None, 8, 8, 8) == 0


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = tmp_path_factory.mktemp("plan") / "plan"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, os.path.join(ROOT, "tests", "host_scaled_plan.cpp"), "-o", str(exe)], check=True)

    def run(calls):
        args = [str(v) for c in calls for v in c]
        lines = subprocess.run([str(exe), *args], capture_output=True, text=True, check=True).stdout.splitlines()
        return [[float(v) for v in ln.split()] for ln in lines]
    return run


def measured():
    for line in open(os.path.join(ROOT, "tests", "golden", "scaled_times.txt")):
        if not line.startswith("#"):
            v = line.split()
            yield [int(x) for x in v[:4]], [None if x == "-" else float(x) for x in v[4:]]


def test_route_is_among_the_fastest_measured(plan):
    # the fit is good to about 10 %, so the chosen route may be that much slower than the best, and the mean much less
    rows = list(measured())
    plans = plan([(*size, 0, 0, 0) for size, _ in rows])
    lost = []
    for (size, times), p in zip(rows, plans):
        best = min(t for t in times if t is not None)
        route, parts = int(p[0]), int(p[1])
        if parts > 1:
            continue
        got = times[route - 1]
        assert got is not None and got <= 1.15 * best, (size, route, times)
        lost.append(got / best)
    assert sum(lost) / len(lost) < 1.04


def test_plans_at_the_ends(plan):
    few, t64, tall, big = 0, 1, 4, 5
    calls = {(0, 1, 4096, 4096, 0, 0, 0): (few, 1, 8), (0, 64, 100, 128, 0, 0, 0): (few, 1, 4), (0, 1, 16, 1 << 20, 0, 0, 0): (few, 16, 16),
             (0, 8192, 8192, 8192, 0, 0, 0): (big, 1, 0), (1, 8192, 8192, 8192, 0, 0, 0): (tall, 1, 0), (0, 96, 2048, 512, 32, 1, 0): (few, 1, 4),
             (0, 65, 1, 1, 0, 0, 0): (None, 1, 0), (0, 256, 256, 16384, 0, 0, 0): (t64, 16, 0)}
    for c, p in zip(calls, plan(list(calls))):
        want = calls[c]
        assert want[0] is None or int(p[0]) == want[0], (c, p)
        assert (int(p[1]), int(p[2])) == want[1:], (c, p)
    # the parts of k are a matter of sizes alone, whatever the types: the workspace is asked for without them
    sizes = [(300, 300, 8192), (1024, 1024, 8192), (100, 3000, 4096), (70, 9000, 1000), (128, 4096, 4096)]
    by_kind = [[p[1] for p in plan([(kind, *s, 0, 0, 0) for s in sizes])] for kind in range(4)]
    assert by_kind[0] == by_kind[1] == by_kind[2] == by_kind[3]


def test_large_kernels_keep_to_their_registers(tmp_path):
    # one wave per SIMD: 512 registers, none of them in memory
    for source in ("oz_scaled_gemm_big", "oz_scaled_gemm_big_f32"):
        for name, (registers, scratch) in resources(source, tmp_path).items():
            assert registers <= 512 and scratch == 0, (name, registers, scratch)
