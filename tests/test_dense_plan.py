"""The rules that cut dense products into tiles and parts (csrc/dense_plan.h), compiled as plain C++, and that the GPU tests' sizes reach
every tile, with whole sums and cut ones."""
import os
import shutil
import subprocess

import pytest
import torch

import test_gpu_more_operators as operators

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <cstdio>
#include <cstring>
#include "dense_plan.h"
using namespace nomad_dense;
int main(int argc, char**) {
    if (argc > 1) {   // rows columns k small few whole -> tile parts
        long long rows, columns, k;
        int small, few, whole;
        while (std::scanf("%lld %lld %lld %d %d %d", &rows, &columns, &k, &small, &few, &whole) == 6) {
            const Plan p = plan(rows, columns, k, small, few, whole, 256);
            std::printf("%d %d\n", (int)p.tile, (int)p.parts);
        }
        return 0;
    }
    const int64_t sizes[] = {1, 2, 7, 16, 17, 64, 65, 129, 256, 768, 2048, 4096, 8192, 1048576};
    const int64_t rows[] = {1, 16, 48, 64, 65, 257, 1000, 20011, 524288, 10000019, 2147483392};
    for (int64_t r : rows) for (int64_t c : sizes) for (int64_t k : sizes) for (int way = 0; way < 8; ++way) {
        for (int turn = 0; turn < 2; ++turn) {   // a long sum over rows too
            const int64_t n = turn ? c : r, m = turn ? k : c, sum = turn ? r : k;
            const Plan p = plan(n, m, sum, way & 1, way & 2, way & 4, 256);
            const int64_t stage = way & 1 ? 64 : 32;
            // the parts hold the whole sum, each of them something of it, in whole stages
            if (p.parts < 1 || p.parts > kMostParts || p.length % stage || p.parts * p.length < sum || (p.parts - 1) * p.length >= sum) return 1;
            if (p.tile == kFew && (n > kFewRows || !(way & 2))) return 2;
            if (p.tile == k256 && !((way & 1) && (way & 4))) return 3;
            if (p.parts > 1 && p.units > 2 * 256) return 4;
        }
        const SlopePlan s = plan_slope(r, c, 256);
        if (s.parts < 1 || s.parts > 512 || s.parts * s.length < r || (s.parts - 1) * s.length >= r) return 5;
    }
    const Plan none = plan(40, 24, 0, 1, 0, 1, 256);   // no rows: the weights' gradient is zeros, of one part
    if (none.parts != 1) return 6;
    std::puts("ok");
    return 0;
}
"""


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no C++ compiler")
    folder = tmp_path_factory.mktemp("plan")
    src, exe = folder / "plan.cpp", folder / "plan"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-I" + os.path.join(ROOT, "paper_2505_15511_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    return str(exe)


def test_plans(planner):
    run = subprocess.run([planner], capture_output=True, text=True)
    assert run.returncode == 0 and run.stdout == "ok\n", run.returncode


def test_sizes_of_the_gpu_tests_reach_every_tile(planner):
    asked = []
    for rows, inner, out, dtype in operators.DENSE:
        chunk, small = (4, 0) if dtype == torch.float32 else (8, 1)
        if rows:
            asked += [(rows, out, inner, small, few, int(inner % chunk == 0 and out % chunk == 0)) for few in (0, 1)]
    for rows, inner, out, dtype in operators.BACK:
        chunk, small = (4, 0) if dtype == torch.float32 else (8, 1)
        whole = int(inner % chunk == 0 and out % chunk == 0)
        if rows:
            asked += [(rows, inner, out, small, 0, whole), (out, inner, rows, small, 0, whole)]
    run = subprocess.run([planner, "sizes"], input="\n".join(" ".join(map(str, a)) for a in asked), capture_output=True, text=True, check=True)
    seen = {(int(tile), int(parts) > 1) for tile, parts in (line.split() for line in run.stdout.splitlines())}
    assert {tile for tile, _ in seen} == set(range(5))
    assert {(tile, cut) for tile in (1, 2, 3, 4) for cut in (False, True)} <= seen, seen
