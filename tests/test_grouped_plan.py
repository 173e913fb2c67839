"""The rules that cut grouped products into tiles and parts (csrc/grouped_plan.h), compiled as plain C++."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <cstdio>
#include "grouped_plan.h"
using namespace nomad_grouped;
int main() {
    const int64_t sizes[] = {1, 2, 7, 16, 17, 64, 65, 129, 256, 768, 2048, 4096};
    const int64_t rows[] = {0, 1, 48, 255, 256, 257, 1000, 20011, 524288, 10000019, 2147483392};
    const int64_t groups[] = {1, 2, 64, 256, 1024, 1048576};
    for (int64_t r : rows) for (int64_t g : groups) for (int64_t in : sizes) for (int64_t out : sizes) for (int small = 0; small < 2; ++small) {
        const GradientPlan p = plan_gradient(r, g, in, out, small, 256);
        if (p.most < 256 || p.tiles < 1) return 1;
        if ((p.slots > 0) != (r > p.most)) return 2;
        // every part of a long group begins in a slot of its own, and the slots are there: groups of every length, one after the other
        if (p.slots > 0 && (r - 1) / (p.most / 2) >= p.slots) return 3;
        if (!small && p.tile == kGradient256) return 4;
        const ProductTile t = plan_product(r, g, in, out, small, 256);
        if ((out <= 16) != (t == kProduct16) || (!small && t == kProduct256)) return 5;
    }
    // parts of a group of n rows, as the kernels cut them
    for (int64_t most : {256, 257, 1001, 4687})
        for (int64_t n : {most + 1, 2 * most, 2 * most + 1, 10 * most + 3, 1000 * most - 1}) {
            const int64_t parts = (n + most - 1) / most;
            int64_t before = -1;
            for (int64_t j = 0; j < parts; ++j) {
                const int64_t begin = 77 + n * j / parts, end = 77 + n * (j + 1) / parts, slot = begin / (most / 2);
                if (end - begin > most || end - begin < most / 2 || slot == before) return 6;
                before = slot;
            }
            if ((77 + n) / (most / 2) == before) return 7;    // the next group's first part
        }
    std::puts("ok");
    return 0;
}
"""


def test_plans(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-I" + os.path.join(ROOT, "paper_2505_15511_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0 and run.stdout == "ok\n", run.returncode
