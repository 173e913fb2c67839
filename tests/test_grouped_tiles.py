"""The sizes of the GPU tests reach every tile of the grouped products and their gradients, in every way in which their rows are loaded
and stored (csrc/grouped_plan.h and csrc/grouped_launch.h; no GPU needed)."""
import os
import shutil
import subprocess

import pytest
import torch

import test_gpu_map_operators as operators
import test_gpu_grouped_instances as instances

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include "grouped_plan.h"
using namespace nomad_grouped;
int main() {
    long long rows, groups, in, out;
    int small;
    while (std::scanf("%lld %lld %lld %lld %d", &rows, &groups, &in, &out, &small) == 5) {
        const GradientPlan p = plan_gradient(rows, groups, in, out, small, 256);
        std::printf("%d %d %d %d %d\n", (int)plan_product(rows, groups, out, small, true, 256), (int)plan_product(rows, groups, out, small, false, 256), (int)p.tile, (int)p.most, p.slots > 0);
    }
    return 0;
}
"""


def test_every_instance_is_reached(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no C++ compiler")
    (tmp_path / "plan.cpp").write_text(SOURCE)
    exe = str(tmp_path / "plan")
    subprocess.run(["g++", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2505_15511_amd", "csrc"), str(tmp_path / "plan.cpp"), "-o", exe], check=True)
    cases = operators.PRODUCTS + instances.NARROW + instances.WIDE
    asked = "".join(f"{total + (37 if total else 0)} {groups} {inner} {out} {int(dtype != torch.float32)}\n" for groups, total, inner, out, dtype, _ in cases)
    said = [[int(v) for v in line.split()] for line in subprocess.run([exe], input=asked, capture_output=True, text=True, check=True).stdout.splitlines()]
    assert len(said) == len(cases)
    products, gradients, parts = set(), set(), set()
    for (groups, total, inner, out, dtype, kind), (straight, turned, tile, most, slots) in zip(cases, said):
        chunk = 4 if dtype == torch.float32 else 8
        whole_in, whole_out = inner % chunk == 0, out % chunk == 0                # rows of whole 16-byte chunks, contiguous tensors
        for turn, which in ((False, straight), (True, turned)):
            loads, stores = whole_in and (not turn or whole_out), whole_out
            if which == 0 and not (loads and stores):                            # (256 x 256 is for whole chunks alone)
                which = 1
            products.add((which, loads and stores, stores) if which != 4 else (4,))
        if tile == 0 and not (whole_in and whole_out):
            tile = 1
        gradients.add((tile, dtype == torch.float32, whole_in and whole_out, whole_in))
        if slots and kind == "one" and total > most:
            parts.add((tile, inner * out < 16384))
    assert {p[0] for p in products} == {0, 1, 2, 3, 4}
    ends = ((True, True), (False, True), (False, False))
    missing = {(which, *end) for which in (1, 2, 3) for end in ends} - products
    assert not missing, missing
    assert (0, False, True, True) in gradients
    missing = {(tile, single, *end) for tile in (1, 2, 3) for single in (False, True) for end in ends} - gradients   # 128, 64 and 128 x 16, in 32 and in 16 bits
    assert not missing, missing
    assert parts >= {(3, True)}, parts
