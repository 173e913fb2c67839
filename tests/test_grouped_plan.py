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
        // every row's slot is there, and a slot has no more rows than half of the longest part
        if (p.slots > 0 && (r - 1) >> p.slot_bits >= p.slots) return 3;
        if ((int64_t)1 << p.slot_bits > p.most / 2) return 8;
        if (!small && p.tile == kGradient256) return 4;
        for (int w_kc = 0; w_kc < 2; ++w_kc) {
            const ProductTile t = plan_product(r, g, out, small, w_kc, 256);
            if ((!small && t == kProduct256) || (!w_kc && t == kProductFew)) return 5;
            if (out <= 16 && t != kProduct16 && t != kProductFew) return 9;
        }
    }
    // parts of a group of n rows, as the kernels cut them: each in a slot of its own, and so is the next group's first
    for (int64_t most : {256, 257, 1001, 4687})
        for (int64_t n : {most + 1, 2 * most, 2 * most + 1, 10 * most + 3, 1000 * most - 1}) {
            const int64_t parts = (n + most - 1) / most, each = n / parts, left = n % parts;
            int bits = 0;
            while ((int64_t)2 << bits <= most / 2) ++bits;
            int64_t before = -1;
            for (int64_t j = 0; j < parts; ++j) {
                const int64_t begin = 77 + j * each + (j < left ? j : left), end = 77 + (j + 1) * each + (j + 1 < left ? j + 1 : left), slot = begin >> bits;
                if (end - begin > most || end - begin < most / 2 || slot == before || (j + 1 == parts && end != 77 + n)) return 6;
                before = slot;
            }
            if ((77 + n) >> bits == before) return 7;
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


LAYOUT = r"""
#include <stdio.h>
#include <stddef.h>
#include "nomad.h"
int main(void) {
    printf("%zu %zu %zu %zu\n", sizeof(nomad_grouped_product_args), sizeof(nomad_grouped_gradient_args), sizeof(nomad_adamw_tensor), sizeof(nomad_adamw_options));
    printf("%zu %zu %zu %zu\n", offsetof(nomad_grouped_product_args, rows), offsetof(nomad_grouped_product_args, w), offsetof(nomad_grouped_product_args, z_stride),
           offsetof(nomad_grouped_product_args, device));
    printf("%zu %zu %zu %zu\n", offsetof(nomad_grouped_gradient_args, rows), offsetof(nomad_grouped_gradient_args, dy), offsetof(nomad_grouped_gradient_args, workspace_bytes),
           offsetof(nomad_grouped_gradient_args, device));
    printf("%zu %zu %zu %zu\n", offsetof(nomad_adamw_tensor, n), offsetof(nomad_adamw_tensor, g_dtype), offsetof(nomad_adamw_options, lr), offsetof(nomad_adamw_options, device));
    return 0;
}
"""


def test_argument_layouts(tmp_path):
    """What the binding packs is what the header declares."""
    import struct

    from paper_2505_15511_amd import binding as b
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text(LAYOUT)
    subprocess.run(["gcc", "-std=c99", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    said = [[int(v) for v in line.split()] for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()]
    assert said[0] == [b.GROUPED_PRODUCT_ARGS.size, b.GROUPED_GRADIENT_ARGS.size, b.ADAMW_TENSOR.size, b.ADAMW_OPTIONS.size]

    def at(fmt, part):                                         # offset of the field behind the first `part` of a format
        return struct.calcsize("@" + part + "0" + fmt)
    assert said[1] == [at("q", "I7i"), at("P", "I7i2q3Pq"), at("q", "I7i2q3PqP3qPqPqPqP"), at("i", "I7i2q3PqP3qPqPqPqPqP")]
    assert said[2] == [at("q", "I6i4x"), at("P", "I6i4x2q2P"), at("q", "I6i4x2q2PPqPqPPP"), at("i", "I6i4x2q2PPqPqPPPqP")]
    assert said[3] == [at("q", "6P"), at("i", "6Pqi"), at("d", "Iiq"), at("i", "Iiq5dPP")]
