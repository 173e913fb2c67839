"""The current device across a call (csrc/device_scope.h), compiled against a runtime of three devices that only keeps count."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_15511_amd", "csrc")

RUNTIME = r"""
#pragma once
typedef int hipError_t;
enum { hipSuccess = 0, hipErrorInvalidDevice = 101 };
static int current = 0, sets = 0, refuse = -1;
static inline hipError_t hipGetDeviceCount(int* n) { *n = 3; return hipSuccess; }
static inline hipError_t hipGetDevice(int* d) { *d = current; return hipSuccess; }
static inline hipError_t hipSetDevice(int d) { ++sets; if (d == refuse) return hipErrorInvalidDevice; current = d; return hipSuccess; }
"""

SOURCE = r"""
#include <initializer_list>
#include "device_scope.h"
int main() {
    { DeviceScope on(0); if (!on.ok() || current != 0) return 1; }
    if (current != 0 || sets != 0) return 2;                 // nothing to change: no calls
    { DeviceScope on(2); if (!on.ok() || current != 2) return 3; { DeviceScope inner(1); if (current != 1) return 4; } if (current != 2) return 5; }
    if (current != 0) return 6;
    current = 1;
    for (int bad : {-1, 3, 100}) { DeviceScope on(bad); if (on.ok() || current != 1) return 7; }
    refuse = 2;
    { DeviceScope on(2); if (on.ok() || current != 1) return 8; }
    return current == 1 ? 0 : 9;
}
"""


def test_the_current_device_comes_back(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no C++ compiler")
    os.makedirs(tmp_path / "hip")
    (tmp_path / "hip" / "hip_runtime.h").write_text(RUNTIME)
    (tmp_path / "scope.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-I" + str(tmp_path), "-I" + CSRC, str(tmp_path / "scope.cpp"), "-o", str(tmp_path / "scope")], check=True)
    assert subprocess.run([str(tmp_path / "scope")]).returncode == 0


@pytest.mark.parametrize("source", ["route.hip", "grouped.hip", "adamw.hip"])
def test_the_operators_of_a_learned_map_set_no_device_by_themselves(source):
    text = open(os.path.join(CSRC, source)).read()
    entries = len(re.findall(r'^extern "C" int nomad_', text, flags=re.M))
    assert "hipSetDevice" not in text and entries > 0 and len(re.findall(r"const DeviceScope on\(", text)) == entries
