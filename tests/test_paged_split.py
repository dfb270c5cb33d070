"""How attention over a paged cache is dealt out to workgroups (csrc/paged_units.h), on the CPU: every tile of every unit once, the parts of units each in a place of
their own within the scratch, joined from those places, and nothing outside of them for starts in no order."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2507_17245_amd", "csrc")

# What the header takes from the device's language.
COMMON = """#pragma once
#include <stdint.h>
#include <algorithm>
#include <cmath>
#define __device__
#define __global__
#define __shared__
#define __launch_bounds__(...)
struct Index { unsigned x; };
inline Index threadIdx, blockIdx;
int __builtin_amdgcn_readlane(int x, int lane);
uint64_t __builtin_amdgcn_ballot_w64(bool x);
int __builtin_amdgcn_update_dpp(int old, int x, int ctrl, int rows, int banks, bool zero);
float __builtin_amdgcn_exp2f(float x);
void __syncthreads();
namespace da {
using std::max;
using std::min;
constexpr int kComputeUnits = 256;
struct f32x4 {
  float v[4];
  float& operator[](int i) { return v[i]; }
  float operator[](int i) const { return v[i]; }
  f32x4& operator*=(float s) {
    for (float& x : v) x *= s;
    return *this;
  }
};
}  // namespace da
"""


@pytest.mark.skipif(os.uname().machine != "x86_64", reason="lanes are switched as on x86-64")
def test_units_are_dealt_out_once(tmp_path):
    shutil.copy(os.path.join(CSRC, "paged_units.h"), tmp_path)
    (tmp_path / "da_common.h").write_text(COMMON)
    (tmp_path / "paged.h").write_text("#pragma once\n#include \"distr_attn.h\"\n")
    exe = str(tmp_path / "paged_split_driver")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wno-attributes", "-U_FORTIFY_SOURCE", "-I", str(tmp_path), "-I", os.path.join(os.path.dirname(HERE), "include"),
                    os.path.join(HERE, "paged_split_driver.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr
