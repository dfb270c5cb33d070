"""How attention over a paged cache of 4-bit codes is dealt out to workgroups (csrc/paged4_split.h), on the CPU: every tile of every unit once in every form, a place
for four tiles of sequences with few rows in mixed batches, kv heads' lines apart, parts joined from where they were left."""
import os
import shutil
import subprocess

import pytest

from test_paged_split import COMMON, CSRC, HERE


@pytest.mark.skipif(os.uname().machine != "x86_64", reason="lanes are switched as on x86-64")
def test_units_are_dealt_out_once(tmp_path):
    for name in ("paged_units.h", "paged4_split.h"):
        shutil.copy(os.path.join(CSRC, name), tmp_path)
    (tmp_path / "da_common.h").write_text(COMMON.replace("inline Index threadIdx, blockIdx;", "inline Index threadIdx, blockIdx, gridDim;"))
    (tmp_path / "paged.h").write_text("#pragma once\n#include \"distr_attn.h\"\n")
    exe = str(tmp_path / "paged4_split_driver")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wno-attributes", "-Wno-unused-function", "-U_FORTIFY_SOURCE", "-I", str(tmp_path), "-I",
                    os.path.join(os.path.dirname(HERE), "include"), "-I", HERE, os.path.join(HERE, "paged4_split_driver.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr
