"""The orthogonalisation's tables against a stand-in for the HIP runtime (ortho_check.cpp), without a GPU."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.join(os.path.dirname(HERE), "paper_1905_05957_amd")


def test_tiles_operands_and_parts_lie_where_they_belong(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    binary = str(tmp_path / "ortho_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", os.path.join(HERE, "ortho_check.cpp"), "-o", binary,
                    "-rdynamic", "-L" + PKG, "-lds_hip", "-Wl,--unresolved-symbols=ignore-in-shared-libs",
                    f"-Wl,-rpath,{PKG}:{rocm}/lib"], check=True)
    r = subprocess.run([binary], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "FAILED" not in r.stdout, r.stdout + r.stderr
