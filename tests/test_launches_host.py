"""The launches of the dense operators' largest calls, without a GPU:
tests/native/launch_driver.cpp, linked with the built library, stands in for the HIP
runtime."""
import os
import subprocess

import pytest

from paper_2108_03917_amd.lattice import LIB_PATH

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("native") / "launch_driver")
    libdir = os.path.dirname(LIB_PATH)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
                    "-I", os.path.join(ROOT, "include"), os.path.join(HERE, "native", "launch_driver.cpp"),
                    LIB_PATH, "-rdynamic", f"-Wl,-rpath,{libdir}", "-Wl,--allow-shlib-undefined", "-o", exe],
                   check=True, timeout=120)
    return exe


@pytest.mark.parametrize("check", ["rotations", "attention", "clipping", "normalisation"])
def test_threads_along_a_side_have_32_bits(driver, check):
    r = subprocess.run([driver, check], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.returncode, r.stdout, r.stderr)
