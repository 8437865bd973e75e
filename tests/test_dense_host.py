"""The dense operators' host side (sizes of the scratch, arguments of the
launches, errors) without a GPU: tests/native/host_driver.cpp, linked with the
built library, stands in for the HIP runtime."""
import os
import subprocess

import pytest

from paper_2108_03917_amd.lattice import LIB_PATH

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("native") / "host_driver")
    libdir = os.path.dirname(LIB_PATH)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
                    "-I", os.path.join(ROOT, "include"), os.path.join(HERE, "native", "host_driver.cpp"),
                    LIB_PATH, "-rdynamic", f"-Wl,-rpath,{libdir}", "-Wl,--allow-shlib-undefined", "-o", exe],
                   check=True, timeout=120)
    return exe


def run(driver, check):
    r = subprocess.run([driver, check], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.returncode, r.stdout, r.stderr)


def test_bias_gradient_of_many_pieces_of_rows(driver):
    """More pieces than one sum takes: no level of it reads outside the scratch."""
    run(driver, "many_pieces")


def test_scratch_of_a_captured_call_is_kept(driver):
    """A larger call frees the scratch only if no graph may use it, and leaves a
    capture that it falls into whole."""
    run(driver, "captured_scratch")


def test_work_is_on_the_handles_device(driver):
    """Allocations, launches and waits, with another device current, which is
    current again after each call."""
    run(driver, "another_current_device")


def test_layer_norm_backward_without_rows(driver):
    """Short and long rows, any of the outputs, or none that has an address."""
    run(driver, "no_rows")


def test_gradient_bits_of_no_handle():
    from paper_2108_03917_amd import lattice as B

    assert B.load_library().lattice_dense_set_gradient_bits(None, 8) == B.E_ARG


def test_work_is_in_the_order_of_the_handles_stream(driver):
    """From the clearing of its status word on: its stream need not wait for the
    null stream."""
    run(driver, "the_handles_stream")


def test_products_read_inside_their_operands(driver):
    """Operands of every product of 3000 losses and updates of random sizes lie
    inside the callers' buffers or the scratch, padding and planes included."""
    run(driver, "products_stay_inside")
