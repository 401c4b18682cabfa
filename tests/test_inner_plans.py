"""Host code of the inner step's operators against stand-ins for the HIP runtime and the kernel launchers."""
import os
import subprocess

import pytest

from conftest import ROOT


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    """Builds the driver; returns a call that runs one of its checks and returns what it printed."""
    csrc = os.path.join(ROOT, "paper_2506_10911_amd", "csrc")
    exe = tmp_path_factory.mktemp("plans") / "inner_plan_driver"
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    "-I", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
                    os.path.join(ROOT, "tests", "inner_plan_driver.cpp"), os.path.join(csrc, "inner_step.cpp"), "-o", str(exe)], check=True)

    def run(*args, text=""):
        done = subprocess.run([str(exe), *map(str, args)], input=text, capture_output=True, text=True, timeout=120)
        assert done.returncode == 0, done.stdout + done.stderr
        return done.stdout
    return run


def test_calls_on_another_device_are_refused(driver):
    driver("devices")


def test_lookup_of_any_number_of_tokens_is_a_grid_that_hip_takes(driver):
    driver("lookup_grid")


def test_arrays_of_nothing_overlap_nothing(driver):
    driver("empty_arrays")
