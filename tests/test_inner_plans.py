"""Host code of the inner step's operators against stand-ins for the HIP runtime and the kernel launchers."""
import os
import subprocess

import pytest

import paper_2506_10911_amd as nl
import test_gpu_muon_general as general
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


def planned(driver, matrices, W, products):
    """({(rows, cols): (tile, how many, parts of X X^T)}, launches of two steps) of a plan; tile 0: in one workgroup."""
    text = f"{W} {products} {len(matrices)}\n" + "\n".join(" ".join(map(str, m[:4])) for m in matrices)
    shapes, launches = {}, 0
    for line in driver("plan", text=text).splitlines():
        words = line.split()
        if words[0] == "launches":
            launches = int(words[1])
        elif len(words) == 5:
            tile, rows, cols, count, parts = map(int, words)
            before = shapes.get((rows, cols), (tile, 0, parts))
            assert before[0] == tile and before[2] == parts
            shapes[rows, cols] = (tile, before[1] + count, parts)
    return shapes, launches


@pytest.mark.parametrize("products", [nl.PRODUCTS_F16, nl.PRODUCTS_PAIRS])
@pytest.mark.parametrize("path", sorted(general.PATHS))
def test_gpu_tests_of_the_general_path_reach_its_tiles(driver, path, products):
    """A rule that moves a threshold may not leave a kernel without its test."""
    matrices, _, W, tile, shared = general.path(path)
    shapes, _ = planned(driver, matrices, W, products)
    assert {s[0] for s in shapes.values()} == {tile}
    assert any(s[2] > 1 for s in shapes.values()) == shared
