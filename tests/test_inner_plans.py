"""Host code of the inner step's operators against stand-ins for the HIP runtime and the kernel launchers."""
import os
import re
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


def side_by_side(*shapes):
    """(offset, rows, cols, row_stride) of `count` matrices of each shape (count, rows, cols), one after the other."""
    found, at = [], 0
    for count, rows, cols in shapes:
        for _ in range(count):
            found.append((at, rows, cols, cols))
            at += rows * cols
    return found


@pytest.mark.parametrize("products", [nl.PRODUCTS_F16, nl.PRODUCTS_PAIRS])
def test_small_matrices_go_along_in_launches_of_their_tile_only(driver, products):
    """Two steps: sums, start and six products of the large ones. Small ones beside tiles of 64 or 128 go along, beside tiles of 256
    alone, where they would need eight launches of their own, they take one."""
    for large, tile in (((2, 260, 516), 64), ((14, 768, 768), 128)):
        shapes, launches = planned(driver, side_by_side(large, (2, 64, 64)), 1, products)
        assert (shapes[64, 64][0], shapes[large[1:]][0], launches) == (tile, tile, 8)
    shapes, launches = planned(driver, side_by_side((8, 4096, 4096), (2, 64, 64)), 1, products)
    assert (shapes[64, 64][0], shapes[4096, 4096][0], launches) == (0, 256, 9)
    # with others of 128 beside those of 256 they go along again
    shapes, launches = planned(driver, side_by_side((8, 4096, 4096), (1, 768, 768), (2, 64, 64)), 1, products)
    assert (shapes[64, 64][0], shapes[768, 768][0], shapes[4096, 4096][0], launches) == (128, 128, 256, 16)


def test_tiles_are_counted_in_the_format_that_is_asked_for(driver):
    """128 x 256 fits one workgroup in single binary16 and goes through launches in pairs, where 256 tiles of 128 and more take these."""
    matrices = side_by_side((255, 128, 256))
    assert planned(driver, matrices, 1, nl.PRODUCTS_PAIRS)[0][128, 256][:2] == (64, 255)
    matrices = side_by_side((256, 128, 256))
    assert planned(driver, matrices, 1, nl.PRODUCTS_F16)[0][128, 256][:2] == (0, 256)
    assert planned(driver, matrices, 1, nl.PRODUCTS_PAIRS)[0][128, 256][:2] == (128, 256)


def test_only_the_loads_to_the_lds_use_m0(tmp_path):
    """They write it in inline assembly, which cannot say so: m0 is reserved. So nothing else may count on what it holds."""
    with open(nl.library_path(), "rb") as f:
        data = f.read()
    kernels, at = 0, data.find(b"\x7fELF", 4)
    while at >= 0:
        if int.from_bytes(data[at + 18:at + 20], "little") == 224:                  # AMDGPU
            table, entry, count = (int.from_bytes(data[at + a:at + b], "little") for a, b in ((40, 48), (58, 60), (60, 62)))
            image = tmp_path / "gfx950.elf"
            image.write_bytes(data[at:at + table + entry * count])
            objdump = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
            text = subprocess.run([objdump, "-d", "--no-show-raw-insn", str(image)], check=True, capture_output=True, text=True).stdout
            for body in re.findall(r"<[^>]*ns_product[^>]*>:\n(.*?)\n\n", text + "\n\n", re.S):
                lines = [line.split("//")[0].strip() for line in body.splitlines()]
                kernels += 1
                for i, line in enumerate(lines):
                    if re.search(r"\bm0\b", line):
                        assert re.match(r"s_mov_b32 m0, s\d+$", line) and lines[i + 1] == "s_nop 0" and lines[i + 2].endswith("offen lds")
                    elif line.endswith(" lds"):
                        assert lines[i - 2].startswith("s_mov_b32 m0")
        at = data.find(b"\x7fELF", at + 4)
    assert kernels == 3 * 2 * 5                                                     # tiles, formats, kinds (the last with two results)
