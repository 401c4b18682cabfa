"""What the inner step's entry points refuse before they touch a GPU, and their host code under AddressSanitizer and UBSan
against stand-ins for the HIP runtime and the kernel launchers."""
import os
import subprocess

import pytest

import paper_2506_10911_amd as nl
from conftest import ROOT

nl.library_path()          # loads libnoloco.so now; a missing library is an error, not a skip


def refused(status, call, *args, **more):
    with pytest.raises(nl.NolocoError) as e:
        call(*args, **more)
    assert e.value.status == status


@pytest.mark.parametrize("status,matrices,stride,W,room", [
    (2, [(0, 4, 4)], 64, 0, 0), (2, [(0, 4, 4)], -64, 1, 0), (2, [(0, 4, 4)], 64, 1, -1), (5, [(0, 4, 4)], 65, 1, 0),
    (7, [(0, 4, 4)], 64, 65537, 0), (2, [(-1, 4, 4)], 64, 1, 0), (2, [(0, -4, 4)], 64, 1, 0), (2, [(0, 4, 4, 3)], 64, 1, 0),
    (2, [(0, 4, 4, 4, float("nan"))], 64, 1, 0), (4, [(0, 4, 17)], 64, 1, 0), (4, [(49, 4, 4)], 64, 1, 0), (4, [(0, 4, 4, 30)], 64, 1, 0),
    (4, [(65, 1, 1)], 64, 1, 0), (4, [(0, 4, 4), (15, 2, 2)], 64, 1, 0), (4, [(0, 4, 4, 10), (3, 1, 2)], 64, 1, 0),
    (4, [(0, 1 << 20, 1, 1 << 50)], 1 << 30, 1, 0), (7, [(0, 1 << 23, 1)], 1 << 30, 1, 0), (7, [(0, 1 << 15, 1 << 14)], 1 << 40, 1, 0),
    (7, [(0, 4, 4)], 1 << 60, 4, 0), (7, [(i, 1, 1) for i in range(512)], 512, 65536, 0),
])
def test_matrix_plans_refused(status, matrices, stride, W, room):
    refused(status, nl.MuonPlan, matrices, stride, W, room)


@pytest.mark.parametrize("status,args", [
    (2, (-1, 4, 4, 64, 1, 1)), (2, (0, 0, 4, 64, 1, 1)), (2, (0, 4, 0, 64, 1, 1)), (2, (0, 4, 4, 64, 0, 1)), (2, (0, 4, 4, 64, 1, -1)),
    (4, (0, 4, 17, 64, 1, 1)), (4, (49, 4, 4, 64, 1, 1)), (4, (65, 1, 1, 64, 1, 1)), (5, (0, 4, 4, 63, 1, 1)), (7, (0, 4, 4, 64, 65537, 1)),
    (7, (0, 4, 4, 64, 1, 1 << 28)), (7, (0, 4, 4, 64, 64, 1 << 26)), (7, (0, (1 << 29) + 1, 1, 1 << 40, 1, 1)), (7, (0, 1, (1 << 24) + 1, 1 << 40, 1, 1)),
])
def test_embedding_plans_refused(status, args):
    refused(status, nl.EmbeddingPlan, *args)


def test_null_plans_refused():
    class NoPlan:
        _address = 0
    refused(1, nl.orthogonalize, NoPlan, 256, nl.F32, 512, nl.F32, stream=0)
    refused(1, nl.muon_step, NoPlan, 256, nl.F32, 512, nl.F32, 1024, (0.1, 0.9, 0.0), stream=0)
    refused(1, nl.embed_lookup, NoPlan, 256, nl.F32, 512, nl.I32, 1, 1.0, 1024, nl.F32, stream=0)
    refused(1, nl.embed_gradient, NoPlan, 256, nl.F32, 512, nl.I32, 1, 1.0, 1024, nl.F32, stream=0)


def test_coefficients_come_in_threes():
    class NoPlan:
        _address = 0
    with pytest.raises(ValueError):
        nl.orthogonalize(NoPlan, 0, nl.F32, 0, nl.F32, coefficients=((1.0, 2.0),), stream=0)


def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    csrc = os.path.join(ROOT, "paper_2506_10911_amd", "csrc")
    exe = tmp_path / "inner_host_driver"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    "-I", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
                    os.path.join(ROOT, "tests", "inner_host_driver.cpp"), os.path.join(csrc, "inner_step.cpp"), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], env=dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1"),
                         capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout + run.stderr
    assert "inner host driver: ok" in run.stdout
