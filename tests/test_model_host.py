"""What layer norm, matrices and log probabilities refuse before they touch a GPU, and their host code under AddressSanitizer and
UBSan against stand-ins for the HIP runtime and the kernel launchers."""
import os
import re
import subprocess

import pytest

import paper_2506_10911_amd as nl
from conftest import ROOT

nl.library_path()          # loads libnoloco.so now; a missing library is an error, not a skip


def refused(status, call, *args, **more):
    with pytest.raises(nl.NolocoError) as e:
        call(*args, **more)
    assert e.value.status == status


@pytest.mark.parametrize("status,args", [
    (2, ([(0, 4, 4)], -64, 1, 1)), (2, ([(0, 4, 4)], 64, 0, 1)), (2, ([(0, 4, 4)], 64, 1, -1)), (5, ([(0, 4, 4)], 65, 1, 1)),
    (7, ([(0, 4, 4)], 64, 65537, 1)), (7, ([(0, 4, 4)], 1 << 60, 4, 1)), (7, ([(0, 4, 4)], 64, 1, 1 << 28)), (7, ([(0, 4, 4)], 64, 64, 1 << 26)),
    (2, ([(-1, 4, 4)], 64, 1, 1)), (2, ([(0, -2, 4)], 64, 1, 1)), (2, ([(0, 4, 0)], 64, 1, 1)), (7, ([(0, -1, (1 << 20) + 1)], 1 << 30, 1, 1)),
    (4, ([(61, 0, 4)], 64, 1, 1)), (4, ([(0, 61, 4)], 64, 1, 1)), (4, ([(65, -1, 1)], 64, 1, 1)), (4, ([(0, 3, 4)], 64, 1, 1)), (4, ([(3, 0, 4)], 64, 1, 1)),
    (4, ([(0, 0, 1)], 64, 1, 1)),
])
def test_norm_plans_refused(status, args):
    refused(status, nl.LayerNormPlan, *args)


@pytest.mark.parametrize("status,layer,more", [
    (2, (0, 4, 4), dict(worker_stride=-64)), (2, (0, 4, 4), dict(W=0)), (2, (0, 4, 4), dict(max_tokens=-1)), (2, (0, 4, 4), dict(workspace_bytes=-1)),
    (5, (0, 4, 4), dict(worker_stride=66)), (7, (0, 4, 4), dict(W=65537)), (7, (0, 4, 4), dict(worker_stride=1 << 60, W=4)),
    (7, (0, 4, 4), dict(max_tokens=(1 << 24) + 1)), (2, (-1, 4, 4), {}), (2, (0, 0, 4), {}), (2, (0, 4, 0), {}), (2, (0, 4, 4, -2), {}),
    (2, (0, 4, 4, -1, 2), {}), (2, (0, 4, 4, -1, 0, 3), {}), (2, (0, 5, 4, -1, 1, 4), {}), (4, (0, 8, 9), {}), (4, (49, 4, 4), {}), (4, (0, 4, 4, 61), {}),
    (4, (0, 4, 4, -1, 0, 21), {}), (4, (65, 1, 1), {}), (4, (0, 4, 4, 15), {}), (4, (4, 4, 4, 1), {}), (4, (0, 4, 4, 7, 0, 10), {}),
    (4, (0, 4, 2, 1, 0, 10), {}), (4, (0, 1 << 20, 1, -1, 0, 1 << 50), dict(worker_stride=1 << 30)),
    (7, (0, (1 << 22) + 1, 1), dict(worker_stride=1 << 30)), (7, (0, 1 << 16, 1 << 15), dict(worker_stride=1 << 40)),
    (7, (0, 1 << 12, 1), dict(worker_stride=1 << 30, max_tokens=(1 << 18) + 1)),
])
def test_linear_plans_refused(status, layer, more):
    refused(status, nl.LinearPlan, [layer], **{**dict(worker_stride=64, W=1, max_tokens=1), **more})


@pytest.mark.parametrize("status,args,more", [
    (2, (0, 1, 1), {}), (2, (4, 0, 1), {}), (2, (4, 1, -1), {}), (2, (4, 1, 1), dict(row_stride=3)), (2, (4, 1, 1), dict(max_top=-1)),
    (7, (4, 1, 1), dict(max_top=33)), (7, ((1 << 24) + 1, 1, 1), {}), (7, (4, 65537, 1), {}), (7, (4, 64, 1 << 26), {}),
    (7, (4, 1, 1 << 30), dict(row_stride=1 << 40)),
])
def test_log_prob_plans_refused(status, args, more):
    refused(status, nl.LogProbPlan, *args, **more)


def test_null_plans_refused():
    class NoPlan:
        _address = 0
    refused(1, nl.layer_norm, NoPlan, 0, 256, nl.F32, 512, nl.F32, 1, 1e-5, 1024, nl.F32, stream=0)
    refused(1, nl.layer_norm_gradient, NoPlan, 0, 256, nl.F32, 512, nl.F32, 768, nl.F32, 1024, 1, 2048, nl.F32, None, nl.F32, stream=0)
    refused(1, nl.linear, NoPlan, 0, 256, nl.F32, 512, nl.F32, 1, 1024, nl.F32, stream=0)
    refused(1, nl.linear_gradient, NoPlan, 0, 256, nl.F32, 512, nl.F32, 768, nl.F32, 1, 1024, nl.F32, None, nl.F32, stream=0)
    refused(1, nl.token_log_probs, NoPlan, 256, nl.F32, 512, nl.I32, 1, 1024, stream=0)
    refused(1, nl.token_log_probs_gradient, NoPlan, 256, nl.F32, 512, nl.I32, 1, 768, 1024, 2048, nl.F32, stream=0)


def test_arguments_of_other_kinds_raise():
    calls = nl.binding._calls
    for call, count in ((calls.layer_norm, 12), (calls.layer_norm_gradient, 17), (calls.linear, 13), (calls.linear_gradient, 18),
                        (calls.token_log_probs, 13), (calls.token_log_probs_gradient, 13)):
        with pytest.raises(TypeError):
            call(*([0] * (count - 1)))
        with pytest.raises((TypeError, ValueError)):
            call(*([0] * (count - 1) + ["x"]))
        assert call(*([0] * count)) == 1               # no plan


def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    csrc = os.path.join(ROOT, "paper_2506_10911_amd", "csrc")
    exe = tmp_path / "model_host_driver"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    "-I", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
                    os.path.join(ROOT, "tests", "model_host_driver.cpp"), os.path.join(csrc, "model_step.cpp"), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], env=dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1"),
                         capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout + run.stderr
    assert "model host driver: ok" in run.stdout


def test_only_the_loads_to_the_lds_use_m0(tmp_path):
    """They write it in inline assembly, which cannot say so: m0 is reserved. So nothing else in these kernels may count on what it holds."""
    with open(nl.library_path(), "rb") as f:
        data = f.read()
    kernels, at = 0, data.find(b"\x7fELF", 4)
    objdump = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
    while at >= 0:
        if int.from_bytes(data[at + 18:at + 20], "little") == 224:                  # AMDGPU
            table, entry, count = (int.from_bytes(data[at + a:at + b], "little") for a, b in ((40, 48), (58, 60), (60, 62)))
            if b"product_direct" in data[at:at + table]:
                image = tmp_path / "gfx950.elf"
                image.write_bytes(data[at:at + table + entry * count])
                text = subprocess.run([objdump, "-d", "--no-show-raw-insn", str(image)], check=True, capture_output=True, text=True).stdout
                for body in re.findall(r"<[^>]*product_direct[^>]*>:\n(.*?)\n\n", text + "\n\n", re.S):
                    lines = [line.split("//")[0].strip() for line in body.splitlines()]
                    kernels += 1
                    for i, line in enumerate(lines):
                        if re.search(r"\bm0\b", line):
                            assert re.match(r"s_mov_b32 m0, s\d+$", line) and lines[i + 1] == "s_nop 0" and lines[i + 2].endswith("offen lds")
                        elif line.endswith(" lds"):
                            assert lines[i - 2].startswith("s_mov_b32 m0")
        at = data.find(b"\x7fELF", at + 4)
    assert kernels == 2 * (3 + 3 + 2)                  # formats; layouts of the operands in tiles of 256, 128, 32 x 256
