"""Which kernels the products of a call of linear or linear_gradient take, from the host code that decides it, compiled for the CPU."""
import functools
import os
import subprocess
import tempfile

from conftest import ROOT

TYPES = {"f32": 0, "bf16": 1}


@functools.lru_cache(None)
def _driver():
    exe = os.path.join(tempfile.mkdtemp(), "product_plan_driver")
    csrc = os.path.join(ROOT, "paper_2506_10911_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    "-I", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
                    os.path.join(ROOT, "tests", "product_plan_driver.cpp"), os.path.join(csrc, "model_step.cpp"), "-o", exe], check=True)
    return exe


def plans(calls):
    """For every call (room of its plan in bytes, its products as dicts). A call: dict(gradient, W, T, layer, stride, act, types,
    accumulate, more) with the layer as LinearPlan takes it, whole, and more: is something added to the result?"""
    lines = []
    for c in calls:
        offset, inputs, outputs, bias, transposed, row_stride = c["layer"]
        types = [TYPES[t] for t in c["types"]] + [0] * (5 - len(c["types"]))
        lines.append(" ".join(str(int(v)) for v in (c["gradient"], c["W"], c["T"], c.get("room", 0), offset, inputs, outputs, row_stride, bias, transposed,
                                                    c["stride"], c["act"], *types, c["accumulate"], c["more"])))
    run = subprocess.run([_driver()], input="\n".join(lines), capture_output=True, text=True, check=True)
    found, room, products = [], 0, []
    for line in run.stdout.splitlines():
        words = line.split()
        if words[0] == "room":
            room, products = int(words[1]), []
        elif words[0] == "product":
            two = {"parts", "along", "packed"}
            p, i = {}, 1
            while i < len(words):
                if words[i] in two:
                    p[words[i]] = (int(words[i + 1]), int(words[i + 2]))
                    i += 3
                else:
                    p[words[i]] = int(words[i + 1])
                    i += 2
            products.append(p)
        else:
            found.append((room, products))
    assert len(found) == len(calls)
    return found
