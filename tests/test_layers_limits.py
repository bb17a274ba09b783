"""The operators beside the sparse product on the host: sizes next to the limits, and tensors that only just go together."""
import os
import subprocess

import numpy as np
import pytest

import paper_2506_15174_amd as spmm

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2506_15174_amd", "csrc")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("layers") / "limits")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__=1", "-I", CSRC, "-I", os.path.join(rocm, "include"),
                    os.path.join(HERE, "layers_limits_on_stand_ins.cpp"), os.path.join(CSRC, "layers", "layers_api.cpp"), "-pthread", "-o", exe], check=True)
    return exe


def run(program, what):
    res = subprocess.run([program, what], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.endswith("ok\n"), res.stdout + res.stderr


def test_groups_of_any_size(program):
    run(program, "groups")
