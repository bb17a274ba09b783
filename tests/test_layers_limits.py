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


def test_one_token_in_columns_with_gaps_and_without(program):
    run(program, "one token")


def test_outputs_between_the_rows_of_inputs(program):
    run(program, "between rows")


@pytest.mark.parametrize("M,K,group", [(6, 300, 2 ** 64 + 128), (6, 300, 2 ** 63), (6, 300, -2 ** 64 + 128), (-2 ** 64 + 6, 300, 128), (6, -2 ** 64 + 300, 128), (2 ** 64 + 6, 300, 128), (6, 2 ** 64 + 300, 128)])
def test_sizes_of_more_than_64_bits(M, K, group):
    """Cut off to 64 bits they would be those of larger arrays."""
    with pytest.raises(ValueError):
        spmm.quant_plan_create(M, K, np.zeros((6, 150), np.uint8), np.ones((6, 1 if group > 0 else 0), np.float32), group=group)


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """The launches' host code, linked with stand-ins for the HIP runtime (the kernels' own code is left out)."""
    made = tmp_path_factory.mktemp("launches")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    objects = []
    for name in ("quant", "rows"):
        objects.append(str(made / (name + ".o")))
        subprocess.run([os.path.join(rocm, "bin", "hipcc"), "--offload-arch=gfx950", "--offload-host-only", "-O1", "-fPIC", "-std=c++17", "-w", "-I", CSRC, "-c", os.path.join(CSRC, "layers", name + ".hip"),
                        "-o", objects[-1]], check=True)
    exe = str(made / "launches")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-D__HIP_PLATFORM_AMD__=1", "-I", CSRC, "-I", os.path.join(rocm, "include"), os.path.join(HERE, "layers_launches_on_stand_ins.cpp"),
                    os.path.join(CSRC, "layers", "layers_api.cpp")] + objects + ["-Wl,--unresolved-symbols=ignore-all", "-pthread", "-o", exe], check=True)
    return exe


def test_launches_of_norm_and_gate_are_within_limits(launches):
    run(launches, "rows")


def test_launches_of_the_product_are_within_limits(launches):
    run(launches, "products")
