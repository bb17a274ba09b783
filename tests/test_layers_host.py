"""The operators beside the sparse product, what of them runs on the host."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

import paper_2506_15174_amd as spmm

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2506_15174_amd", "csrc")


def test_library_exports_every_declared_symbol():
    with open(os.path.join(ROOT, "include", "spmm_layers.h")) as f:
        header = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = set(re.findall(r"\b(spmm_[a-z_]+)\s*\(", header))
    assert declared == set(spmm.LAYER_EXPORTS)
    lib = ctypes.CDLL(spmm.LIB_PATH)
    for name in declared:
        assert getattr(lib, name) is not None


def test_header_is_plain_c(tmp_path):
    source = tmp_path / "client.c"
    source.write_text('#include "spmm_layers.h"\nint main(void) { spmm_norm_t n = {0}; return n.eps != 0 || SPMM_ACT_SILU; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-c", str(source), "-o", str(tmp_path / "client.o")],
                   check=True)


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("layers") / "layers")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__=1", "-I", CSRC, "-I", os.path.join(rocm, "include"),
                    os.path.join(HERE, "layers_on_stand_ins.cpp"), os.path.join(CSRC, "layers", "layers_api.cpp"), "-pthread", "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("what", ["layouts", "failures", "product", "rows"])
def test_host_source_on_stand_ins(program, what):
    res = subprocess.run([program, what], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.endswith("ok\n"), res.stdout + res.stderr


def test_what_creation_refuses():
    """Shapes and types of the arrays, before the library is asked."""
    codes, scales, zeros = np.zeros((6, 5), np.uint8), np.ones((6, 1), np.float32), np.zeros((6, 1), np.uint8)
    for bad in (dict(codes=codes[:, :4]), dict(codes=codes.astype(np.int32)), dict(scales=scales[:5]), dict(scales=scales.astype(np.float64)), dict(scales=np.ones((6, 2), np.float32)),
                dict(zeros=zeros[:5]), dict(zeros=zeros.astype(np.float32))):
        with pytest.raises(ValueError):
            spmm.quant_plan_create(6, 10, **{**dict(codes=codes, scales=scales, zeros=zeros, group=32), **bad})
    for M, K, group, status in ((-1, 10, 32, spmm.binding.SPMM_ERR_INVALID_ARG), (6, 10, 0, spmm.binding.SPMM_ERR_INVALID_ARG)):
        with pytest.raises(spmm.SpmmError) as err:
            spmm.quant_plan_create(M, K, codes, np.ones((6, 0), np.float32) if group == 0 else scales, group=group)
        assert err.value.status == status
    with pytest.raises(spmm.SpmmError) as err:
        spmm.quant_plan_create(6, 10, codes, scales, group=48)
    assert err.value.status == spmm.binding.SPMM_ERR_UNSUPPORTED


def test_weights_of_the_benchmarks_blocks():
    """Seeded, in the plan's form, and of the standard deviation that they are asked for."""
    from workloads import generators as gen
    codes, scales = gen.weights_4bit(64, 321, 128, 5)
    assert codes.shape == (64, 161) and codes.dtype == np.uint8 and scales.shape == (64, 3) and scales.dtype == np.float32
    again = gen.weights_4bit(64, 321, 128, 5)
    assert np.array_equal(codes, again[0]) and np.array_equal(scales, again[1])
    values = (codes & 15).astype(np.float64) - 8
    values *= np.repeat(scales, 64, 1)[:, :161]
    # uniform codes have a variance of 21.25 about -0.5, scales a mean square of 1.0133 (0.02 / 4.6)^2; 10304 draws are off by 5 % at most
    assert abs(np.sqrt((values ** 2).mean()) / 0.02 - np.sqrt(21.5 * 1.0133) / 4.6) < 0.05
