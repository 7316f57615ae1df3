"""By which rules a call on frozen layers becomes launches (csrc/lora_experts.h), without a GPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2511_22880_amd", "csrc")
HIP_INCLUDE = "/opt/rocm/include"
pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(HIP_INCLUDE), reason="needs g++ and the HIP headers")


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("rules") / "libexperts_rules.so")
    cmd = ["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I" + HIP_INCLUDE, "-I" + CSRC, "-o", so,
           os.path.join(ROOT, "tests", "experts_rules.cpp")]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-2000:]
    lib = ctypes.CDLL(so)
    lib.rule_quantize_rows_at_once.restype = ctypes.c_longlong
    return lib


def test_a_launch_that_rounds_rows_has_fewer_than_32_bits_of_threads(rules):
    """256 threads, 16 of them a block of 128, for every 16 kQuantizeBlocks blocks; the last launch of a call may have fewer"""
    per_group = 16 * rules.rule_quantize_blocks()
    for blocks in [1, 2, 3, 5, 7, 32, 1000, 4097, (1 << 17) - 1, 1 << 17]:  # up to LORA_EXPERTS_MAX_FEATURES
        rows = rules.rule_quantize_rows_at_once(blocks)
        assert rows >= 1
        assert -(-rows * blocks // per_group) * 256 < 2 ** 32
