"""By which rules a call of attention becomes launches (csrc/lora_attention.h), without a GPU."""
import ctypes
import math
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2511_22880_amd", "csrc")
HIP_INCLUDE = "/opt/rocm/include"
needs_headers = pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(HIP_INCLUDE), reason="needs g++ and the HIP headers")


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("rules") / "libattention_rules.so")
    cmd = ["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I" + HIP_INCLUDE, "-I" + CSRC, "-o", so,
           os.path.join(ROOT, "tests", "attention_rules.cpp")]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-2000:]
    lib = ctypes.CDLL(so)
    sizes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_longlong]
    for name, rest, result in (("rule_forms", [ctypes.c_longlong, ctypes.c_int, ctypes.c_int], ctypes.c_char_p),
                               ("rule_shares", [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int], ctypes.c_int),
                               ("rule_bytes", [ctypes.c_longlong, ctypes.c_int, ctypes.c_int], ctypes.c_longlong),
                               ("rule_most_bytes", [ctypes.c_int, ctypes.c_int], ctypes.c_longlong)):
        getattr(lib, name).argtypes, getattr(lib, name).restype = sizes + rest, result
    return lib


def calls(n, seed=1):
    """(tokens, group, key heads, requests, keys, most rows, dim, bits), sizes spread by their logarithm"""
    r = random.Random(seed)
    size = lambda least, most: round(math.exp(r.uniform(math.log(least), math.log(most))))  # noqa: E731
    for _ in range(n):
        tokens, group, heads = size(1, 50000), r.choice([1, 2, 3, 4, 7, 8, 12, 16, 17, 40, 64]), r.choice([1, 2, 4, 8, 9, 32, 600])
        yield tokens, group, heads, min(size(1, 3000), 2 * tokens), 16 * size(1, 20000), r.choice([0, 1, size(1, 64), size(1, tokens)]), r.choice([64, 128]), r.choice([8, 16])


@needs_headers
def test_a_workspace_is_enough_whatever_most_says(rules):
    for *sizes, most, dim, bits in calls(20000):
        said = rules.rule_most_bytes(*sizes, dim, bits)
        for rows in (most, 0, 1, max(1, 16 // sizes[1]), max(1, 40 // sizes[1]), max(1, 128 // sizes[1]), max(1, 2 * sizes[0] // sizes[3])):
            assert rules.rule_bytes(*sizes, rows, dim, bits) <= said, (sizes, rows, dim, bits)
