"""By which rules a call on frozen layers becomes launches (csrc/lora_experts.h), without a GPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2511_22880_amd", "csrc")
HIP_INCLUDE = "/opt/rocm/include"
needs_headers = pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(HIP_INCLUDE), reason="needs g++ and the HIP headers")

# Sizes that take each kernel of the products, which test_gpu_experts_forms.py runs.  By experts: rows of each, picks a token has,
# picks without an expert, in and out features.
EXPERTS_FORMS = {
    ("thin 1x1/8", 16): ([3, 0, 1], 1, 2, 320, 256), ("thin 1x1/8", 8): ([0, 3, 1], 2, 1, 1088, 256),
    ("thin 1x2/8", 16): ([40, 0, 41], 3, 9, 704, 768), ("thin 1x2/8", 8): ([2, 1], 1, 0, 2112, 2304),
    ("thin 1x4/4", 16): ([2, 1], 2, 0, 1088, 4736), ("thin 1x4/4", 8): ([1, 3], 2, 1, 192, 4736),
    ("thin 1x4/4 once", 16): ([3, 1, 0, 2], 1, 0, 4160, 8192), ("thin 1x4/4 once", 8): ([1, 0, 2], 2, 1, 4160, 10752),
    ("thin 2x4/4", 16): ([20, 16], 2, 1, 448, 3200), ("thin 2x4/4", 8): ([1, 33], 2, 1, 1088, 3200),
    ("thin 2x4/4 once", 16): ([33, 17, 9], 2, 4, 4160, 5504), ("thin 2x4/4 once", 8): ([19], 2, 0, 11776, 12544),
    ("mid 2x2/1", 16): ([33, 4, 0], 2, 6, 448, 6272), ("mid 2x2/1", 8): ([2, 32], 2, 1, 1088, 9216),
    ("mid 2x2/2", 16): ([70, 33], 2, 4, 1088, 3712), ("mid 2x2/2", 8): ([7, 13], 2, 1, 2112, 9344),
    ("mid 2x2/1 once", 16): ([5, 9, 0, 8, 17, 12, 1, 4] * 8, 8, 8, 2048, 1536), ("mid 2x2/1 once", 8): ([13, 0, 33, 2] * 24, 4, 7, 960, 1536),
    ("mid 2x2/2 once", 16): ([3, 1, 0, 6], 2, 0, 3008, 7424), ("mid 2x2/2 once", 8): ([4, 1, 3], 1, 0, 4160, 10752),
    ("mid 4x2/1", 16): ([129, 22, 0, 2], 2, 6, 704, 4608), ("mid 4x2/1", 8): ([63, 1], 2, 0, 1088, 9344),
    ("mid 4x2/2", 16): ([65, 85], 2, 3, 1088, 4608), ("mid 4x2/2", 8): ([21, 40], 2, 0, 2112, 9344),
    ("mid 4x2/1 once", 16): ([33, 64, 0, 40, 2, 65, 1, 31, 20], 2, 9, 704, 10624), ("mid 4x2/1 once", 8): ([48, 2, 25, 0, 64, 10, 21, 30] * 6, 2, 9, 192, 11136),
    ("mid 4x2/2 once", 16): ([47, 13], 2, 4, 3008, 11392), ("mid 4x2/2 once", 8): ([33, 65, 1], 2, 1, 4160, 10880),
    ("mid 4x4/1", 16): ([65, 64, 22], 1, 1, 704, 9216), ("mid 4x4/1", 8): ([129, 20], 2, 1, 1088, 9216),
    ("mid 4x4/2", 16): ([130, 30], 2, 1, 1088, 9216), ("mid 4x4/2", 8): ([17, 133], 2, 1, 2112, 9216),
    ("wide", 16): ([129, 70, 300], 2, 1, 320, 9344), ("wide", 8): ([60, 1, 256, 130], 2, 3, 704, 9344),
    ("wide large", 16): ([200, 256, 130], 2, 2, 2112, 10880), ("wide large", 8): ([140, 256, 0, 255, 200, 129, 300, 33] * 2, 2, 2, 4160, 2176),
}
# .. and of one layer in 8 bits: rows, in and out features
LAYER_FORMS = {
    "thin 1x1/8": (3, 1088, 256), "thin 1x2/8": (9, 2112, 4736), "thin 1x4/4": (5, 320, 9344), "thin 1x4/4 once": (3, 8512, 16128), "thin 2x4/4": (18, 1088, 9600),
    "thin 2x4/4 once": (19, 8896, 15616), "mid 2x2/1": (35, 704, 9472), "mid 2x2/2": (61, 2112, 9472), "mid 4x2/1": (67, 1088, 10624), "mid 4x2/2": (127, 2112, 10624),
    "mid 4x4/1": (133, 448, 12800), "mid 4x4/2": (200, 2112, 9472), "wide": (260, 704, 14208), "wide large": (200, 8192, 16512),
}


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("rules") / "libexperts_rules.so")
    cmd = ["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I" + HIP_INCLUDE, "-I" + CSRC, "-o", so,
           os.path.join(ROOT, "tests", "experts_rules.cpp")]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-2000:]
    lib = ctypes.CDLL(so)
    lib.rule_quantize_rows_at_once.restype = ctypes.c_longlong
    lib.rule_product_form.restype = ctypes.c_char_p
    return lib


@needs_headers
def test_a_launch_that_rounds_rows_has_fewer_than_32_bits_of_threads(rules):
    """256 threads, 16 of them a block of 128, for every 16 kQuantizeBlocks blocks; the last launch of a call may have fewer"""
    per_group = 16 * rules.rule_quantize_blocks()
    for blocks in [1, 2, 3, 5, 7, 32, 1000, 4097, (1 << 17) - 1, 1 << 17]:  # up to LORA_EXPERTS_MAX_FEATURES
        rows = rules.rule_quantize_rows_at_once(blocks)
        assert rows >= 1
        assert -(-rows * blocks // per_group) * 256 < 2 ** 32


def form(rules, bits, rows, experts, in_f, out_f):
    return rules.rule_product_form(bits, rows, experts, in_f, out_f).decode()


@needs_headers
@pytest.mark.parametrize("name, bits", EXPERTS_FORMS)
def test_these_experts_take_the_kernel_they_stand_for(rules, name, bits):
    sizes, picks, idle, in_f, out_f = EXPERTS_FORMS[name, bits]
    assert form(rules, bits, -(-(sum(sizes) + idle) // picks) * picks, len(sizes), in_f, out_f) == name


@needs_headers
@pytest.mark.parametrize("name", LAYER_FORMS)
def test_these_layers_take_the_kernel_they_stand_for(rules, name):
    rows, in_f, out_f = LAYER_FORMS[name]
    assert form(rules, 8, rows, 0, in_f, out_f) == name


@needs_headers
def test_no_call_takes_a_kernel_that_is_not_among_them(rules):
    """over sizes spread by their logarithm, 1 to 20000 rows of 1 to 512 experts and of one layer"""
    import math
    import random
    r = random.Random(1)
    size = lambda least, most, unit: unit * max(1, round(math.exp(r.uniform(math.log(least), math.log(most))) / unit))  # noqa: E731
    seen, seen_one = set(), set()
    for _ in range(60000):
        bits, experts, rows, in_f, out_f = r.choice((8, 16)), size(1, 512, 1), size(1, 20000, 1), size(64, 16384, 64), size(128, 16384, 128)
        seen.add((form(rules, bits, rows, experts, in_f, out_f), bits))
        seen_one.add(form(rules, 8, rows, 0, in_f, out_f))
    assert seen == set(EXPERTS_FORMS)
    assert seen_one <= set(LAYER_FORMS)
