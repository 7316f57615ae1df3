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


# Calls that take each kind of launch, which test_gpu_attention_forms.py runs: requests of (rows, keys), most rows as the host says.  8 query heads on 2 key heads.
LONG = {"cut": 2500, "whole": 300}
MORE = [(1, 7 * i + 1) for i in range(28)]  # (up to 32 requests with little to read are one launch, and up to 256 of few steps here)
FORMS = {f"few {c} {how}": ([(1, keys), (rows, 40), (0, 9), (rows, keys - 7), (1, 1)], rows) for c, rows in ((16, 4), (32, 8)) for how, keys in LONG.items()}
FORMS |= {f"wide {c} {how}": ([(rows, keys), (rows, rows), (rows - 3, 80), (1, 17)], rows) for c, rows in ((128, 32), (256, 77)) for how, keys in LONG.items()}
FORMS |= {f"few 16 {how}, wide {c} {how}": ([(1, keys), (1, 1), (rows, keys), (3, 290), (0, 0), (4, 4), (5, 5), (1, 33), (2, 100), (rows, 90)] + MORE * (10 if how == "whole" else 1), rows)
          for c, rows in ((128, 27), (256, 91)) for how, keys in LONG.items()}
# .. with a table that has room for more: tiles of many columns have more keys in 16 steps than those of few in 4
FORMS |= {f"few 16 cut, wide {c} whole": ([(1, 1020), (1, 1), (rows, 1000), (3, 290), (4, 4), (5, 5), (1, 33), (2, 100)] + MORE, rows) for c, rows in ((128, 31), (256, 300))}


def form_of(rules, name, dim, bits, page=16):
    sizes, most = FORMS[name]
    keys = -(-max(k for _, k in sizes) // page) * page
    return rules.rule_forms(sum(n for n, _ in sizes), 4, 2, len(sizes), keys, most, dim, bits).decode()


def taken(name, bits):
    return bits == 16 or name.split(",")[0] != "few 16 cut" or "whole" not in name  # (few columns in 8 bits take 256 keys a step: 1020 are 4)


@needs_headers
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("name, bits", [(name, bits) for name in FORMS for bits in (8, 16) if taken(name, bits)])
def test_these_calls_take_the_launches_they_stand_for(rules, name, dim, bits):
    assert form_of(rules, name, dim, bits) == name


@needs_headers
def test_no_call_takes_launches_that_are_not_among_them(rules):
    seen = {rules.rule_forms(*c).decode() for c in calls(20000, seed=2)}
    # (few columns whole and many cut, by the number of their tiles alone: each is among them)
    assert {form for forms in seen for form in forms.split(", ")} == {f"{kind} {c} {how}" for kind, c in (("few", 16), ("few", 32), ("wide", 128), ("wide", 256))
                                                                    for how in ("cut", "whole")}
    assert set(FORMS) <= seen


@needs_headers
def test_launches_have_work_groups_for_what_there_may_be_and_no_more_than_a_grid_has(rules):
    """whole tiles: one work group for each that the host cannot rule out; cut ones: a share of a key head's is never empty by rule alone"""
    for c in calls(20000, seed=3):
        tokens, group, heads, requests, keys, most, dim, bits = c
        for i, form in enumerate(rules.rule_forms(*c).decode().split(", ")):
            columns, shares = int(form.split()[1]), rules.rule_shares(*c, i)
            assert shares >= 1 and shares * heads * 512 < 2 ** 32
            if form.endswith("whole"):
                # requests of one token each, and one of all others
                filled, up = min(requests, tokens), lambda n: -(-n * group // columns)  # noqa: E731
                if "," not in rules.rule_forms(*c).decode():
                    assert shares >= (filled - 1) * up(1) + up(tokens - filled + 1)
            else:
                assert shares <= max(1, 512 // heads)


@needs_headers
def test_a_table_without_pages_has_its_launches_too(rules):
    """no request has a key then, and every row is written, with zeros: a tile is a step for that, in as many launches of a work group at least, with room for what they leave"""
    for tokens, group, heads, requests, _, most, dim, bits in calls(20000, seed=4):
        sizes = tokens, group, heads, requests, 0
        forms = rules.rule_forms(*sizes, most, dim, bits).decode().split(", ")
        assert all(1 <= rules.rule_shares(*sizes, most, dim, bits, i) <= 2 ** 23 // heads for i in range(len(forms))), (sizes, most, dim, bits, forms)
        assert rules.rule_bytes(*sizes, most, dim, bits) <= rules.rule_most_bytes(*sizes, dim, bits)
