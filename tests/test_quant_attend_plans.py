"""Shared memory for the scores of summed rows (csrc/launch_plans.h), which the host reserves and the kernel asks again with the lengths it
finds: exact up to the longest cache, where the bytes pass what 32 bits hold."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_13587_b200", "csrc")
SHIM = """
#include "launch_plans.h"
extern "C" int ld(int keys) { return vvs::quant_score_ld(keys); }
extern "C" long long bytes(int rows, int keys) { return vvs::quant_score_bytes(rows, keys); }
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    src, lib = str(d / "shim.cc"), str(d / "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", lib], check=True)
    so = ctypes.CDLL(lib)
    so.bytes.restype = ctypes.c_longlong
    return so


def test_scores_of_summed_rows_are_counted_exactly(plans):
    slices = list(range(0, 200)) + [2 ** k + d for k in range(8, 27) for d in (-1, 0, 1) if 2 ** k + d <= 2 ** 26]
    for n in slices:
        keys = 16 * n
        ld = plans.ld(keys)
        assert ld >= keys and ld % 32 == 8 and ld < keys + 40, keys
        for rows in (1, 2, 15, 16, 17, 31, 32):
            assert plans.bytes(rows, keys) == rows * ld * 4, (rows, keys)
    # 32 rows of 2^24 keys: as a product of 32-bit numbers it is negative, and less than any shared memory
    assert plans.bytes(32, 1 << 24) > 227 * 1024


def test_the_kernel_asks_the_same_arithmetic():
    with open(os.path.join(CSRC, "quant_attend.cu")) as f:
        text = f.read()
    assert text.count("quant_score_bytes(") == 2 and "score_ld * 4" not in text
