"""How a product of 8-bit rows and weights is cut up (csrc/block_plans.h): every plan covers its rows and fits the device."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_13587_b200", "csrc")
SHIM = """
#include "block_plans.h"
extern "C" void plan(long long m, long long n, long long k, int sms, int* out) {
  const vvs::BlockMatmulPlan p = vvs::plan_block_matmul(m, n, k, sms);
  out[0] = p.pairs; out[1] = p.tn; out[2] = p.passes; out[3] = p.splits; out[4] = p.stages;
}
"""
SIZES = [1, 2, 15, 16, 17, 32, 33, 64, 65, 96, 97, 128, 129, 191, 192, 193, 255, 256, 257, 300, 511, 512, 1000, 5460, 70001, 1 << 24]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    src, lib = str(d / "shim.cc"), str(d / "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", lib], check=True)
    so = ctypes.CDLL(lib)
    so.plan.argtypes = [ctypes.c_longlong] * 3 + [ctypes.c_int, ctypes.c_void_p]

    def call(m, n, k, sms=148):
        out = (ctypes.c_int * 5)()
        so.plan(m, n, k, sms, out)
        return dict(zip(("pairs", "tn", "passes", "splits", "stages"), out))
    return call


def test_plans_cover_their_rows_and_fit(plan):
    for m in SIZES:
        for n in (1, 127, 128, 129, 1280, 4096, 22016, 65535 * 128):
            for k in (16, 128, 144, 1280, 4096, 11008, 1 << 20):
                p = plan(m, n, k)
                if p["pairs"]:
                    continue
                assert p["tn"] in (16, 32, 64, 96, 128) and 1 <= p["passes"] <= 65535 and p["tn"] * p["passes"] >= m, (m, n, k)
                assert p["tn"] * (p["passes"] - 1) < m                              # no pass without rows
                assert 1 <= p["splits"] <= 8 and p["splits"] <= -(-k // 128)        # no CTA without a block of K
                stage = 16384 + p["tn"] * 128
                smem = p["stages"] * stage + 1024
                # two CTAs of a pass of 64 rows at most on an SM, one otherwise (1 KB each is the system's; factors and barriers are static)
                per_sm = 2 if p["tn"] <= 64 else 1
                assert 2 <= p["stages"] <= 8 and smem + 64 * p["tn"] + 256 <= min(227, (228 - per_sm) / per_sm) * 1024
                assert p["tn"] * 512 <= p["stages"] * stage                         # the sums go where the stages were


@pytest.mark.parametrize("m,k,n", [(2100, 400, 1290), (1025, 272, 3001), (5000, 16, 1000), (1300, 1296, 2056), (300, 640, 22000), (3000, 128, 17000)])
def test_sizes_of_the_gpu_tests_on_pairs(plan, m, k, n):
    assert plan(m, n, k)["pairs"]


def test_few_rows_stay_with_the_weights_and_many_go_on_pairs(plan):
    assert not plan(1, 1280, 1280)["pairs"] and plan(1, 1280, 1280)["splits"] == 4
    assert not plan(18, 22016, 4096)["pairs"] and plan(18, 22016, 4096)["splits"] == 1
    assert not plan(288, 1280, 3456)["pairs"] and plan(5460, 12288, 4096)["pairs"] and plan(1 << 24, 16, 128)["pairs"]
