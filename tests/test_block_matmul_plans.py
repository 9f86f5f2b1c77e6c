"""How a product of 8-bit rows and weights is cut up (csrc/block_plans.h): every plan covers its rows and fits the device."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_13587_b200", "csrc")
SHIM = """
#include "block_plans.h"
extern "C" void plan(long long m, long long n, long long k, int sms, const int* clusters, long long* out) {
  const vvs::BlockMatmulPlan p = vvs::plan_block_matmul(m, n, k, sms, clusters);
  out[0] = p.pairs; out[1] = p.tn; out[2] = p.passes;
  for (int i = 0; i < 2; ++i) out[3 + 3 * i] = p.part[i].first, out[4 + 3 * i] = p.part[i].count, out[5 + 3 * i] = p.part[i].splits;
}
extern "C" int stages(int tn, int splits) { return vvs::matmul_stages(tn, splits); }
extern "C" int recv(int tn, int splits) { return vvs::matmul_recv_bytes(tn, splits); }
extern "C" int places(int tn) { return vvs::matmul_places(tn); }
extern "C" int columns(int tn) { return vvs::matmul_columns(tn); }
extern "C" int pair_smem() { return vvs::kMatmulPairSmem; }
extern "C" int room(int tn) { return vvs::matmul_room(tn) + 1024; }
extern "C" int smem(int tn, int splits) { return vvs::matmul_smem(tn, splits); }
"""
SIZES = [1, 2, 15, 16, 17, 32, 33, 48, 49, 64, 65, 96, 97, 128, 129, 191, 192, 193, 255, 256, 257, 300, 511, 512, 1000, 5460, 70001, 1 << 24]
# clusters of 0 .. 8 CTAs that a device holds at once, an SM each, and of a device that holds none of more than one
CLUSTERS = {None: [0, 148, 74, 45, 33, 26, 22, 15, 15], 0: [0, 148] + [0] * 7}


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    src, lib = str(d / "shim.cc"), str(d / "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", lib], check=True)
    so = ctypes.CDLL(lib)
    so.plan.argtypes = [ctypes.c_longlong] * 3 + [ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]

    def call(m, n, k, held=None):
        clusters = (ctypes.c_int * 9)(*CLUSTERS[held])
        out = (ctypes.c_longlong * 9)()
        so.plan(m, n, k, 148, clusters, out)
        p = dict(zip(("pairs", "tn", "passes"), out))
        call.lib = so
        return dict(p, parts=[tuple(out[3 + 3 * i:6 + 3 * i]) for i in range(2)], clusters=list(clusters))
    return call


@pytest.mark.parametrize("held", [None, 0])
def test_plans_cover_their_rows_and_weights_and_fit(plan, held):
    for m in SIZES:
        for n in (1, 127, 128, 129, 1280, 4096, 18944, 22016, 37889, 65535 * 128):
            for k in (16, 128, 144, 1280, 4096, 11008, 1 << 20):
                p = plan(m, n, k, held)
                if p["pairs"]:
                    continue
                assert p["tn"] in (16, 32, 48, 64, 96, 128) and 1 <= p["passes"] <= 65535 and p["tn"] * p["passes"] >= m, (m, n, k)
                assert p["tn"] * (p["passes"] - 1) < m                              # no pass without rows
                (first, count, splits), (first_2, count_2, splits_2) = p["parts"]
                assert first == 0 and count >= 1 and count + count_2 == -(-n // 128) <= 65535
                assert count_2 == 0 or (first_2 == count and p["passes"] == 1)
                # no CTA without a block of K, clusters that are all there at once; the second launch's beside the first one's CTAs
                for c, s, slots in ((count * p["passes"], splits, 2 if p["tn"] <= 64 else 1), (count_2, splits_2, 1)):
                    assert c == 0 or 1 <= s <= 8 and s <= -(-k // 128)
                    assert c == 0 or s == 1 or c <= p["clusters"][s] * slots


def test_shared_memory_of_a_cta(plan):
    plan(1, 128, 128)
    for tn in (16, 32, 48, 64, 96, 128):
        for splits in range(1, 9):
            stages, recv, smem = (f(tn, splits) for f in (plan.lib.stages, plan.lib.recv, plan.lib.smem))
            stage = 16384 + tn * 128
            assert 2 <= stages <= 8 and smem == stages * stage + recv + 1024 <= plan.lib.room(tn)
            assert plan.lib.places(tn) <= stages                                    # a stage's barrier never completes twice unseen
            # two CTAs of a pass of 64 rows at most on an SM, one otherwise (1 KB each is the system's; factors and barriers are static)
            per_sm = 2 if tn <= 64 else 1
            assert smem + 64 * tn + 256 <= min(227, (228 - per_sm) / per_sm) * 1024
            if splits == 1:
                assert tn * 512 <= stages * stage                                   # the sums go where the stages were
            else:                                                                   # the last place that is written to
                most = max(rank * -(-(tn // 4) // splits) + q // splits for rank in range(splits) for q in range(tn // 4))
                assert (most * 128 + 127) * 16 + 16 <= recv


def test_shares_of_tensor_memory(plan):
    """At least as large a share of shared memory as of tensor memory; beside a CTA that has all 512 columns nothing fits that wants 32."""
    plan(1, 128, 128)
    for tn in (16, 32, 48, 64, 96, 128):
        for splits in range(1, 9):
            assert plan.lib.smem(tn, splits) + 1024 >= plan.lib.columns(tn) / 512 * 228 * 1024
    assert 228 * 1024 - (plan.lib.pair_smem() + 1024) < 32 / 512 * 228 * 1024 - 2048 and plan.lib.pair_smem() + 512 <= 227 * 1024


@pytest.mark.parametrize("m,k,n", [(2100, 400, 1290), (1025, 272, 3001), (5000, 16, 1000), (1300, 1296, 2056), (300, 640, 22000), (3000, 128, 17000), (20000, 16, 1000), (9000, 272, 1288)])
def test_sizes_of_the_gpu_tests_on_pairs(plan, m, k, n):
    assert plan(m, n, k)["pairs"]


def test_few_rows_stay_with_the_weights_and_many_go_on_pairs(plan):
    assert not plan(1, 1280, 1280)["pairs"] and plan(1, 1280, 1280)["parts"][0] == (0, 10, 4)
    assert not plan(18, 22016, 4096)["pairs"] and plan(18, 22016, 4096)["parts"] == [(0, 148, 1), (148, 24, 5)]
    assert not plan(288, 1280, 3456)["pairs"] and plan(288, 1280, 3456)["parts"][0] == (0, 10, 4)
    assert plan(5460, 12288, 4096)["pairs"] and plan(1 << 24, 16, 128)["pairs"]


@pytest.mark.parametrize("m,k,n", [(18, 4096, 19000), (3, 4000, 20001), (36, 4096, 19000), (100, 4096, 20001)])
def test_sizes_of_the_gpu_tests_in_two_launches(plan, m, k, n):
    assert plan(m, n, k)["parts"][1][1] > 0
