"""How many clusters of the 8-bit product's CTAs the device is said to hold: of CTAs that have an SM each, as the plans take it, whatever the rows of a pass
and although two of the smaller CTAs fit an SM."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2511_13587_b200 import build

pytestmark = pytest.mark.gpu
SHIM = """
#include "block_matmul.cu"
namespace vvs {
int launch_block_matmul_pair(const BlockMatmulArgs&, cudaStream_t) { return VVS_OK; }
int make_tmap_bytes_2d(CUtensorMap*, const void*, uint64_t, uint64_t, uint64_t, uint32_t, uint32_t) { return VVS_OK; }
}
template <typename T>
static const int* table(int tn) {
  switch (tn) {
    case 16: return vvs::clusters_of<8, T>();
    case 32: return vvs::clusters_of<16, T>();
    case 48: return vvs::clusters_of<24, T>();
    case 64: return vvs::clusters_of<32, T>();
    case 96: return vvs::clusters_of<48, T>();
    default: return vvs::clusters_of<64, T>();
  }
}
extern "C" int clusters(int tn, int f32, int* out) {
  const int* t = f32 ? table<float>(tn) : table<__nv_bfloat16>(tn);
  for (int i = 1; t && i <= 8; ++i) out[i] = t[i];
  return t != nullptr;
}
"""


def test_clusters_of_ctas_that_have_an_sm_each(tmp_path):
    src, lib = str(tmp_path / "shim.cu"), str(tmp_path / "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-shared", src, "-o", lib], check=True)
    torch.zeros(1, device="cuda")
    so = ctypes.CDLL(lib)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    got = {}
    for tn in (16, 32, 48, 64, 96, 128):
        for f32 in (0, 1):
            t = (ctypes.c_int * 9)()
            assert so.clusters(tn, f32, t)
            got[tn, f32] = list(t)[1:]
    for key, t in got.items():
        assert t == got[128, 0], key                           # of whose CTAs two could not lie on an SM
        assert t[0] == sms and all(1 <= (c + 1) * n <= sms for c, n in enumerate(t))
