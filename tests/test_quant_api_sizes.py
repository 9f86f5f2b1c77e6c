"""Host checks of the 8-bit cache's entry points (csrc/quant_api.cu) at the ends of their ranges: compiled with launchers that do nothing but say that
they were reached, so sizes that no memory holds can be asked for without a GPU."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2511_13587_b200 import binding as vb
from paper_2511_13587_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
REACHED, SHAPE = 77, -2
STAND_INS = """
#include "quant_cache.cuh"
namespace vvs {
template <typename T> int launch_rotate_axes(const RotateArgs&, cudaStream_t) { return 77; }
template <typename T> int launch_quant_append(const QAppendArgs&, cudaStream_t) { return 77; }
template <typename T> int launch_quant_attend(const QAttendArgs&, cudaStream_t) { return 77; }
int launch_quant_evict(const QEvictArgs&, cudaStream_t) { return 77; }
template int launch_rotate_axes<float>(const RotateArgs&, cudaStream_t);
template int launch_rotate_axes<__nv_bfloat16>(const RotateArgs&, cudaStream_t);
template int launch_quant_append<float>(const QAppendArgs&, cudaStream_t);
template int launch_quant_append<__nv_bfloat16>(const QAppendArgs&, cudaStream_t);
template int launch_quant_attend<float>(const QAttendArgs&, cudaStream_t);
template int launch_quant_attend<__nv_bfloat16>(const QAttendArgs&, cudaStream_t);
}  // namespace vvs
extern "C" void* a_context() {
  static vvs_ctx c;
  c.desc.dtype = VVS_DTYPE_BF16;
  return &c;
}
"""


@pytest.fixture(scope="module")
def api(tmp_path_factory):
    d = tmp_path_factory.mktemp("api")
    src, lib = str(d / "stand_ins.cu"), str(d / "api.so")
    with open(src, "w") as f:
        f.write(STAND_INS)
    subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-O0", "-shared", os.path.join(build.CSRC, "quant_api.cu"), src, "-o", lib], check=True)
    so = C.CDLL(lib)
    for name in ("vvs_rotate_axes", "vvs_quant_cache_append", "vvs_quant_cache_attend", "vvs_quant_cache_evict"):
        getattr(so, name).argtypes = getattr(vb.lib, name).argtypes
    so.a_context.restype = C.c_void_p
    return so


def heads():
    return C.byref(vb.vvs_heads(16, 0, 0, 0))


def cache(n_seqs=1, n_heads=1, cap=128):
    return C.byref(vb.vvs_qcache(16, 16, 16, 16, 16, 16, n_seqs, n_heads, 64, cap, 128))


def attend(api, n_rows, n_heads, kv):
    return api.vvs_quant_cache_attend(api.a_context(), cache(n_heads=kv), heads(), heads(), 16, n_rows, n_heads, None, None, None, None, 0.0, 0, 1.0, 0, None)


def test_attention_fills_the_grid_at_most(api):
    """Cached heads x tiles of rows are one dimension of the grid: 16 rows a tile where there are no more, else 32 (128 in the kernel for many)."""
    for kv, share, n_rows in [(65535, 1, 1), (65535, 1, 16), (32767, 2, 8), (61680, 1, 17), (30840, 1, 34), (1, 1, 65535 * 16), (4, 4, 65535)]:
        rows = share * n_rows
        assert kv * (1 if rows <= 16 else -(-rows // 32)) <= 65535
        assert attend(api, n_rows, kv * share, kv) == REACHED, (kv, share, n_rows)
    for kv, share, n_rows in [(65536, 1, 1), (70000, 1, 1), (65536, 2, 4), (1048560, 1, 1), (61681, 1, 17), (1, 1, 65535 * 16 + 1)]:
        assert attend(api, n_rows, kv * share, kv) == SHAPE, (kv, share, n_rows)


def test_rows_of_queries_are_counted_in_32_bits(api):
    rope = vb.vvs_rope_axes(16, 16, 16, 1, 32, 0)

    def append(n_seqs, n_rows, q):
        return api.vvs_quant_cache_append(api.a_context(), cache(n_seqs=n_seqs), heads(), heads(), 16, n_rows, None, None, None, C.byref(rope), 1,
                                          heads() if q else None, heads() if q else None, None)
    assert append(65535, 32768, True) == REACHED and append(65535, 32769, True) == SHAPE and append(65535, 32769, False) == REACHED
    assert append(128, 1 << 24, True) == SHAPE and append(127, 1 << 24, True) == REACHED

    def rotate(n_seqs, n_rows):
        return api.vvs_rotate_axes(api.a_context(), C.byref(rope), n_seqs, n_rows, 1, 0, 64, heads(), heads(), None, None, None)
    assert rotate(65535, 32768) == REACHED and rotate(65535, 32769) == SHAPE
