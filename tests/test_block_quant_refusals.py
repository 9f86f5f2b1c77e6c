"""What the entry points of 8-bit rows, weights and products refuse, on the CPU: the binding by the tensors, the library by what the host sees (its
checks compiled with launchers that do nothing but say that they were reached, so sizes that no memory holds can be asked for)."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from paper_2511_13587_b200 import binding as vb
from paper_2511_13587_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
REACHED, INVALID, SHAPE, ALIGN = 77, -1, -2, -3
ROWS, COLS, OUTS = 5, 144, 200
STAND_INS = """
#include "block_quant.cuh"
namespace vvs {
template <typename T> int launch_norm_quant(const NormQuantArgs&, cudaStream_t) { return 77; }
template <typename T> int launch_rows_quant(const RowsQuantArgs&, cudaStream_t) { return 77; }
template <typename T> int launch_weight_quant(const RowsQuantArgs&, cudaStream_t) { return 77; }
int launch_block_matmul(const BlockMatmulArgs&, cudaStream_t) { return 77; }
template int launch_norm_quant<float>(const NormQuantArgs&, cudaStream_t);
template int launch_norm_quant<__nv_bfloat16>(const NormQuantArgs&, cudaStream_t);
template int launch_rows_quant<float>(const RowsQuantArgs&, cudaStream_t);
template int launch_rows_quant<__nv_bfloat16>(const RowsQuantArgs&, cudaStream_t);
template int launch_weight_quant<float>(const RowsQuantArgs&, cudaStream_t);
template int launch_weight_quant<__nv_bfloat16>(const RowsQuantArgs&, cudaStream_t);
}  // namespace vvs
extern "C" void* a_context() {
  static vvs_ctx c;
  c.desc.dtype = VVS_DTYPE_BF16;
  return &c;
}
"""


# ---- the library ---------------------------------------------------------------------------------------------------------------


@pytest.fixture(scope="module")
def api(tmp_path_factory):
    d = tmp_path_factory.mktemp("api")
    src, lib = str(d / "stand_ins.cu"), str(d / "api.so")
    with open(src, "w") as f:
        f.write(STAND_INS)
    subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-O0", "-shared", os.path.join(build.CSRC, "block_api.cu"), src, "-o", lib], check=True)
    so = C.CDLL(lib)
    for name in ("vvs_norm_quant", "vvs_rows_quant", "vvs_weight_quant", "vvs_block_matmul"):
        getattr(so, name).argtypes = getattr(vb.lib, name).argtypes
    so.a_context.restype = C.c_void_p
    return so


def rows(data=16, row=1 << 20):
    return C.byref(vb.vvs_rows(data, row))


def qrows(codes=16, row=1 << 20, scale=16):
    return C.byref(vb.vvs_qrows(codes, row, scale))


def qweight(codes=16, row=1 << 20, scale=16, n_rows=OUTS, n_cols=COLS):
    return C.byref(vb.vvs_qweight(codes, row, scale, n_rows, n_cols))


def test_norm(api):
    def call(n=ROWS, c=COLS, x=rows(), res=None, weight=16, eps=1e-5, s=None, y=None, out=qrows(), ctx=api.a_context()):
        return api.vvs_norm_quant(ctx, n, c, x, res, weight, eps, s, y, out, None)
    assert call() == REACHED and call(res=rows(), s=rows(), y=rows()) == REACHED and call(eps=0.0) == REACHED
    assert call(c=32768) == REACHED and call(c=32784) == SHAPE and call(c=16) == REACHED
    assert call(n=1 << 30, c=16) == REACHED and call(n=(1 << 30) + 1, c=16) == SHAPE and call(n=1 << 29, c=256) == REACHED and call(n=(1 << 29) + 1, c=256) == SHAPE
    for n, c in [(0, 128), (-1, 128), (5, 0), (5, 8), (5, 129), (5, -128)]:
        assert call(n=n, c=c) == SHAPE, (n, c)
    for bad in (dict(x=None), dict(x=rows(0)), dict(weight=None), dict(out=None), dict(out=qrows(0)), dict(out=qrows(scale=0)), dict(eps=-1e-5),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(res=rows(0)), dict(s=rows(0)), dict(y=rows(0)), dict(ctx=None)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(x=rows(24)), dict(weight=8), dict(out=qrows(8)), dict(out=qrows(scale=18)), dict(x=rows(row=148)), dict(out=qrows(row=152)),
                dict(res=rows(row=1 << 20 | 4)), dict(s=rows(8)), dict(y=rows(row=148))):
        assert call(**bad) == ALIGN, bad
    for bad in (dict(s=rows(row=136)), dict(y=rows(row=0)), dict(out=qrows(row=128)), dict(out=qrows(row=1 << 40))):       # rows that would overlap
        assert call(**bad) == SHAPE, bad
    assert call(n=1, x=rows(row=3), out=qrows(row=1), s=rows(row=0)) == REACHED      # the stride of one row is not looked at
    assert call(x=rows(row=0)) == REACHED and call(out=qrows(scale=20)) == REACHED   # the same row again and again may be read


def test_rows_and_weights(api):
    ctx = api.a_context()
    call = lambda n=ROWS, c=COLS, x=rows(), g=None, out=qrows(), ctx=ctx: api.vvs_rows_quant(ctx, n, c, x, g, out, None)  # noqa: E731
    assert call() == REACHED and call(g=rows()) == REACHED and call(c=1 << 16) == REACHED
    assert call(ctx=None) == INVALID and call(g=rows(0)) == INVALID and call(x=None) == INVALID and call(out=None) == INVALID
    assert call(n=1, c=1 << 30) == REACHED and call(n=1, c=(1 << 30) + 16) == SHAPE
    assert call(n=0) == SHAPE and call(c=100) == SHAPE and call(g=rows(8)) == ALIGN and call(out=qrows(row=143)) == SHAPE
    call = lambda w=rows(), ctx=ctx, **kw: api.vvs_weight_quant(ctx, w, qweight(**kw), None)  # noqa: E731
    assert call() == REACHED and call(n_rows=1, row=0) == REACHED and call(n_rows=65535 * 128) == REACHED
    assert call(n_rows=1, n_cols=1 << 30) == REACHED and call(n_rows=1, n_cols=(1 << 30) + 16) == SHAPE
    assert call(n_rows=65535 * 128 + 1) == SHAPE and call(n_rows=0) == SHAPE and call(n_cols=24) == SHAPE and call(row=128) == SHAPE
    assert call(w=None) == INVALID and call(codes=0) == INVALID and call(scale=0) == INVALID and call(ctx=None) == INVALID
    assert call(w=rows(8)) == ALIGN and call(codes=8) == ALIGN and call(scale=6) == ALIGN and call(row=150) == ALIGN
    assert api.vvs_weight_quant(ctx, rows(), None, None) == INVALID


def test_product(api):
    def call(n=ROWS, a=qrows(), out=rows(), ctx=api.a_context(), **kw):
        return api.vvs_block_matmul(ctx, n, a, qweight(**kw), out, None)
    assert call() == REACHED and call(out=rows(row=OUTS + 1)) == REACHED and call(n=1, a=qrows(row=0), out=rows(row=0)) == REACHED
    assert call(ctx=None) == INVALID and call(a=None) == INVALID and call(out=None) == INVALID and call(out=rows(0)) == INVALID and call(codes=0) == INVALID
    assert call(n=0) == SHAPE and call(n_cols=130) == SHAPE and call(out=rows(row=OUTS - 1)) == SHAPE and call(a=qrows(row=0)) == SHAPE
    assert call(out=rows(2)) == ALIGN and call(a=qrows(row=150)) == ALIGN and call(row=150) == ALIGN
    assert api.vvs_block_matmul(api.a_context(), ROWS, qrows(), None, rows(), None) == INVALID


def test_structures_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "vvs.h")).read(), flags=re.S)
    for struct in (vb.vvs_rows, vb.vvs_qrows, vb.vvs_qweight):
        body = re.search(r"typedef struct %s \{(.*?)\}" % struct.__name__, text, flags=re.S).group(1)
        assert re.findall(r"(\w+)\s*;", body) == [f[0] for f in struct._fields_], struct.__name__


# ---- the binding ---------------------------------------------------------------------------------------------------------------


def t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


CODES, SCALE = t(ROWS, COLS, dtype=torch.uint8), t(ROWS, 2)
CODED = [(dict(codes=t(ROWS, COLS)), "codes.*e4m3"), (dict(codes=t(ROWS, COLS, dtype=torch.float8_e5m2)), "codes.*e4m3"),
         (dict(codes=t(ROWS, COLS, dtype=torch.int8)), "codes.*e4m3"), (dict(codes=t(ROWS, COLS - 16, dtype=torch.uint8)), "codes.*dimension 1"),
         (dict(codes=t(COLS, ROWS, dtype=torch.uint8).t()), "codes.*side by side"), (dict(codes=t(COLS, dtype=torch.uint8)), "codes.*2 dimensions"),
         (dict(scale=t(ROWS, 1)), "scale.*dimension 1"), (dict(scale=t(ROWS - 1, 2)), "scale.*dimension 0"),
         (dict(scale=t(ROWS, 2, dtype=torch.float64)), "scale.*float32"), (dict(scale=t(2, ROWS).t()), "scale.*contiguous"),
         (dict(scale=t(ROWS, 4)[:, :2]), "scale.*contiguous"), ({}, "CUDA")]


@pytest.mark.parametrize("wrong,told", CODED)
def test_what_rows_are_written_to(wrong, told):
    for codes in (CODES, CODES.view(torch.float8_e4m3fn)):
        a = dict(dict(codes=codes, scale=SCALE), **wrong)
        with pytest.raises(ValueError, match=told):
            vb.vvs_rows_quant(None, t(ROWS, COLS), a["codes"], a["scale"], stream=0)
        with pytest.raises(ValueError, match=told):
            vb.vvs_norm_quant(None, t(ROWS, COLS), t(COLS), 1e-5, a["codes"], a["scale"], stream=0)


@pytest.mark.parametrize("name", ["residual", "sum_out", "norm_out"])
def test_norm_tensors(name):
    for wrong in (t(ROWS, COLS + 16), t(ROWS + 1, COLS), t(COLS, ROWS).t(), t(ROWS * COLS)):
        with pytest.raises(ValueError, match=name):
            vb.vvs_norm_quant(None, t(ROWS, COLS), t(COLS), 1e-5, CODES, SCALE, stream=0, **{name: wrong})
    for wrong in (t(COLS - 1), t(1, COLS), t(2 * COLS)[::2]):
        with pytest.raises(ValueError, match="weight"):
            vb.vvs_norm_quant(None, t(ROWS, COLS), wrong, 1e-5, CODES, SCALE, stream=0)


def test_weights():
    w8, ws = t(OUTS, COLS, dtype=torch.uint8), t(2, 2)
    for a, told in (((t(OUTS, COLS), ws), "codes"), ((w8, t(1, 2)), "scale.*dimension 0"), ((w8, t(OUTS, 2)), "scale"), ((w8, ws), "CUDA")):
        with pytest.raises(ValueError, match=told):
            vb.make_qweight(*a)
        with pytest.raises(ValueError, match=told):
            vb.vvs_weight_quant(None, t(OUTS, COLS), *a, stream=0)
    with pytest.raises(TypeError, match="codes"):
        vb.make_qweight(0, ws)


def test_product_tensors():
    w = vb.vvs_qweight(16, COLS, 16, OUTS, COLS)
    for a, told in (((CODES, SCALE, w, t(ROWS, OUTS - 1)), "out.*dimension 1"), ((CODES, SCALE, w, t(ROWS + 1, OUTS)), "out.*dimension 0"),
                    ((CODES[:, :128], SCALE, w, t(ROWS, OUTS)), "codes.*dimension 1"), ((CODES, SCALE, w, t(ROWS, OUTS)), "CUDA")):
        with pytest.raises(ValueError, match=told):
            vb.vvs_block_matmul(None, *a, stream=0)
    for wrong in (vb.vvs_qrows(), b"x" * 12):
        with pytest.raises(TypeError, match="vvs_qweight"):
            vb.vvs_block_matmul(None, CODES, SCALE, wrong, t(ROWS, OUTS), stream=0)
    with pytest.raises(vb.VvsError, match="-2"):
        vb.vvs_block_matmul(None, CODES, SCALE, vb.vvs_qweight(16, COLS, 16, 0, COLS), t(ROWS, OUTS), stream=0)
