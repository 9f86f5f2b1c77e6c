"""Products whose scales are as far from one as may be: the product of a row's and a weight's scale is a float32 number, normal or 0, and nothing is lost
on the way.  Every kernel; the bound is that of tests/test_gpu_block_quant.py, to which a result that is no normal number adds half of the smallest
number for each block."""
import numpy as np
import pytest
import torch

from paper_2511_13587_b200 import binding as vb
from test_gpu_block_matmul_rewritten import product64
from test_gpu_block_quant import F32, ctxs, dev  # noqa: F401
from vvs_synth import gen

pytestmark = pytest.mark.gpu
SIZES = [(20, 512, 300), (100, 1296, 400), (18, 4096, 19000), (1300, 1296, 2056)]         # few rows, a pass of 128, two parts, pairs


@pytest.mark.parametrize("rows,cols,outs", SIZES)
@pytest.mark.parametrize("a_power,w_power", [(-62, -63), (-140, 30), (60, -60), (-126, 1), (40, 50), (100, -4), (-60, 127)])
def test_product_of_scales(ctxs, rows, cols, outs, a_power, w_power):  # noqa: F811
    rng = gen.rng_for(94, f"scales{rows}{cols}{outs}{a_power}")
    blocks = -(-cols // 128)
    a, w = (rng.integers(0, 0x7F, n, np.uint8) | rng.integers(0, 2, n, np.uint8) << 7 for n in ((rows, cols), (outs, cols)))
    a_scale = (rng.uniform(1, 2, (rows, blocks)) * np.exp2(a_power)).astype(np.float32)
    w_scale = (rng.uniform(1, 2, (-(-outs // 128), blocks)) * np.exp2(w_power)).astype(np.float32)
    a_scale[0], w_scale[0, 0] = 0.0, 0.0
    assert np.isfinite(a_scale).all() and np.isfinite(w_scale).all()
    ops = [dev(t) for t in (a, a_scale, w, w_scale)]
    out = torch.full((rows, outs), float("nan"), device="cuda")
    vb.vvs_block_matmul(ctxs[F32], ops[0], ops[1], vb.make_qweight(ops[2], ops[3]), out)
    want, room = product64(*ops)
    bound = (2.0 ** -16 + 3 * blocks * 2.0 ** -24) * room + 2.0 ** -24 * want.abs() + blocks * 2.0 ** -150
    assert ((out.double() - want).abs() <= bound).all() and (out[0] == 0).all()
    assert vb.vvs_device_status(ctxs[F32]) == 0
