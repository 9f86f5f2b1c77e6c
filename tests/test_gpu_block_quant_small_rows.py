"""The norm into 8 bits of rows whose squares float32 does not hold, with little or nothing added to their mean.

Tolerance: that of tests/test_gpu_block_quant.py, 2^-17 of y; a row that is scaled by a power of two is so without rounding."""
import numpy as np
import pytest
import torch

from oracle import block_quant_oracle as B
from paper_2511_13587_b200 import binding as vb
from test_gpu_block_quant import BF16, F32, HALF_STEP, check_codes, coded, ctxs, dev, host  # noqa: F401
from vvs_synth import gen

pytestmark = pytest.mark.gpu


def normed(ctx, x, w, eps, residual=None):
    codes, scale = coded(*x.shape)
    s, y = torch.zeros_like(x), torch.zeros_like(x)
    vb.vvs_norm_quant(ctx, x, w, eps, codes, scale, residual=residual, sum_out=s, norm_out=y)
    return codes, scale, s, y, vb.vvs_device_status(ctx)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-38, 1e-32, 1e-30, 1e-5])
@pytest.mark.parametrize("cols", [16, 144, 272, 4096, 16400])
def test_rows_of_small_numbers(ctxs, dtype, eps, cols):  # noqa: F811
    rng = gen.rng_for(91, f"small{cols}")
    size = np.array([1.0, 1e-10, 1e-15, 2e-16, 1e-18, 1e-20, 1e-25, 1e-30, 1e-36, 1e-38])[:, None]
    x = dev(rng.standard_normal((10, cols)) * size, dtype)
    w = dev(1 + 0.2 * rng.standard_normal(cols), dtype)
    for residual in (None, dev(rng.standard_normal((10, cols)) * size, dtype)):
        codes, scale, s, y, status = normed(ctxs[dtype], x, w, eps, residual)
        total, want = B.norm(host(x) + 0.0, None if residual is None else host(residual), host(w), float(np.float32(eps)))
        assert status == 0
        if dtype == F32 and residual is not None:              # (the sum is a float32 number: what is normalised is that)
            total = (host(x).astype(np.float32) + host(residual).astype(np.float32)).astype(np.float64)
            want = B.norm(total, None, host(w), float(np.float32(eps)))[1]
        check_codes(codes, scale, want, 2.0 ** -17)
        assert (np.abs(host(y) - want) <= (HALF_STEP[dtype] + 2.0 ** -17) * np.abs(want) + 2.0 ** -133).all()       # (half a step of bf16's smallest numbers)
        assert (np.abs(host(s) - total) <= HALF_STEP[dtype] * np.abs(total) + 2.0 ** -134).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_smallest_numbers_and_zeros(ctxs, dtype):  # noqa: F811
    x = torch.zeros((4, 400), dtype=F32, device="cuda")
    x[0], x[1, ::2], x[2, 7] = 2.0 ** -133, -2.0 ** -133, 2.0 ** -133
    x, w = x.to(dtype), torch.ones(400, dtype=dtype, device="cuda")
    codes, scale, _, y, status = normed(ctxs[dtype], x[:3], w, 0.0)
    want = B.norm(host(x[:3]), None, host(w), 0.0)[1]
    assert status == 0 and np.abs(want[0] - 1).max() < 1e-12
    check_codes(codes, scale, want, 2.0 ** -17)
    # nothing over nothing
    codes, scale, s, y, status = normed(ctxs[dtype], x[3:], w, 0.0)
    assert status == vb.VVS_DEV_NONFINITE and (codes == 0).all() and (scale == 2.0 ** -60).all() and y.isnan().all() and (s == 0).all()
    # and beside the smallest number that may be added
    codes, scale, s, y, status = normed(ctxs[dtype], x[3:], w, 1e-45)
    assert status == 0 and (codes == 0).all() and (y == 0).all()
