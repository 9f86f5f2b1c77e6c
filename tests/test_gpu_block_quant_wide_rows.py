"""The norm into 8 bits of wide rows: every number of units that a thread may have, in both types."""
import numpy as np
import pytest

from oracle import block_quant_oracle as B
from test_gpu_block_quant import BF16, EPS, F32, HALF_STEP, check_codes, ctxs, dev, host  # noqa: F401
from test_gpu_block_quant_small_rows import normed
from vvs_synth import gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,dtype", [(3, 9008, F32), (700, 12304, F32), (2, 16384, F32), (301, 16384, BF16), (5, 24592, F32), (3, 20000, BF16)])
def test_wide_rows(ctxs, rows, cols, dtype):  # noqa: F811
    rng = gen.rng_for(92, f"wide{rows}{cols}")
    x, r = (dev(rng.standard_normal((rows, cols)), dtype) for _ in range(2))
    w = dev(1 + 0.2 * rng.standard_normal(cols), dtype)
    codes, scale, s, y, status = normed(ctxs[dtype], x, w, EPS, r)
    total, want = B.norm(host(x), host(r), host(w), EPS)
    assert status == 0
    check_codes(codes, scale, want, 2.0 ** -17)
    assert (np.abs(host(s) - total) <= HALF_STEP[dtype] * np.abs(total)).all()
    assert (np.abs(host(y) - want) <= (HALF_STEP[dtype] + 2.0 ** -17) * np.abs(want)).all()
