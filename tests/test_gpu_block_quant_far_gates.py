"""SwiGLU into 8 bits of large elements and gates far below zero: exact to the last gate whose reciprocal is a normal float32 number, 0 beyond.

Tolerance: the exponent of e^-gate is below 126, its product and constant round, 1.3 * 2^-24 of it, times ln 2: 2^-17.2 of y; the exponential, the
reciprocal and two products add 2^-22 each: 2^-17."""
import numpy as np
import pytest
import torch

from oracle import block_quant_oracle as B
from paper_2511_13587_b200 import binding as vb
from test_gpu_block_quant import BF16, F32, check_codes, coded, ctxs, dev, host  # noqa: F401
from vvs_synth import gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("power", [127, 100, 60, 20, 0, -20])
def test_large_elements(ctxs, dtype, power):  # noqa: F811
    rng = gen.rng_for(93, f"far{power}")
    gates = np.concatenate([np.linspace(-87.3, -84, 128), np.linspace(-87, -60, 128), rng.uniform(-87, 87, 128)])
    gates = np.concatenate([gates, rng.permutation(gates)]).reshape(6, 128).astype(np.float32)
    x = (np.exp2(power) * rng.uniform(0.5, 1.0, gates.shape) * rng.choice([-1.0, 1.0], gates.shape)).astype(np.float32)
    gate, x = dev(np.maximum(gates, -87.3), dtype), dev(x, dtype)
    gate.clamp_(min=-87.0 if dtype == BF16 else -87.3)         # (bf16 has -87 and -87.5 there)
    y = B.gated(host(x), host(gate))
    over = np.abs(y) > 3.4e38
    y = np.where(over, np.copysign(np.inf, y), y)
    codes, scale = coded(6, 128)
    vb.vvs_rows_quant(ctxs[dtype], x, codes, scale, gate=gate)
    check_codes(codes, scale, y, 2.0 ** -17)
    assert vb.vvs_device_status(ctxs[dtype]) == (vb.VVS_DEV_NONFINITE if over.any() else 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gates_beyond(ctxs, dtype):  # noqa: F811
    gate = dev(np.concatenate([np.linspace(-200, -87.5, 120), [-1e4, -3e38]]).astype(np.float32), dtype)
    gate = torch.cat([gate, gate[:6]]).repeat(3, 1)
    x = torch.full((3, 128), 2.0 ** 100, device="cuda").to(dtype)
    x[1], x[2] = -3e38, 1.0
    codes, scale = coded(3, 128)
    vb.vvs_rows_quant(ctxs[dtype], x, codes, scale, gate=gate)
    assert (host(codes) & 0x7F == 0).all() and (scale == 2.0 ** -60).all() and vb.vvs_device_status(ctxs[dtype]) == 0
