"""Scales and codes bit for bit: a scale is max / 448 and a code the nearest to element / scale, both as float32 divisions round them (numpy's), ties to
the even code.  bf16's elements lie on borders between codes often, and there a quotient that is off by its last bit is another code."""
import numpy as np
import pytest
import torch

from oracle.quant_cache_oracle import e4m3_decode, e4m3_encode
from paper_2511_13587_b200 import binding as vb
from test_gpu_block_quant import BF16, EPS, F32, coded, ctxs, host  # noqa: F401
from vvs_synth import gen

pytestmark = pytest.mark.gpu
CODES = e4m3_decode(np.arange(127, dtype=np.uint8))                     # 0 .. 448
BORDERS = (CODES[1:] + CODES[:-1]) / 2


def by_division(y, block_rows=1):
    """y float32 [rows, cols] -> (codes, scale) by float32 divisions."""
    rows, cols = y.shape
    padded = np.zeros((-(-rows // block_rows) * block_rows, -(-cols // 128) * 128), np.float32)
    padded[:rows, :cols] = y
    blocks = padded.reshape(-1, block_rows, padded.shape[1] // 128, 128)
    scale = np.maximum(np.abs(blocks).max((1, 3)) / np.float32(448), np.float32(2.0 ** -60))
    quotient = blocks / scale[:, None, :, None]
    assert scale.dtype == np.float32 and quotient.dtype == np.float32
    return e4m3_encode(quotient.astype(np.float64)).reshape(padded.shape)[:rows, :cols], scale


def check(codes, scale, y, block_rows=1):
    want, s = by_division(y, block_rows)
    assert np.array_equal(scale.cpu().numpy(), s)
    got = host(codes)
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]


def on_borders(rng, rows, cols):
    """Elements at and right beside the borders of two codes and the codes themselves, of each block's own scale."""
    at = np.concatenate([BORDERS, CODES[:-1]])
    y = rng.choice(at, (rows, cols)) * rng.choice([-1.0, 1.0], (rows, cols))
    y = y.reshape(rows, -1, 16 if cols % 128 else 128)
    y[:, :, 0] = 448.0
    power = rng.uniform(-30, 30, y.shape[:2])
    power = np.where(rng.random(power.shape) < 0.5, np.round(power), power)
    y = (y * np.exp2(power)[:, :, None]).astype(np.float32)
    y[:, :, 1:] = np.nextafter(y[:, :, 1:], y[:, :, 1:] * rng.choice([0.0, 1.0, 2.0], y[:, :, 1:].shape).astype(np.float32))
    return y.reshape(rows, cols)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 16), (18, 1280), (301, 1376), (2000, 1024)])
def test_rows(ctxs, dtype, rows, cols):  # noqa: F811
    rng = gen.rng_for(71, f"codes{rows}{cols}")
    for y in (rng.standard_normal((rows, cols)).astype(np.float32), on_borders(rng, rows, cols)):
        x = torch.from_numpy(y).cuda().to(dtype)
        codes, scale = coded(rows, cols)
        vb.vvs_rows_quant(ctxs[dtype], x, codes, scale)
        check(codes, scale, x.float().cpu().numpy())
    assert vb.vvs_device_status(ctxs[dtype]) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 16), (130, 1280), (1000, 2064)])
def test_weights(ctxs, dtype, rows, cols):  # noqa: F811
    rng = gen.rng_for(72, f"codes{rows}{cols}")
    w = torch.from_numpy((0.02 * rng.standard_normal((rows, cols))).astype(np.float32)).cuda().to(dtype)
    codes, scale = coded(rows, cols, True)
    vb.vvs_weight_quant(ctxs[dtype], w, codes, scale)
    check(codes, scale, w.float().cpu().numpy(), 128)
    assert vb.vvs_device_status(ctxs[dtype]) == 0


@pytest.mark.parametrize("rows,cols", [(1, 128), (77, 1376), (700, 4096)])
def test_norm(ctxs, rows, cols):  # noqa: F811
    """Against the normalised rows that the call gives: in float32 they are what it rounds."""
    rng = gen.rng_for(73, f"codes{rows}{cols}")
    x = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)).cuda()
    w = torch.from_numpy((1 + 0.2 * rng.standard_normal(cols)).astype(np.float32)).cuda()
    codes, scale = coded(rows, cols)
    y = torch.zeros_like(x)
    vb.vvs_norm_quant(ctxs[F32], x, w, EPS, codes, scale, norm_out=y)
    check(codes, scale, y.cpu().numpy())


def test_scales_of_many_maxima(ctxs):  # noqa: F811
    """Maxima of every magnitude whose quotient is above the least scale, the widest and those around powers of two among them."""
    rng = gen.rng_for(74, "maxima")
    m = rng.integers(0x24000000, 0x7F7FFFFF, 1 << 20, dtype=np.int64)          # 2^-55 .. the largest float32
    m[:16] = 0x7F7FFFFF - np.arange(16)
    near = np.arange(0x49, 0xFF)[:, None] * (1 << 23) + np.arange(-64, 64)[None, :]
    m[16:16 + near.size] = near.reshape(-1)
    y = np.zeros((1 << 12, 1 << 15), np.float32).reshape(-1, 128)
    y[:, 77] = m.astype(np.int32).view(np.float32)
    x = torch.from_numpy(y.reshape(1 << 12, -1)).cuda()
    codes, scale = torch.zeros(x.shape, dtype=torch.uint8, device="cuda"), torch.zeros((1 << 12, 1 << 8), device="cuda")
    vb.vvs_rows_quant(ctxs[F32], x, codes, scale)
    want = y[:, 77] / np.float32(448)
    assert want.min() >= 2.0 ** -64 and np.array_equal(scale.cpu().numpy().reshape(-1), np.maximum(want, np.float32(2.0 ** -60)))
    assert (codes.view(-1, 128)[:, 77].cpu().numpy()[want >= 2.0 ** -60] == 0x7E).all()
    assert vb.vvs_device_status(ctxs[F32]) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinities_beside_large_and_small_numbers_and_zeros_with_signs(ctxs, dtype):  # noqa: F811
    for most in (3.3e38, 1e30, 1.0, 1e-18, 0.0):
        y = np.zeros((3, 128), np.float32)
        y[:, 1:5], y[:, 5], y[:, 6], y[:, 7], y[:, 8] = [most, -most, most / 2, -0.0], np.inf, -np.inf, np.nan, -0.0
        x = torch.from_numpy(y).cuda().to(dtype)
        finite = x.float().cpu().numpy()
        inf, nan = np.isinf(finite), np.isnan(finite)
        finite[inf | nan] = 0
        want, s = by_division(finite)
        want[inf] = np.where(np.signbit(y[inf]), 0xFE, 0x7E)
        w, ws = by_division(finite, 128)
        w[inf] = want[inf]
        for call, codes, scale, a, b in ((vb.vvs_rows_quant, *coded(3, 128), want, s), (vb.vvs_weight_quant, *coded(3, 128, True), w, ws)):
            call(ctxs[dtype], x, codes, scale)
            assert np.array_equal(host(codes), a) and np.array_equal(scale.cpu().numpy(), b)
            assert vb.vvs_device_status(ctxs[dtype]) == vb.VVS_DEV_NONFINITE
