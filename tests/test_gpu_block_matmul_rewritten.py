"""Products in two parts whose rows, scales and weights are written by the calls right before them, into the same buffers again and again: every
result is that of what was written last.  The scales of the sets lie far apart, so that one set's scale beside another's codes is a result far off."""
import pytest
import torch

from paper_2511_13587_b200 import binding as vb
from test_gpu_block_quant import BF16, E4M3, EPS, F32, HALF_STEP, coded, ctxs, dev  # noqa: F401
from vvs_synth import gen

pytestmark = pytest.mark.gpu


def product64(a, a_scale, w, w_scale):
    """(out, sum of magnitudes) in float64, on the device: the oracle's loops take seconds for a matrix of this size."""
    cols = a.shape[1]
    a = a.view(E4M3).double() * a_scale.double().repeat_interleave(128, 1)[:, :cols]
    w = w.view(E4M3).double() * w_scale.double().repeat_interleave(128, 0)[:len(w)].repeat_interleave(128, 1)[:, :cols]
    return a @ w.T, a.abs() @ w.abs().T


def check_product(out, ops):
    want, room = product64(*ops)
    off = (out.double() - want).abs()
    assert (off <= (2.0 ** -16 + 3 * ops[1].shape[1] * 2.0 ** -24) * room + HALF_STEP[out.dtype] * want.abs()).all()


@pytest.mark.parametrize("dtype,rows,cols,outs", [(BF16, 18, 4096, 19000), (F32, 18, 4096, 19000), (BF16, 36, 4096, 20001), (BF16, 100, 4096, 20001),
                                                  (F32, 65, 4096, 22016)])
def test_rows_that_the_call_before_writes(ctxs, dtype, rows, cols, outs):  # noqa: F811
    ctx, rng = ctxs[dtype], gen.rng_for(81, f"rewritten{rows}{cols}{outs}")
    sets = [dev(rng.standard_normal((rows, cols)) * s, dtype) for s in (1.0, 1e4, 1e-4)]
    one = torch.ones(cols, dtype=dtype, device="cuda")
    w, ws = coded(outs, cols, True)
    vb.vvs_weight_quant(ctx, dev(0.05 * rng.standard_normal((outs, cols)), dtype), w, ws)
    weight = vb.make_qweight(w, ws)
    codes, scale = coded(rows, cols)

    def written(i, codes, scale):
        if i % 2:                                             # normalised rows are of one size whatever the set's: their weight tells them apart
            vb.vvs_norm_quant(ctx, sets[i], one * float(8 ** i), EPS, codes, scale)
        else:
            vb.vvs_rows_quant(ctx, sets[i], codes, scale)

    want = []
    for i in range(3):
        q = coded(rows, cols)
        written(i, *q)
        torch.cuda.synchronize()
        want.append(torch.full((rows, outs), float("nan"), dtype=dtype, device="cuda"))
        vb.vvs_block_matmul(ctx, *q, weight, want[i])
        check_product(want[i], [*q, w, ws])
    results = [torch.zeros((rows, outs), dtype=dtype, device="cuda") for _ in range(12)]

    def run():
        for j, out in enumerate(results):
            written(j % 3, codes, scale)
            vb.vvs_block_matmul(ctx, codes, scale, weight, out)

    def check():
        for j, out in enumerate(results):
            assert torch.equal(out, want[j % 3]), j
            out.zero_()
    for _ in range(5):
        run()
        check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for _ in range(5):
        g.replay()
        check()
    assert vb.vvs_device_status(ctx) == 0


@pytest.mark.parametrize("rows", [18, 100])
def test_weights_and_their_scales_that_the_call_before_writes(ctxs, rows):  # noqa: F811
    ctx, rng, cols, outs = ctxs[BF16], gen.rng_for(82, f"weights{rows}"), 4096, 19000
    sets = [dev(rng.standard_normal((outs, cols)) * s, BF16) for s in (1.0, 1e3)]
    codes, scale = coded(rows, cols)
    vb.vvs_rows_quant(ctx, dev(rng.standard_normal((rows, cols)), BF16), codes, scale)
    w, ws = coded(outs, cols, True)
    weight = vb.make_qweight(w, ws)
    results = [torch.zeros((rows, outs), dtype=BF16, device="cuda") for _ in range(6)]
    for j, out in enumerate(results):
        vb.vvs_weight_quant(ctx, sets[j % 2], w, ws)
        vb.vvs_block_matmul(ctx, codes, scale, weight, out)
    for i in (0, 1):
        vb.vvs_weight_quant(ctx, sets[i], w, ws)
        torch.cuda.synchronize()
        check_product(results[i], [codes, scale, w, ws])
        assert all(torch.equal(out, results[i]) for out in results[i::2])
    assert vb.vvs_device_status(ctx) == 0
