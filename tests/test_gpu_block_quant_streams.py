"""Products of 8-bit rows and weights beside verification steps on another stream, whose kernels hold tensor memory and come in clusters too: every
call gives the bits that it gives alone.  And calls that are the first of their process while a stream is captured."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2511_13587_b200 import binding as vb
from test_gpu_block_quant import BF16, ctxs, dev, operands  # noqa: F401
from test_gpu_same_bits import _weights
from test_gpu_two_streams import SHAPE, _Program
from vvs_synth import gen

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Products:
    """Few rows in clusters, a pass of 128 rows, two launches, pairs of CTAs: one after the other, each followed by a norm of its result."""

    SIZES = [(18, 1280, 640), (130, 1040, 1290), (10, 4096, 19000), (1300, 1296, 2056)]

    def __init__(self, ctx):
        self.ctx, self.calls = ctx, []
        for rows, cols, outs in self.SIZES:
            rng = gen.rng_for(61, f"beside{rows}{cols}{outs}")
            if rows * outs < 1e5:
                ops = operands(rng, rows, cols, outs)
            else:
                codes = [dev(rng.integers(0, 0x7F, n, np.uint8)) for n in ((rows, cols), (outs, cols))]
                scale = [dev(np.exp(rng.standard_normal((n, -(-cols // 128)))).astype(np.float32)) for n in (rows, -(-outs // 128))]
                ops = [codes[0], scale[0], codes[1], scale[1]]
            out = torch.zeros((rows, outs), dtype=BF16, device="cuda")
            self.calls.append((ops[0], ops[1], vb.make_qweight(ops[2], ops[3]), out))

    def step(self, stream):
        for a in self.calls:
            vb.vvs_block_matmul(self.ctx, *a, stream=stream)

    def result(self):
        return [a[3].clone() for a in self.calls]

    def reset(self):
        for a in self.calls:
            a[3].zero_()


@pytest.mark.parametrize("images,drafts", [(1, 8), (6, 8), (8, 13)])
def test_beside_verification_steps(ctxs, images, drafts):  # noqa: F811
    program = _Program(_weights(SHAPE, 9300), images, 2, drafts, 9400 + images)
    products = Products(ctxs[BF16])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    program.step(streams[0])
    torch.cuda.synchronize()
    products.step(streams[1])
    torch.cuda.synchronize()
    alone, want = program.result(), products.result()
    program.hidden.zero_()
    products.reset()
    torch.cuda.synchronize()
    for _ in range(15):
        program.step(streams[0])
        products.step(streams[1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(program.result(), alone)) and all(torch.equal(a, b) for a, b in zip(products.result(), want))
    assert vb.vvs_device_status(ctxs[BF16]) == 0
    program.vb.vvs_destroy(program.ctx)


def test_products_of_two_streams(ctxs):  # noqa: F811
    """One context, two streams, the same weights."""
    one, two = Products(ctxs[BF16]), Products(ctxs[BF16])
    one.step(None)
    want = one.result()
    one.reset()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(15):
        for p, s in zip((one, two), streams):
            p.step(s)
    torch.cuda.synchronize()
    for p in (one, two):
        assert all(torch.equal(a, b) for a, b in zip(p.result(), want))
    assert vb.vvs_device_status(ctxs[BF16]) == 0


FIRST = """
import sys, torch
sys.path.insert(0, sys.argv[1])
from paper_2511_13587_b200 import binding as vb
from vvs_synth.configs import ModelShape
ctx = vb.vvs_create(vb.make_desc(ModelShape("rows", 0, 64, 0, 0, 0, 128), 1, 1))
g = torch.Generator(device="cuda")
g.manual_seed(5)
sizes = [(18, 256, 640), (1300, 640, 2056)]
calls = []
for m, k, n in sizes:
    x, r, w = (torch.randn(s, generator=g, device="cuda").to(torch.bfloat16) for s in ((m, k), (m, k), (n, k)))
    q, s = torch.zeros((m, k), dtype=torch.uint8, device="cuda"), torch.zeros((m, -(-k // 128)), device="cuda")
    wq, ws = torch.zeros((n, k), dtype=torch.uint8, device="cuda"), torch.zeros((-(-n // 128), -(-k // 128)), device="cuda")
    calls.append((x, r, torch.ones(k, dtype=torch.bfloat16, device="cuda"), w, q, s, wq, ws, vb.make_qweight(wq, ws), torch.zeros((m, n), dtype=torch.bfloat16, device="cuda")))
def step():
    for x, r, one, w, q, s, wq, ws, qw, out in calls:
        vb.vvs_weight_quant(ctx, w, wq, ws)
        vb.vvs_norm_quant(ctx, x, one, 1e-5, q, s, residual=r)
        vb.vvs_block_matmul(ctx, q, s, qw, out)
        vb.vvs_rows_quant(ctx, x, q, s, gate=r)
        vb.vvs_block_matmul(ctx, q, s, qw, out)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
graph.replay()
torch.cuda.synchronize()
got = [c[-1].clone() for c in calls]
for c in calls:
    c[-1].zero_()
step()
torch.cuda.synchronize()
assert all(torch.equal(a, c[-1]) and a.isfinite().all() and a.any() for a, c in zip(got, calls)) and vb.vvs_device_status(ctx) == 0
print("the same")
"""


def test_first_calls_of_a_process_in_a_capture(ctxs):  # noqa: F811
    r = subprocess.run([sys.executable, "-c", FIRST, ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "the same" in r.stdout, r.stderr[-2000:]
