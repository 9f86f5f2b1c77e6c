"""Attention over the 8-bit cache for many rows, whose CTAs take an SM each: in a CUDA graph, and on a stream of its own beside verification steps,
whose kernels hold tensor memory too.  Every call gives the bits that it gives alone."""
import numpy as np
import pytest
import torch

from paper_2511_13587_b200 import binding as vb
from test_gpu_quant_cache import BF16, ctxs, dev, make_cache, rope_of, tree_masks  # noqa: F401
from test_gpu_same_bits import _weights
from test_gpu_two_streams import SHAPE, _Program
from vvs_synth import gen

pytestmark = pytest.mark.gpu


class Steps:
    """Appends and attends a tree of 27 rows; every step from the same cache."""

    def __init__(self, ctx, mass_rows, seed):
        rng = gen.rng_for(91, f"beside{mass_rows}{seed}")
        self.ctx, self.mass_rows, self.fills, b, kv, h, hd, t = ctx, mass_rows, [1500, 37], 2, 2, 8, 128, 27
        self.start = [dev(x) for x in make_cache(rng, b, kv, 1600, hd, 32, self.fills)]
        self.cache = [x.clone() for x in self.start] + [torch.zeros((b, kv, 1600), device="cuda")]
        self.qc = vb.make_qcache(*self.cache)
        self.q, self.k, self.v = dev(rng.standard_normal((b, t, h + 2 * kv, hd)), BF16).split((h, kv, kv), dim=2)
        self.rope = vb.make_rope_axes(*(dev(x) for x in rope_of(rng, hd, 3, hd // 2, b, t)))
        self.lens, self.visible = dev(np.array(self.fills, np.int32)), dev(tree_masks(rng, b, t).view(np.int32))
        self.turned, self.out = (torch.zeros((b, t, h, hd), dtype=BF16, device="cuda") for _ in range(2))
        self.lse = torch.zeros((b, t, h), device="cuda")

    def reset(self):
        for x, y in zip(self.cache, self.start):
            x.copy_(y)
        self.cache[4].zero_()
        self.out.zero_()

    def step(self, stream):
        # (an append over the same slots again: the block's scales have grown to what they grow to, the codes are the same)
        vb.vvs_quant_cache_append(self.ctx, self.qc, self.k, self.v, self.lens, rope=self.rope, q=self.q, q_out=self.turned, stream=stream)
        vb.vvs_quant_cache_attend(self.ctx, self.qc, self.turned, self.out, self.lens, visible=self.visible, lse=self.lse, mass_rows=self.mass_rows,
                                  mass_decay=0.0, stream=stream)

    def result(self):
        return [x.clone() for x in (self.out, self.lse, self.turned, *self.cache)]


def same(a, b):
    """By bits: scales of blocks that hold nothing are NaN."""
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("mass_rows", [0, 5])
def test_in_a_graph(ctxs, mass_rows):  # noqa: F811
    steps = Steps(ctxs[BF16], mass_rows, 1)
    steps.step(None)
    want = steps.result()
    steps.reset()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        steps.step(None)
    steps.reset()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert same(steps.result(), want) and vb.vvs_device_status(ctxs[BF16]) == 0
    del g


@pytest.mark.parametrize("mass_rows,images,drafts", [(0, 1, 8), (5, 6, 8), (0, 8, 13)])
def test_beside_verification_steps(ctxs, mass_rows, images, drafts):  # noqa: F811
    program = _Program(_weights(SHAPE, 9100), images, 2, drafts, 9200 + images)
    steps = Steps(ctxs[BF16], mass_rows, 2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    program.step(streams[0])
    steps.step(streams[1])
    torch.cuda.synchronize()
    alone = program.result()
    torch.cuda.synchronize()
    want = steps.result()
    program.hidden.zero_()
    steps.reset()
    torch.cuda.synchronize()
    for _ in range(20):
        program.step(streams[0])
        steps.step(streams[1])
    torch.cuda.synchronize()
    assert same(program.result(), alone) and same(steps.result(), want)
    assert vb.vvs_device_status(ctxs[BF16]) == 0
    program.vb.vvs_destroy(program.ctx)
