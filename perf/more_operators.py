"""The measured work of the 8-bit rows, weights and products, through the public entry points of `paper_2511_13587_b200.binding`, and the
same operators in plain torch.

A case is a dict of plain values; `op` names the operator:

  norm     `vvs_norm_quant`: a residual is added, the sum normalised by its root mean square, and the row rounded to e4m3 with one scale
           for each 128 columns
  rows     `vvs_rows_quant`: rows, or silu(gate) * rows, rounded the same way
  weight   `vvs_weight_quant`: a weight matrix rounded to e4m3 with one scale for each block of 128 x 128
  product  `vvs_block_matmul`: rows in 8 bits times the transpose of weights in 8 bits, by the scales of their blocks

Definitions.  sum = x + residual; y = sum / sqrt(mean(sum^2) + eps) * weight, from the sum before it is rounded.  A scale is the block's
largest magnitude / 448, 2^-60 at least; a code is the nearest e4m3 value to element / scale.  The last block of a row (of the rows, too, in
a weight matrix) may be short.  out[m, n] = sum over the blocks b of a_scale[m, b] * w_scale[n / 128, b] * sum over b's columns of
a[m, k] * w[n, k].
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
EPS = 1e-5


# ---------------------------------------------------------------------------------------------
# the cases


def listed():
    def c(name, op, rows, cols, **more):
        return dict(name=name, op=op, rows=rows, cols=cols, f32=False, **more)
    return [
        # the nine rows of a verified block, one image with guidance, at the width of 1280: latency is what counts
        c("norm step xl", "norm", 18, 1280, residual=True, keep=False),
        # a prompt of several clips at the width of 4096, the sum kept for the next layer
        c("norm prompt 7b", "norm", 10408, 4096, residual=True, keep=False),
        # a float32 context, an odd number of rows, a last block of 96 columns; the first norm of a model (no residual), its rows wanted too
        dict(c("norm odd float32", "norm", 77, 1376, residual=False, keep=True), f32=True),
        # the inner rows of the same step's SwiGLU: gate and up side by side, as one projection leaves them
        c("gate step xl", "rows", 18, 3456, gate=True),
        # those of a prompt at the inner width of 11008
        c("gate prompt 7b", "rows", 5460, 11008, gate=True),
        # attention's output of sixteen images with guidance, on its way to the output projection
        c("rows batch 7b", "rows", 288, 4096, gate=False),
        # weights as a program loads them: the output projection of the narrow model
        c("weight out xl", "weight", 1280, 1280),
        # gate and up of the wide one
        c("weight gate up 7b", "weight", 22016, 4096),
        # one token through an output projection: the smallest product
        c("product token xl", "product", 1, 1280, outs=1280),
        # a verified block through gate and up
        c("product step 7b", "product", 18, 4096, outs=22016),
        # sixteen images with guidance, the same block, through the narrow model's down projection
        c("product batch xl", "product", 288, 3456, outs=1280),
        # a prompt of four clips through the wide model's q, k and v
        c("product prompt 7b", "product", 5460, 4096, outs=12288),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(("norm", "rows", "weight", "product", "product"))
    cols = rng.choice((256, 320, 1280, 4096, 16 * _log_int(rng, 4, 688), 16 * _log_int(rng, 4, 688)))
    c = dict(op=op, rows=_log_int(rng, 1, 10408), cols=cols, f32=rng.random() < 0.25)
    if op == "norm":
        c.update(residual=rng.random() < 0.7, keep=rng.random() < 0.3)
        c["rows"] = min(c["rows"], 10408 * 4096 // cols // (2 if c["f32"] else 1) // (2 if c["keep"] else 1))
    elif op == "rows":
        c["gate"] = rng.random() < 0.6
        c["rows"] = min(c["rows"], 5460 * 11008 // cols // (2 if c["f32"] else 1))
    elif op == "weight":
        c["rows"] = min(_log_int(rng, 1, 22016), 22016 * 4096 // cols // (2 if c["f32"] else 1))
    else:
        c["outs"] = _log_int(rng, 16, 22016)
        c["rows"] = max(1, min(c["rows"], 5460 * 12288 * 4096 // (cols * c["outs"]), 5460 * 12288 // c["outs"] // (2 if c["f32"] else 1)))
    return c


# ---------------------------------------------------------------------------------------------
# the inputs


class State:
    pass


def _blocks(cols):
    return -(-cols // BLOCK)


def _rows_scaled(y):
    """32-bit rows -> (codes, scale [rows, blocks]): a scale for each 128 columns."""
    rows, cols = y.shape
    n = _blocks(cols)
    padded = torch.nn.functional.pad(y, (0, n * BLOCK - cols)).view(rows, n, BLOCK)
    scale = (padded.abs().amax(-1) / 448.0).clamp(min=2.0 ** -60)
    codes = (padded / scale.unsqueeze(-1)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return codes.view(rows, n * BLOCK)[:, :cols].contiguous(), scale


def _weight_scaled(w):
    """A 32-bit matrix -> (codes, scale [blocks of rows, blocks of columns])."""
    rows, cols = w.shape
    m, n = _blocks(rows), _blocks(cols)
    padded = torch.nn.functional.pad(w, (0, n * BLOCK - cols, 0, m * BLOCK - rows)).view(m, BLOCK, n, BLOCK)
    scale = (padded.abs().amax(dim=(1, 3)) / 448.0).clamp(min=2.0 ** -60)
    codes = (padded / scale[:, None, :, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return codes.view(m * BLOCK, n * BLOCK)[:rows, :cols].contiguous(), scale


def prepare(case, seed):
    s = State()
    s.case = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    rows, cols, op = case["rows"], case["cols"], case["op"]
    s.dtype = torch.float32 if case["f32"] else torch.bfloat16

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def empty(*shape, dtype=None):
        return torch.zeros(shape, dtype=dtype or s.dtype, device="cuda")

    channel = torch.exp(0.5 * normal(cols))                 # some channels are larger than others,
    token = torch.exp(0.5 * normal(rows, 1))                # and some tokens
    if op == "product":
        s.a_codes, s.a_scale = _rows_scaled(normal(rows, cols) * channel * token)
        s.w_codes, s.w_scale = _weight_scaled(0.02 * normal(case["outs"], cols))
        s.out, s.w = empty(rows, case["outs"]), None
        return s
    if op == "weight":
        s.x = (0.02 * normal(rows, cols) * torch.exp(0.3 * normal(rows, 1))).to(s.dtype)
        s.codes, s.scale = empty(rows, cols, dtype=torch.float8_e4m3fn), empty(_blocks(rows), _blocks(cols), dtype=torch.float32)
        return s
    s.codes, s.scale = empty(rows, cols, dtype=torch.float8_e4m3fn), empty(rows, _blocks(cols), dtype=torch.float32)
    if op == "norm":
        s.x = (normal(rows, cols) * channel * token).to(s.dtype)
        s.residual = (2.0 * normal(rows, cols) * channel * token).to(s.dtype) if case["residual"] else None
        s.weight = (1.0 + 0.2 * normal(cols)).to(s.dtype)
        s.sum_out = empty(rows, cols) if case["residual"] else None
        s.norm_out = empty(rows, cols) if case["keep"] else None
    elif case["gate"]:
        both = normal(rows, 2 * cols) * token
        both[:, cols:] *= channel
        s.gate, s.x = both.to(s.dtype).split((cols, cols), dim=1)
    else:
        s.gate, s.x = None, (normal(rows, cols) * channel * token).to(s.dtype)
    return s


# ---------------------------------------------------------------------------------------------
# plain forms, in 32 bits


def _plain(s):
    case = s.case
    if case["op"] == "norm":
        total = s.x.float() if s.residual is None else s.x.float() + s.residual.float()
        y = total * torch.rsqrt(total.square().mean(-1, keepdim=True) + EPS) * s.weight.float()
        codes, scale = _rows_scaled(y)
        more = {} if s.residual is None else dict(sum=total.to(s.dtype))
        if case["keep"]:
            more["norm"] = y.to(s.dtype)
        return dict(codes=codes, scale=scale, **more)
    if case["op"] == "rows":
        y = s.x.float()
        if s.gate is not None:
            gate = s.gate.float()
            y = gate / (1.0 + torch.exp(-gate)) * y
        codes, scale = _rows_scaled(y)
        return dict(codes=codes, scale=scale)
    if case["op"] == "weight":
        codes, scale = _weight_scaled(s.x.float())
        return dict(codes=codes, scale=scale)
    cols, outs = case["cols"], case["outs"]
    a = s.a_codes.float() * s.a_scale.repeat_interleave(BLOCK, dim=1)[:, :cols]
    w = s.w_codes.float() * s.w_scale.repeat_interleave(BLOCK, dim=0)[:outs].repeat_interleave(BLOCK, dim=1)[:, :cols]
    return dict(out=torch.matmul(a, w.t()).to(s.dtype))


# ---------------------------------------------------------------------------------------------
# the framework's calls

_contexts = {}


def _context(dtype):
    """A decoding program has one context; these operators need its storage type and its status word."""
    from paper_2511_13587_b200 import binding as vb
    from vvs_synth.configs import DTYPE_BF16, DTYPE_FP32, ModelShape
    if dtype not in _contexts:
        shape = ModelShape("rows", 0, 64, 0, 0, 0, 128, dtype=DTYPE_FP32 if dtype == torch.float32 else DTYPE_BF16)
        _contexts[dtype] = vb, vb.vvs_create(vb.make_desc(shape, 1, 1))
    return _contexts[dtype]


def _own(s):
    vb, ctx = _context(s.dtype)
    case = s.case
    if case["op"] == "norm":
        vb.vvs_norm_quant(ctx, s.x, s.weight, EPS, s.codes, s.scale, residual=s.residual, sum_out=s.sum_out, norm_out=s.norm_out)
        more = {} if s.residual is None else dict(sum=s.sum_out)
        if case["keep"]:
            more["norm"] = s.norm_out
        return dict(codes=s.codes, scale=s.scale, **more)
    if case["op"] == "rows":
        vb.vvs_rows_quant(ctx, s.x, s.codes, s.scale, gate=s.gate)
        return dict(codes=s.codes, scale=s.scale)
    if case["op"] == "weight":
        vb.vvs_weight_quant(ctx, s.x, s.codes, s.scale)
        return dict(codes=s.codes, scale=s.scale)
    if s.w is None:
        s.w = vb.make_qweight(s.w_codes, s.w_scale)
    vb.vvs_block_matmul(ctx, s.a_codes, s.a_scale, s.w, s.out)
    return dict(out=s.out)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    rows, cols = case["rows"], case["cols"]
    es = 4 if case["f32"] else 2
    n = rows * cols
    if case["op"] == "norm":
        return {"bytes": n * (es * (1 + 2 * case["residual"] + case["keep"]) + 1) + cols * es + rows * _blocks(cols) * 4, "flops": 8 * n}
    if case["op"] == "rows":
        return {"bytes": n * (es * (1 + case["gate"]) + 1) + rows * _blocks(cols) * 4, "flops": (8 if case["gate"] else 3) * n}
    if case["op"] == "weight":
        return {"bytes": n * (es + 1) + _blocks(rows) * _blocks(cols) * 4, "flops": 3 * n}
    outs = case["outs"]
    return {"bytes": n + outs * cols + rows * outs * es + (rows + _blocks(outs)) * _blocks(cols) * 4, "flops": 2.0 * n * outs}


# ---------------------------------------------------------------------------------------------
# from the definitions, in 64 bits.  A code is given as the number that it was rounded from, element / scale.


def _exact_blocks(y, dims):
    """y / scale and scale, block by block; `dims`: the dimensions that are cut into blocks."""
    scale = y.abs()
    for d in dims:
        scale = torch.stack([part.amax(dim=d) for part in scale.split(BLOCK, dim=d)], dim=d)
    scale = torch.clamp(scale / 448.0, min=2.0 ** -60)
    spread = scale
    for d in dims:
        at = torch.arange(y.shape[d], device=y.device) // BLOCK
        spread = spread.index_select(d, at)
    return dict(codes=y / spread, scale=scale)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "weight":
        return _exact_blocks(s.x.double(), (0, 1))
    if case["op"] == "rows":
        y = s.x.double()
        if s.gate is not None:
            y = y * torch.nn.functional.silu(s.gate.double())
        return _exact_blocks(y, (1,))
    if case["op"] == "norm":
        total = s.x.double()
        if s.residual is not None:
            total = total + s.residual.double()
        length = torch.linalg.vector_norm(total, dim=1, keepdim=True)
        y = total * s.weight.double() / torch.sqrt(length * length / case["cols"] + EPS)
        out = _exact_blocks(y, (1,))
        if s.residual is not None:
            out["sum"] = total
        if case["keep"]:
            out["norm"] = y
        return out
    out = torch.zeros((case["rows"], case["outs"]), dtype=torch.float64, device="cuda")
    for b in range(_blocks(case["cols"])):
        at = slice(b * BLOCK, min(case["cols"], (b + 1) * BLOCK))
        w_scale = s.w_scale[:, b].double()[torch.arange(case["outs"], device="cuda") // BLOCK]
        out += torch.matmul(s.a_codes[:, at].double(), s.w_codes[:, at].double().t()) * s.a_scale[:, b:b + 1].double() * w_scale
    return dict(out=out)
