"""Rows and weights in 8 bits with scales for each 128, the norm that makes them and their product, through the public entry points against the
float64 oracle.

Tolerances.  Norm: the sum of squares is a float32 sum whose longest chain has 64 additions and ten shuffles (74 * 2^-24 of it, half of that
of the root), rsqrtf is within 2 units of the last place and the two products round: 2^-17 of y.  Gate: __expf is within 2 + 1.2 |z| units
(2^-16 at |z| = 88), the division within 2: 2^-15 of y; beyond, where e^-z passes float32, |y| is below 2^-115 |x|.  A scale is as far off as y
and rounds once.  A code is the nearest to y / scale: half a step, 2^-4 of the value or 2^-10 of the scale, beside y's own error.  Product: a
block's products are exact in float32 and its 128 additions are within 2^-23 each, 2^-16 of the sum of magnitudes; a scale product and the
addition of a block round, 3 * 2^-24 for each block.  T's own rounding is half a step of it: 2^-8 for bf16, 2^-24 for float32."""
import numpy as np
import pytest
import torch

from oracle import block_quant_oracle as B
from oracle.quant_cache_oracle import e4m3_decode, e4m3_encode
from paper_2511_13587_b200 import binding as vb
from vvs_synth import gen
from vvs_synth.configs import DTYPE_BF16, DTYPE_FP32, ModelShape

pytestmark = pytest.mark.gpu
BF16, F32, E4M3, U8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.uint8
HALF_STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
EPS = 1e-5


@pytest.fixture(scope="module")
def ctxs():
    made = {dt: vb.vvs_create(vb.make_desc(ModelShape("rows", 0, 64, 0, 0, 0, 128, dtype=code), 1, 1))
            for dt, code in ((BF16, DTYPE_BF16), (F32, DTYPE_FP32))}
    yield made
    for c in made.values():
        vb.vvs_destroy(c)


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.view(U8).cpu().numpy() if t.dtype in (E4M3, U8) else t.double().cpu().numpy()


def coded(rows, cols, of_weight=False):
    """Where codes and scales go, filled with what must not stay."""
    s = (-(-rows // 128) if of_weight else rows, -(-cols // 128))
    return torch.full((rows, cols), 0x7F, dtype=U8, device="cuda"), torch.full(s, float("nan"), device="cuda")


def strided(x, more):
    """The same rows, `more` elements further apart, with NaNs between."""
    wide = torch.full((x.shape[0], x.shape[1] + more), 0x7F if x.dtype == U8 else float("nan"), dtype=x.dtype, device="cuda")
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def check_codes(codes, scale, y, rel, block_rows=1, room=0.0):
    """y: what was to be rounded (float64); rel: how far off the kernel's own value may be."""
    codes, scale = host(codes), host(scale)
    _, want = B.quantise(y, block_rows)
    assert (np.abs(scale - want) <= (rel + 2.0 ** -22) * want).all()
    spread = np.repeat(np.repeat(scale, block_rows, axis=0)[:len(y)], 128, axis=1)[:, :y.shape[1]]
    got = e4m3_decode(codes) * spread
    finite = np.isfinite(y)
    to = np.abs(np.where(finite, y, 0.0))
    off = np.abs(got - np.where(finite, y, 0.0))
    assert (off <= np.where(finite, np.maximum(2.0 ** -4 * to, 2.0 ** -10 * spread) * (1 + 2.0 ** -10) + rel * to + room, np.inf)).all()
    assert (codes[y == np.inf] == 0x7E).all() and (codes[y == -np.inf] == 0xFE).all() and (codes[np.isnan(y)] == 0).all()


# ---- norm ----------------------------------------------------------------------------------------------------------------------

SIZES = [(1, 16), (1, 128), (2, 144), (3, 256), (4, 272), (5, 1280), (18, 1376), (77, 4096), (1, 8192), (2, 16400), (1, 32768), (650, 2064), (1500, 320)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", SIZES + [(2500, 1040), (1300, 4096)])
def test_norm(ctxs, dtype, rows, cols):
    rng = gen.rng_for(21, f"norm{rows}{cols}")
    x, r = (dev(rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1))), dtype) for _ in range(2))
    w = dev(1 + 0.3 * rng.standard_normal(cols), dtype)
    for residual in (None, r):
        s, y = B.norm(host(x), None if residual is None else host(residual), host(w), EPS)
        codes, scale = coded(rows, cols)
        sum_out, norm_out = (strided(torch.zeros((rows, cols), dtype=dtype, device="cuda"), 16) for _ in range(2))
        vb.vvs_norm_quant(ctxs[dtype], strided(x, 32), w, EPS, codes, scale, residual=None if residual is None else strided(residual, 8),
                          sum_out=sum_out, norm_out=norm_out)
        check_codes(codes, scale, y, 2.0 ** -17)
        assert (np.abs(host(sum_out) - s) <= HALF_STEP[dtype] * np.abs(s)).all()
        assert (np.abs(host(norm_out) - y) <= (HALF_STEP[dtype] + 2.0 ** -17) * np.abs(y)).all()
        assert sum_out._base[:, cols:].isnan().all() and norm_out._base[:, cols:].isnan().all()
        # outputs that are not asked for, codes behind a stride, outputs in the inputs' places
        codes2, scale2 = strided(codes, 16), torch.zeros_like(scale)
        vb.vvs_norm_quant(ctxs[dtype], x, w, EPS, codes2.view(E4M3) if cols % 16 == 0 else codes2, scale2, residual=residual)
        assert torch.equal(codes2, codes) and torch.equal(scale2, scale) and (codes2._base[:, cols:] == 0x7F).all()
        x2, r2 = x.clone(), r.clone()
        vb.vvs_norm_quant(ctxs[dtype], x2, w, EPS, codes, scale, residual=None if residual is None else r2, sum_out=r2 if residual is not None else None,
                          norm_out=x2)
        assert torch.equal(x2, norm_out) and torch.equal(codes2, codes) and (residual is None or torch.equal(r2, sum_out))
    assert vb.vvs_device_status(ctxs[dtype]) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_of_what_is_not_ordinary(ctxs, dtype):
    rows, cols = 6, 400
    rng = gen.rng_for(22, "odd")
    x = rng.standard_normal((rows, cols)).astype(np.float32)
    x[0], x[1, 300], x[2, 7], x[3], x[4] = 0.0, np.inf, np.nan, 1e30, 1e-30
    x, w = dev(x, dtype), torch.ones(cols, dtype=dtype, device="cuda")
    w[::3] = 0.0
    codes, scale = coded(rows, cols)

    def run(at):
        codes.fill_(0x7F)
        vb.vvs_norm_quant(ctxs[dtype], x[at:at + 1], w, EPS, codes[at:at + 1], scale[at:at + 1])
        return vb.vvs_device_status(ctxs[dtype])
    assert run(0) == 0 and (codes[0] == 0).all() and (scale[0] == 2.0 ** -60).all()      # zeros over sqrt(eps)
    assert run(1) == vb.VVS_DEV_NONFINITE and (codes[1] & 0x7F == 0).all()                # everything is nothing beside an infinity, inf * 0 a NaN
    assert run(2) == vb.VVS_DEV_NONFINITE and (codes[2] & 0x7F == 0).all()
    assert run(3) == vb.VVS_DEV_NONFINITE and (codes[3] & 0x7F == 0).all()                # squares beyond float32
    assert run(4) == 0                                                                    # squares of 0
    check_codes(codes[4:5], scale[4:5], host(x[4:5]) / np.sqrt(EPS) * host(w), 2.0 ** -17)
    assert run(5) == 0
    check_codes(codes[5:], scale[5:], B.norm(host(x[5:]), None, host(w), EPS)[1], 2.0 ** -17)


# ---- rows and weights ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", SIZES + [(9, 11008), (1, 40000), (3000, 1360)])
def test_rows(ctxs, dtype, rows, cols):
    rng = gen.rng_for(23, f"rows{rows}{cols}")
    both = dev(rng.standard_normal((rows, 2 * cols)) * 3, dtype)              # gate and up, side by side
    gate, x = both.split((cols, cols), dim=1)
    for g in (None, gate):
        y = host(x) if g is None else B.gated(host(x), host(g))
        codes, scale = coded(rows, cols)
        codes = strided(codes, 16)
        vb.vvs_rows_quant(ctxs[dtype], x, codes, scale, gate=g)
        check_codes(codes, scale, y, 0.0 if g is None else 2.0 ** -15)
        assert (codes._base[:, cols:] == 0x7F).all()
    assert vb.vvs_device_status(ctxs[dtype]) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gates_far_from_zero(ctxs, dtype):
    z = np.concatenate([np.linspace(-120, 120, 241), [-1e4, 1e4, -3e38, 3e38, 0.0, -0.0, 1e-38], np.zeros(8)]).astype(np.float32)[None, :256]
    x = np.ones_like(z) * np.exp2(np.arange(256) % 7 - 3).astype(np.float32)
    gate, x = dev(z, dtype), dev(x, dtype)
    codes, scale = coded(1, 256)
    vb.vvs_rows_quant(ctxs[dtype], x, codes, scale, gate=gate)
    y = B.gated(host(x), host(gate))
    over = np.abs(y) > 3.4e38                              # 3e38 times a number above 1.1: an infinity in float32
    y = np.where(over, np.copysign(np.inf, y), y)
    check_codes(codes, scale, y, 2.0 ** -15, room=2.0 ** -115 * 16)
    assert vb.vvs_device_status(ctxs[dtype]) == (vb.VVS_DEV_NONFINITE if over.any() else 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 16), (127, 128), (128, 144), (129, 16), (1, 4096), (300, 1376), (1000, 400), (257, 640)])
def test_weights(ctxs, dtype, rows, cols):
    rng = gen.rng_for(24, f"weight{rows}{cols}")
    w = strided(dev(rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1))), dtype), 8)
    codes, scale = coded(rows, cols, True)
    codes = strided(codes, 32)
    vb.vvs_weight_quant(ctxs[dtype], w, codes, scale)
    check_codes(codes, scale, host(w), 0.0, 128)
    assert (codes._base[:, cols:] == 0x7F).all() and vb.vvs_device_status(ctxs[dtype]) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values_that_are_codes_stay_and_what_is_not_finite_is_told(ctxs, dtype):
    """Every e4m3 value times a power of two, 448 of them among each block: the codes themselves.  Between two codes, ties go to the even one."""
    all_codes = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    x = np.zeros((130, 256))
    x[:, :254] = e4m3_decode(all_codes)
    x[:, 255] = 448.0
    x = x * np.exp2(np.arange(130) % 40 - 20)[:, None]
    tie = (e4m3_decode(np.arange(126, dtype=np.uint8)) + e4m3_decode(np.arange(1, 127, dtype=np.uint8))) / 2
    x[1, :126], x[1, 127], x[1, 128:] = tie, 448.0, 0.0
    codes, scale = coded(130, 256)
    vb.vvs_rows_quant(ctxs[dtype], dev(x, dtype), codes, scale)
    for i in range(130):
        for j in (0, 128):
            amax = np.abs(x[i, j:j + 128]).max()
            s = host(scale)[i, j // 128]
            assert s == max(np.float32(amax) / np.float32(448), 2.0 ** -60)
            if amax and np.log2(s) == np.round(np.log2(s)):
                assert (host(codes)[i, j:j + 128] & 0x7F == e4m3_encode(x[i, j:j + 128] / s) & 0x7F).all()
    odd = torch.randn((140, 144), device="cuda")
    odd[3, 5], odd[3, 6], odd[139, 143] = float("inf"), float("nan"), -float("inf")
    odd = odd.to(dtype)
    for call, block_rows in ((vb.vvs_rows_quant, 1), (vb.vvs_weight_quant, 128)):
        assert vb.vvs_device_status(ctxs[dtype]) == 0
        codes, scale = coded(140, 144, block_rows == 128)
        call(ctxs[dtype], odd, codes, scale)
        assert vb.vvs_device_status(ctxs[dtype]) == vb.VVS_DEV_NONFINITE
        check_codes(codes, scale, host(odd), 0.0, block_rows)


# ---- product -------------------------------------------------------------------------------------------------------------------


def operands(rng, rows, cols, outs):
    a = B.quantise(rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1))))
    w = B.quantise(rng.standard_normal((outs, cols)) * np.exp(rng.standard_normal((outs, 1))), 128)
    return [dev(x, F32 if i % 2 else None) for i, x in enumerate((*a, *w))]


def check_product(out, ops, rows=None):
    a_codes, a_scale, w_codes, w_scale = (host(x) for x in ops)
    if rows is not None:
        a_codes, a_scale, out = a_codes[rows], a_scale[rows], out[rows]
    if len(a_codes) * len(w_codes) > 4e6:                    # of large results every seventh row, and the last ones
        rows = np.r_[0:len(a_codes):7, len(a_codes) - 9:len(a_codes)]
        a_codes, a_scale, out = a_codes[rows], a_scale[rows], out[torch.from_numpy(rows).to(out.device)]
    want, room = B.product(a_codes, a_scale, w_codes, w_scale)
    bound = (2.0 ** -16 + 3 * a_scale.shape[1] * 2.0 ** -24) * room + HALF_STEP[out.dtype] * np.abs(want)
    assert (np.abs(host(out) - want) <= bound).all()


PRODUCTS = [(1, 16, 1), (1, 128, 128), (1, 1280, 1280), (2, 144, 127), (8, 112, 129), (15, 4096, 200), (16, 256, 640), (17, 1376, 999), (18, 2064, 384),
            (32, 128, 3000), (33, 320, 130), (40, 5984, 4000), (36, 1280, 1280), (45, 144, 1290), (48, 11008, 512), (49, 640, 300), (64, 1280, 257),
            (64, 11008, 512), (30, 6000, 520), (100, 7008, 400), (10, 8016, 130), (65, 1296, 512), (96, 640, 100), (97, 256, 64), (128, 3456, 300), (129, 128, 1000),
            (200, 1360, 700), (257, 512, 640), (300, 2048, 1000), (513, 384, 520), (1030, 272, 650), (1500, 1040, 1290), (2100, 128, 260),
            # on pairs of CTAs: odd blocks of K, results that end anywhere, tiles of rows and weights that are not full, one tile and many
            (2100, 400, 1290), (1025, 272, 3001), (5000, 16, 1000), (1300, 1296, 2056), (300, 640, 22000), (3000, 128, 17000), (20000, 16, 1000), (9000, 272, 1288)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,outs", PRODUCTS)
def test_product(ctxs, dtype, rows, cols, outs):
    ops = operands(gen.rng_for(25, f"product{rows}{cols}{outs}"), rows, cols, outs)
    out = torch.full((rows + 1, outs), float("nan"), dtype=dtype, device="cuda")[:rows]
    vb.vvs_block_matmul(ctxs[dtype], ops[0], ops[1], vb.make_qweight(ops[2], ops[3]), out)
    check_product(out, ops)
    assert out._base[rows:].isnan().all()
    # rows of codes and of the result further apart: the same bits, nothing between them
    for more in (8, 3):
        far = strided(torch.zeros((rows, outs), dtype=dtype, device="cuda"), more)
        vb.vvs_block_matmul(ctxs[dtype], strided(ops[0], 48).view(E4M3), ops[1], vb.make_qweight(strided(ops[2], 16), ops[3]), far)
        assert torch.equal(far, out) and far._base[:, outs:].isnan().all()
    assert vb.vvs_device_status(ctxs[dtype]) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,outs", [(18, 4096, 19000), (3, 4000, 20001), (36, 4096, 19000), (100, 4096, 20001)])
def test_few_rows_of_many_weights(ctxs, dtype, rows, cols, outs):
    """Two launches: tiles for all SMs, and those left over dealt to all of them.  Right behind other calls on the stream, and in a graph."""
    rng = gen.rng_for(25, f"many{rows}{cols}{outs}")
    codes = [rng.integers(0, 0x7F, n, np.uint8) | rng.integers(0, 2, n, np.uint8) << 7 for n in ((rows, cols), (outs, cols))]
    scale = [np.exp(rng.standard_normal((n, -(-cols // 128)))).astype(np.float32) for n in (rows, -(-outs // 128))]
    ops = [dev(x) for x in (codes[0], scale[0], codes[1], scale[1])]
    w = vb.make_qweight(ops[2], ops[3])
    out, other = (torch.zeros((rows, outs), dtype=dtype, device="cuda") for _ in range(2))
    vb.vvs_block_matmul(ctxs[dtype], ops[0], ops[1], w, out)
    check_product(out, ops)
    g = torch.cuda.CUDAGraph()
    a = torch.zeros_like(ops[0])
    x = torch.zeros((rows, cols), dtype=dtype, device="cuda")
    s = torch.zeros_like(ops[1])
    with torch.cuda.graph(g):
        for _ in range(3):                                    # rows that change right before, results that are overwritten right behind
            a.zero_()
            vb.vvs_block_matmul(ctxs[dtype], a, ops[1], w, other)
            vb.vvs_rows_quant(ctxs[dtype], x, a, s)
            a.copy_(ops[0])
            vb.vvs_block_matmul(ctxs[dtype], a, ops[1], w, other)
            vb.vvs_block_matmul(ctxs[dtype], a, ops[1], w, other)
    for _ in range(3):
        g.replay()
        assert torch.equal(other, out)
    assert vb.vvs_device_status(ctxs[dtype]) == 0


def test_product_of_scales_far_apart_and_of_nan(ctxs):
    rng = gen.rng_for(26, "far")
    ops = operands(rng, 40, 512, 300)
    ops[1] *= torch.exp2(torch.randint(-40, 40, ops[1].shape, device="cuda").float())
    ops[3] *= torch.exp2(torch.randint(-40, 20, ops[3].shape, device="cuda").float())
    out = torch.zeros((40, 300), device="cuda")
    vb.vvs_block_matmul(ctxs[F32], ops[0], ops[1], vb.make_qweight(ops[2], ops[3]), out)
    check_product(out, ops)
    ops[0][7, 300] = 0x7F                                    # a NaN in row 7, one in weight 128
    ops[2][128, 5] = 0xFF
    got = torch.zeros((40, 300), device="cuda")
    vb.vvs_block_matmul(ctxs[F32], ops[0], ops[1], vb.make_qweight(ops[2], ops[3]), got)
    bad = torch.zeros((40, 300), dtype=torch.bool, device="cuda")
    bad[7], bad[:, 128] = True, True
    assert got[bad].isnan().all() and torch.equal(got[~bad], out[~bad])


def test_rows_and_products_beyond_32_bits(ctxs):
    """Rows more than 2^31 elements apart, and a result of more than 2^31 elements."""
    far = (1 << 31) + 64
    rng = gen.rng_for(27, "far apart")
    x = torch.zeros(2 * far + 256, dtype=BF16, device="cuda").as_strided((3, 256), (far, 1))
    x.copy_(torch.randn((3, 256), device="cuda"))
    codes = torch.zeros(2 * far + 256, dtype=U8, device="cuda").as_strided((3, 256), (far, 1))
    scale = torch.zeros((3, 2), device="cuda")
    vb.vvs_rows_quant(ctxs[BF16], x, codes, scale)
    check_codes(codes.contiguous(), scale, host(x.contiguous()), 0.0)
    _, _, w_codes, w_scale = operands(rng, 1, 256, 200)
    out = torch.zeros((3, 200), dtype=BF16, device="cuda")
    vb.vvs_block_matmul(ctxs[BF16], codes, scale, vb.make_qweight(w_codes, w_scale), out)
    check_product(out, [codes.contiguous(), scale, w_codes, w_scale])
    del x, codes
    rows, outs = 70001, 32700
    ops = operands(rng, 64, 128, outs)
    a, s = ops[0].repeat(1094, 1)[:rows].contiguous(), ops[1].repeat(1094, 1)[:rows].contiguous()
    out = torch.zeros((rows, outs), dtype=BF16, device="cuda")
    vb.vvs_block_matmul(ctxs[BF16], a, s, vb.make_qweight(ops[2], ops[3]), out)
    at = [0, 1, 65535, 65700, 69999, 70000]
    check_product(out, [a, s, ops[2], ops[3]], at)
    assert torch.equal(out[64 * 1000:64 * 1001], out[:64]) and torch.equal(out[64 * 1093 - 64:64 * 1093], out[:64])


# ---- together ------------------------------------------------------------------------------------------------------------------


class Layer:
    """Norm, gate / up product, gate, down product: what a layer's second half calls, weights rounded on the way."""

    def __init__(self, ctx, dtype, rows, d, ff, seed):
        rng = gen.rng_for(28, f"layer{rows}{d}{ff}{seed}")
        self.ctx, self.dtype, self.d, self.ff = ctx, dtype, d, ff
        self.x, self.res = (dev(rng.standard_normal((rows, d)), dtype) for _ in range(2))
        self.w, self.w_in, self.w_out = dev(1 + 0.2 * rng.standard_normal(d), dtype), dev(0.05 * rng.standard_normal((2 * ff, d)), dtype), \
            dev(0.05 * rng.standard_normal((d, ff)), dtype)
        self.q_in, self.q_out, self.a, self.h = coded(2 * ff, d, True), coded(d, ff, True), coded(rows, d), coded(rows, ff)
        self.sum, self.y, self.both = self.x.clone(), torch.zeros_like(self.x), torch.zeros((rows, 2 * ff), dtype=dtype, device="cuda")

    def step(self, stream=None):
        vb.vvs_norm_quant(self.ctx, self.x, self.w, EPS, *self.a, residual=self.res, sum_out=self.sum, stream=stream)
        vb.vvs_weight_quant(self.ctx, self.w_in, *self.q_in, stream=stream)         # right before the product that reads it
        vb.vvs_block_matmul(self.ctx, *self.a, vb.make_qweight(*self.q_in), self.both, stream=stream)
        vb.vvs_weight_quant(self.ctx, self.w_out, *self.q_out, stream=stream)
        vb.vvs_rows_quant(self.ctx, self.both[:, self.ff:], *self.h, gate=self.both[:, :self.ff], stream=stream)
        vb.vvs_block_matmul(self.ctx, *self.h, vb.make_qweight(*self.q_out), self.y, stream=stream)

    def result(self):
        return [x.clone() for x in (self.sum, self.y, self.both, *self.a, *self.h)]

    def clear(self):
        for x in (self.y, self.both, *self.a, *self.h, *self.q_in, *self.q_out):
            x.zero_()

    def check(self):
        s, y = B.norm(host(self.x), host(self.res), host(self.w), EPS)
        check_codes(*self.a, y, 2.0 ** -17)
        check_codes(*self.q_in, host(self.w_in), 0.0, 128)
        check_product(self.both, [*self.a, *self.q_in])
        check_codes(*self.h, B.gated(host(self.both[:, self.ff:]), host(self.both[:, :self.ff])), 2.0 ** -15)
        check_product(self.y, [*self.h, *self.q_out])


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype,rows,d,ff", [(BF16, 18, 1280, 3456), (F32, 5, 256, 1024), (BF16, 300, 640, 1376), (BF16, 1100, 512, 864), (BF16, 1, 4096, 1408)])
def test_a_layers_second_half(ctxs, dtype, rows, d, ff):
    """Together, again, in a graph, and on a stream of its own beside another on the same context: the same bits."""
    one, two = (Layer(ctxs[dtype], dtype, rows, d, ff, seed) for seed in (1, 2))
    one.step()
    one.check()
    want = one.result()
    two.step()
    want_two = two.result()
    one.clear()
    one.step()
    assert same(one.result(), want)
    one.clear()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        one.step()
    for _ in range(3):
        one.clear()
        g.replay()
        assert same(one.result(), want)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for layer, s in zip((one, two), streams):
            with torch.cuda.stream(s):
                layer.clear()
                layer.step()
    torch.cuda.synchronize()
    assert same(one.result(), want) and same(two.result(), want_two)
    assert vb.vvs_device_status(ctxs[dtype]) == 0
