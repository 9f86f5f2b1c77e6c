"""Attention over blocks whose scales lie at the ends of what the entry point takes: values' scales of 2^-80 to 2^120 side by side, keys' down to 2^-60,
both kernels, with and without several warps and CTAs for the keys.  Tolerances are the operator's; the sums of p |v| that they are relative to come from
the oracle.  A row's weight on small values has to be right although large ones decide its output: the summed weights show it."""
import numpy as np
import pytest
import torch

from oracle import quant_cache_oracle as Q
from paper_2511_13587_b200 import binding as vb
from test_gpu_quant_cache import BF16, F32, check_attend, ctxs, dev, host, make_cache  # noqa: F401
from vvs_synth import gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows", [(BF16, 3), (F32, 3), (BF16, 40), (F32, 40)])
@pytest.mark.parametrize("v_log2", [[-80] * 16, [120] * 16, [-80, -80, 0, -80, 120, -60, 0, 30] * 2, [-60, 60] * 8])
def test_scales_at_the_ends(ctxs, dtype, rows, v_log2):  # noqa: F811
    rng = gen.rng_for(71, f"ends{rows}{v_log2[:5]}")
    kc, vc, ks, vs = make_cache(rng, 1, 1, 256, 64, 16, [256])
    vc[(vc & 127) > 0x40] = 0x38                               # codes of 2 at most: the largest value is 2^121
    vs[0, 0] = 2.0 ** np.array(v_log2, float)
    ks[0, 0, ::5] = 2.0 ** -60
    q = dev(rng.standard_normal((1, rows, 1, 64)), dtype)
    out, lse = torch.zeros_like(q), torch.zeros((1, rows, 1), device="cuda")
    mass = torch.zeros((1, 1, 256), device="cuda")
    fill = 256 - rows - 1
    lens = torch.tensor([fill], dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_attend(ctxs[dtype], vb.make_qcache(dev(kc), dev(vc), dev(ks), dev(vs), mass), q, out, lens, lse=lse, mass_rows=rows)
    want = Q.attend(kc, vc, ks, vs, host(q), [fill], 16, mass=np.zeros((1, 1, 256)), mass_rows=rows)
    assert vb.vvs_device_status(ctxs[dtype]) == 0
    check_attend(ctxs[dtype], dtype, q, out, lse, mass, want, rows)


@pytest.mark.parametrize("dtype,rows,decay", [(BF16, 2, 1.0), (F32, 2, 0.5), (BF16, 40, 1.0), (BF16, 27, 0.0)])
@pytest.mark.parametrize("order", ["mixed", "rising", "falling", "one large", "one small"])
def test_long_caches_of_scales_far_apart(ctxs, dtype, rows, decay, order):  # noqa: F811
    rng = gen.rng_for(72, f"apart{rows}{order}")
    b, h, cap, block = 1, 2, 2560, 32
    kc, vc, ks, vs = make_cache(rng, b, 1, cap, 64, block, [cap])
    vc[(vc & 127) > 0x40] = 0x38
    n = cap // block
    e = {"mixed": rng.integers(-80, 121, n), "rising": np.linspace(-80, 120, n).astype(int), "falling": np.linspace(120, -80, n).astype(int),
         "one large": np.where(np.arange(n) == 37, 110, -60), "one small": np.where(np.arange(n) == 41, -80, 100)}[order]
    vs[0, 0] = 2.0 ** e.astype(float)
    q = dev(rng.standard_normal((b, rows, h, 64)), dtype)
    out, lse = torch.zeros_like(q), torch.zeros((b, rows, h), device="cuda")
    m0 = np.abs(rng.standard_normal((b, 1, cap))).astype(np.float32)
    mass = dev(m0)
    fill, summed = cap - rows - 5, min(rows, 9)
    lens = torch.tensor([fill], dtype=torch.int32, device="cuda")
    for max_len in (0, 1):
        vb.vvs_quant_cache_attend(ctxs[dtype], vb.make_qcache(dev(kc), dev(vc), dev(ks), dev(vs), mass), q, out, lens, lse=lse, mass_rows=summed,
                                  mass_decay=decay, max_len=max_len)
        want = Q.attend(kc, vc, ks, vs, host(q), [fill], block, mass=m0, mass_rows=summed, mass_decay=decay)
        assert vb.vvs_device_status(ctxs[dtype]) == 0
        check_attend(ctxs[dtype], dtype, q, out, lse, mass, want, rows)
        mass = dev(m0)
