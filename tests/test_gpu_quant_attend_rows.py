"""Attention over the 8-bit cache for many query rows of a cached head (the kernel that has 128 of them a tile), against the float64 oracle.
Tolerances are those of the few rows' tests: the operator is the same."""
import numpy as np
import pytest
import torch

from oracle import quant_cache_oracle as Q
from paper_2511_13587_b200 import binding as vb
from test_gpu_quant_cache import BF16, check_attend, ctxs, dev, host, make_cache, tree_masks  # noqa: F401
from vvs_synth import gen

pytestmark = pytest.mark.gpu

# (rows, heads, cached heads, hd, block, fills, row counts, first slots, tree, mass rows, decay)
MANY = [
    (33, 1, 1, 128, 16, [0], None, None, False, 0, 1.0),
    (33, 2, 2, 64, 16, [1, 30], [33, 0], None, False, 0, 1.0),
    (27, 8, 2, 128, 128, [700, 129], None, None, True, 0, 1.0),
    (27, 8, 2, 128, 128, [700, 129], [27, 11], [13, 129], True, 1, 0.5),
    (32, 8, 2, 64, 32, [64, 63, 0], [32, 1, 17], [16, 63, 0], True, 32, 0.0),
    (64, 4, 2, 128, 64, [64, 1000], [64, 63], [0, 640], False, 0, 1.0),
    (64, 4, 2, 64, 64, [64, 1000], [5, 64], [0, 999], False, 3, 1.0),
    (129, 1, 1, 128, 32, [300], None, [33], False, 129, 0.75),
    (43, 6, 2, 64, 16, [2500, 17], None, [0, 1], False, 2, 0.0),
    (5, 40, 1, 128, 128, [3000], [4], [100], True, 5, 1.0),
    (50, 2, 1, 128, 64, [5000, 77], [50, 49], [0, 3], False, 50, 0.25),
    (30, 8, 2, 64, 16, [4000], None, [1777], True, 9, 0.0),
]


@pytest.mark.parametrize("t,h,kv,hd,block,fills,counts,firsts,tree,mass_rows,decay", MANY)
def test_many_rows(ctxs, t, h, kv, hd, block, fills, counts, firsts, tree, mass_rows, decay):  # noqa: F811
    rng = gen.rng_for(41, f"many{t}{h}{kv}{hd}{block}{tree}")
    b, cap = len(fills), -(-(max(fills) + t) // block) * block + block
    n = [t] * b if counts is None else counts
    kc, vc, ks, vs = make_cache(rng, b, kv, cap, hd, block, np.array(fills) + n)
    for i in range(b):                                     # codes of NaN where no row looks
        lo = 0 if firsts is None else firsts[i]
        kc[i, :, :lo], vc[i, :, :lo] = 0x7f, 0xff
        kc[i, :, fills[i] + n[i]:], vc[i, :, fills[i] + n[i]:] = 0xff, 0x7f
    q = dev(rng.standard_normal((b, t, h, hd)) * 2.0, BF16)
    m0 = np.abs(rng.standard_normal((b, kv, cap))).astype(np.float32)
    vis = tree_masks(rng, b, t) if tree else None
    i32 = lambda x: None if x is None else dev(np.array(x, np.int32))
    want = Q.attend(kc, vc, ks, vs, host(q), fills, block, row_count=counts, first_slot=firsts, visible=vis, mass=m0, mass_rows=mass_rows,
                    mass_decay=decay)
    bits = None
    for max_len in (0, 1, 200, max(fills) + t, 0):
        out, lse = torch.full((b, t, h, hd), float("nan"), dtype=BF16, device="cuda"), torch.full((b, t, h), float("nan"), device="cuda")
        mass = dev(m0)
        vb.vvs_quant_cache_attend(ctxs[BF16], vb.make_qcache(dev(kc), dev(vc), dev(ks), dev(vs), mass), q, out, i32(fills), row_count=i32(counts),
                                  first_slot=i32(firsts), visible=None if vis is None else dev(vis.view(np.int32)), lse=lse, mass_rows=mass_rows,
                                  mass_decay=decay, max_len=max_len)
        assert vb.vvs_device_status(ctxs[BF16]) == 0
        check_attend(ctxs[BF16], BF16, q, out, lse, mass, want, mass_rows)
        if max_len == 0:
            assert bits is None or all(torch.equal(x, y) for x, y in zip(bits, (out, lse, mass)))
            bits = (out, lse, mass)


def test_scores_that_climb(ctxs):  # noqa: F811
    """Every tile's largest score far above the last one's: references move again and again, weights of 2^-40 and 1 in one row."""
    rng = gen.rng_for(42, "climb")
    hd, block, fill, t, h = 128, 64, 1500, 40, 2
    kc, vc, ks, vs = make_cache(rng, 1, 1, 1600, hd, block, np.array([fill + t]))
    ks[:] = np.float32(2.0) ** (np.arange(ks.shape[-1]) - 16)
    vs[:] = np.float32(2.0) ** rng.integers(-30, 30, vs.shape)
    q = dev(rng.standard_normal((1, t, h, hd)), BF16)
    q[:, 3] = float("nan")
    q[:, 5] = 0
    out, lse = torch.zeros((1, t, h, hd), dtype=BF16, device="cuda"), torch.zeros((1, t, h), device="cuda")
    lens = dev(np.array([fill], np.int32))
    vb.vvs_quant_cache_attend(ctxs[BF16], vb.make_qcache(dev(kc), dev(vc), dev(ks), dev(vs)), q, out, lens, lse=lse)
    assert out[:, 3].isnan().all()
    live = [r for r in range(t) if r != 3]
    qh = host(q)
    qh[:, 3] = 0
    want = Q.attend(kc, vc, ks, vs, qh, [fill], block)
    spread = want[3][:, live]
    room = 2.0 ** -8 * np.abs(want[0][:, live]) + (2.0 ** -11 + 2.0 ** -13) * spread
    assert (np.abs(host(out)[:, live] - want[0][:, live]) <= room).all()
    # log-sum-exp of scores up to thousands: float32 holds 24 bits of them
    np.testing.assert_allclose(host(lse)[:, live], want[1][:, live], rtol=2.0 ** -20, atol=2.0 ** -15)
