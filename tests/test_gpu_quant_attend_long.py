"""Weights summed over a cache so long that the bytes of its scores pass 32 bits, with a `max_len` that says less than the truth: one CTA walks
17 million keys.  Checked against the same operator in float64 on the device, a part of the keys at a time.

Tolerances: a lane adds the weights of 2^20 keys one by one to a float32 sum.  Every addition rounds by 2^-24 of the sum at most; as a random walk
that is 2^10 * 2^-24 of it, and 2^-9 is kept for a row's log-sum and for a weight relative to its value.  Outputs: 2^-8 |out| for bf16 and 2^-9 + 2^-11 of
sum p|v| (weights as halves, 2^-11, beside the sums)."""
import numpy as np
import pytest
import torch

from paper_2511_13587_b200 import binding as vb
from test_gpu_quant_cache import BF16, ctxs  # noqa: F401

pytestmark = pytest.mark.gpu


def test_scores_that_pass_32_bits(ctxs):  # noqa: F811
    cap, hd, rows, block = (1 << 24) + 4096, 64, 32, 128
    fill = cap - rows - 5
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    k, v = (torch.randint(0, 256, (1, 1, cap, hd), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
    for c in (k, v):
        c[(c & 127) > 0x58] = 0x30                             # codes up to 16, no NaN
    ks, vs = (torch.full((1, 1, cap // block), 2.0 ** -4, device="cuda") for _ in range(2))
    q = (torch.randn((1, rows, 1, hd), generator=g, device="cuda") * 0.5).to(BF16)
    mass = torch.zeros((1, 1, cap), device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros((1, rows, 1), device="cuda")
    lens = torch.tensor([fill], dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_attend(ctxs[BF16], vb.make_qcache(k, v, ks, vs, mass), q, out, lens, lse=lse, mass_rows=rows, max_len=1)
    assert vb.vvs_device_status(ctxs[BF16]) == 0
    end, part = fill + rows, 1 << 20
    qd = q[0, :, 0].double() / 8.0

    def scores(lo, hi):
        s = qd @ (k[0, 0, lo:hi].view(torch.float8_e4m3fn).double() * 2.0 ** -4).T
        at, t = torch.arange(lo, hi, device="cuda"), torch.arange(rows, device="cuda").view(-1, 1)
        return s.masked_fill(at - fill > t, -np.inf)

    parts = [(lo, min(end, lo + part)) for lo in range(0, end, part)]
    want = torch.stack([torch.logsumexp(scores(*p), dim=1) for p in parts]).logsumexp(dim=0)
    assert (lse[0, :, 0].double() - want).abs().max() <= 2.0 ** -9
    o, spread = torch.zeros((rows, hd), dtype=torch.float64, device="cuda"), torch.zeros((rows, hd), dtype=torch.float64, device="cuda")
    for lo, hi in parts:
        p = torch.exp(scores(lo, hi) - want.view(-1, 1))
        vd = v[0, 0, lo:hi].view(torch.float8_e4m3fn).double() * 2.0 ** -4
        o += p @ vd
        spread += p @ vd.abs()
        got = mass[0, 0, lo:hi].double()
        assert ((got - p.sum(0)).abs() <= 2.0 ** -9 * p.sum(0)).all()
    assert (mass[0, 0, end:] == 0).all()
    assert ((out[0, :, 0].double() - o).abs() <= 2.0 ** -8 * o.abs() + (2.0 ** -9 + 2.0 ** -11) * spread).all()
