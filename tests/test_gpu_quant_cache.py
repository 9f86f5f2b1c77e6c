"""The 8-bit cache, its attention and eviction, and the rotation with several axes, through the public entry points against the
float64 oracle.

Tolerances.  Rotation: cosine and sine are within 2 units of the last place (2^-23 absolutely), each product and the sum rounds once
(2^-24 relative): 2^-22 (|x0| + |x1|); bf16 outputs (8 bits) round once more, 2^-8 of the value.  Codes: exactly the oracle's, except that
a turned key lies 2^-22 (|x0| + |x1|) off and may then round to the other side of a tie: its stored value is within half a step (2^-4 of
the value, 2^-10 of the scale) plus that.  Attention: a score is off by float32 sums of head_dim exact products and one 2-based exponential;
at |score| up to 2^5 that is 2^-17 of its weight (a few units of 2^-24 * 2^5, and 2^-22 of the exponential).  A weight goes
into the second product as a half (2^-11 of it) in bf16 contexts, as two of them (2^-22) in float32 ones.  So outputs are within
2^-8 |out| + (2^-11 + 2^-13) sum p|v| in bf16 and 2^-15 sum p|v| in float32, a log-sum is within 2^-15, an accumulated weight within 2^-15 of it.
Eviction is exact."""
import numpy as np
import pytest
import torch

from oracle import quant_cache_oracle as Q
from paper_2511_13587_b200 import binding as vb
from vvs_synth import gen
from vvs_synth.configs import DTYPE_BF16, DTYPE_FP32, ModelShape

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctxs():
    made = {dt: vb.vvs_create(vb.make_desc(ModelShape("cache", 0, 64, 0, 0, 0, 128, dtype=code), 1, 1))
            for dt, code in ((BF16, DTYPE_BF16), (F32, DTYPE_FP32))}
    yield made
    for c in made.values():
        vb.vvs_destroy(c)


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def rope_of(rng, hd, n_axes, n_pairs, b, t, hi=2000):
    axis = np.sort(rng.integers(0, n_axes, n_pairs)).astype(np.int32)
    f = (10000.0 ** (-np.arange(n_pairs) / n_pairs)).astype(np.float32)
    return f, axis, rng.integers(0, hi, (n_axes, b, t)).astype(np.int32)


def pair_room(x, n, halves):
    """|x0| + |x1| of the pair that an element belongs to; 0 behind the last pair."""
    room = np.zeros_like(x)
    e0, e1 = (slice(0, n), slice(n, 2 * n)) if halves else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    room[..., e0] = room[..., e1] = np.abs(x[..., e0]) + np.abs(x[..., e1])
    return room


# ---- rotation --------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b,t,h,kv,hd,n_axes,n_pairs,halves", [
    (1, 1, 1, 1, 8, 1, 4, False), (1, 1, 1, 1, 8, 1, 4, True), (2, 9, 20, 20, 64, 2, 32, False), (3, 7, 5, 0, 64, 3, 21, False),
    (2, 33, 8, 2, 128, 3, 64, True), (1, 130, 3, 1, 128, 4, 24, True), (2, 3, 2, 2, 256, 2, 128, False), (1, 5, 1, 1, 24, 1, 1, False),
    (40, 65, 40, 3, 128, 2, 64, False)])
def test_rotation(ctxs, dtype, b, t, h, kv, hd, n_axes, n_pairs, halves):
    rng = gen.rng_for(11, f"rot{b}{t}{h}{hd}{halves}")
    f, axis, pos = rope_of(rng, hd, n_axes, n_pairs, b, t, 40000)
    qkv = dev(rng.standard_normal((b, t, h + 2 * kv, hd)), dtype)            # heads of a row side by side: strides of their own
    q, k = qkv[:, :, :h], qkv[:, :, h:h + kv]
    rope = vb.make_rope_axes(dev(f), dev(axis), dev(pos), halves)
    # outputs with another order of dimensions: [T][B][H]
    q_out = torch.zeros((t, b, h, hd), dtype=dtype, device="cuda").transpose(0, 1)
    k_out = torch.zeros((t, b, kv, hd), dtype=dtype, device="cuda").transpose(0, 1) if kv else None
    vb.vvs_rotate_axes(ctxs[dtype], rope, q, q_out, k if kv else None, k_out)
    for x, y in ((q, q_out), (k, k_out))[:2 if kv else 1]:
        xd = host(x)
        want = Q.rotate_axes(xd, f, axis, pos, halves)
        room = pair_room(xd, n_pairs, halves) * 2.0 ** -22 + (np.abs(want) * 2.0 ** -8 if dtype == BF16 else 0)
        assert (np.abs(host(y) - want) <= room).all()
    before = qkv.clone()
    vb.vvs_rotate_axes(ctxs[dtype], rope, q, q, k if kv else None, k if kv else None)      # in place
    assert torch.equal(q, q_out) and (not kv or torch.equal(k, k_out))
    assert torch.equal(qkv[:, :, h + kv:], before[:, :, h + kv:])
    assert vb.vvs_device_status(ctxs[dtype]) == 0


def test_rotation_of_unknown_axes_is_left_out_and_told(ctxs):
    x = torch.randn((1, 2, 1, 16), device="cuda")
    f, pos = torch.ones(8, device="cuda"), torch.full((1, 1, 2), 3, dtype=torch.int32, device="cuda")
    axis = torch.tensor([0, 1, -1, 0, 0, 0, 0, 0], dtype=torch.int32, device="cuda")
    out = torch.zeros_like(x)
    vb.vvs_rotate_axes(ctxs[F32], vb.make_rope_axes(f, axis, pos), x, out)
    assert torch.equal(out[..., 2:6], x[..., 2:6]) and not torch.equal(out[..., :2], x[..., :2])
    assert vb.vvs_device_status(ctxs[F32]) == vb.VVS_DEV_BAD_ARG


# ---- append ------------------------------------------------------------------------------------------------------------------------


def make_cache(rng, b, kv, cap, hd, block, fills, spread=1.0):
    """Codes and scales of filled slots; what lies behind them is NaN codes and NaN scales."""
    kc, vc = (np.full((b, kv, cap, hd), 0x7f, np.uint8) for _ in range(2))
    ks, vs = (np.full((b, kv, cap // block), np.nan, np.float32) for _ in range(2))
    for c, s in ((kc, ks), (vc, vs)):
        for i in range(b):
            for h in range(kv):
                x = rng.standard_normal((int(fills[i]), hd)) * np.exp(spread * rng.standard_normal((int(fills[i]), 1)))
                Q.append_rows(c[i, h], s[i, h], x, 0, block)
    return kc, vc, ks, vs


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t,h,kv,hd,block,fills,counts,turn,halves", [
    (1, 4, 4, 64, 16, [0, 15, 16], None, True, False),
    (9, 8, 2, 128, 16, [3, 0, 23], [9, 0, 4], True, True),
    (9, 4, 1, 64, 64, [60, 63, 64], None, True, False),
    (33, 2, 2, 128, 128, [1, 100, 127], [33, 30, 1], False, False),
    (150, 2, 1, 64, 32, [0, 7, 31], None, True, True),
    (300, 1, 1, 128, 128, [5, 0, 120], [300, 299, 150], True, False)])
def test_append(ctxs, dtype, t, h, kv, hd, block, fills, counts, turn, halves):
    rng = gen.rng_for(12, f"app{t}{h}{kv}{hd}{block}")
    b, cap = len(fills), -(-(max(fills) + t) // block) * block
    kc, vc, ks, vs = make_cache(rng, b, kv, cap, hd, block, fills)
    x = rng.standard_normal((b, t, h + 2 * kv, hd)) * np.exp(rng.standard_normal((b, t, 1, 1)))
    qkv = dev(x, dtype)
    q, k, v = qkv.split((h, kv, kv), dim=2)
    f, axis, pos = rope_of(rng, hd, 3, hd // 2 - 4, b, t)
    rope = vb.make_rope_axes(dev(f), dev(axis), dev(pos), halves)
    lens = dev(np.array(fills, np.int32))
    mass, age = torch.full((b, kv, cap), float("nan"), device="cuda"), torch.full((b, kv, cap), -7, dtype=torch.int32, device="cuda")
    tk, tv, tks, tvs = dev(kc), dev(vc), dev(ks), dev(vs)
    qc = vb.make_qcache(tk, tv, tks, tvs, mass, age)
    q_out = torch.zeros((b, t, h, hd), dtype=dtype, device="cuda")
    count = None if counts is None else dev(np.array(counts, np.int32))
    more = dict(rope=rope, q=q, q_out=q_out) if turn else {}
    vb.vvs_quant_cache_append(ctxs[dtype], qc, k, v, lens, row_count=count, next_age=lens + 1000, **more)
    assert vb.vvs_device_status(ctxs[dtype]) == 0
    kd, vd = host(k), host(v)
    kt = Q.rotate_axes(kd, f, axis, pos, halves) if turn else kd
    off = pair_room(kd, len(f), halves) * 2.0 ** -22 if turn else np.zeros_like(kd)
    for i in range(b):
        n = t if counts is None else counts[i]
        for j in range(kv):
            for got_c, got_s, c, s, rows, err in ((tk, tks, kc, ks, kt, off), (tv, tvs, vc, vs, vd, None)):
                Q.append_rows(c[i, j], s[i, j], rows[i, :n, j], fills[i], block)
                g_c, g_s = got_c[i, j].cpu().numpy(), got_s[i, j].cpu().numpy()
                np.testing.assert_array_equal(g_s, s[i, j])
                if err is None or not turn:
                    np.testing.assert_array_equal(g_c, c[i, j])
                    continue
                lo, hi = fills[i], fills[i] + n
                np.testing.assert_array_equal(np.delete(g_c, np.s_[lo:hi], 0), np.delete(c[i, j], np.s_[lo:hi], 0))
                sc = g_s[np.arange(lo, hi) // block][:, None]
                room = np.maximum(np.abs(rows[i, :n, j]) * 2.0 ** -4, sc * 2.0 ** -10) + 1.0625 * err[i, :n, j]
                assert (np.abs(Q.e4m3_decode(g_c[lo:hi]) * sc - rows[i, :n, j]) <= room).all()
            assert (mass[i, j, fills[i]:fills[i] + n] == 0).all() and mass[i, j, fills[i] + n:].isnan().all()
            assert age[i, j, fills[i]:fills[i] + n].tolist() == list(range(fills[i] + 1000, fills[i] + 1000 + n))
            assert (age[i, j, :fills[i]] == -7).all() and (age[i, j, fills[i] + n:] == -7).all()
    if turn:
        want = Q.rotate_axes(host(q), f, axis, pos, halves)
        room = pair_room(host(q), len(f), halves) * 2.0 ** -22 + (np.abs(want) * 2.0 ** -8 if dtype == BF16 else 0)
        assert (np.abs(host(q_out) - want) <= room).all()


def test_append_again_along_an_accepted_path(ctxs):
    """A tree's rows are appended, then those on the accepted path again from the same fill: the cache holds the path side by side."""
    rng = gen.rng_for(13, "path")
    b, t, kv, hd, block, fills = 2, 7, 2, 64, 16, [13, 16]
    kc, vc, ks, vs = make_cache(rng, b, kv, 48, hd, block, fills)
    k, v = (dev(rng.standard_normal((b, t, kv, hd)), BF16) for _ in range(2))
    f, axis, pos = rope_of(rng, hd, 2, 32, b, t)
    rope = vb.make_rope_axes(dev(f), dev(axis), dev(pos))
    path = np.array([[0, 2, 5, -1, -1, -1, -1], [0, 1, 3, 4, -1, -1, -1]], np.int32)
    count = np.array([3, 4], np.int32)
    lens = dev(np.array(fills, np.int32))
    tk, tv, tks, tvs = dev(kc), dev(vc), dev(ks), dev(vs)
    qc = vb.make_qcache(tk, tv, tks, tvs)
    vb.vvs_quant_cache_append(ctxs[BF16], qc, k, v, lens, rope=rope)
    vb.vvs_quant_cache_append(ctxs[BF16], qc, k, v, lens, rope=rope, row_index=dev(path), row_count=dev(count))
    assert vb.vvs_device_status(ctxs[BF16]) == 0
    kt = Q.rotate_axes(host(k), f, axis, pos, False)
    for i in range(b):
        lo, n = fills[i], int(count[i])
        for j in range(kv):
            for got, sc, rows in ((tk, tks, kt), (tv, tvs, host(v))):
                s = sc[i, j].cpu().numpy()[np.arange(lo, lo + n) // block][:, None]
                want = rows[i, path[i, :n], j]
                room = np.maximum(np.abs(want) * 2.0 ** -4, s * 2.0 ** -10) * (1 + 1e-5) + 1e-5
                assert (np.abs(Q.e4m3_decode(got[i, j, lo:lo + n].cpu().numpy()) * s - want) <= room).all()


def test_append_of_infinities_and_nans(ctxs):
    """They neither reach the block's scale nor the other rows, and the caller is told."""
    x = torch.randn((1, 3, 1, 64), device="cuda")
    clean = x.clone()
    x[0, 1, 0, 5], x[0, 1, 0, 6], x[0, 2, 0, 7] = float("inf"), float("-inf"), float("nan")
    clean[0, 1, 0, 5] = clean[0, 1, 0, 6] = clean[0, 2, 0, 7] = 0
    caches = []
    for rows in (x, clean):
        c = [torch.zeros((1, 1, 16, 64), dtype=torch.uint8, device="cuda") for _ in range(2)] + \
            [torch.zeros((1, 1, 1), device="cuda") for _ in range(2)]
        vb.vvs_quant_cache_append(ctxs[F32], vb.make_qcache(*c), rows, rows, torch.zeros(1, dtype=torch.int32, device="cuda"))
        caches.append(c)
        assert vb.vvs_device_status(ctxs[F32]) == (vb.VVS_DEV_NONFINITE if rows is x else 0)
    a, b = caches
    assert torch.equal(a[2], b[2]) and torch.equal(a[3], b[3])
    assert a[0][0, 0, 1, 5] == 0x7e and a[0][0, 0, 1, 6] == 0xfe and a[0][0, 0, 2, 7] == 0
    a[0][0, 0, 1, 5:7] = b[0][0, 0, 1, 5:7]
    assert torch.equal(a[0], b[0])


def test_append_skips_sequences_that_do_not_fit(ctxs):
    c = [torch.full((3, 2, 32, 64), 9, dtype=torch.uint8, device="cuda") for _ in range(2)] + \
        [torch.ones((3, 2, 2), device="cuda") for _ in range(2)]
    rows = torch.randn((3, 4, 2, 64), device="cuda")
    lens = torch.tensor([29, -1, 28], dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_append(ctxs[F32], vb.make_qcache(*c), rows, rows, lens)
    assert vb.vvs_device_status(ctxs[F32]) == vb.VVS_DEV_CACHE_OVERFLOW
    assert (c[0][:2] == 9).all() and (c[1][:2] == 9).all() and (c[0][2, :, 28:] != 9).any()
    count = torch.tensor([3, 5, -2], dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_append(ctxs[F32], vb.make_qcache(*c), rows, rows, torch.zeros_like(lens) + 29, row_count=count)
    assert vb.vvs_device_status(ctxs[F32]) == vb.VVS_DEV_BAD_ARG
    assert (c[0][0, :, 29:] != 9).any() and (c[0][1] == 9).all()


# ---- attention ------------------------------------------------------------------------------------------------------------------------


ATTEND = [
    # t, h, kv, hd, block, fills, counts, firsts, tree, mass_rows, decay, dtype
    (1, 1, 1, 64, 16, [0], None, None, False, 0, 1.0, BF16),
    (1, 4, 4, 128, 16, [0, 1, 15, 16, 17, 40], None, None, False, 1, 1.0, BF16),
    (1, 2, 2, 64, 32, [0, 100, 31], None, [0, 99, 31], False, 1, 0.5, F32),
    (9, 20, 20, 64, 64, [311, 5], None, None, False, 9, 1.0, BF16),
    (9, 4, 4, 128, 64, [0, 200, 63], [9, 0, 4], [0, 13, 63], False, 5, 0.0, BF16),
    (16, 2, 2, 64, 16, [33, 0], None, None, False, 16, 1.0, F32),
    (17, 2, 2, 128, 128, [120, 0], None, None, False, 3, 1.0, BF16),
    (33, 2, 1, 64, 16, [70, 1], [33, 20], [16, 0], False, 33, 0.25, BF16),
    (27, 8, 2, 128, 128, [500, 100], None, None, True, 0, 1.0, BF16),
    (32, 8, 1, 64, 32, [90, 0], None, None, True, 32, 1.0, BF16),
    (8, 16, 2, 128, 16, [48, 7], None, None, True, 2, 0.9, F32),
    (40, 16, 2, 64, 64, [130, 64], None, None, False, 40, 1.0, BF16),
    (5, 1, 1, 64, 16, [3000, 2999], None, [0, 2990], False, 1, 1.0, BF16),
    (200, 2, 2, 64, 64, [0, 17], [200, 131], None, False, 0, 1.0, BF16),
    (130, 4, 2, 128, 32, [0, 300], None, None, False, 2, 1.0, BF16),
]


def tree_masks(rng, b, t):
    out = np.zeros((b, t), np.uint32)
    for i in range(b):
        for j in range(t):
            out[i, j] = (0 if j == 0 else out[i, rng.integers(max(0, j - 5), j)]) | np.uint32(1 << j)
    return out


def check_attend(ctx, dtype, q, out, lse, mass, want, n_masses):
    want_out, want_lse, want_mass, spread = want
    got = host(out)
    room = (2.0 ** -8 * np.abs(want_out) + (2.0 ** -11 + 2.0 ** -13) * spread) if dtype == BF16 else 2.0 ** -15 * spread
    assert np.isfinite(got).all()
    worst = (np.abs(got - want_out) - room).max()
    assert worst <= 0, worst
    gl = host(lse)
    np.testing.assert_array_equal(np.isfinite(gl), np.isfinite(want_lse))
    f = np.isfinite(gl)
    assert np.abs(gl[f] - want_lse[f]).max(initial=0.0) <= 2.0 ** -15
    if n_masses:
        np.testing.assert_allclose(host(mass), want_mass, rtol=2.0 ** -15, atol=2.0 ** -30)


@pytest.mark.parametrize("t,h,kv,hd,block,fills,counts,firsts,tree,mass_rows,decay,dtype", ATTEND)
def test_attention(ctxs, t, h, kv, hd, block, fills, counts, firsts, tree, mass_rows, decay, dtype):
    rng = gen.rng_for(14, f"att{t}{h}{kv}{hd}{block}{tree}")
    b, cap = len(fills), -(-(max(fills) + t) // block) * block + block
    n = [t] * b if counts is None else counts
    kc, vc, ks, vs = make_cache(rng, b, kv, cap, hd, block, np.array(fills) + n)
    wide = dev(rng.standard_normal((b, t, h + 1, hd)) * 1.5, dtype)
    q = wide[:, :, :h]
    out = torch.full((t, b, h, hd), float("nan"), dtype=dtype, device="cuda").transpose(0, 1)
    lse = torch.full((b, t, h), float("nan"), device="cuda")
    m0 = np.abs(rng.standard_normal((b, kv, cap))).astype(np.float32)
    mass = dev(np.full_like(m0, np.nan) if decay == 0 else m0)
    vis = tree_masks(rng, b, t) if tree else None
    i32 = lambda x: None if x is None else dev(np.array(x, np.int32))
    qc = vb.make_qcache(dev(kc), dev(vc), dev(ks), dev(vs), mass)
    vb.vvs_quant_cache_attend(ctxs[dtype], qc, q, out, i32(fills), row_count=i32(counts), first_slot=i32(firsts),
                              visible=None if vis is None else dev(vis.view(np.int32)), lse=lse, mass_rows=mass_rows, mass_decay=decay)
    assert vb.vvs_device_status(ctxs[dtype]) == 0
    want = Q.attend(kc, vc, ks, vs, host(q), fills, block, row_count=counts, first_slot=firsts, visible=vis, mass=m0, mass_rows=mass_rows,
                    mass_decay=decay)
    got_mass = mass.clone()
    if decay == 0:                                         # slots that the call does not reach are not touched
        for i in range(b):
            assert mass[i, :, fills[i] + n[i]:].isnan().all()
            got_mass[i, :, fills[i] + n[i]:] = dev(m0)[i, :, fills[i] + n[i]:]
    check_attend(ctxs[dtype], dtype, q, out, lse, got_mass, want, mass_rows)
    # the same bits again, and with whatever the caller says of the lengths
    for max_len in (0, 1, 64, max(fills) + t):
        o2, l2, m2 = torch.zeros_like(out), torch.zeros_like(lse), dev(np.full_like(m0, np.nan) if decay == 0 else m0)
        vb.vvs_quant_cache_attend(ctxs[dtype], vb.make_qcache(qc._keep[0], qc._keep[1], qc._keep[2], qc._keep[3], m2), q, o2, i32(fills),
                                  row_count=i32(counts), first_slot=i32(firsts), visible=None if vis is None else dev(vis.view(np.int32)),
                                  lse=l2, mass_rows=mass_rows, mass_decay=decay, max_len=max_len)
        if max_len == 0:
            assert torch.equal(o2, out) and torch.equal(l2, lse) and torch.equal(m2.view(torch.int32), mass.view(torch.int32))
        else:
            m3 = torch.where(m2.isnan(), dev(m0), m2) if decay == 0 else m2
            check_attend(ctxs[dtype], dtype, q, o2, l2, m3, want, mass_rows)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_of_rows_that_see_nothing(ctxs, dtype):
    rng = gen.rng_for(15, "nothing")
    kc, vc, ks, vs = make_cache(rng, 2, 1, 32, 64, 16, [20, 9])
    q = dev(rng.standard_normal((2, 3, 2, 64)), dtype)
    vis = np.array([[0, 2, 0], [0, 0, 0]], np.uint32)          # row 0 and 2 of sequence 0 see no row of the block, nor itself
    out, lse = torch.full_like(q, 7), torch.zeros((2, 3, 2), device="cuda")
    mass = torch.zeros((2, 1, 32), device="cuda")
    first = torch.tensor([17, 6], dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_attend(ctxs[dtype], vb.make_qcache(dev(kc), dev(vc), dev(ks), dev(vs), mass), q, out, first.clone(), first_slot=first,
                              visible=dev(vis.view(np.int32)), lse=lse, mass_rows=3)
    want = Q.attend(kc, vc, ks, vs, host(q), [17, 6], 16, first_slot=[17, 6], visible=vis, mass=np.zeros((2, 1, 32)), mass_rows=3)
    check_attend(ctxs[dtype], dtype, q, out, lse, mass, want, 3)
    assert (out[0, 0] == 0).all() and (out[1] == 0).all() and lse[1].isneginf().all() and abs(mass.sum().item() - 2) < 1e-5


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_of_extreme_scales_and_queries(ctxs, dtype):
    """Blocks whose values are 2^40 apart, queries of 2^60 and 2^-60 (scaled back by `scale`), a row of NaN beside rows that are not."""
    rng = gen.rng_for(16, "extreme")
    kc, vc, ks, vs = make_cache(rng, 1, 1, 64, 64, 16, [64])
    vs[0, 0] = [2.0 ** -40, 1.0, 2.0 ** 20, 2.0 ** -60]
    for e in (60, -60):
        q = dev(rng.standard_normal((1, 4, 1, 64)) * 2.0 ** e, dtype)
        out, lse = torch.zeros_like(q), torch.zeros((1, 4, 1), device="cuda")
        lens = torch.tensor([60], dtype=torch.int32, device="cuda")
        scale = 0.125 * 2.0 ** -e
        vb.vvs_quant_cache_attend(ctxs[dtype], vb.make_qcache(dev(kc), dev(vc), dev(ks), dev(vs)), q, out, lens, lse=lse, scale=scale)
        want = Q.attend(kc, vc, ks, vs, host(q), [60], 16, scale=scale)
        check_attend(ctxs[dtype], dtype, q, out, lse, None, want, 0)
        bad = q.clone()
        bad[0, 1] = float("nan")
        o2 = torch.zeros_like(q)
        vb.vvs_quant_cache_attend(ctxs[dtype], vb.make_qcache(dev(kc), dev(vc), dev(ks), dev(vs)), bad, o2, lens, scale=scale)
        assert o2[0, 1].isnan().all() and torch.equal(o2[0, 2:], out[0, 2:]) and torch.equal(o2[0, 0], out[0, 0])


def test_attention_told_of_bad_lengths(ctxs):
    rng = gen.rng_for(17, "lens")
    kc, vc, ks, vs = make_cache(rng, 4, 1, 32, 64, 16, [32, 32, 32, 32])
    q = dev(rng.standard_normal((4, 2, 1, 64)), BF16)
    out, lse = torch.full_like(q, 7), torch.zeros((4, 2, 1), device="cuda")
    lens = torch.tensor([31, -1, 30, 30], dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_attend(ctxs[BF16], vb.make_qcache(dev(kc), dev(vc), dev(ks), dev(vs)), q, out, lens, lse=lse)
    assert vb.vvs_device_status(ctxs[BF16]) == vb.VVS_DEV_CACHE_OVERFLOW
    assert (out[:2] == 0).all() and lse[:2].isneginf().all() and (out[2:] != 0).any()
    count = torch.tensor([2, 2, 3, 2], dtype=torch.int32, device="cuda")
    first = torch.tensor([0, -4, 0, 31], dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_attend(ctxs[BF16], vb.make_qcache(dev(kc), dev(vc), dev(ks), dev(vs)), q, out, torch.full_like(lens, 30), row_count=count,
                              first_slot=first, lse=lse)
    assert vb.vvs_device_status(ctxs[BF16]) == vb.VVS_DEV_BAD_ARG
    want = Q.attend(kc, vc, ks, vs, host(q), [30] * 4, 16, row_count=[2, 2, 0, 2], first_slot=[0, 0, 0, 30])
    check_attend(ctxs[BF16], BF16, q, out, lse, None, want, 0)


def test_cache_beyond_32_bit_offsets(ctxs):
    """A cache of more than 2^31 bytes of keys: its last head, in its last slots."""
    heads, cap, hd, block = 132, 131072, 128, 128
    k, v = (torch.zeros((1, heads, cap, hd), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.ones((1, heads, cap // block), device="cuda") for _ in range(2))
    mass = torch.zeros((1, heads, cap), device="cuda")
    qc = vb.make_qcache(k, v, ks, vs, mass)
    rng = gen.rng_for(18, "long")
    t, fill = 4, cap - 9
    x = dev(rng.standard_normal((1, t, heads, hd)), BF16)
    lens = torch.tensor([fill], dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_append(ctxs[BF16], qc, x, x, lens)
    q = dev(rng.standard_normal((1, t, heads, hd)) * 2, BF16)
    out, lse = torch.zeros_like(q), torch.zeros((1, t, heads), device="cuda")
    first = lens - 100
    vb.vvs_quant_cache_attend(ctxs[BF16], qc, q, out, lens, first_slot=first, lse=lse, mass_rows=t)
    for h in (0, 65, heads - 1):
        c = [z[:, h:h + 1].cpu().numpy() for z in (k, v, ks, vs)]
        np.testing.assert_allclose(Q.e4m3_decode(c[0][0, 0, fill:fill + t]) * c[2][0, 0, -1], host(x[0, :, h]), rtol=2.0 ** -4, atol=2.0 ** -7)
        lo = fill - 100
        c = [c[0][:, :, lo - lo % block:], c[1][:, :, lo - lo % block:], c[2][:, :, lo // block:], c[3][:, :, lo // block:]]
        want = Q.attend(*c, host(q[:, :, h:h + 1]), [100 + lo % block], block, first_slot=[lo % block],
                        mass=np.zeros((1, 1, c[0].shape[2])), mass_rows=t)
        check_attend(ctxs[BF16], BF16, q, out[:, :, h:h + 1], lse[:, :, h:h + 1], mass[:, h:h + 1, lo - lo % block:], want, t)
    mass_out, kept = torch.zeros_like(mass), torch.zeros((1, heads, 256), dtype=torch.int32, device="cuda")
    new_len = torch.zeros_like(lens)
    vb.vvs_quant_cache_evict(ctxs[BF16], qc, lens + t, 256, 0, 8, None, mass_out, None, new_len, kept)
    assert new_len.item() == 256 and vb.vvs_device_status(ctxs[BF16]) == 0
    stay = kept[0, heads - 1].long()
    assert set(range(fill - 4, fill + t)) <= set(stay.tolist())
    assert torch.equal(mass_out[0, heads - 1, :256], mass[0, heads - 1, stay])


# ---- eviction --------------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("heads,hd,block,cap,fills,keep,sink,recent,kind", [
    (1, 64, 16, 32, [0, 1, 20], 1, 0, 1, "plain"), (2, 64, 16, 64, [64, 33, 40], 32, 1, 4, "plain"), (3, 128, 32, 96, [96, 95, 50], 49, 0, 0, "ties"),
    (2, 128, 128, 640, [600, 576, 448], 448, 1, 64, "plain"), (1, 64, 64, 2112, [2100, 1000, 1500], 999, 10, 500, "odd"),
    (2, 64, 16, 4096, [4096, 4001, 3000], 2050, 64, 300, "ties"), (1, 128, 128, 9088, [9000, 8999, 1], 1, 0, 0, "plain"),
    (1, 64, 32, 9088, [9000, 8191, 8200], 8192, 100, 1000, "odd"), (2, 64, 16, 48, [48, 48, 47], 47, 20, 27, "plain")])
def test_eviction(ctxs, heads, hd, block, cap, fills, keep, sink, recent, kind):
    rng = gen.rng_for(19, f"evict{heads}{hd}{block}{cap}{kind}")
    b = len(fills)
    kc, vc = (rng.integers(0, 256, (b, heads, cap, hd)).astype(np.uint8) for _ in range(2))
    for c in (kc, vc):
        c[(c & 127) == 127] = 1
    ks, vs = ((2.0 ** rng.integers(-9, -4, (b, heads, cap // block))).astype(np.float32) for _ in range(2))
    mass = rng.standard_normal((b, heads, cap)).astype(np.float32)
    if kind == "ties":
        mass = rng.integers(0, 3, mass.shape).astype(np.float32) * rng.choice([1.0, -1.0], mass.shape).astype(np.float32)
    if kind == "odd":
        pick = rng.integers(0, 6, mass.shape)
        mass[pick == 0], mass[pick == 1], mass[pick == 2], mass[pick == 3] = np.nan, np.inf, -np.inf, -0.0
    fills = np.array(fills, np.int32)
    ages = np.sort(rng.permuted(np.broadcast_to(np.arange(2 * cap), (b, heads, 2 * cap)), axis=2)[:, :, :cap], axis=2).astype(np.int32)
    ages = rng.permuted(ages, axis=2)                                     # a cache that was shrunk before has its ages in any order
    nxt = np.full(b, 2 * cap, np.int32)
    t = [dev(x) for x in (kc, vc, ks, vs, mass, ages)]
    mass_out, age_out = torch.full_like(t[4], 5), torch.full_like(t[5], 5)
    new_len, kept = torch.zeros(b, dtype=torch.int32, device="cuda"), torch.zeros((b, heads, keep), dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_evict(ctxs[BF16], vb.make_qcache(*t), dev(fills), keep, sink, recent, dev(nxt), mass_out, age_out, new_len, kept)
    assert vb.vvs_device_status(ctxs[BF16]) == 0
    assert np.array_equal(host(t[4]), mass.astype(np.float64), equal_nan=True) and np.array_equal(host(t[5]), ages)   # inputs stay
    w_kept, w_mass, w_age, w_len = Q.evict(kc, vc, ks, vs, mass, ages, fills, nxt, keep, sink, recent, block)
    np.testing.assert_array_equal(host(kept), w_kept)
    np.testing.assert_array_equal(host(new_len), w_len)
    for got, want in zip(t[:4], (kc, vc, ks, vs)):
        np.testing.assert_array_equal(got.cpu().numpy(), want)
    for i in range(b):
        n = fills[i]
        np.testing.assert_array_equal(mass_out[i, :, :n].cpu().numpy(), w_mass[i, :, :n])
        np.testing.assert_array_equal(age_out[i, :, :n].cpu().numpy(), w_age[i, :, :n])
        assert (mass_out[i, :, n:] == 5).all() and (age_out[i, :, n:] == 5).all()
    # once more on what it left
    w_kept, *_ = Q.evict(kc, vc, ks, vs, mass, ages, fills, nxt, keep, sink, recent, block)
    vb.vvs_quant_cache_evict(ctxs[BF16], vb.make_qcache(*t), dev(fills), keep, sink, recent, dev(nxt), mass_out, age_out, new_len, kept)
    np.testing.assert_array_equal(host(kept), w_kept)
    for got, want in zip(t[:4], (kc, vc, ks, vs)):
        np.testing.assert_array_equal(got.cpu().numpy(), want)


def test_eviction_without_ages_and_of_bad_lengths(ctxs):
    rng = gen.rng_for(20, "noage")
    c = [dev(rng.integers(0, 100, (3, 2, 48, 64)).astype(np.uint8)) for _ in range(2)] + [torch.ones((3, 2, 3), device="cuda") for _ in range(2)]
    mass = dev(rng.random((3, 2, 48)).astype(np.float32))
    before = [x.clone() for x in c]
    lens = torch.tensor([40, -1, 49], dtype=torch.int32, device="cuda")
    mass_out, new_len = torch.zeros_like(mass), torch.full((3,), 9, dtype=torch.int32, device="cuda")
    kept = torch.zeros((3, 2, 20), dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_evict(ctxs[F32], vb.make_qcache(*c, mass), lens, 20, 2, 5, None, mass_out, None, new_len, kept)
    assert vb.vvs_device_status(ctxs[F32]) == vb.VVS_DEV_CACHE_OVERFLOW
    assert new_len.tolist() == [20, 9, 9] and all(torch.equal(x[1:], y[1:]) for x, y in zip(c, before))
    arr = [x.cpu().numpy() for x in before]
    w_kept, w_mass, _, _ = Q.evict(*[a[:1] for a in arr], mass.cpu().numpy()[:1], np.broadcast_to(np.arange(48, dtype=np.int32), (1, 2, 48)),
                                   np.array([40]), np.array([40]), 20, 2, 5, 16)
    np.testing.assert_array_equal(kept[:1].cpu().numpy(), w_kept)
    np.testing.assert_array_equal(mass_out[0, :, :20].cpu().numpy(), w_mass[0, :, :20])


# ---- refusals, streams ---------------------------------------------------------------------------------------------------------------------


def test_refusals(ctxs):
    ctx = ctxs[BF16]
    f, axis, pos = (dev(x) for x in rope_of(gen.rng_for(21, "r"), 64, 1, 32, 2, 3))
    rope = vb.make_rope_axes(f, axis, pos)
    q, k = (torch.zeros((2, 3, n, 64), dtype=BF16, device="cuda") for n in (4, 2))
    c = [torch.zeros((2, 2, 48, 64), dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.ones((2, 2, 3), device="cuda") for _ in range(2)]
    mass = torch.zeros((2, 2, 48), device="cuda")
    qc, qm = vb.make_qcache(*c), vb.make_qcache(*c, mass)
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    kept = torch.zeros((2, 2, 16), dtype=torch.int32, device="cuda")
    pad = torch.zeros(2 * 3 * 4 * 64 + 8, dtype=BF16, device="cuda")

    def shifted(t, by):
        return pad[by:by + t.numel()].view(t.shape)

    def status(call):
        with pytest.raises(vb.VvsError) as e:
            call()
        return e.value.status

    inv, shape, align = -1, -2, -3
    assert status(lambda: vb.vvs_rotate_axes(ctx, rope, q, q, k, None)) == inv
    assert status(lambda: vb.vvs_rotate_axes(None, rope, q, q)) == inv
    assert status(lambda: vb.vvs_rotate_axes(ctx, rope, shifted(q, 4), q)) == align
    assert status(lambda: vb.vvs_rotate_axes(ctx, rope, q[..., :12], q[..., :12])) == shape
    odd = torch.zeros((2, 3, 4, 68), dtype=BF16, device="cuda")[..., :64]
    assert status(lambda: vb.vvs_rotate_axes(ctx, rope, odd, q)) == align
    many = vb.make_rope_axes(torch.ones(33, device="cuda"), torch.zeros(33, dtype=torch.int32, device="cuda"), pos)
    assert status(lambda: vb.vvs_rotate_axes(ctx, many, q, q)) == shape
    part = vb.make_rope_axes(f[:30].contiguous(), axis[:30].contiguous(), pos, halves=True)
    assert status(lambda: vb.vvs_rotate_axes(ctx, part, q, q)) == shape
    with pytest.raises(ValueError):
        vb.vvs_rotate_axes(ctx, rope, q.float(), q.float())                    # not the context's type
    with pytest.raises(ValueError):
        vb.vvs_rotate_axes(ctx, rope, q.transpose(2, 3).contiguous().transpose(2, 3), q)
    with pytest.raises(ValueError):
        vb.vvs_rotate_axes(ctx, rope, q, q[:1])
    with pytest.raises(TypeError):
        vb.vvs_rotate_axes(ctx, qc, q, q)

    assert status(lambda: vb.vvs_quant_cache_append(ctx, qc, k, k, None)) == inv
    assert status(lambda: vb.vvs_quant_cache_append(ctx, qc, k, k, n, q=q, q_out=q)) == inv          # nothing to turn q by
    assert status(lambda: vb.vvs_quant_cache_append(ctx, qc, k, k, n, rope=rope, q=q)) == inv
    assert status(lambda: vb.vvs_quant_cache_append(ctx, qc, k, k, n, rope=rope, q=q, q_out=q, row_index=n)) == inv
    assert status(lambda: vb.vvs_quant_cache_append(ctx, qc, shifted(k, 1), k, n)) == align
    with pytest.raises(ValueError):
        vb.vvs_quant_cache_append(ctx, qc, q, q, n)
    bad = vb.make_qcache(*c)
    bad.block = 48
    assert status(lambda: vb.vvs_quant_cache_append(ctx, bad, k, k, n)) == shape
    bad = vb.make_qcache(*c)
    bad.cap = 40
    assert status(lambda: vb.vvs_quant_cache_append(ctx, bad, k, k, n)) == shape
    bad = vb.make_qcache(*c)
    bad.k_scale = None
    assert status(lambda: vb.vvs_quant_cache_append(ctx, bad, k, k, n)) == inv
    with pytest.raises(ValueError):
        vb.make_qcache(c[0], c[1][:1], c[2], c[3])
    with pytest.raises(ValueError):
        vb.make_qcache(c[0], c[1], c[2], c[3], mass[:, :, :47])

    out = torch.zeros_like(q)
    assert status(lambda: vb.vvs_quant_cache_attend(ctx, qc, q, out, n, mass_rows=1)) == inv
    assert status(lambda: vb.vvs_quant_cache_attend(ctx, qm, q, out, n, mass_rows=-1)) == shape
    assert status(lambda: vb.vvs_quant_cache_attend(ctx, qm, q, out, n, mass_rows=1, mass_decay=-0.5)) == inv
    assert status(lambda: vb.vvs_quant_cache_attend(ctx, qm, q, out, n, scale=float("nan"))) == inv
    assert status(lambda: vb.vvs_quant_cache_attend(ctx, qm, q, out, n, max_len=-1)) == shape
    assert status(lambda: vb.vvs_quant_cache_attend(ctx, qm, q[:, :, :3], out[:, :, :3], n)) == shape
    long = torch.zeros((2, 33, 4, 64), dtype=BF16, device="cuda")
    assert status(lambda: vb.vvs_quant_cache_attend(ctx, qm, long, long.clone(), n, visible=kept)) == shape

    good = dict(mass_out=torch.zeros_like(mass), age_out=None, new_len=torch.zeros_like(n), kept=kept)
    assert status(lambda: vb.vvs_quant_cache_evict(ctx, qc, n, 16, 0, 0, None, **good)) == inv          # no weights
    assert status(lambda: vb.vvs_quant_cache_evict(ctx, qm, n, 16, 0, 0, None, **dict(good, mass_out=mass))) == inv
    assert status(lambda: vb.vvs_quant_cache_evict(ctx, qm, n, 16, 0, 0, None, **dict(good, new_len=n))) == inv
    assert status(lambda: vb.vvs_quant_cache_evict(ctx, qm, n, 0, 0, 0, None, **good)) == shape
    assert status(lambda: vb.vvs_quant_cache_evict(ctx, qm, n, 49, 0, 0, None, **good)) == shape
    assert status(lambda: vb.vvs_quant_cache_evict(ctx, qm, n, 16, 9, 8, None, **good)) == shape
    assert vb.vvs_device_status(ctx) == 0


def test_on_another_stream_and_captured(ctxs):
    """Append and attention run where the caller says, and inside a graph."""
    ctx = ctxs[BF16]
    rng = gen.rng_for(22, "stream")
    kc, vc, ks, vs = make_cache(rng, 2, 2, 160, 64, 32, [100, 37])
    x = dev(rng.standard_normal((2, 9, 8, 64)), BF16)
    q, k, v = x.split((4, 2, 2), dim=2)
    f, axis, pos = (dev(z) for z in rope_of(rng, 64, 2, 32, 2, 9))
    rope = vb.make_rope_axes(f, axis, pos)
    lens = torch.tensor([100, 37], dtype=torch.int32, device="cuda")

    def buffers():
        return [dev(z) for z in (kc, vc, ks, vs)] + [torch.zeros((2, 2, 160), device="cuda")]

    def step(c, q_out, out, stream=None):
        qc = vb.make_qcache(*c)
        vb.vvs_quant_cache_append(ctx, qc, k, v, lens, rope=rope, q=q, q_out=q_out, stream=stream)
        vb.vvs_quant_cache_attend(ctx, qc, q_out, out, lens, mass_rows=9, mass_decay=0.0, stream=stream)

    a, qa, oa = buffers(), torch.zeros_like(q), torch.zeros((2, 9, 4, 64), dtype=BF16, device="cuda")
    step(a, qa, oa)
    side = torch.cuda.Stream()
    b, qb, ob = buffers(), torch.zeros_like(q), torch.zeros_like(oa)
    torch.cuda.synchronize()
    step(b, qb, ob, side)
    side.synchronize()
    assert torch.equal(oa, ob) and torch.equal(qa, qb)
    assert all(torch.equal(y.view(torch.uint8), z.view(torch.uint8)) for y, z in zip(a, b))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(b, qb, ob)
    ob.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(oa, ob)
    del g
