"""Pins of the oracle of the 8-bit cache and of rotary positions with several axes (CPU)."""
import numpy as np
import pytest
import torch

from oracle import quant_cache_oracle as Q
from vvs_synth import gen


def test_e4m3_codes_are_torchs():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes.copy()).view(torch.float8_e4m3fn).double().numpy()
    got = Q.e4m3_decode(codes)
    np.testing.assert_array_equal(got, want)
    rng = gen.rng_for(3, "e4m3")
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-14, 8, 4000), got[np.isfinite(got)],
                        0.5 * (Q._POSITIVE[1:] + Q._POSITIVE[:-1]), -0.5 * (Q._POSITIVE[1:] + Q._POSITIVE[:-1])]).astype(np.float32)
    x = x[np.abs(x) <= 448.0]
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(Q.e4m3_encode(x), want)
    assert list(Q.e4m3_encode(np.array([np.inf, -np.inf, np.nan, 1e9, -500.0]))) == [0x7e, 0xfe, 0, 0x7e, 0xfe]


@pytest.mark.parametrize("amax,want", [(448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (1.75, 2.0 ** -8),
                                       (0.0, 2.0 ** -60), (1e-30, 2.0 ** -60), (3e38, 2.0 ** 120)])
def test_scale_is_the_smallest_power_that_holds_the_block(amax, want):
    assert Q.block_scale(amax) == want


def test_rotation_of_one_axis_and_of_a_grid():
    """One axis: rotations compose and keep lengths, and q.k depends on the distance alone; a grid of two axes is one axis per half."""
    rng = gen.rng_for(5, "axes")
    f = (10000.0 ** (-np.arange(8) / 8)).astype(np.float32)
    x = rng.standard_normal((1, 6, 2, 16))
    pos = np.arange(6, dtype=np.int32).reshape(1, 1, 6)
    y = Q.rotate_axes(x, f, np.zeros(8, int), pos, False)
    np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-12)
    same = np.repeat(x[:, :1], 6, axis=1)
    r = Q.rotate_axes(same, f, np.zeros(8, int), pos, False)
    assert abs((r[0, 1, 0] * r[0, 3, 0]).sum() - (r[0, 2, 0] * r[0, 4, 0]).sum()) < 1e-5     # (angles are float32)
    axis = np.array([0] * 4 + [1] * 4)
    grid = np.stack([pos[0] // 3, pos[0] % 3])
    both = Q.rotate_axes(x, f, axis, grid, False)
    np.testing.assert_array_equal(both[..., :8], Q.rotate_axes(x[..., :8], f[:4], np.zeros(4, int), grid[:1], False))
    np.testing.assert_array_equal(both[..., 8:], Q.rotate_axes(x[..., 8:], f[4:], np.zeros(4, int), grid[1:], False))
    split = Q.rotate_axes(x, f, axis, grid, True)
    order = np.arange(16).reshape(2, 8).T.reshape(-1)                     # pair i's elements side by side
    np.testing.assert_array_equal(split[..., order], Q.rotate_axes(x[..., order], f, axis, grid, False))


def test_append_row_by_row_holds_what_one_append_holds():
    """The scales are those of the whole block at the end; the values are within one rounding of theirs."""
    rng = gen.rng_for(6, "append")
    x = rng.standard_normal((37, 8)) * np.exp(rng.standard_normal((37, 1)))
    whole = np.full((64, 8), 0x7f, np.uint8), np.full(4, np.nan, np.float32)
    single = np.full((64, 8), 0x7f, np.uint8), np.full(4, np.nan, np.float32)
    Q.append_rows(*whole, x, 0, 16)
    for i in range(37):
        Q.append_rows(*single, x[i:i + 1], i, 16)
    np.testing.assert_array_equal(whole[1][:3], single[1][:3])
    for codes, scales in (whole, single):
        y = Q.e4m3_decode(codes[:37]) * scales[np.arange(37) // 16][:, None]
        half = np.maximum(np.abs(x) * 2.0 ** -4, scales[np.arange(37) // 16][:, None] * 2.0 ** -10)
        assert (np.abs(y - x) <= half * (1 + 1e-12)).all()
    assert (whole[0][37:] == 0x7f).all()


def test_attention_of_wide_codes_is_torchs():
    rng = gen.rng_for(7, "attend")
    b, t, h, kv, hd, cap = 2, 5, 4, 2, 16, 32
    kc, vc = (Q.e4m3_encode(rng.standard_normal((b, kv, cap, hd)) * 50) for _ in range(2))
    ks, vs = (2.0 ** rng.integers(-8, -4, (b, kv, 2)) for _ in range(2))
    q = rng.standard_normal((b, t, h, hd))
    lens = [20, 11]
    out, lse, mass, _ = Q.attend(kc, vc, ks, vs, q, lens, 16, mass=np.ones((b, kv, cap)), mass_rows=2, mass_decay=0.5)
    for i in range(b):
        n = lens[i] + t
        k, v = (torch.from_numpy(Q.e4m3_decode(c[i]) * np.repeat(s[i], 16, axis=1)[..., None])[:, :n].repeat_interleave(2, dim=0)
                for c, s in ((kc, ks), (vc, vs)))
        mask = torch.ones(t, n, dtype=torch.bool).tril(diagonal=lens[i])
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[i]).transpose(0, 1), k, v, attn_mask=mask)
        np.testing.assert_allclose(out[i], want.transpose(0, 1).numpy(), atol=1e-12)
        assert abs(mass[i].sum() - (kv * 0.5 * n + kv * (cap - n) + 2 * h)) < 1e-9
    chain = np.array([[(2 << j) - 1 for j in range(t)]] * b)
    again, _, _, _ = Q.attend(kc, vc, ks, vs, q, lens, 16, visible=chain)
    np.testing.assert_array_equal(out, again)


def test_eviction_by_hand():
    """Slots 0 .. 7, keep 5, the first and the last token guarded: 3 has the least weight, 1 and 6 tie behind it."""
    mass = np.array([[[0.0, 2.0, 5.0, 1.0, 4.0, 3.0, 2.0, 0.5, 9.0, 9.0]]], np.float32)
    age = np.arange(10, dtype=np.int32).reshape(1, 1, 10)
    k = np.arange(10, dtype=np.uint8).reshape(1, 1, 10, 1) + 40
    v = k + 1
    ks, vs = np.array([[[1.0, 4.0]]]), np.array([[[2.0, 1.0]]])
    kept, m, a, n = Q.evict(k, v, ks, vs, mass, age, np.array([8]), np.array([8]), 5, 1, 1, 5)
    # stay: 0, 7 (guarded), 2, 4, 5 -> slots 5, 7 move into the holes 1, 3
    assert kept.tolist() == [[[0, 5, 2, 7, 4]]] and n.tolist() == [5]
    assert m[0, 0, :5].tolist() == [0.0, 3.0, 5.0, 0.5, 4.0] and a[0, 0].tolist() == [0, 5, 2, 7, 4, -1, -1, -1, -1, -1]
    assert ks.tolist() == [[[4.0, 4.0]]] and vs.tolist() == [[[2.0, 1.0]]]
    dec = Q.e4m3_decode(np.arange(256, dtype=np.uint8))
    assert Q.e4m3_decode(k[0, 0, :5, 0]).tolist() == [dec[40] / 4, dec[45], dec[42] / 4, dec[47], dec[44] / 4]
    assert Q.e4m3_decode(v[0, 0, :5, 0]).tolist() == [dec[41], dec[46] / 2, dec[43], dec[48] / 2, dec[45]]


def test_eviction_keeps_all_where_all_fit():
    mass = np.array([[[1.0, np.nan, 3.0, 0.0]]], np.float32)
    age = np.arange(4, dtype=np.int32).reshape(1, 1, 4)
    k = np.zeros((1, 1, 4, 1), np.uint8)
    s = np.ones((1, 1, 1))
    kept, m, a, n = Q.evict(k, k.copy(), s, s.copy(), mass, age, np.array([3]), np.array([3]), 3, 0, 0, 4)
    assert kept.tolist() == [[[0, 1, 2]]] and n.tolist() == [3]
    kept, *_ = Q.evict(k, k.copy(), s, s.copy(), mass, age, np.array([3]), np.array([3]), 2, 0, 0, 4)
    assert kept.tolist() == [[[0, 2]]]                                     # the NaN goes first
