"""A tree's rows put again along the accepted path: keys, values, ages and the weights that the tree's attention gave them, on every layer.

Weights are moved, not computed again: compared by their bits with those of the rows before.  Codes: a value's code under the place's scale is the
oracle's of the same bf16 value; a turned key lies 2^-22 (|k0| + |k1|) off and may round to the other side of a tie (half a step: 2^-4 of the value, 2^-10 of
the scale)."""
import numpy as np
import pytest
import torch

from oracle import quant_cache_oracle as Q
from paper_2511_13587_b200 import binding as vb
from paper_2511_13587_b200 import bounded_cache as bc
from test_gpu_bounded_cache import host
from vvs_synth import gen
from vvs_synth.configs import ModelShape

pytestmark = pytest.mark.gpu

# 0 - 1 - 2 and 0 - 3 - (4, 5)
MASKS = np.array([1, 3, 7, 9, 25, 41], np.uint32)


@pytest.mark.parametrize("mass_rows", [1, 6])
def test_rows_keep_their_weights(mass_rows):
    rng = gen.rng_for(61, f"trees{mass_rows}")
    n_seqs, layers, heads, kv, hd, rows, block = 4, 3, 4, 2, 64, 6, 16
    ctx = vb.vvs_create(vb.make_desc(ModelShape("clip", 0, 64, 0, 0, 0, 128), 1, 1))
    axis, f = np.zeros(hd // 2, np.int32), (1000.0 ** (-np.arange(hd // 2) / (hd // 2))).astype(np.float32)
    cache = bc.BoundedCache(ctx, layers, n_seqs, heads, kv, hd, 40, rows, torch.from_numpy(f).cuda(), torch.from_numpy(axis).cuda(), slack=10,
                            block=block, n_sink=2, n_recent=8)
    paths = np.array([[0, 3, 5, -1, -1, -1], [0, 1, -1, -1, -1, -1], [0, 3, 4, -1, -1, -1], [-1] * 6], np.int32)
    count = np.array([3, 2, 3, 0], np.int32)
    evicted = 0
    for step in range(24):
        evicted += cache.make_room()
        fill, ages = host(cache.fill).copy(), host(cache.next_age).copy()
        rope = cache.rope(cache.next_age.view(1, -1, 1) + torch.arange(rows, device="cuda", dtype=torch.int32).view(1, 1, -1))
        before, kt, vs = [], [], []
        for i in range(layers):
            qkv = torch.from_numpy(rng.standard_normal((n_seqs, rows, heads + 2 * kv, hd)) * np.exp(rng.standard_normal((n_seqs, rows, 1, 1))))
            q, k, v = qkv.cuda().to(torch.bfloat16).split((heads, kv, kv), dim=2)
            turned = cache.append(i, q, k, v, rope)
            cache.attend(i, turned, torch.zeros_like(turned), mass_rows=mass_rows,
                         visible=torch.from_numpy(np.tile(MASKS, (n_seqs, 1)).view(np.int32)).cuda())
            before.append(host(cache.mass[cache.turn][i]).copy())
            cache.put_again(i, k, v, rope, torch.from_numpy(paths).cuda(), torch.from_numpy(count).cuda())
            kt.append(Q.rotate_axes(host(k), f, axis, host(rope._keep[2]), False))
            vs.append(host(v))
        cache.commit(torch.from_numpy(count).cuda(), 3)
        np.testing.assert_array_equal(host(cache.fill), fill + count)
        for i in range(layers):
            mass, age = host(cache.mass[cache.turn][i]), host(cache.age[cache.turn][i])
            for b in range(n_seqs):
                lo, n = fill[b], count[b]
                picked = lo + paths[b, :n]
                np.testing.assert_array_equal(mass[b, :, :lo], before[i][b, :, :lo])
                np.testing.assert_array_equal(mass[b, :, lo:lo + n], before[i][b][:, picked])
                assert (age[b, :, lo:lo + n] == ages[b] + np.arange(n)).all()
                at = np.arange(lo, lo + n)
                for codes, scales, rows_of in ((cache.k, cache.k_scale, kt[i]), (cache.v, cache.v_scale, vs[i])):
                    s = host(scales[i])[b][:, at // block][..., None]
                    x, got = rows_of[b, paths[b, :n]].transpose(1, 0, 2), host(codes[i])[b][:, at]
                    assert (np.abs(Q.e4m3_decode(got) * s - x) <= np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10) * (1 + 1e-5) + 1e-5).all()
                    if codes is cache.v:
                        np.testing.assert_array_equal(got, Q.e4m3_encode(x / s))
    assert evicted >= 1 and vb.vvs_device_status(ctx) == 0
    vb.vvs_destroy(ctx)


def test_a_tree_weighs_as_much_as_the_chain_of_its_path():
    """The same tokens decoded as a chain, and as the path of a tree whose other rows are rejected, have the same weights."""
    rng = gen.rng_for(62, "chain")
    n_seqs, heads, kv, hd = 1, 2, 2, 64
    ctx = vb.vvs_create(vb.make_desc(ModelShape("clip", 0, 64, 0, 0, 0, 128), 1, 1))
    caches = [bc.BoundedCache(ctx, 1, n_seqs, heads, kv, hd, 100, 6, torch.ones(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"),
                              slack=10) for _ in range(2)]
    for step in range(10):
        x = torch.from_numpy(rng.standard_normal((n_seqs, 6, heads + 2 * kv, hd))).cuda().to(torch.bfloat16)
        x[:, 1:, :, :2] = 0                                    # (positions do not matter: the one pair that is turned is 0)
        x[:, 0, :, :2] = 0
        path = torch.tensor([[0, 3, 5, -1, -1, -1]], dtype=torch.int32, device="cuda")
        n = torch.tensor([3], dtype=torch.int32, device="cuda")
        for cache, block, masks in ((caches[0], x[:, [0, 3, 5]].contiguous(), None), (caches[1], x, MASKS)):
            rows = block.shape[1]
            rope = cache.rope(torch.zeros((1, n_seqs, rows), dtype=torch.int32, device="cuda"))
            q, k, v = block.split((heads, kv, kv), dim=2)
            turned = cache.append(0, q, k, v, rope)
            cache.attend(0, turned, torch.zeros_like(turned), mass_rows=1, visible=None if masks is None else torch.from_numpy(
                np.tile(masks, (n_seqs, 1)).view(np.int32)).cuda())
            if masks is not None:
                cache.put_again(0, k, v, rope, path, n)
            cache.commit(n, 3)
    a, b = (host(c.mass[c.turn][0])[:, :, :30] for c in caches)
    # a block put again and not committed, and another one in its place that is a chain: nothing moves
    last = caches[1]
    fill = int(host(last.fill)[0])
    masses = []
    for tree in (True, False):
        turned = last.append(0, q, k, v, rope)
        last.attend(0, turned, torch.zeros_like(turned), mass_rows=6, visible=torch.from_numpy(MASKS.view(np.int32)).view(1, 6).cuda() if tree else None)
        if tree:
            last.put_again(0, k, v, rope, path, n)
        masses.append(host(last.mass[last.turn][0])[:, :, fill:fill + 6].copy())
    last.commit(n, 3)
    np.testing.assert_array_equal(host(last.mass[last.turn][0])[:, :, fill:fill + 6], masses[1])
    # (a rejected row may have made a block's scale grow: keys of one step then differ by their roundings, 2^-4 of them, and scores by some of that)
    assert (a > 0).sum() == (b > 0).sum() and (b[:, :, ::3] > 0).all()
    np.testing.assert_allclose(a.sum(), b.sum(), rtol=1e-5)
    vb.vvs_destroy(ctx)
