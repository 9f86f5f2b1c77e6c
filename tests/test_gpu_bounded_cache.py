"""The bounded 8-bit cache as a decoding program runs it: blocks appended, attended, committed and evicted over many steps and layers, against
the float64 oracle of the same steps.

Tolerances.  The oracle's cache starts every step from the codes, scales, weights and ages on the device, so that a key that rounds to the
other side of a tie does not count twice; a step is then held to the bounds of its operators: outputs 2^-8 |out| + (2^-11 + 2^-13)
sum p|v|, weights 2^-15 of theirs, evictions exactly."""
import numpy as np
import pytest
import torch

from oracle import quant_cache_oracle as Q
from paper_2511_13587_b200 import binding as vb
from paper_2511_13587_b200 import bounded_cache as bc
from vvs_synth import gen
from vvs_synth.configs import ModelShape

pytestmark = pytest.mark.gpu


def host(t):
    if t.dtype == torch.float8_e4m3fn:
        return t.view(torch.uint8).cpu().numpy()
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


@pytest.mark.parametrize("hd,heads,kv,block,tree", [(64, 4, 2, 16, False), (128, 6, 3, 32, True)])
def test_steps_of_a_clip(hd, heads, kv, block, tree):
    rng = gen.rng_for(31, f"clip{hd}{tree}")
    n_seqs, layers, rows, budget, steps = 2, 2, 6, 40, 40
    ctx = vb.vvs_create(vb.make_desc(ModelShape("clip", 0, 64, 0, 0, 0, 128), 1, 1))
    pairs = hd // 2
    axis = np.sort(rng.integers(0, 3, pairs)).astype(np.int32)
    f = (1000.0 ** (-np.arange(pairs) / pairs)).astype(np.float32)
    cache = bc.BoundedCache(ctx, layers, n_seqs, heads, kv, hd, budget, rows, torch.from_numpy(f).cuda(), torch.from_numpy(axis).cuda(), slack=10,
                            block=block, n_sink=2, n_recent=8)
    # a tree of six rows: 0 - 1 - 2 and 0 - 3 - (4, 5); accepted paths 0, 3, 5 and 0, 1
    masks = np.array([[1, 3, 7, 9, 25, 41]] * n_seqs, np.uint32)
    paths = np.array([[0, 3, 5, -1, -1, -1], [0, 1, -1, -1, -1, -1]], np.int32)
    evicted = 0
    for step in range(steps):
        fill, age_end = host(cache.fill), host(cache.next_age)
        before = [[host(x).copy() for x in (cache.k[i], cache.v[i], cache.k_scale[i], cache.v_scale[i], cache.mass[cache.turn][i],
                                            cache.age[cache.turn][i])] for i in range(layers)]
        if cache.make_room():
            evicted += 1
            for i in range(layers):
                k, v, ks, vs, mass, age = before[i]
                kept, m, a, n = Q.evict(k, v, ks, vs, mass, age, fill, age_end, budget, 2, 8, block)
                np.testing.assert_array_equal(host(cache.fill), n)
                np.testing.assert_array_equal(host(cache.k[i]), k)
                np.testing.assert_array_equal(host(cache.v[i]), v)
                np.testing.assert_array_equal(host(cache.k_scale[i]), ks)
                for b in range(n_seqs):
                    np.testing.assert_array_equal(host(cache.mass[cache.turn][i])[b, :, :fill[b]], m[b, :, :fill[b]])
                    np.testing.assert_array_equal(host(cache.age[cache.turn][i])[b, :, :fill[b]], a[b, :, :fill[b]])
        fill = host(cache.fill)
        assert (fill <= cache.fill_most).all() and (fill + rows <= cache.cap).all()
        pos = bc.clip_positions(cache.next_age, rows, 4, 5)
        rope = cache.rope(pos)
        count = np.array([3, 2], np.int32) if tree else rng.integers(1, rows + 1, n_seqs).astype(np.int32)
        for i in range(layers):
            qkv = torch.from_numpy(rng.standard_normal((n_seqs, rows, heads + 2 * kv, hd))).cuda().to(torch.bfloat16)
            q, k, v = qkv.split((heads, kv, kv), dim=2)
            m0 = host(cache.mass[cache.turn][i]).copy()
            turned = cache.append(i, q, k, v, rope)
            out = torch.zeros_like(turned)
            cache.attend(i, turned, out, mass_rows=1, visible=torch.from_numpy(masks.view(np.int32)).cuda() if tree else None)
            for b in range(n_seqs):
                m0[b, :, fill[b]:fill[b] + rows] = 0
            want, _, mass, spread = Q.attend(host(cache.k[i]), host(cache.v[i]), host(cache.k_scale[i]), host(cache.v_scale[i]), host(turned), fill,
                                             block, visible=masks if tree else None, mass=m0, mass_rows=1)
            assert (np.abs(host(out) - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -13) * spread).all()
            np.testing.assert_allclose(host(cache.mass[cache.turn][i]), mass, rtol=2.0 ** -15, atol=2.0 ** -30)
            if tree:
                cache.put_again(i, k, v, rope, torch.from_numpy(paths).cuda(), torch.from_numpy(count).cuda())
                kt = Q.rotate_axes(host(k), f, axis, host(pos), False)
                for b in range(n_seqs):
                    at = np.arange(fill[b], fill[b] + count[b])
                    s = host(cache.k_scale[i])[b][:, at // block][..., None]
                    got, x = Q.e4m3_decode(host(cache.k[i])[b][:, at]) * s, kt[b, paths[b, :count[b]]].transpose(1, 0, 2)
                    assert (np.abs(got - x) <= np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10) * (1 + 1e-5) + 1e-5).all()
        cache.commit(torch.from_numpy(count).cuda(), rows if not tree else 3)
    assert evicted >= 2 and vb.vvs_device_status(ctx) == 0
    vb.vvs_destroy(ctx)


def test_demo_stays_within_its_budget():
    got = bc.demo(steps=150, verbose=False)
    assert got["status"] == 0 and got["finite"] and got["evictions"] >= 2
    assert all(n > 600 for n in got["tokens"]) and all(n <= 448 + 256 + 9 for n in got["fill"])
