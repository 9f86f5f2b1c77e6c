"""Eviction of more heads than the device has SMs (selected by CTAs of 256 or 512 threads, several on an SM, by digits of eight bits), against the
oracle; and a cache that is evicted and rounded again many times, against the values that were put into it.

Evictions are exact.  A stored value is within half a step of the code (2^-4 of the value, 2^-10 of the scale) when it is put; a scale that grows is a power of
two times the old one, which changes codes by their exponent and rounds those below 2^-6 again, by half a step of the new scale at most: all of these
together less than twice the last, 2^-9 of the scale."""
import numpy as np
import pytest
import torch

from oracle import quant_cache_oracle as Q
from paper_2511_13587_b200 import binding as vb
from paper_2511_13587_b200 import bounded_cache as bc
from test_gpu_quant_cache import BF16, ctxs, dev, host  # noqa: F401
from vvs_synth import gen
from vvs_synth.configs import ModelShape

pytestmark = pytest.mark.gpu


# heads of a sequence, blocks, slots, what stays, guarded, kind of weights: (times the SMs that heads are more than)
MANY = [(8, 16, 640, 448, 1, 64, "plain", 1), (8, 32, 1504, 1001, 3, 100, "ties", 1), (4, 64, 2048, 700, 0, 0, "odd", 1), (8, 16, 1024, 333, 4, 50, "odd", 2),
        (10, 128, 640, 129, 0, 129, "plain", 2), (8, 16, 96, 33, 1, 2, "ties", 2), (8, 32, 1024, 1023, 5, 300, "ties", 2), (4, 16, 3008, 1, 1, 0, "plain", 1)]


@pytest.mark.parametrize("heads,block,cap,keep,sink,recent,kind,times", MANY)
def test_more_heads_than_sms(ctxs, heads, block, cap, keep, sink, recent, kind, times):  # noqa: F811
    rng = gen.rng_for(81, f"many{heads}{block}{cap}{kind}")
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    b, hd = times * sms // heads + 1, 64
    assert b * heads > times * sms and cap <= 8192
    fills = rng.integers(keep + 1, cap + 1, b).astype(np.int32) if keep < cap else np.full(b, cap, np.int32)
    fills[0], fills[1], fills[2], fills[3] = cap, keep, max(0, keep - 1), 0
    c = [rng.integers(0, 256, (b, heads, cap, hd)).astype(np.uint8) for _ in range(2)]
    for x in c:
        x[(x & 127) == 127] = 1
    c += [(2.0 ** rng.integers(-9, -4, (b, heads, cap // block))).astype(np.float32) for _ in range(2)]
    mass = rng.standard_normal((b, heads, cap)).astype(np.float32)
    if kind == "ties":
        mass = rng.integers(0, 3, mass.shape).astype(np.float32) * rng.choice([1.0, -1.0], mass.shape).astype(np.float32)
    if kind == "odd":
        pick = rng.integers(0, 6, mass.shape)
        mass[pick == 0], mass[pick == 1], mass[pick == 2], mass[pick == 3] = np.nan, np.inf, -np.inf, -0.0
    ages = np.stack([np.stack([rng.permutation(2 * cap)[:cap] for _ in range(heads)]) for _ in range(b)]).astype(np.int32)
    nxt = np.full(b, 2 * cap, np.int32)
    t = [dev(x) for x in c + [mass, ages]]
    mass_out, age_out = torch.full_like(t[4], 5), torch.full_like(t[5], 5)
    new_len, kept = torch.zeros(b, dtype=torch.int32, device="cuda"), torch.zeros((b, heads, keep), dtype=torch.int32, device="cuda")
    vb.vvs_quant_cache_evict(ctxs[BF16], vb.make_qcache(*t), dev(fills), keep, sink, recent, dev(nxt), mass_out, age_out, new_len, kept)
    assert vb.vvs_device_status(ctxs[BF16]) == 0
    w_kept, w_mass, w_age, w_len = Q.evict(*c, mass, ages, fills, nxt, keep, sink, recent, block)
    np.testing.assert_array_equal(host(kept), w_kept)
    np.testing.assert_array_equal(host(new_len), w_len)
    for got, want in zip(t[:4], c):
        np.testing.assert_array_equal(got.cpu().numpy(), want)
    for i in range(b):
        n = fills[i]
        np.testing.assert_array_equal(mass_out[i, :, :n].cpu().numpy(), w_mass[i, :, :n])
        np.testing.assert_array_equal(age_out[i, :, :n].cpu().numpy(), w_age[i, :, :n])
        assert (mass_out[i, :, n:] == 5).all() and (age_out[i, :, n:] == 5).all()


@pytest.mark.parametrize("block,grow", [(16, 1.0), (64, 1.03)])
def test_values_after_many_evictions(block, grow):
    """Tokens that stay for hundreds of steps are still the ones that were put, whatever their blocks went through; with rows that become larger, so that
    scales grow."""
    rng = gen.rng_for(82, f"drift{block}")
    n_seqs, heads, hd, rows, budget = 2, 2, 64, 5, 96
    ctx = vb.vvs_create(vb.make_desc(ModelShape("clip", 0, 64, 0, 0, 0, 128), 1, 1))
    f = (1000.0 ** (-np.arange(32) / 32)).astype(np.float32)
    cache = bc.BoundedCache(ctx, 1, n_seqs, heads, heads, hd, budget, rows, dev(f), torch.zeros(32, dtype=torch.int32, device="cuda"), slack=11, block=block,
                            n_sink=7, n_recent=20)
    put = [[{} for _ in range(n_seqs)] for _ in range(2)]      # of keys and values: age -> [heads, hd]
    ends, evicted = np.zeros(n_seqs, int), 0
    for step in range(160):
        evicted += cache.make_room()
        pos = cache.next_age.view(1, -1, 1) + torch.arange(rows, device="cuda", dtype=torch.int32).view(1, 1, -1)
        x = rng.standard_normal((n_seqs, rows, 3 * heads, hd)) * np.exp(0.5 * rng.standard_normal((n_seqs, rows, 1, 1))) * grow ** step
        qkv = dev(x, BF16)
        q, k, v = qkv.split((heads, heads, heads), dim=2)
        turned = cache.append(0, q, k, v, cache.rope(pos.contiguous()))
        cache.attend(0, turned, torch.zeros_like(turned))
        n = rng.integers(1, rows + 1, n_seqs).astype(np.int32)
        kt = Q.rotate_axes(host(k), f, np.zeros(32, int), host(pos), False)
        for b in range(n_seqs):
            for t in range(n[b]):
                put[0][b][ends[b] + t], put[1][b][ends[b] + t] = kt[b, t], host(v)[b, t]
        ends += n
        cache.commit(dev(n), rows)
    assert evicted >= 10 and vb.vvs_device_status(ctx) == 0
    ages, fill = host(cache.age[cache.turn][0]), host(cache.fill)
    for codes, scales, rows_of in ((cache.k, cache.k_scale, put[0]), (cache.v, cache.v_scale, put[1])):
        got, s = Q.e4m3_decode(codes[0].view(torch.uint8).cpu().numpy()), host(scales[0])
        for b in range(n_seqs):
            for h in range(heads):
                a = ages[b, h, :fill[b]]
                assert len(set(a.tolist())) == fill[b] and set(range(7)) <= set(a.tolist()) and set(range(ends[b] - 5, ends[b])) <= set(a.tolist())
                want = np.stack([rows_of[b][i][h] for i in a])
                each = s[b, h][np.arange(fill[b]) // block][:, None]
                room = np.abs(want) * 2.0 ** -4 + each * 2.0 ** -9
                assert (np.abs(got[b, h, :fill[b]] * each - want) <= room * (1 + 1e-5)).all()
    vb.vvs_destroy(ctx)
