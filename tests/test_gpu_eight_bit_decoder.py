"""Decoder layers in 8 bits over the bounded cache, as a program runs them: a step is the sequence of calls that it says (the same bits from calls
made by hand on buffers of their own, with every product and rounding held to its bounds), in a graph too; and a clip decoded to its end."""
import numpy as np
import pytest
import torch

from oracle import block_quant_oracle as B
from paper_2511_13587_b200 import binding as vb
from paper_2511_13587_b200 import eight_bit_decoder as ed
from paper_2511_13587_b200.bounded_cache import BoundedCache, clip_positions
from test_gpu_block_quant import BF16, F32, check_codes, check_product, coded, ctxs, host  # noqa: F401

pytestmark = pytest.mark.gpu
LAYERS, SEQS, ROWS = 2, 2, 9


def decoder(ctx, dtype, d, heads, kv, hd, ff, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    pairs = hd // 2
    inv_freq = torch.pow(1000.0, -torch.arange(pairs, device="cuda").float() / pairs)
    cache = BoundedCache(ctx, LAYERS, SEQS, heads, kv, hd, 64, ROWS, inv_freq, torch.zeros(pairs, dtype=torch.int32, device="cuda"),
                         n_recent=16, dtype=dtype)
    weights = ed.random_weights(g, LAYERS, d, heads, kv, hd, ff, dtype)
    x = [torch.randn((SEQS, ROWS, d), generator=g, device="cuda").to(dtype) for _ in range(3)]
    return ed.EightBitDecoder(ctx, weights, cache, ff), weights, x


def by_hand(ctx, dtype, weights, cache, x, d, heads, kv, hd, ff):
    """The step's calls, each checked against the oracle from what the device holds before it."""
    n = SEQS * ROWS
    rope = cache.rope(clip_positions(cache.next_age, ROWS, 4, 4)[:1].contiguous())
    new = lambda cols: torch.zeros((n, cols), dtype=dtype, device="cuda")  # noqa: E731

    def weight(w):
        q = coded(*w.shape, True)
        vb.vvs_weight_quant(ctx, w.contiguous(), *q)
        check_codes(*q, host(w), 0.0, 128)
        return q

    def normed(t, residual, w):
        q, s = coded(n, d), new(d)
        vb.vvs_norm_quant(ctx, t, w, 1e-5, *q, residual=residual, sum_out=s)
        check_codes(*q, B.norm(host(t), None if residual is None else host(residual), host(w), 1e-5)[1], 2.0 ** -17)
        return q, s

    def product(a, w):
        out = new(w[0].shape[0])
        vb.vvs_block_matmul(ctx, *a, vb.make_qweight(*w), out)
        check_product(out, [*a, *w])
        return out
    stream, delta = x.reshape(n, d), None
    for i, w in enumerate(weights["layers"]):
        q, stream = normed(stream, None, w["norm1"]) if delta is None else normed(delta, stream, w["norm1"])
        qkv = product(q, weight(w["w_qkv"])).view(SEQS, ROWS, heads + 2 * kv, hd)
        out = torch.zeros((SEQS, ROWS, heads, hd), dtype=dtype, device="cuda")
        cache.attend(i, cache.append(i, *qkv.split((heads, kv, kv), dim=2), rope), out)
        a = coded(n, heads * hd)
        vb.vvs_rows_quant(ctx, out.view(n, heads * hd), *a)
        check_codes(*a, host(out.view(n, heads * hd)), 0.0)
        delta = product(a, weight(w["w_o"]))
        q, stream = normed(delta, stream, w["norm2"])
        both = product(q, weight(torch.cat((w["w_gate"], w["w_up"]))))
        h = coded(n, ff)
        vb.vvs_rows_quant(ctx, both[:, ff:], *h, gate=both[:, :ff])
        check_codes(*h, B.gated(host(both[:, ff:]), host(both[:, :ff])), 2.0 ** -15)
        delta = product(h, weight(w["w_down"]))
    features, q = new(d), coded(n, d)
    vb.vvs_norm_quant(ctx, delta, weights["norm_f"], 1e-5, *q, residual=stream, norm_out=features)
    return features.view(SEQS, ROWS, d)


def state(cache):
    return [x.clone() for x in (cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale, cache.v_scale, cache.mass, cache.age)]


@pytest.mark.parametrize("dtype,d,heads,kv,hd,ff", [(BF16, 320, 5, 5, 64, 864), (BF16, 512, 4, 2, 128, 1376), (F32, 256, 4, 4, 64, 1024)])
def test_a_step_is_its_calls(ctxs, dtype, d, heads, kv, hd, ff):  # noqa: F811
    one, weights, x = decoder(ctxs[dtype], dtype, d, heads, kv, hd, ff)
    two = decoder(ctxs[dtype], dtype, d, heads, kv, hd, ff)[0]                    # its cache, for the calls by hand
    count = torch.full((SEQS,), 4, dtype=torch.int32, device="cuda")
    for block in x[:2]:
        got = one.step(block, clip_positions(one.cache.next_age, ROWS, 4, 4)[:1].contiguous()).clone()
        want = by_hand(ctxs[dtype], dtype, weights, two.cache, block, d, heads, kv, hd, ff)
        assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(state(one.cache), state(two.cache)))
        for c in (one.cache, two.cache):
            c.commit(count, 4)
    # once more, captured: nothing of the step depends on when it is launched
    pos = clip_positions(one.cache.next_age, ROWS, 4, 4)[:1].contiguous()
    before = state(one.cache)
    want = one.step(x[2], pos).clone()
    after = state(one.cache)
    for a, b in zip((one.cache.k.view(torch.uint8), one.cache.v.view(torch.uint8), one.cache.k_scale, one.cache.v_scale, one.cache.mass,
                     one.cache.age), before):
        a.copy_(b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = one.step(x[2], pos)
    out.zero_()
    g.replay()
    assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(state(one.cache), after))
    assert vb.vvs_device_status(ctxs[dtype]) == 0


def test_a_clip(ctxs):  # noqa: F811
    got = ed.demo(steps=70, n_layers=2, d_model=320, n_heads=5, n_kv_heads=5, d_ff=864, budget=128, verbose=False)
    assert got["status"] == 0 and got["finite"] and got["evictions"] >= 1 and max(got["fill"]) <= 128 + 256 + 9
    per_layer = (3 + 1) * 320 * 320 + 3 * 320 * 864
    blocks = 8 * 3 + 3 * 3 + 14 * 3 + 3 * 7
    assert got["weight_bytes"] == 2 * (per_layer + 4 * blocks)


def test_what_does_not_fit_is_refused(ctxs):  # noqa: F811
    one, weights, x = decoder(ctxs[BF16], BF16, 320, 5, 5, 64, 864)
    with pytest.raises(ValueError, match="expected"):
        one.step(torch.zeros((SEQS, ROWS + 1, 320), dtype=BF16, device="cuda"), torch.zeros((1, SEQS, ROWS + 1), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="w_down"):
        bad = dict(weights, layers=[dict(w, w_down=w["w_down"].t()) for w in weights["layers"]])
        ed.EightBitDecoder(ctxs[BF16], bad, one.cache, 864)
    with pytest.raises(ValueError, match="layers"):
        ed.EightBitDecoder(ctxs[BF16], dict(weights, layers=weights["layers"][:1]), one.cache, 864)
