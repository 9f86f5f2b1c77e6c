"""Elements that a rotation leaves alone (behind the last pair, or of an unknown axis) come out bit for bit, next to infinities, NaN and
zeros of either sign: through `vvs_rotate_axes` and through `vvs_quant_cache_append` with positions.

No tolerances: unturned elements are compared by their bits, codes with the oracle's of the same values."""
import numpy as np
import pytest
import torch

from oracle import quant_cache_oracle as Q
from paper_2511_13587_b200 import binding as vb
from test_gpu_quant_cache import BF16, F32, ctxs, dev, host  # noqa: F401
from vvs_synth import gen

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == BF16 else torch.int32)


def unturned_elements(hd, n_pairs, halves, axis, n_axes):
    """Elements that stay, and the partner of each that is in a pair of an unknown axis."""
    stay = list(range(2 * n_pairs, hd))
    for i, a in enumerate(axis):
        if not 0 <= a < n_axes:
            stay += [i, i + n_pairs] if halves else [2 * i, 2 * i + 1]
    return sorted(stay)


def planted(rng, b, t, h, hd, stay, dtype):
    """Normal values; of the elements that stay every other one of each row is an infinity, a NaN or -0, its neighbours are finite."""
    x = dev(rng.standard_normal((b, t, h, hd)), dtype)
    for n, e in enumerate(stay):
        if (e + n) % 2 == 0:
            x[:, n % t::3, :, e] = (INF, -INF, NAN, -0.0)[n % 4]
        elif n % 4 == 1:
            x[:, :, :, e] = -0.0
    return x


# (hd, pairs, halves, axes of some pairs outside 0 .. 1)
PARTS = [(64, 30, False, []), (64, 21, False, []), (64, 1, False, []), (64, 24, True, []), (128, 50, False, [3, 17, 49]), (128, 64, False, [0, 63]),
         (128, 32, True, [5, 6, 31]), (64, 32, True, [0])]


def rope_parts(rng, hd, n_pairs, unknown, b, t):
    axis = rng.integers(0, 2, n_pairs).astype(np.int32)
    axis[unknown] = rng.choice([-1, 2, 1000], len(unknown))
    f = (10000.0 ** (-np.arange(n_pairs) / n_pairs)).astype(np.float32)
    return f, axis, rng.integers(0, 500, (2, b, t)).astype(np.int32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,n_pairs,halves,unknown", PARTS)
def test_rotation_leaves_unturned_elements_alone(ctxs, dtype, hd, n_pairs, halves, unknown):  # noqa: F811
    rng = gen.rng_for(51, f"stay{hd}{n_pairs}{halves}{len(unknown)}")
    b, t, h, kv = 2, 7, 5, 2
    f, axis, pos = rope_parts(rng, hd, n_pairs, unknown, b, t)
    stay = unturned_elements(hd, n_pairs, halves, axis, 2)
    q, k = planted(rng, b, t, h, hd, stay, dtype), planted(rng, b, t, kv, hd, stay, dtype)
    rope = vb.make_rope_axes(dev(f), dev(axis), dev(pos), halves)
    q_out, k_out = torch.zeros_like(q), torch.zeros_like(k)
    vb.vvs_rotate_axes(ctxs[dtype], rope, q, q_out, k, k_out)
    assert vb.vvs_device_status(ctxs[dtype]) == (vb.VVS_DEV_BAD_ARG if unknown else 0)
    turned = sorted(set(range(hd)) - set(stay))
    for x, y in ((q, q_out), (k, k_out)):
        assert torch.equal(bits(y)[..., stay], bits(x)[..., stay])
        assert y[..., turned].isfinite().all() and not torch.equal(y[..., turned], x[..., turned])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t,block", [(9, 64), (70, 128)])             # one launch of a warp for a head, and a prompt's launches
@pytest.mark.parametrize("hd,n_pairs,halves,unknown", PARTS)
def test_append_leaves_unturned_elements_alone(ctxs, dtype, t, block, hd, n_pairs, halves, unknown):  # noqa: F811
    rng = gen.rng_for(52, f"stay{hd}{n_pairs}{halves}{len(unknown)}{t}")
    b, h, kv, cap = 2, 3, 2, 128
    f, axis, pos = rope_parts(rng, hd, n_pairs, unknown, b, t)
    stay = unturned_elements(hd, n_pairs, halves, axis, 2)
    q, k = planted(rng, b, t, h, hd, stay, dtype), planted(rng, b, t, kv, hd, stay, dtype)
    v = dev(rng.standard_normal((b, t, kv, hd)), dtype)
    rope = vb.make_rope_axes(dev(f), dev(axis), dev(pos), halves)
    c = [torch.zeros((b, kv, cap, hd), dtype=torch.uint8, device="cuda") for _ in range(2)] + \
        [torch.zeros((b, kv, cap // block), device="cuda") for _ in range(2)]
    q_out = torch.zeros_like(q)
    vb.vvs_quant_cache_append(ctxs[dtype], vb.make_qcache(*c), k, v, torch.zeros(b, dtype=torch.int32, device="cuda"), rope=rope, q=q, q_out=q_out)
    told = vb.vvs_device_status(ctxs[dtype])
    assert told == (0 if k.isfinite().all() else vb.VVS_DEV_NONFINITE) | (vb.VVS_DEV_BAD_ARG if unknown else 0)
    assert torch.equal(bits(q_out)[..., stay], bits(q)[..., stay])
    # codes of the elements that stay: the oracle's of their values under the block's scale
    each = np.arange(t) // block
    want = Q.e4m3_encode(host(k).transpose(0, 2, 1, 3) / c[2].cpu().numpy()[:, :, each][..., None])
    np.testing.assert_array_equal(c[0][:, :, :t].cpu().numpy()[..., stay], want[..., stay])
    # and the scale is that of the finite values
    turned = Q.rotate_axes(np.nan_to_num(host(k), nan=0.0, posinf=0.0, neginf=0.0), f, np.where((axis >= 0) & (axis < 2), axis, 0), pos, halves)
    kept = np.where(np.isfinite(host(k)), host(k), 0.0)
    turned[..., stay] = kept[..., stay]
    most = np.abs(turned)[:, :block].max(axis=(1, 3))
    got = c[2][:, :, 0].cpu().numpy()
    assert all(got[i, j] in (Q.block_scale(most[i, j] * (1 - 1e-5)), Q.block_scale(most[i, j] * (1 + 1e-5))) for i in range(b) for j in range(kv))
