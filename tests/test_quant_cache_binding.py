"""What the binding of the 8-bit cache's entry points refuses: tensors of another type, shape or layout than the kernels would take them for, and
tensors that are not on the device.  On the CPU: no call comes as far as the library."""
import pytest
import torch

from paper_2511_13587_b200 import binding as vb

N_SEQS, ROWS, HEADS, KV, HD, CAP, BLOCK, KEEP = 2, 3, 4, 2, 64, 48, 16, 20
I32 = torch.int32


def rope_args(**other):
    a = dict(inv_freq=torch.ones(32), axis=torch.zeros(32, dtype=I32), pos=torch.zeros((2, N_SEQS, ROWS), dtype=I32))
    return dict(a, **other)


# What is wrong, and what the message names; CPU tensors are told of once everything else is right.
ROPE = [(dict(pos=torch.zeros((2, 2, 3), dtype=torch.int64)), "pos.*int32"), (dict(axis=torch.zeros(32, dtype=torch.int64)), "axis.*int32"),
        (dict(inv_freq=torch.ones(32, dtype=torch.float64)), "inv_freq.*float32"),
        (dict(inv_freq=torch.ones(32).to(torch.bfloat16)), "inv_freq.*float32"),
        (dict(axis=torch.zeros(31, dtype=I32)), "axis.*32"), (dict(pos=torch.zeros((2, 3, 2), dtype=I32).transpose(1, 2)), "pos.*contiguous"),
        (dict(pos=torch.zeros((2, 6), dtype=I32)), "pos"), (dict(pos=torch.zeros((2, 2, 3))), "pos.*int32"),
        (dict(inv_freq=torch.ones(64)[::2]), "contiguous"), ({}, "CUDA")]


@pytest.mark.parametrize("wrong,told", ROPE)
def test_positions_and_frequencies(wrong, told):
    with pytest.raises(ValueError, match=told):
        vb.make_rope_axes(**rope_args(**wrong))


def test_what_is_no_tensor():
    for name in ("inv_freq", "pos"):
        with pytest.raises(TypeError, match=name):
            vb.make_rope_axes(**rope_args(**{name: 0}))


CACHE = [(dict(mass=torch.zeros((N_SEQS, KV, CAP), dtype=I32)), "mass"), (dict(age=torch.zeros((N_SEQS, KV, CAP))), "age"),
         (dict(k_scale=torch.ones((N_SEQS, KV, 3), dtype=I32)), "k_scale"),
         (dict(k=torch.zeros((N_SEQS, KV, CAP, HD), dtype=torch.int16)), "k"), ({}, "CUDA")]


@pytest.mark.parametrize("wrong,told", CACHE)
def test_a_cache(wrong, told):
    a = dict(k=torch.zeros((N_SEQS, KV, CAP, HD), dtype=torch.uint8), k_scale=torch.ones((N_SEQS, KV, CAP // BLOCK)))
    a.update(v=a["k"], v_scale=a["k_scale"], mass=torch.zeros((N_SEQS, KV, CAP)), age=torch.zeros((N_SEQS, KV, CAP), dtype=I32))
    with pytest.raises(ValueError, match=told):
        vb.make_qcache(**dict(a, **wrong))


def qcache():
    return vb.vvs_qcache(n_seqs=N_SEQS, n_heads=KV, head_dim=HD, cap=CAP, block=BLOCK)


def rows(heads, **kw):
    return torch.zeros((N_SEQS, ROWS, heads, HD), **kw)


def lens(n=N_SEQS, dtype=I32):
    return torch.zeros(n, dtype=dtype)


ARRAYS = [(lens(dtype=torch.int64), "int32"), (lens(N_SEQS - 1), r"int32 \[2\]"), (torch.zeros(N_SEQS), "int32"),
          (torch.zeros((N_SEQS, 2), dtype=I32)[:, 0], "contiguous"), (torch.zeros((N_SEQS, 2), dtype=I32), r"int32 \[2\]"), (lens(), "CUDA")]


@pytest.mark.parametrize("name", ["cache_len", "row_count", "next_age"])
@pytest.mark.parametrize("wrong,told", ARRAYS)
def test_append(name, wrong, told):
    a = dict(cache_len=lens(), row_count=lens(), next_age=lens())
    with pytest.raises(ValueError, match=told if told == "CUDA" else name + ".*" + told):
        vb.vvs_quant_cache_append(None, qcache(), rows(KV), rows(KV), stream=0, **dict(a, **{name: wrong}))


def test_append_of_picked_rows():
    for wrong in (torch.zeros((N_SEQS, ROWS - 1), dtype=I32), torch.zeros((N_SEQS, ROWS), dtype=torch.int64),
                  torch.zeros((ROWS, N_SEQS), dtype=I32).T):
        with pytest.raises(ValueError, match="row_index"):
            vb.vvs_quant_cache_append(None, qcache(), rows(KV), rows(KV), lens(), row_index=wrong, stream=0)


@pytest.mark.parametrize("name", ["cache_len", "row_count", "first_slot"])
@pytest.mark.parametrize("wrong,told", ARRAYS)
def test_attend(name, wrong, told):
    a = dict(cache_len=lens(), row_count=lens(), first_slot=lens())
    with pytest.raises(ValueError, match=told if told == "CUDA" else name + ".*" + told):
        vb.vvs_quant_cache_attend(None, qcache(), rows(HEADS), rows(HEADS), stream=0, **dict(a, **{name: wrong}))


def test_attend_masks_and_sums():
    for name, wrong in (("visible", torch.zeros((N_SEQS, ROWS), dtype=torch.int64)), ("visible", torch.zeros((N_SEQS, ROWS - 1), dtype=I32)),
                        ("visible", torch.zeros((N_SEQS, ROWS, ROWS), dtype=torch.bool)), ("lse", torch.zeros((N_SEQS, ROWS, HEADS - 1))),
                        ("lse", torch.zeros((N_SEQS, ROWS, HEADS), dtype=torch.float64)),
                        ("lse", torch.zeros((N_SEQS, HEADS, ROWS)).transpose(1, 2))):
        with pytest.raises(ValueError, match=name):
            vb.vvs_quant_cache_attend(None, qcache(), rows(HEADS), rows(HEADS), lens(), stream=0, **{name: wrong})


def test_evict():
    good = dict(cache_len=lens(), keep=KEEP, n_sink=1, n_recent=2, next_age=lens(), mass_out=torch.zeros((N_SEQS, KV, CAP)),
                age_out=torch.zeros((N_SEQS, KV, CAP), dtype=I32), new_len=lens(), kept=torch.zeros((N_SEQS, KV, KEEP), dtype=I32))
    for name, wrong in (("cache_len", lens(dtype=torch.int64)), ("next_age", lens(1)), ("new_len", lens(1)), ("new_len", lens(dtype=torch.int64)),
                        ("mass_out", torch.zeros((N_SEQS, KV, KEEP))), ("mass_out", torch.zeros((N_SEQS, KV, CAP), dtype=I32)),
                        ("age_out", torch.zeros((N_SEQS, KV, CAP), dtype=torch.int64)), ("age_out", torch.zeros((N_SEQS, CAP), dtype=I32)),
                        ("kept", torch.zeros((N_SEQS, KV, KEEP - 1), dtype=I32)), ("kept", torch.zeros((N_SEQS, KEEP), dtype=I32)),
                        ("kept", torch.zeros((N_SEQS, KV, KEEP), dtype=torch.int64))):
        with pytest.raises(ValueError, match=name):
            vb.vvs_quant_cache_evict(None, qcache(), stream=0, **dict(good, **{name: wrong}))
    with pytest.raises(ValueError, match="CUDA"):
        vb.vvs_quant_cache_evict(None, qcache(), stream=0, **good)


def test_rotation_of_another_block():
    rope = vb._RopeOfRows(n_axes=2, n_pairs=32, n_seqs=N_SEQS, n_rows=ROWS)
    for q in (torch.zeros((N_SEQS, ROWS + 1, HEADS, HD)), torch.zeros((N_SEQS + 1, ROWS, HEADS, HD))):
        with pytest.raises(ValueError, match="rope: positions of 2 sequences and 3 rows"):
            vb.vvs_rotate_axes(None, rope, q, q, stream=0)
    k = torch.zeros((N_SEQS, ROWS + 1, KV, HD))
    with pytest.raises(ValueError, match="rope: positions of 2 sequences and 3 rows"):
        vb.vvs_quant_cache_append(None, qcache(), k, k, lens(), rope=rope, stream=0)
    with pytest.raises(ValueError, match="CUDA"):
        vb.vvs_rotate_axes(None, rope, rows(HEADS), rows(HEADS), stream=0)
    with pytest.raises(TypeError, match="vvs_rope_axes"):
        vb.vvs_rotate_axes(None, vb.vvs_heads(), rows(HEADS), rows(HEADS), stream=0)
    with pytest.raises(ValueError, match="4 dimensions"):
        vb.vvs_rotate_axes(None, rope, rows(HEADS)[0], rows(HEADS)[0], stream=0)
    with pytest.raises(ValueError, match="side by side"):
        vb.vvs_rotate_axes(None, rope, torch.zeros((N_SEQS, ROWS, HD, HEADS)).transpose(2, 3), rows(HEADS), stream=0)
