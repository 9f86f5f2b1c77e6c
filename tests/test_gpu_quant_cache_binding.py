"""Tensors that the binding of the 8-bit cache's entry points takes (any order of dimensions of rows of heads, flat and longer arrays, addresses) and
element types that it refuses, on the device; and that a refused call leaves everything as it was."""
import pytest
import torch

from paper_2511_13587_b200 import binding as vb
from test_gpu_quant_cache import BF16, F32, ctxs  # noqa: F401

pytestmark = pytest.mark.gpu
I32 = torch.int32


def zeros(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def small():
    c = [zeros(2, 2, 48, 64, dtype=torch.uint8) for _ in range(2)] + [torch.ones((2, 2, 3), device="cuda") for _ in range(2)]
    return c, vb.make_qcache(*c, zeros(2, 2, 48), zeros(2, 2, 48, dtype=I32))


@pytest.mark.parametrize("dtype,others", [(BF16, (torch.float16, torch.int16, F32)), (F32, (torch.int32, BF16, torch.float64))])
def test_rows_of_heads_of_another_type(ctxs, dtype, others):  # noqa: F811
    ctx = ctxs[dtype]
    c, qc = small()
    before = [x.clone() for x in c]
    rope = vb.make_rope_axes(torch.ones(32, device="cuda"), zeros(32, dtype=I32), zeros(1, 2, 3, dtype=I32))
    lens, good = zeros(2, dtype=I32), zeros(2, 3, 2, 64, dtype=dtype)
    for other in others:
        x = zeros(2, 3, 2, 64, dtype=other)
        for call in (lambda: vb.vvs_rotate_axes(ctx, rope, x, x), lambda: vb.vvs_rotate_axes(ctx, rope, good, x),
                     lambda: vb.vvs_quant_cache_append(ctx, qc, x, good, lens), lambda: vb.vvs_quant_cache_append(ctx, qc, good, x, lens),
                     lambda: vb.vvs_quant_cache_append(ctx, qc, good, good, lens, rope=rope, q=x, q_out=good),
                     lambda: vb.vvs_quant_cache_attend(ctx, qc, x, good, lens), lambda: vb.vvs_quant_cache_attend(ctx, qc, good, x, lens)):
            with pytest.raises(ValueError, match="elements"):
                call()
    assert vb.vvs_device_status(ctx) == 0 and all(torch.equal(x, y) for x, y in zip(c, before))


def test_arrays_that_are_taken(ctxs):  # noqa: F811
    """Longer flat arrays, arrays of other dimensions with as many elements, and addresses give what exact ones give."""
    ctx = ctxs[F32]
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn((2, 3, 2, 64), generator=g, device="cuda")
    exact = torch.tensor([7, 20], dtype=I32, device="cuda")
    longer = torch.tensor([7, 20, 99, -5], dtype=I32, device="cuda")
    got = []
    for lens in (exact, longer, exact.view(2, 1), exact.data_ptr(), exact.view(torch.uint32)):
        c, qc = small()
        vb.vvs_quant_cache_append(ctx, qc, x, x, lens)
        out, lse = zeros(2, 3, 2, 64), zeros(2, 3, 2)
        vb.vvs_quant_cache_attend(ctx, qc, x, out, lens, first_slot=lens, lse=lse if lens is exact else lse.view(-1))
        got.append(c + [out, lse])
        new_len, kept = zeros(2, dtype=I32), zeros(2, 2, 5, dtype=I32)
        vb.vvs_quant_cache_evict(ctx, qc, lens, 5, 0, 1, lens, zeros(2, 2, 48), None, new_len, kept if lens is exact else kept.view(-1))
        got[-1] += [new_len, kept]
    assert vb.vvs_device_status(ctx) == 0
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_positions_that_go_before_the_call(ctxs):  # noqa: F811
    """What make_rope_axes was given stays alive with its result."""
    ctx = ctxs[F32]
    x, a, b = torch.ones((2, 3, 1, 64), device="cuda"), zeros(2, 3, 1, 64), zeros(2, 3, 1, 64)
    freq, axis, pos = torch.full((32,), 0.5, device="cuda"), zeros(32, dtype=I32), torch.full((1, 2, 3), 3, dtype=I32, device="cuda")
    rope = vb.make_rope_axes(freq, axis, pos)
    assert rope._keep == (freq, axis, pos) and (rope.n_axes, rope.n_pairs, rope.halves, rope.n_seqs, rope.n_rows) == (1, 32, 0, 2, 3)
    vb.vvs_rotate_axes(ctx, rope, x, a)
    rope = vb.make_rope_axes(freq.clone(), axis.clone(), pos=pos.clone(), halves=False)
    torch.zeros(1 << 20, device="cuda")
    vb.vvs_rotate_axes(ctx, rope, x, b)
    assert torch.equal(a, b) and not torch.equal(a, x)
