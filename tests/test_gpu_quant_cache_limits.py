"""Sizes that no launch takes are refused as such, and leave no error behind for the next call of the program."""
import pytest
import torch

from paper_2511_13587_b200 import binding as vb
from test_gpu_quant_cache import BF16, ctxs  # noqa: F401

pytestmark = pytest.mark.gpu
SHAPE = -2


def many_heads(n):
    c = [torch.zeros((1, n, 16, 64), dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.ones((1, n, 1), device="cuda") for _ in range(2)]
    return vb.make_qcache(*c, torch.zeros((1, n, 16), device="cuda"))


@pytest.mark.parametrize("mass_rows", [0, 1])
def test_cached_heads(ctxs, mass_rows):  # noqa: F811
    ctx = ctxs[BF16]
    lens = torch.full((1,), 3, dtype=torch.int32, device="cuda")
    for n, fits in ((65535, True), (65536, False), (70001, False)):
        q = torch.ones((1, 1, n, 64), dtype=BF16, device="cuda")
        out = torch.full_like(q, 7)
        if fits:
            vb.vvs_quant_cache_attend(ctx, many_heads(n), q, out, lens, mass_rows=mass_rows)
            assert (out == 0).all()
            continue
        with pytest.raises(vb.VvsError) as e:
            vb.vvs_quant_cache_attend(ctx, many_heads(n), q, out, lens, mass_rows=mass_rows)
        assert e.value.status == SHAPE
        assert (out + 1 == 8).all()                            # (torch asks for the last error behind its launches)
    assert vb.vvs_device_status(ctx) == 0

