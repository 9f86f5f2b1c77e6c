"""What a bounded cache refuses when it is made, not when it is full (on the CPU: nothing is allocated before)."""
import os
import re

import pytest
import torch

from paper_2511_13587_b200 import binding as vb
from paper_2511_13587_b200.bounded_cache import BoundedCache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GOOD = dict(ctx=0, n_layers=2, n_seqs=1, n_heads=4, n_kv_heads=2, head_dim=64, budget=512, max_rows=9, inv_freq=torch.ones(4),
            axis=torch.zeros(4, dtype=torch.int32), device="cpu")


@pytest.mark.parametrize("wrong,told", [
    (dict(budget=131072), "131072"), (dict(budget=130000, slack=1064), "131072"), (dict(budget=100, max_rows=131000), "131072"),
    (dict(budget=130999, slack=0, max_rows=9, block=128), None), (dict(budget=0), "budget"), (dict(max_rows=0), "max_rows"), (dict(slack=-1), "slack"),
    (dict(n_heads=3), "multiple"), (dict(n_kv_heads=0), "heads"), (dict(n_layers=0), "layers"), (dict(block=48), "block"), (dict(head_dim=96), "head"),
    (dict(n_sink=-1), "n_sink"), (dict(n_recent=-1), "n_recent"), (dict(n_sink=500, n_recent=13), "budget"), (dict(mass_decay=-0.5), "mass_decay"),
    (dict(mass_decay=float("nan")), "mass_decay")])
def test_a_cache_that_could_not_run(wrong, told):
    # what passes the checks ends at the first tensor that is not on a device
    with pytest.raises(ValueError, match=told or "CUDA"):
        BoundedCache(**dict(GOOD, **wrong))


def test_the_limit_is_the_library_s():
    with open(os.path.join(ROOT, "include", "vvs.h")) as f:
        assert int(re.search(r"#define VVS_QCACHE_EVICT_CAP (\d+)", f.read()).group(1)) == vb.VVS_QCACHE_EVICT_CAP
