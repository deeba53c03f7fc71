"""The operators around a paged cache where calls go wrong or run long: bad entries and words that are up, waits that run out, other streams,
and the kernels' forms for many units, many rows and long ranges, against the float64 oracle.  Tolerances: see test_gpu_paged.py."""
import numpy as np
import pytest
import torch

from paper_2608_03682_b200 import binding
from tests.test_gpu_paged import Paged, ints, normal

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------------------
# what a call finds wrong on the device
# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("q_len", [1, 3])
def test_fp32_blocks_that_begin_while_others_raise_the_word(q_len):
    """Every request of several waves of blocks has a bad entry, so that blocks begin before, while and after the word goes up: all threads of
    a block go by one value of it."""
    batch, kv = 600, 48
    p = Paged(81, [q_len] * batch, [kv] * batch, 2, 128, 16, "f32", layers=1, layer=0)
    q, args = normal(p.rng, (p.T, 4, 128), "f32").cuda(), p.device_args()
    want = p.cache.attend(0, q, *args)
    assert p.cache.poll_status() == 0
    table = p.table.copy()
    table[:, 1] = p.cache.n_pages
    bad = ints(table)
    for _ in range(50):
        p.cache.attend(0, q, *args[:2], bad)
        assert p.cache.poll_status() == binding.ERR_INVALID_ARG
    assert torch.equal(want, p.cache.attend(0, q, *args)) and p.cache.poll_status() == 0
