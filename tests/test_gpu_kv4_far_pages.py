"""Pages behind 32-bit offsets, in every way of cutting the contexts: outputs and
lse are the bits that the same division gives over a small cache."""

import pytest
import torch

from tests.gpu_cases import d2sd
from tests.test_gpu_kv4_attention import Batch
from tests.test_gpu_kv4_shares import chain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_pages_give_the_bits_of_near_ones(dtype):
    m = d2sd()
    b = Batch([chain(9), chain(3)], [700, 50], 16, 8, dtype, seed=81)
    near, table, n = b.cache, b.d[0], b.cache.num_pages
    pages = (1 << 32) // (8 * 1024) + 1000
    far = m.Kv4Cache(*(torch.empty((pages, *t.shape[1:]), dtype=torch.uint8, device="cuda")
                       for t in (near.k, near.v, near.k_scale, near.v_scale)))
    for x, y in ((far.k, near.k), (far.v, near.v), (far.k_scale, near.k_scale), (far.v_scale, near.v_scale)):
        x.fill_(255)                                   # any other page: NaN blocks
        x[pages - n:] = y
    for kw in (dict(), dict(kv_split=128), dict(kv_split=64)):
        b.cache, b.d[0] = near, table
        want = [t.clone() for t in b.run(**kw)]
        b.check(*want)
        b.cache, b.d[0] = far, table + (pages - n)
        for got, x in zip(b.run(**kw), want):
            assert torch.equal(got, x), kw
