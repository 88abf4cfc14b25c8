"""lse of bf16 calls over a 4-bit cache: what the queries are held in does not
show, whatever the keys' mean, the spread of a query's dims, the context's
length, the others in the batch and the bound on their contexts."""

import numpy as np
import pytest

from tests.gpu_cases import d2sd
from tests.kv4_cases import dev, gather
from tests.test_gpu_kv4_attention import TYPES, Batch, tokens

pytestmark = pytest.mark.gpu


def check_lse(b, lse):
    """Against float64, within what follows from the arithmetic.

    Four terms of five bits hold a query element down to 2^-19 of P, the power
    of two above its block's largest magnitude: one whose last bit (of eight) is
    no less is held exactly, another is off by at most half of that. A score is a sum of
    128 products through at most 16 accumulations in fp32; its scaling and its
    difference to the reference are two roundings, the exponential one more
    unit. The weights of a row are summed in 16 at a time, 8 to a chain, then
    in chains of one per 32 keys, and the parts (at most 16 pieces of 4 waves) in
    another; the logarithm and its sum with the reference are 4 roundings."""
    q, lse = b.q.double().cpu().numpy(), lse.double().cpu().numpy()
    for r, C in enumerate(int(c) for c in b.ctx):
        k = gather(b.host, "k", b.table[r], 0, C)
        for h in range(b.hq):
            key = k[:, h // (b.hq // b.hkv)]
            s = key @ q[r, h] / np.sqrt(128.0)
            want = s.max() + np.log(np.exp(s - s.max()).sum())
            x = np.abs(q[r, h]).reshape(4, 32)
            last = np.exp2(np.frexp(x)[1] - 8.0)                   # an element's last bit
            unit = np.exp2(np.frexp(x.max(1, keepdims=True))[1] - 19.0)
            lost = np.where(last < unit, unit / 2, 0.0).reshape(128)
            cut = (np.abs(key) @ lost).max() / np.sqrt(128.0)
            size = (np.abs(key) @ np.abs(q[r, h])).max() / np.sqrt(128.0)
            sums = 8 + C / 32 + 64
            tol = cut + 2.0 ** -24 * (16 * size + 4 * np.abs(s).max() + 2 + sums + 4 * abs(want))
            assert abs(lse[r, h] - want) <= tol, (r, h, C, lse[r, h] - want, tol)


def positive_keys(b):
    """Every key's elements are made positive: their mean is far from 0."""
    b.host["k"] &= 0x77
    b.cache.k.copy_(dev(b.host["k"]))


def spread_queries(b):
    """One dim of every 32 is 32 times the others."""
    q = b.q.float()
    q[..., ::32] *= 32
    b.q.copy_(q.to(TYPES["bf16"]))


CONTEXTS = [1, 17, 300, 4000]


@pytest.mark.parametrize("spread", [False, True])
@pytest.mark.parametrize("positive", [False, True])
@pytest.mark.parametrize("kv_split", [0, 256])
def test_lse_of_a_ragged_batch(kv_split, positive, spread):
    m = d2sd()
    b = Batch(tokens(len(CONTEXTS)), CONTEXTS, 8, 2, "bf16", seed=[61, spread, positive])
    if positive:
        positive_keys(b)
    if spread:
        spread_queries(b)
    _, lse = b.run(stage=m.STAGE_PREFIX, kv_split=kv_split)
    check_lse(b, lse)


def test_lse_with_a_padded_bound():
    """The bound on the contexts does not change what a query is held in."""
    m = d2sd()
    b = Batch(tokens(3), [1, 16, 100], 8, 2, "bf16", seed=62, pad_pages=300)
    spread_queries(b)
    for bound in (100, 4800):
        _, lse = b.run(stage=m.STAGE_PREFIX, max_ctx_len=bound)
        check_lse(b, lse)
