"""fp32 tree keys and values next to the largest finite number: they are split into
bf16 terms, of which the first must not round to infinity."""

import numpy as np
import pytest
import torch

from tests.kv4_cases import dev
from tests.test_gpu_kv4_attention import Batch, Rows, canonical, mask_of

pytestmark = pytest.mark.gpu
MOST = float(np.finfo(np.float32).max)
OVER = float(np.float32(2.0 ** 128 - 2.0 ** 119))      # the least that rounds to a bf16 infinity


@pytest.mark.parametrize("kv_split", [0, 64])
@pytest.mark.parametrize("value", [MOST, -MOST, OVER, -OVER])
def test_a_largest_value_stays_with_the_rows_that_see_it(value, kv_split):
    trees = canonical(16, [[3, 9]])
    b = Batch(trees, [100], 4, 2, "f32", seed=71)
    ref, ref_lse = (t.clone() for t in b.run(kv_split=kv_split))
    node = trees[0].N - 1
    b.vt[node, 1, 37] = value
    out, lse = b.run(kv_split=kv_split)
    assert torch.equal(lse, ref_lse)
    touched = torch.zeros_like(ref, dtype=torch.bool)
    touched[:, 2:, 37] = dev(trees[0].visible()[:, node])[:, None]
    assert touched.any() and torch.equal(out[~touched], ref[~touched])
    b.check(out, lse)


@pytest.mark.parametrize("kv_split", [0, 64])
@pytest.mark.parametrize("value", [MOST, OVER])
def test_a_largest_key_takes_all_or_nothing(value, kv_split):
    """Its score is finite and some 1e37, of either sign: the row is that node's
    value, or what it is without the node."""
    trees = canonical(16, [[3, 9]])
    b = Batch(trees, [100], 4, 2, "f32", seed=72)
    vis, node = trees[0].visible(), trees[0].N - 1
    sees = np.flatnonzero(vis[:, node])
    b.q[:, :2, 5] = 0.5
    b.q[:, 1, 5] = -0.5
    b.kt[node, 0, 5] = 0.0
    ref, ref_lse = (t.clone() for t in b.run(kv_split=kv_split))
    b.kt[node, 0, 5] = value
    out, lse = b.run(kv_split=kv_split)
    unseen = np.flatnonzero(~vis[:, node])
    assert torch.equal(out[unseen], ref[unseen]) and torch.equal(lse[unseen], ref_lse[unseen])
    assert torch.equal(out[:, 2:], ref[:, 2:])
    for r in sees:
        assert torch.equal(out[r, 0], b.vt[node, 0])    # one weight of 1 and a sum of 1
        want = 0.5 * value / np.sqrt(128.0)
        assert abs(float(lse[r, 0]) / want - 1) < 8 * 2.0 ** -24
    # without the node: its mask bit taken away
    without = vis.copy()
    without[:, node] = False
    b.mask = dev(mask_of([Rows(without)], b.W))
    ref, ref_lse = b.run(kv_split=kv_split)
    assert torch.equal(out[:, 1], ref[:, 1]) and torch.equal(lse[:, 1], ref_lse[:, 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
def test_an_infinite_key_stays_with_the_rows_that_see_it(value, dtype):
    """Rows that see it are NaN in fp32; in bf16 where its score is +inf, and without the node where it is -inf."""
    trees = canonical(16, [[3, 9]])
    b = Batch(trees, [100], 4, 2, dtype, seed=73)
    vis, node = trees[0].visible(), trees[0].N - 1
    b.q[:, 0, 5], b.q[:, 1, 5] = 0.5, -0.5
    ref, ref_lse = (t.clone() for t in b.run())
    b.kt[node, 0, 5] = value
    out, lse = b.run()
    sees, unseen = np.flatnonzero(vis[:, node]), np.flatnonzero(~vis[:, node])
    assert torch.equal(out[unseen], ref[unseen]) and torch.equal(lse[unseen], ref_lse[unseen])
    assert torch.equal(out[:, 2:], ref[:, 2:]) and torch.equal(lse[:, 2:], ref_lse[:, 2:])
    up = 0 if value > 0 else 1                          # the head whose score is +inf
    assert out[sees, up].isnan().all()
    if dtype == "f32":
        assert out[sees, 1 - up].isnan().all() and lse[sees, 1 - up].isnan().all()
        return
    without = vis.copy()
    without[:, node] = False
    b.kt[node, 0, 5] = 0.0
    b.mask = dev(mask_of([Rows(without)], b.W))
    ref, ref_lse = b.run()
    assert torch.equal(out[:, 1 - up], ref[:, 1 - up]) and torch.equal(lse[:, 1 - up], ref_lse[:, 1 - up])
