"""Logit adjustment with lists longer than a workgroup, and many nodes per
workgroup, against the float64 oracle (bounds in tests/test_gpu_logits.py)."""

import numpy as np
import pytest
import torch

from oracle.tree import build_tree
from tests.test_gpu_logits import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [37, 2048, 2049])
def test_long_histories_and_bias_lists(V, dtype):
    """9000 tokens of history, 700 biases, most of them for the same few tokens: summed in list order."""
    b = Batch([build_tree(8, p) for p in ([3, 7], [])], V, dtype, seed=[50, V], hist=9000, bias=700, few=9)
    b.kw["history_len"][:] = [9000, 4097]
    b.kw["prompt_len"][:] = [4500, 4096]
    b.kw["bias_len"][:] = [700, 257]
    b.check(b.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_requests_are_what_each_is_alone(dtype):
    """A batch large enough for eight nodes per workgroup, bit for bit what its requests give by themselves."""
    tree = build_tree(16, [3, 7, 12])
    n, V = 64, 16001
    b = Batch([tree] * n, V, dtype, seed=51, hist=300, bias=20, masks=4, few=60)
    got = b.run()
    for i in (0, 31, n - 1):
        s, e = int(b.ip[i]), int(b.ip[i + 1])
        one = Batch([tree], V, dtype, seed=52)
        one.draft, one.x = b.draft[s:e], b.x[s:e].clone()          # rows of an odd vocabulary start unaligned
        one.kw = {k: v[s:e] if k == "mask_row" else v if k == "token_mask" else v[i:i + 1] for k, v in b.kw.items()}
        alone = one.run()
        assert torch.equal(got[s:e], alone)
        one.check(alone)


@pytest.mark.parametrize("most", [1, 2, 3, 5, 64, 600])
def test_bias_lists_that_repeat(most):
    """Up to `most` entries of a token in a row and far apart, among single ones; a list padded with one id."""
    b = Batch([build_tree(8, p) for p in ([3, 7], [])], 2500, "f32", seed=[55, most], bias=600, masks=0)
    rng = np.random.default_rng([56, most])
    tokens = np.repeat(rng.permutation(2500)[:600], most)[:600]
    b.kw["bias_token"][0] = tokens
    b.kw["bias_token"][1] = rng.permutation(tokens)
    b.kw["bias_token"][1, 200:450] = 7
    b.kw["bias_value"][1, 300:450] = 0.0
    b.kw["bias_len"][:] = 600
    b.check(b.run())
