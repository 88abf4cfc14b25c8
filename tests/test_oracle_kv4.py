"""Pins of the 4-bit cache and logit oracles: worked values and closed bounds."""

import numpy as np
import pytest

from oracle import kv4, logits


def block(*head):
    x = np.zeros(32)
    x[:len(head)] = head
    return x


def test_levels_ties_and_signs():
    # scale 2^0: the largest magnitude lies in (3.5, 7]
    x = block(6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.26, -5.01, 6.9, 7, -0.0)
    codes, scale = kv4.quantise(x)
    assert scale[0] == 127
    got = kv4.values(codes, scale)[:14]
    assert got.tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -0.5, -6, 6, 6, 0]
    assert codes[4] & 15 == 8 and codes[6] >> 4 == 8        # negative zeros keep their sign
    assert codes[0] == 7                                    # 6 in the low half, 0.25 -> 0 in the high


@pytest.mark.parametrize("top, e", [(7.0, 0), (7.0001, 1), (3.5, -1), (3.5001, 0), (1.0, -2), (0.875, -3), (0.0, -124),
                                    (2.0 ** -130, -124), (7 * 2.0 ** 125, 125), (2.0 ** 128 * (1 - 2.0 ** -24), 125)])
def test_block_exponent(top, e):
    assert kv4.block_exponent(top) == e


def test_half_a_step_is_the_most_an_element_is_off():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 128)) * 2.0 ** rng.integers(-20, 20, (200, 1))
    codes, scales = kv4.quantise(x)
    y = kv4.values(codes, scales)
    u = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=-1)
    a = np.abs(x) / u
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    assert (np.abs(x - y) <= step / 2 * u).all()
    again = kv4.quantise(y)
    assert np.array_equal(kv4.values(*again), y)            # values are their own nearest


def test_nonfinite_blocks_are_nan_and_others_are_not():
    x = np.ones((1, 128))
    x[0, 40] = np.inf
    x[0, 100] = np.nan
    codes, scales = kv4.quantise(x)
    assert scales[0].tolist() == [125, 255, 125, 255]
    y = kv4.values(codes, scales)
    assert np.isnan(y[0, 32:64]).all() and np.isnan(y[0, 96:]).all() and (y[0, :32] == 1).all() and (y[0, 64:96] == 1).all()


def test_adjusted_row_by_hand():
    x = np.array([2.0, -2.0, 1.0, 0.5, 3.0, -1.0])
    y = logits.adjust_row(x, prompt=[0, 1, 1], answered=[2, 2, 9], path=[2, 3], repetition=2.0, presence=0.25,
                          frequency=0.5, biases=[(4, 1.0), (4, 0.5), (5, -np.inf)], allowed=[1, 1, 1, 1, 1, 0])
    assert y.tolist() == [1.0, -4.0, 0.5 - 3 * 0.5 - 0.25, 0.25 - 0.5 - 0.25, 4.5, -np.inf]


def test_the_root_is_not_on_the_path():
    parent, draft = [-1, 0, 1, 0], [10, 11, 12, 13]
    assert logits.path_tokens(parent, draft, 0) == []
    assert sorted(logits.path_tokens(parent, draft, 2)) == [11, 12]
    assert logits.path_tokens(parent, draft, 3) == [13]
