"""The 64-bit reference of the 4-bit cache against the format's definition, values written out by hand."""
import numpy as np
import pytest

import paged_reference as R


def block(*first):
    x = np.zeros(64, np.float32)
    x[:len(first)] = first
    return x


def test_every_code_stands_for_its_value_and_back():
    values = [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]
    c, s = R.encode(block(*values))
    assert list(s) == [127, 27]
    assert [(c[i // 2] >> (4 * (i % 2))) & 15 for i in range(16)] == list(range(16))
    assert (R.decode(c, s)[:16] == values).all()


@pytest.mark.parametrize("x,code", [(0.25, 0), (0.2500001, 1), (0.75, 2), (0.7499999, 1), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (5.0000005, 7)])
def test_ties_go_to_the_even_code(x, code):
    c, _ = R.encode(block(6.0, x))
    assert c[0] >> 4 == code


@pytest.mark.parametrize("top,e,code", [(4.0, 127, 6), (6.0, 127, 7), (7.0, 127, 7), (7.0000005, 128, 6), (7.9, 128, 6), (8.0, 128, 6), (0.0, 27, 0),
                                        (2.0 ** -126, 27, 0), (2.0 ** -98, 27, 6)])
def test_the_exponent_goes_by_the_largest_value(top, e, code):
    c, s = R.encode(block(top))
    assert s[0] == e and c[0] & 15 == code


def test_a_block_with_a_value_that_is_not_finite_is_not_a_number():
    for bad in (np.nan, np.inf, -np.inf):
        c, s = R.encode(block(1.0, bad))
        assert list(s) == [255, 27] and not c.any()
        d = R.decode(c, s)
        assert np.isnan(d[:32]).all() and not d[32:].any()


def test_attention_of_one_visible_slot_is_its_value():
    rng = np.random.default_rng(0)
    c = R.Cache(rng, 1, 1, 2, 16, 64, [0], 3)
    q = rng.standard_normal((1, 3, 4, 64))
    out = c.attend(0, q, [[[1, 0, 0], [0, 0, 0], [0, 0, 1]]], 0.125)
    v = c.values("v", 0, 0, 0, 3)
    assert np.allclose(out[0, 0], v[0, [0, 0, 1, 1]]) and not out[0, 1].any() and np.allclose(out[0, 2], v[2, [0, 0, 1, 1]])
