"""Pins of the words oracle (8-bit rows, rules, best words, draws): closed forms and
identities, and torch's own 8-bit type."""
import math

import numpy as np
import pytest
import torch

from oracle import words as ow


def test_values_are_the_8_bit_types():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).to(torch.float64).numpy()
    np.testing.assert_array_equal(ow.value8(codes.numpy()), want)


@pytest.mark.parametrize("amax,e", [(0.0, -127), (448.0, 0), (449.0, 1), (448.0000001, 1), (1.0, -8),
                                    (0.875, -9), (0.8750001, -8), (1e300, 127), (1e-300, -127),
                                    (448 * 2.0 ** -127, -127), (449 * 2.0 ** -127, -126)])
def test_scale_exponent(amax, e):
    assert ow.scale_exponent(amax) == e


def test_pack_is_nearest_even():
    # halves between neighbouring codes at scale 1 (448 fixes it) go to the even code
    mid = (ow.VALUES8[:-1] + ow.VALUES8[1:]) / 2
    x = np.concatenate([[448.0], mid[:126]])
    q, e = ow.pack8(x[None])
    assert e[0, 0] == 127 and q[0, 0] == 126
    assert all(q[0, 1 + i] == (i if i % 2 == 0 else i + 1) for i in range(126))
    back = ow.unpack8(q, e)[0, :127]
    # half a step of 3 fraction bits at most
    assert np.all(np.abs(back - x) <= np.maximum(x * 2.0 ** -4, 2.0 ** -10))


def test_pack_of_values_without_a_number():
    q, e = ow.pack8(np.array([[np.nan, np.inf, -np.inf, 2.0, -1.0]]))
    assert list(q[0, :3] & 127) == [127] * 3 and e[0, 0] == ow.scale_exponent(2.0) + 127
    assert list(ow.unpack8(q, e)[0, 3:5]) == [2.0, -1.0] and not q[0, 5:].any()


def test_rules_by_hand():
    x = np.array([[1.0, -2.0, 0.5, 3.0, np.nan]])
    y = ow.adjusted(x, listed=[[0, 1, 1, 9, -1]], penalties=np.array([[2.0, 0.25, 0.5]]),
                    bias=np.array([[0, 0, 1.0, 0, 0]]),
                    allowed=np.array([[True, True, True, False, False]]))
    # 1 / 2 - (0.25 + 0.5), -2 * 2 - (0.25 + 2 * 0.5), 0.5 + 1, masked, masked NaN
    assert list(y[0]) == [-0.25, -5.25, 1.5, -np.inf, -np.inf]


def test_top_ties_and_missing():
    x = np.array([[1.0, 2.0, 2.0, -np.inf, np.nan], [-np.inf] * 5], np.float32)
    word, value = ow.top(x, 4)
    assert word.tolist() == [[1, 2, 0, -1], [-1] * 4]
    assert value[0].tolist() == [2.0, 2.0, 1.0, -np.inf]


def test_draw_frequencies_and_borders():
    x = np.log(np.array([[0.5, 0.0 + 1e-300, 0.25, 0.25]]))
    u = np.array([[0.0, 0.49, 0.51, 0.74, 0.76, 0.999, 1.0, -1.0, np.nan]])
    word, logp, _ = ow.drawn(x, u)
    assert word.tolist() == [[0, 0, 2, 2, 3, 3, 3, 0, 3]]
    np.testing.assert_allclose(logp[0, :3], [math.log(.5), math.log(.5), math.log(.25)], rtol=1e-12)
    # at half the temperature weights are squared
    u = (np.arange(1000)[None] + 0.5) / 1000
    word, _, _ = ow.drawn(x, u, 0.5)
    got = np.bincount(word[0], minlength=4) / 1000
    np.testing.assert_allclose(got, np.array([4, 0, 1, 1]) / 6, atol=1e-3)
    for row in ([-np.inf, -np.inf], [0.0, np.nan], [0.0, np.inf]):
        word, logp, _ = ow.drawn(np.array([row]), np.array([[0.3]]))
        assert word[0, 0] == -1 and np.isnan(logp[0, 0])
