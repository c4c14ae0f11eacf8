"""The tests' own mxfp4 definitions, pinned: rounding of hand values, the place of every nibble, and the
round trip of a packed cache."""
import numpy as np
import pytest

from tests import _mx


def test_rounding_of_hand_values():
    x = np.zeros((1, 32))
    x[0, :12] = [6.9, -0.25, 0.75, 0.76, -1.25, 1.75, 2.5, 3.5, 5.0, -5.1, 0.24, -0.0]
    codes, scales = _mx.quantize(x)
    assert scales.tolist() == [[127]]                              # 6.9 rounds to 6, not to 8
    got = _mx.values(codes, scales)[0, :12]
    assert got.tolist() == [6.0, 0.0, 1.0, 1.0, -1.0, 2.0, 2.0, 4.0, 4.0, -6.0, 0.0, 0.0]
    x[0, 0] = 7.0                                                  # rounds to 8: the next scale
    codes, scales = _mx.quantize(x)
    assert scales.tolist() == [[128]] and _mx.values(codes, scales)[0, 0] == 8.0


@pytest.mark.parametrize("top,byte", [(0.0, 8), (1e-38, 8), (2.0 ** -119, 8), (2.0 ** -117, 8), (2.0 ** -116, 9),
                                      (3.3e38, 252), (np.inf, 255), (np.nan, 255)])
def test_scales_at_the_ends(top, byte):
    x = np.zeros((2, 32))
    x[1, 5] = top
    codes, scales = _mx.quantize(x)
    assert scales.tolist() == [[8], [byte]] and (byte != 255 or not codes.any())


@pytest.mark.parametrize("ps,D", [(16, 64), (64, 64), (16, 128), (32, 128)])
@pytest.mark.parametrize("which", ["k", "v"])
def test_every_nibble_has_one_place(ps, D, which):
    at, high, sc = _mx.places(ps, D, which)
    nib = at * 2 + high
    assert np.array_equal(np.sort(nib.ravel()), np.arange(ps * D))
    groups = sc[:, ::32]
    assert np.array_equal(np.sort(groups.ravel()), ps * D // 2 + np.arange(ps * D // 32))
    assert (sc == np.repeat(groups, 32, axis=1)).all()
    x = np.random.default_rng(D + ps).normal(size=(2, 3, ps, D))
    codes, scales = _mx.quantize(x)
    assert np.array_equal(_mx.unpack(_mx.pack(x, which), which), _mx.values(codes, scales))
