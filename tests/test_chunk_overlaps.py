"""Overlaps that the rotation into the cache refuses, before any launch (no GPU needed): addresses only."""
import pytest

from tests.test_chunk_refusals import _at, _kv, _msg, _rope

OUT = _at(8)                                                   # q_out: 4 rows of 32 heads of 128 channels
SIZE = 2 * 4 * 4096
END = OUT + SIZE


# address of the first axis from q_out's, stride of the axes in entries: 4 positions an axis
@pytest.mark.parametrize("pos,stride", [(-2 * 8 * 1000, 1000), (-8, 4), (SIZE + 8 * 1000, -1000), (SIZE + 2 * 8 * 500 - 8, -500), (-8 * 3, 0),
                                        (-2 * (8 << 40), 1 << 40), (SIZE - 8 + (8 << 40), -(1 << 40))])
def test_positions_of_any_axis(pos, stride):
    assert _rope(axes=3, pos=OUT + pos, pstride=stride) == 1 and "q_out and positions" in _msg(), _msg()


def test_positions_of_the_last_of_many_axes():
    assert _rope(axes=(1 << 20) + 1, pos=OUT - (8 << 20), pstride=1) == 1 and "q_out and positions" in _msg()
    assert _rope(axes=2 ** 31 - 1, pos=OUT - 8 * (2 ** 31 - 2), pstride=1) == 1 and "q_out and positions" in _msg()


@pytest.mark.parametrize("pos,stride,axes", [(-8 * 1000, 1000, 1), (SIZE, 1000, 3), (-8 * 4, -4, 3), (-8 * 12, 4, 3), (-8 * 4, 4 + SIZE // 8, 3),
                                             (SIZE + 8 * 100, -100, 2), (SIZE + 8 * 100, -104 - SIZE // 8, 2), (-8 * 1004, 1000, 2)])
def test_positions_that_end_before_it_or_lie_around_it(pos, stride, axes):
    """Passed on to the check that comes after theirs."""
    assert _rope(axes=axes, pos=OUT + pos, pstride=stride, freq=OUT) == 1 and "q_out and inv_freq overlap" in _msg(), _msg()


def test_frequencies_and_axes():
    for at in (OUT, OUT - 4 * 63, END - 4):                    # 64 pairs
        assert _rope(freq=at) == 1 and "q_out and inv_freq overlap" in _msg(), _msg()
        assert _rope(axis=at, axes=2, pstride=1 << 20) == 1 and "q_out and axis overlap" in _msg(), _msg()


def test_keys_in_the_place_of_queries_rotated_in_place():
    """q_out may be q itself; keys or values at the same address are another input."""
    rows = dict(q=OUT, qs=(4096, 128), qo=OUT, os=(4096, 128))
    assert _rope(**rows, k=OUT, ks=(4096, 128)) == 1 and "q_out and k_new overlap" in _msg(), _msg()
    assert _rope(**rows, v=OUT, vs=(4096, 128)) == 1 and "q_out and v_new overlap" in _msg(), _msg()
    assert _rope(**rows, Hq=8, kv=_kv(), k=OUT, ks=(4096, 128)) == 1 and "q_out and k_new overlap" in _msg(), _msg()
