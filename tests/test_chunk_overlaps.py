"""Overlaps that the rotation into the cache refuses, before any launch (no GPU needed): addresses only."""
from tests.test_chunk_refusals import _at, _kv, _msg, _rope

OUT = _at(8)                                                   # q_out: 4 rows of 32 heads of 128 channels
END = OUT + 2 * 4 * 4096


def test_keys_in_the_place_of_queries_rotated_in_place():
    """q_out may be q itself; keys or values at the same address are another input."""
    rows = dict(q=OUT, qs=(4096, 128), qo=OUT, os=(4096, 128))
    assert _rope(**rows, k=OUT, ks=(4096, 128)) == 1 and "q_out and k_new overlap" in _msg(), _msg()
    assert _rope(**rows, v=OUT, vs=(4096, 128)) == 1 and "q_out and v_new overlap" in _msg(), _msg()
    assert _rope(**rows, Hq=8, kv=_kv(), k=OUT, ks=(4096, 128)) == 1 and "q_out and k_new overlap" in _msg(), _msg()
