"""The descriptions of rotations that the binding hands to the library follow the tensors they describe (no GPU
needed: the tensors are the host's, as GPU -1)."""
import pytest
import torch

from paper_2606_06453_amd import vx

HOST = -1


def _told(rope):
    st = rope.current(HOST)._obj
    return {n: getattr(st, n) for n, _ in vx._Rope._fields_}


def test_frequencies_that_turn_into_a_view_are_refused():
    base = torch.rand(64)
    rope = vx.Rope(base[:32])
    assert _told(rope)["dim"] == 64
    rope.inv_freq = base[::2]                                          # the same address, length and type
    with pytest.raises(ValueError, match="inv_freq must be contiguous"):
        rope.current(HOST)
    rope.inv_freq = base[:32]
    assert _told(rope)["inv_freq"] == base.data_ptr()


def test_axes_that_turn_into_a_view_are_refused():
    base = torch.zeros(64, dtype=torch.int32)
    rope = vx.Rope(torch.rand(32), axis=base[:32], num_axes=3)
    assert _told(rope)["axis"] == base.data_ptr()
    rope.axis = base[::2]
    with pytest.raises(ValueError, match="axis must be contiguous"):
        rope.current(HOST)


def test_frequencies_strided_in_place_are_refused():
    f = torch.rand(64)
    rope = vx.Rope(f)
    f.resize_(32)
    assert _told(rope)["dim"] == 64
    f.set_(f.untyped_storage(), 0, (32,), (2,))
    with pytest.raises(ValueError, match="inv_freq must be contiguous"):
        rope.current(HOST)


def test_each_field_that_a_rotation_holds():
    rope = vx.Rope(torch.rand(32))
    for name, value in (("num_axes", 3), ("first", 64), ("interleaved", True), ("scale", 0.5)):
        _told(rope)
        setattr(rope, name, value)
        assert _told(rope)[name] == value
    other = torch.rand(16)
    rope.inv_freq = other
    assert _told(rope)["inv_freq"] == other.data_ptr() and _told(rope)["dim"] == 32
    rope.axis = torch.zeros(16, dtype=torch.int32)
    assert _told(rope)["axis"] == rope.axis.data_ptr()
    rope.axis = torch.zeros(32, dtype=torch.int32)
    with pytest.raises(ValueError, match="axis has 32 entries, 16 are needed"):
        rope.current(HOST)
