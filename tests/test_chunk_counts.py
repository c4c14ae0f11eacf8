"""Counts past 31 bits in the chunk calls: refused, or taken as what they mean, never cut to their low bits (no GPU
needed: the library and the device checks are stood in for)."""
import ctypes

import pytest
import torch

from paper_2606_06453_amd import vx

BIG = (2 ** 31, 2 ** 32 + 3, 2 ** 63, -2 ** 32 + 1, -2 ** 31 - 1)


class _Calls:
    """The library's calls, which note the arguments they would have been given as C values."""

    def __init__(self, real):
        self.real, self.seen = real, []

    def __getattr__(self, name):
        types = getattr(self.real, name).argtypes

        def call(*args):
            assert len(args) == len(types)
            self.seen.append((name, [t(a).value if t in (ctypes.c_int32, ctypes.c_int64) else a for t, a in zip(types, args)]))
            return 0
        return call


@pytest.fixture
def calls(monkeypatch):
    c = _Calls(vx.lib())
    monkeypatch.setattr(vx, "lib", lambda: c)
    monkeypatch.setattr(vx, "_gpu_of", lambda t: -1)
    monkeypatch.setattr(vx, "_stream", lambda *a: None)
    return c


def _args():
    kv = vx.PagedKV(torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16))
    i = torch.zeros(2, dtype=torch.int32)
    return kv, vx.BatchSpec(i, i, i[:1].clone(), 1), torch.zeros((1, 1, 64), dtype=torch.bfloat16), i, torch.zeros(64, dtype=torch.uint8)


def test_windows(calls):
    kv, b, q, i, ws = _args()
    for window in (0, 1, 2 ** 31 - 1):
        vx.chunk_attention(q, kv, b, i, 0.1, q.clone(), ws, window=window)
        assert calls.seen[-1][1][7] == window
    for window in (2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63 - 1):          # longer than any request: all of it
        vx.chunk_attention(q, kv, b, i, 0.1, q.clone(), ws, window=window)
        assert calls.seen[-1][1][7] == 2 ** 31 - 1
    n = len(calls.seen)
    for window in (-2 ** 32, -2 ** 32 + 1, -2 ** 63):
        with pytest.raises(ValueError, match="window"):
            vx.chunk_attention(q, kv, b, i, 0.1, q.clone(), ws, window=window)
    assert len(calls.seen) == n


@pytest.mark.parametrize("name", ["kind", "n_sink", "n_local"])
@pytest.mark.parametrize("value", BIG)
def test_selection(calls, name, value):
    kv, b, q, i, ws = _args()
    rest = dict(kind=0, n_sink=0, n_local=1)
    rest[name] = value
    with pytest.raises(ValueError, match=name):
        vx.chunk_score_topk(q, kv, b, i, rest["kind"], torch.zeros((2, 1, 64)), i[:1].clone(), rest["n_sink"], rest["n_local"], 1,
                            torch.zeros((1, 1, 1), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), ws)
    assert not calls.seen


@pytest.mark.parametrize("name", ["stage", "num_rows", "num_q_heads", "max_sel"])
@pytest.mark.parametrize("value", BIG)
def test_sizes(calls, name, value):
    kv, b, _, _, _ = _args()
    rest = dict(stage=0, num_rows=1, num_q_heads=1, max_sel=1)
    rest[name] = value
    with pytest.raises(ValueError, match=name):
        vx.chunk_workspace_size(rest["stage"], kv, b, rest["num_rows"], rest["num_q_heads"], rest["max_sel"])
    assert not calls.seen


@pytest.mark.parametrize("value", BIG)
def test_pages_of_a_request(calls, value):
    kv, b, q, i, ws = _args()
    b.max_pages_per_seq = value
    with pytest.raises(ValueError, match="max_pages_per_seq"):
        vx.chunk_attention(q, kv, b, i, 0.1, q.clone(), ws)
    assert not calls.seen


@pytest.mark.parametrize("name", ["num_axes", "first"])
@pytest.mark.parametrize("value", BIG)
def test_rotations(name, value):
    rope = vx.Rope(torch.rand(32))
    setattr(rope, name, value)
    with pytest.raises(ValueError, match=name):
        rope.current(-1)
