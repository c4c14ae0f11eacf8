"""Refusals of the chunk calls, before any launch (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2606_06453_amd import vx

BUF = torch.zeros(1 << 16, dtype=torch.uint8)
P = BUF.data_ptr() + (-BUF.data_ptr()) % 64
FAR = 1 << 40                                                  # arrays that do not meet: addresses only


def _at(n):
    return P + n * FAR


def _kv(dtype=vx.KV_BF16, D=128, H=8, ps=16, k=_at(1), v=_at(2), Dv=None, block=0):
    return vx._Cache(k, v, 4, H, ps, D, D if Dv is None else Dv, dtype, 1.0, 1.0, block)


def _batch(batch=2, pages=5, indptr=_at(3), idx=_at(4), lens=_at(5)):
    return vx._Batch(batch, pages, indptr, idx, lens)


def _msg():
    return vx.lib().vx_last_error().decode()


def _rope(kv=None, freq=_at(6), axis=None, axes=1, first=0, dim=128, inter=0, scale=1.0, q=_at(7), qs=(4096, 128), Hq=32, qo=_at(8), os=(4096, 128),
          k=_at(9), ks=(1024, 128), v=_at(10), vs=(1024, 128), pos=_at(11), pstride=0, slots=_at(12), n=4, rope=True):
    kv = kv or _kv()
    r = vx._Rope(freq, axis, axes, first, dim, inter, scale)
    return vx.lib().vx_rope_kv_write(ctypes.byref(kv), ctypes.byref(r) if rope else None, q, *qs, Hq, qo, *os, k, *ks, v, *vs, pos, pstride, slots, n,
                                     None)


def test_rope():
    assert _rope(n=0) == 0
    for kw, word in ((dict(rope=False), "rope"), (dict(freq=None), "inv_freq"), (dict(freq=_at(6) + 2), "aligned"), (dict(axes=0), "num_axes"),
                     (dict(inter=2), "interleaved"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
                     (dict(n=-1), "num_rows"), (dict(qo=None), "together"), (dict(q=None), "together"), (dict(Hq=30), "num_q_heads"),
                     (dict(k=None), "k_new"), (dict(v=None), "v_new"), (dict(pos=None), "positions"), (dict(slots=None), "slots"),
                     (dict(pos=_at(11) + 4), "aligned"), (dict(slots=_at(12) + 4), "aligned"), (dict(q=_at(7) + 2), "aligned"),
                     (dict(ks=(1020, 128)), "strides"), (dict(os=(4096, 100)), "strides"), (dict(qs=(1 << 44, 128)), "2^40"),
                     (dict(os=(0, 128)), "overlap"), (dict(os=(4096, 64)), "overlap"), (dict(qo=_at(7) + 64), "overlap"),
                     (dict(qo=_at(7), os=(4096 + 8, 128)), "overlap"), (dict(qo=_at(9)), "overlap"), (dict(qo=_at(1)), "overlap"),
                     (dict(qo=_at(2)), "overlap"), (dict(qo=_at(12)), "overlap"), (dict(qo=_at(11) - 256), "overlap"),
                     (dict(kv=_kv(k=_at(1) + 8)), "aligned")):
        assert _rope(**kw) == 1 and word in _msg(), (kw, _msg())
    for kw in (dict(first=4), dict(dim=8), dict(dim=24), dict(dim=144), dict(first=8), dict(first=-8), dict(Hq=256), dict(kv=_kv(D=96))):
        assert _rope(**kw) == 2, (kw, _msg())
    mla = _kv(D=576, Dv=512, H=1, v=None)
    assert _rope(kv=mla, Hq=16, dim=64, first=512) == 1 and "aliased" in _msg()
    # slices of one projection lie between each other: told apart by their columns
    fused = _at(13)
    apart = dict(q=fused, qs=(48 * 128, 128), k=fused + 2 * 32 * 128, ks=(48 * 128, 128), v=fused + 2 * 40 * 128, vs=(48 * 128, 128))
    assert _rope(**apart, qo=fused + 2 * 128, os=(48 * 128, 128)) == 1 and "q_out and q overlap" in _msg()
    assert _rope(**apart, qo=fused + 2 * 8 * 128, Hq=8, os=(48 * 128, 128), slots=None) == 1 and "slots" in _msg()
    assert _rope(**apart, qo=fused + 2 * 28 * 128, Hq=8, os=(48 * 128, 128)) == 1 and "q_out and k_new overlap" in _msg()


def _chunk(c=True, indptr=_at(6), lens=None, n=8):
    return ctypes.byref(vx._Chunk(indptr, lens, n)) if c else None


def _size(stage, kv=None, b=None, n=8, Hq=32, M=4):
    out = ctypes.c_size_t()
    kv, b = kv or _kv(), b or _batch()
    st = vx.lib().vx_chunk_workspace_size(stage, ctypes.byref(kv), ctypes.byref(b), n, Hq, M, ctypes.byref(out))
    return st, out.value


def test_workspace_size():
    for stage in (0, 1, 2):
        st, n = _size(stage)
        assert st == 0 and n > 0
        assert _size(stage, n=0)[0] == 0
        assert _size(stage, n=-1)[0] == 1 and _size(stage, n=1 << 30)[0] == 2 and _size(stage, Hq=30)[0] == 1
        assert _size(stage, kv=_kv(D=96))[0] == 2 and _size(stage, b=_batch(pages=0))[0] == 1
    assert _size(3)[0] == 1
    assert _size(1, M=0)[0] == 1 and _size(0, M=0)[0] == 0
    mla = _kv(D=576, Dv=512, H=1, v=None)
    assert _size(0, kv=mla, Hq=16)[0] == 0 and _size(1, kv=mla, Hq=16)[0] == 2 and _size(2, kv=mla, Hq=16)[0] == 2
    assert _size(2, b=_batch(pages=16385))[0] == 2 and _size(2, b=_batch(pages=16384))[0] == 0
    assert _size(2, kv=_kv(ps=64, block=16), b=_batch(pages=4097))[0] == 2


COMMON = (((dict(c=False)), 1, "chunk"), (dict(indptr=None), 1, "q_indptr"), (dict(n=-1), 1, "num_rows"), (dict(n=(1 << 19) + 1), 2, "num_rows"),
          (dict(indptr=_at(6) + 2), 1, "aligned"), (dict(lens=_at(6) + 1), 1, "aligned"))


def _shared(call):
    """What every chunk call refuses."""
    for kw, st, word in COMMON:
        assert call(chunk=_chunk(**kw)) == st and word in _msg(), (kw, _msg())
    for kw, st, word in ((dict(q=None), 1, "q "), (dict(q=_at(7) + 2), 1, "aligned"), (dict(qs=(4095, 128)), 1, "strides"), (dict(qs=(4096, 1 << 44)), 1, "2^40"),
                         (dict(Hq=30), 1, "num_q_heads"), (dict(Hq=256), 2, "group"), (dict(kv=_kv(D=96)), 2, "head_dim"), (dict(kv=_kv(k=_at(1) + 8)), 1, "aligned"),
                         (dict(b=_batch(batch=-1)), 1, "batch"), (dict(b=_batch(lens=None)), 1, "seq_lens"), (dict(b=_batch(indptr=_at(3) + 2)), 1, "aligned"),
                         (dict(ws=None), 3, "workspace"), (dict(ws_bytes=0), 3, "workspace"), (dict(ws=_at(20) + 8), 1, "aligned"),
                         (dict(ws=_at(7)), 1, "overlap"), (dict(ws=_at(6)), 1, "overlap"), (dict(ws=_at(3)), 1, "overlap"), (dict(ws=_at(5)), 1, "overlap")):
        assert call(**kw) == st and word in _msg(), (kw, _msg())
    assert call(chunk=_chunk(n=0), q=None, ws=None) == 0 and call(b=_batch(batch=0), ws=None) == 0


def test_chunk_attention():
    def call(q=_at(7), qs=(4096, 128), Hq=32, kv=None, b=None, chunk=None, window=0, causal=1, scale=0.1, out=_at(8), lse=_at(9), ws=_at(20),
             ws_bytes=1 << 30):
        kv, b = kv or _kv(), b or _batch()
        return vx.lib().vx_chunk_attention(q, *qs, Hq, ctypes.byref(kv), ctypes.byref(b), _chunk() if chunk is None else chunk, window, causal, scale,
                                           out, lse, ws, ws_bytes, None)

    def with_chunk(**kw):
        if "chunk" in kw and kw["chunk"] is None:
            kv, b = _kv(), _batch()
            return vx.lib().vx_chunk_attention(_at(7), 4096, 128, 32, ctypes.byref(kv), ctypes.byref(b), None, 0, 1, 0.1, _at(8), None, _at(20), 1 << 30, None)
        return call(**kw)

    _shared(with_chunk)
    for kw, st, word in ((dict(window=-1), 1, "window"), (dict(causal=2), 1, "causal"), (dict(scale=0.0), 1, "sm_scale"), (dict(scale=-1.0), 1, "sm_scale"),
                         (dict(scale=float("nan")), 1, "sm_scale"), (dict(scale=float("inf")), 1, "sm_scale"), (dict(out=None), 1, "out"),
                         (dict(out=_at(8) + 8), 1, "aligned"), (dict(lse=_at(9) + 2), 1, "aligned"), (dict(lse=_at(8)), 1, "overlap"),
                         (dict(out=_at(7)), 1, "overlap"), (dict(out=_at(1)), 1, "overlap"), (dict(out=_at(2)), 1, "overlap"), (dict(lse=_at(5)), 1, "overlap"),
                         (dict(ws=_at(8)), 1, "overlap"), (dict(kv=_kv(v=None)), 2, "V"), (dict(kv=_kv(D=576, Dv=512, H=1, v=None)), 2, "group")):
        assert call(**kw) == st and word in _msg(), (kw, _msg())
    # queries of a strided projection reach past their own rows: results behind them are apart
    assert call(out=_at(7) + 2 * 4096 * 7 + 2 * 31 * 128, Hq=32) == 1 and "overlap" in _msg()


def test_sparse_chunk_attention():
    def call(q=_at(7), qs=(4096, 128), Hq=32, kv=None, b=None, chunk=None, sel=_at(10), count=_at(11), M=4, scale=0.1, out=_at(8), lse=_at(9), ws=_at(20),
             ws_bytes=1 << 30, null=False):
        kv, b = kv or _kv(), b or _batch()
        return vx.lib().vx_sparse_chunk_attention(q, *qs, Hq, ctypes.byref(kv), ctypes.byref(b), None if null else chunk or _chunk(), sel, count, M, scale,
                                                  out, lse, ws, ws_bytes, None)

    _shared(lambda **kw: call(null="chunk" in kw and kw["chunk"] is None, **kw))
    for kw, st, word in ((dict(sel=None), 1, "sel_pages"), (dict(count=None), 1, "sel_count"), (dict(M=0), 1, "max_sel"), (dict(sel=_at(10) + 2), 1, "aligned"),
                         (dict(scale=0.0), 1, "sm_scale"), (dict(out=_at(10)), 1, "overlap"), (dict(lse=_at(11)), 1, "overlap"),
                         (dict(kv=_kv(D=576, Dv=512, H=1, v=None), Hq=16), 2, "GQA"), (dict(b=_batch(pages=20000)), 2, "blocks")):
        assert call(**kw) == st and word in _msg(), (kw, _msg())


def test_chunk_score_topk():
    def call(q=_at(7), qs=(4096, 128), Hq=32, kv=None, b=None, chunk=None, kind=0, mean=_at(10), budget=_at(12), sink=1, local=1, M=4, sel=_at(13),
             count=_at(14), ws=_at(20), ws_bytes=1 << 30, null=False):
        kv, b = kv or _kv(), b or _batch()
        return vx.lib().vx_chunk_score_topk(q, *qs, Hq, ctypes.byref(kv), ctypes.byref(b), None if null else chunk or _chunk(), kind, mean, budget, sink,
                                            local, M, sel, count, ws, ws_bytes, None)

    _shared(lambda **kw: call(null="chunk" in kw and kw["chunk"] is None, **kw))
    for kw, st, word in ((dict(kind=1), 2, "kind"), (dict(kind=7), 2, "kind"), (dict(kind=-1), 1, "kind"), (dict(kind=9), 1, "kind"), (dict(mean=None), 1, "mean"),
                         (dict(budget=None), 1, "budget"), (dict(sel=None), 1, "sel_pages"), (dict(count=None), 1, "sel_count"), (dict(local=0), 1, "n_local"),
                         (dict(sink=-1), 1, "n_sink"), (dict(sink=4), 1, "max_sel"), (dict(M=0), 1, "max_sel"), (dict(mean=_at(10) + 4), 1, "aligned"),
                         (dict(sel=_at(10)), 1, "overlap"), (dict(count=_at(12)), 1, "overlap"), (dict(sel=_at(14)), 1, "overlap"),
                         (dict(kv=_kv(D=576, Dv=512, H=1, v=None), Hq=16), 2, "GQA"), (dict(b=_batch(pages=20000)), 2, "blocks")):
        assert call(**kw) == st and word in _msg(), (kw, _msg())


def test_the_binding_asks_for_the_gpu():
    """Host tensors are refused by the binding, whatever their shapes."""
    kv = vx.PagedKV(torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16))
    i = torch.zeros(2, dtype=torch.int32)
    b = vx.BatchSpec(i, i, i[:1], 1)
    q = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    with pytest.raises((ValueError, AssertionError, RuntimeError)):
        vx.chunk_attention(q, kv, b, i, 0.1, q, BUF)
    with pytest.raises((ValueError, AssertionError, RuntimeError)):
        vx.rope_kv_write(kv, vx.Rope(torch.zeros(32)), q, q, q, torch.zeros(1, dtype=torch.int64), torch.zeros(1, dtype=torch.int64), q)
