"""Refusals of the cache's own operators and of mxfp4 caches, before any launch (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2606_06453_amd import vx

BUF = torch.zeros(1 << 16, dtype=torch.uint8)
P = BUF.data_ptr() + (-BUF.data_ptr()) % 64


def _kv(dtype=vx.KV_MXFP4, D=128, H=8, ps=16, k=P, v=P, Dv=None, block=0):
    return vx._Cache(k, v, 4, H, ps, D, D if Dv is None else Dv, dtype, 1.0, 1.0, block)


def _msg():
    return vx.lib().vx_last_error().decode()


def _rows(kv, k=P, ks=(1024, 128), v=P, vs=(1024, 128), slots=P, n=4, fn="vx_kv_write"):
    return getattr(vx.lib(), fn)(ctypes.byref(kv) if kv else None, k, *ks, v, *vs, slots, n, None)


@pytest.mark.parametrize("fn", ["vx_kv_write", "vx_kv_read"])
def test_rows(fn):
    assert _rows(None, fn=fn) == 1
    assert _rows(_kv(), n=0, slots=None, k=None, v=None, fn=fn) == 0          # nothing to do
    for kw, word in ((dict(n=-1), "num_rows"), (dict(k=None), "k_"), (dict(v=None), "v_"), (dict(slots=None), "slots"),
                     (dict(k=P + 2), "aligned"), (dict(ks=(1020, 128)), "strides"), (dict(vs=(1024, 12)), "strides")):
        assert _rows(_kv(), fn=fn, **kw) == 1 and word in _msg(), (kw, _msg())
    assert _rows(_kv(v=None), fn=fn) == 2                                     # GQA needs a separate V
    assert _rows(_kv(k=P + 8), fn=fn) == 1 and "aligned" in _msg()
    assert _rows(_kv(dtype=vx.KV_BF16, k=P + 8), fn=fn) == 1 and "aligned" in _msg()
    assert _rows(_kv(dtype=vx.KV_BF16, D=576, Dv=512, H=1, v=None), fn=fn) == 1 and "aliased" in _msg()
    assert _rows(_kv(dtype=4), fn=fn) == 1
    assert _rows(_kv(D=96), fn=fn) == 2


def test_mxfp4_caches():
    size = ctypes.c_size_t()
    b = vx._Batch(2, 5, P, P, P)
    ask = lambda kv: vx.lib().vx_workspace_size(vx.STAGE_DECODE, ctypes.byref(kv), ctypes.byref(b), 16, 8, ctypes.byref(size))  # noqa: E731
    assert ask(_kv()) == 0 and ask(_kv(D=64)) == 0
    assert ask(_kv(D=576, Dv=512, H=1, v=None)) == 2 and "GQA" in _msg()
    assert ask(_kv(v=P + 4)) == 1 and "aligned" in _msg()
    assert ask(_kv(block=8)) == 2
    kv = vx.PagedKV(vx.mxfp4_cache(3, 8, 16, 128, "cpu"), vx.mxfp4_cache(3, 8, 16, 128, "cpu"))
    st = kv.struct()
    assert (st.head_dim_qk, st.head_dim_v, st.kv_dtype, kv.head_dim_qk) == (128, 128, vx.KV_MXFP4, 128)
    assert kv.row_dtype == torch.bfloat16
    with pytest.raises(ValueError):
        vx.PagedKV(torch.zeros((2, 1, 16, 64), dtype=torch.uint8), None).struct()
    with pytest.raises(TypeError):
        vx.PagedKV(vx.mxfp4_cache(3, 8, 16, 128, "cpu"), torch.zeros((3, 8, 16, 128), dtype=torch.bfloat16)).struct()
    with pytest.raises(TypeError):                                            # codes are not rows
        vx.kv_append_summarize(kv, vx.BatchSpec(*[torch.zeros(3, dtype=torch.int32)] * 3, 1),
                               torch.zeros((2, 8, 128), dtype=torch.uint8), None)


def _pool(**kw):
    f = dict(free_pages=P, free_count=P, table=P, lens=P, num_phys_pages=10, table_rows=4, table_stride=8, page_size=16,
             block_size=0)
    f.update(kw)
    return vx._Pool(**f)


def test_page_plans():
    need = vx.page_workspace_size(4)
    with pytest.raises(vx.VxError):
        vx.page_workspace_size(-1)
    with pytest.raises(vx.VxError):
        vx.page_workspace_size(65536)
    L = vx.lib()

    def extend(pool=None, batch=4, rows=P, new=P, seq=P, indptr=P, idx=P, cap=9, tok=P, slots=P, scap=9, granted=P, ws=P,
               ws_bytes=need):
        p = pool or _pool()
        return L.vx_page_extend(ctypes.byref(p), batch, rows, new, seq, indptr, idx, cap, tok, slots, scap, granted, None,
                                ws, ws_bytes, None)

    def release(pool=None, batch=4, rows=P, keep=P, ws=P, ws_bytes=need):
        p = pool or _pool()
        return L.vx_page_release(ctypes.byref(p), batch, rows, keep, ws, ws_bytes, None)

    for call in (extend, release):
        for kw in (dict(free_pages=None), dict(free_count=None), dict(table=None), dict(lens=None), dict(num_phys_pages=0),
                   dict(table_rows=0), dict(table_stride=0)):
            assert call(pool=_pool(**kw)) == 1, kw
        for kw in (dict(page_size=8), dict(block_size=8), dict(page_size=32, block_size=64), dict(table_stride=1 << 27)):
            assert call(pool=_pool(**kw)) == 2, kw
        assert call(batch=-1) == 1 and call(batch=65536) == 1 and call(rows=None) == 1
        assert call(ws=None) == 3 and call(ws_bytes=need - 1) == 3 and "workspace" in _msg()
        assert call(batch=0) == 0                                             # nothing to do
    for kw in (dict(new=None), dict(seq=None), dict(indptr=None), dict(idx=None), dict(tok=None), dict(slots=None),
               dict(granted=None), dict(cap=-1), dict(scap=-1)):
        assert extend(**kw) == 1, kw
    assert L.vx_page_extend(None, 4, P, P, P, P, P, 9, P, P, 9, P, None, P, need, None) == 1
    assert L.vx_page_release(None, 4, P, P, P, need, None) == 1


def test_the_binding_checks_types_and_places():
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    pool = vx.PagePool.empty(6, 3, 4, 16, device="cpu")
    assert pool.free_pages.tolist() == [5, 4, 3, 2, 1, 0] and pool.free_count.item() == 6
    batch, ws = vx.BatchSpec(i32(4), i32(6), i32(3), 4), i32(64)
    ok = [i32(3), i32(3), batch, i32(4), torch.zeros(9, dtype=torch.int64), i32(3), ws]
    for at, bad in ((0, torch.zeros(3)), (1, i32(2)), (3, i32(3)), (4, i32(9)), (5, i32(4))):
        args = list(ok)
        args[at] = bad
        with pytest.raises((TypeError, ValueError)):
            vx.page_extend(pool, *args)
    with pytest.raises(ValueError, match="GPU"):                              # host tensors would fault the GPU
        vx.page_extend(pool, *ok)
    with pytest.raises(ValueError, match="GPU"):
        vx.page_release(pool, i32(3), None, ws)
    with pytest.raises(ValueError):
        vx.page_release(pool, i32(3), i32(2), ws)
    with pytest.raises(ValueError):
        vx.PagePool(i32(4), i32(1), i32((3, 4)), i32(2), 16).struct()
    kv = vx.PagedKV(vx.mxfp4_cache(3, 2, 16, 64, "cpu"), vx.mxfp4_cache(3, 2, 16, 64, "cpu"))
    rows, slots = torch.zeros((5, 2, 64), dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        vx.kv_write(kv, rows, rows, slots)
    for k, s in ((rows.float(), slots), (rows[:4], slots), (rows[..., :32], slots), (rows, slots.int()),
                 (rows.transpose(1, 2).contiguous().transpose(1, 2), slots)):
        with pytest.raises((TypeError, ValueError)):
            vx.kv_write(kv, k, rows, s)
        with pytest.raises((TypeError, ValueError)):
            vx.kv_read(kv, s, k, rows)


def test_keys_alone():
    kv = vx.PagedKV(vx.mxfp4_cache(3, 2, 16, 64, "cpu"), None)
    assert (kv.struct().head_dim_qk, kv.struct().head_dim_v) == (64, 64)


def test_a_replaced_cache_is_described_anew():
    new = lambda P: torch.zeros((P, 2, 16, 64), dtype=torch.float8_e4m3fn)  # noqa: E731
    kv = vx.PagedKV(new(3), new(3), k_scale=0.5)
    kv.current()
    assert (kv._st.num_phys_pages, kv._st.k_scale, kv._st.k) == (3, 0.5, kv.k.data_ptr())
    kept = kv.current()
    assert kv.current() is kept
    kv.k, kv.v, kv.k_scale = new(4), new(4), 0.25
    kv.current()
    assert (kv._st.num_phys_pages, kv._st.k_scale, kv._st.k, kv._st.v) == (4, 0.25, kv.k.data_ptr(), kv.v.data_ptr())
