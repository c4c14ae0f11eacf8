"""The descriptions of caches and pools that the binding hands to the library follow the tensors they
describe (no GPU needed)."""
import pytest
import torch

from paper_2606_06453_amd import vx
from paper_2606_06453_amd.decoder import SparseDecoder

BF16, E4M3, E5M2 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e5m2


def _kv(P=3, H=2, ps=16, D=64, dtype=BF16, room=1 << 18):
    """K and V at the starts of two buffers that other caches can take over."""
    bufs = [torch.zeros(room, dtype=torch.uint8) for _ in range(2)]
    kv = vx.PagedKV(*(_on(b, P, H, ps, D, dtype) for b in bufs), k_scale=0.5, v_scale=0.5)
    return kv, bufs


def _on(buf, P, H, ps, D, dtype):
    n = P * H * ps * D * torch.empty(0, dtype=dtype).element_size()
    return buf[:n].view(dtype).view(P, H, ps, D)


def _told(kv):
    kv.current()
    return {n: getattr(kv._st, n) for n, _ in vx._Cache._fields_}


def _fresh(kv):
    st = kv.struct()
    return {n: getattr(st, n) for n, _ in vx._Cache._fields_}


@pytest.mark.parametrize("first,second", [(BF16, E4M3), (E4M3, E5M2), (E5M2, BF16)])
def test_another_type_on_the_same_address_and_shape(first, second):
    kv, bufs = _kv(dtype=first)
    _told(kv)
    kv.k, kv.v = (_on(b, 3, 2, 16, 64, second) for b in bufs)
    assert _told(kv)["kv_dtype"] == vx.kv_dtype_code(kv.k) and _told(kv) == _fresh(kv)


def test_each_field_that_a_description_holds():
    kv, bufs = _kv(ps=32)
    _told(kv)
    for name, value in (("block_size", 16), ("k_scale", 0.25), ("v_scale", 0.125)):
        setattr(kv, name, value)
        assert _told(kv)[name] == value and _told(kv) == _fresh(kv)
    kv.v = _on(bufs[1][64:], 3, 2, 32, 64, BF16)                       # V alone
    assert _told(kv)["v"] == kv.v.data_ptr()
    latent = vx.PagedKV(torch.zeros((2, 1, 16, 576), dtype=BF16), None, 512)
    _told(latent)
    latent.head_dim_v = 576
    assert _told(latent)["head_dim_v"] == 576


def test_a_cache_turned_into_a_view_is_refused():
    kv, bufs = _kv(H=16, ps=16)
    _told(kv)
    kv.k = kv.k.transpose(1, 2)                                        # same address, same shape
    with pytest.raises(AssertionError):
        kv.current()


def test_a_tensor_that_changes_in_place():
    kv, bufs = _kv(dtype=E4M3)
    _told(kv)
    kv.k.data, kv.v.data = (_on(b, 3, 2, 16, 64, E5M2) for b in bufs)
    assert _told(kv)["kv_dtype"] == vx.KV_FP8_E5M2 and _told(kv) == _fresh(kv)
    kv.k.data, kv.v.data = (_on(b, 2, 2, 16, 64, E5M2) for b in bufs)
    assert _told(kv)["num_phys_pages"] == 2 and _told(kv) == _fresh(kv)


def test_an_unchanged_cache_keeps_its_description():
    kv, _ = _kv()
    assert kv.current() is kv.current()


def test_v_must_have_the_pages_of_k():
    """Slots and page ids are bounded by K's pages: a V cache with fewer would be written past its end."""
    for dtype in (BF16, torch.uint8):
        D = 68 if dtype == torch.uint8 else 128
        new = lambda P, H, ps: torch.zeros((P, H, ps, D), dtype=dtype)  # noqa: E731
        for shape in ((8, 2, 16), (9, 1, 16), (9, 2, 8), (9, 4, 16)):
            kv = vx.PagedKV(new(9, 2, 16), new(*shape))
            for describe in (kv.struct, kv.ref, kv.current):
                with pytest.raises(ValueError, match="V cache"):
                    describe()
        assert vx.PagedKV(new(9, 2, 16), new(11, 2, 16)).struct().num_phys_pages == 9     # more pages do no harm


def test_k_and_v_on_two_devices():
    kv = vx.PagedKV(torch.zeros((3, 2, 16, 64), dtype=BF16), torch.zeros((3, 2, 16, 64), dtype=BF16, device="meta"))
    for describe in (kv.struct, kv.current):
        with pytest.raises(ValueError, match="one device"):
            describe()


def _pool_told(monkeypatch, pool):
    """The pool that page_extend and page_release describe to the library, from a call that gets no further."""
    told = []

    class Lib:
        @staticmethod
        def vx_page_extend(p, *a):
            told.append({n: getattr(p._obj, n) for n, _ in vx._Pool._fields_})
            return 0

        vx_page_release = vx_page_extend

    monkeypatch.setattr(vx, "lib", lambda: Lib)
    monkeypatch.setattr(vx, "_gpu_of", lambda t: t.get_device())
    monkeypatch.setattr(vx, "_stream", lambda *a: None)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    vx.page_extend(pool, i32(2), i32(2), vx.BatchSpec(i32(3), i32(6), i32(2), 4), i32(3),
                   torch.zeros(9, dtype=torch.int64), i32(2), i32(64))
    vx.page_release(pool, i32(2), None, i32(64))
    return told


def test_a_pool_is_described_as_it_is_now(monkeypatch):
    pool = vx.PagePool.empty(6, 3, 4, 16, device="cpu")
    first = _pool_told(monkeypatch, pool)
    assert first[0] == first[1] and (first[0]["table"], first[0]["table_stride"]) == (pool.table.data_ptr(), 4)
    pool.table, pool.lens = torch.zeros((5, 8), dtype=torch.int32), torch.zeros(5, dtype=torch.int32)      # it has grown
    pool.free_pages, pool.block_size, pool.page_size = torch.zeros(9, dtype=torch.int32), 16, 32
    for told in _pool_told(monkeypatch, pool):
        assert told == dict(free_pages=pool.free_pages.data_ptr(), free_count=pool.free_count.data_ptr(),
                            table=pool.table.data_ptr(), lens=pool.lens.data_ptr(), num_phys_pages=9, table_rows=5,
                            table_stride=8, page_size=32, block_size=16)


def test_pools_that_do_not_fit_are_refused(monkeypatch):
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    pool = vx.PagePool.empty(6, 3, 4, 16, device="cpu")
    _pool_told(monkeypatch, pool)
    for name, bad in (("lens", i32(2)), ("free_count", i32(0)), ("table", i32((4, 3)).t()), ("lens", i32(6)[::2]),
                      ("free_pages", torch.zeros(6)), ("free_pages", i32(12)[::2])):
        was = getattr(pool, name)
        setattr(pool, name, bad)
        with pytest.raises((TypeError, ValueError, AssertionError)):
            _pool_told(monkeypatch, pool)
        setattr(pool, name, was)
    _pool_told(monkeypatch, pool)


class _Recorder:
    """The library's calls, recorded instead of made: the cache and the batch that each is given."""

    def __init__(self):
        self.told, self.real = [], vx.lib()

    def __getattr__(self, name):
        if name == "vx_workspace_size":
            return self.real.vx_workspace_size

        def call(*args):
            given = [a._obj for a in args if hasattr(a, "_obj")]
            cache = next(g for g in given if isinstance(g, vx._Cache))
            batch = next(g for g in given if isinstance(g, vx._Batch))
            self.told.append((name, cache.k, cache.v, cache.k_scale, batch.page_indptr, batch.page_indices, batch.seq_lens))
            return 0
        return call


def _decoder(monkeypatch, dtype=BF16):
    rec = _Recorder()
    monkeypatch.setattr(vx, "lib", lambda: rec)
    monkeypatch.setattr(vx, "_stream", lambda *a: None)
    D = 68 if dtype == torch.uint8 else 128
    cache = lambda P=6: torch.zeros((P, 2, 16, D), dtype=dtype)  # noqa: E731
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    kv, batch = vx.PagedKV(cache(), cache(), k_scale=0.5), vx.BatchSpec(i32(3), i32(6), i32(2), 3)
    dec = SparseDecoder(kv, batch, 4, vx.MEAN_DOT, 1, 1, 3, 0.1)
    row = lambda t: torch.zeros((2, 2, 128), dtype=t)  # noqa: E731
    q, new, budget = torch.zeros((2, 4, 128), dtype=BF16), (row(kv.row_dtype), row(kv.row_dtype)), i32(2)

    def every_call():
        rec.told.clear()
        dec.summarize()
        dec.summarize(i32(2))
        dec.append(*new)
        dec.select(q, budget)
        dec.append_select(*new, q, budget)
        dec.step(q, budget, None, kv_new=new)
        assert len(rec.told) == 7
        return {t[1:] for t in rec.told}
    return dec, cache, i32, every_call


def _now(dec):
    kv, b = dec.kv, dec.batch
    return {(kv.k.data_ptr(), kv.v.data_ptr(), kv.k_scale, b.page_indptr.data_ptr(), b.page_indices.data_ptr(),
             b.seq_lens.data_ptr())}


def test_a_decoder_follows_replaced_tensors(monkeypatch):
    dec, cache, i32, every_call = _decoder(monkeypatch)
    assert every_call() == _now(dec)
    keep = [dec.kv.k, dec.kv.v, dec.batch.seq_lens]                     # so that no address is used again
    dec.kv.k, dec.kv.v = cache(), cache()
    assert every_call() == _now(dec)
    dec.kv.k_scale = 0.25
    assert every_call() == _now(dec)
    dec.batch.seq_lens, dec.batch.page_indices, dec.batch.page_indptr = i32(2), i32(9), i32(3)
    assert every_call() == _now(dec)
    keep.append(dec.kv.k.data)
    dec.kv.k.data = cache()                                             # the same tensor, other memory
    assert every_call() == _now(dec)
    assert len({t.data_ptr() for t in keep}) == 4


def test_a_decoder_follows_the_batch_in_place(monkeypatch):
    dec, _, i32, every_call = _decoder(monkeypatch)
    every_call()
    b = dec.batch
    keep = [t.data for t in (b.page_indptr, b.page_indices, b.seq_lens)]
    b.page_indptr.data, b.page_indices.data, b.seq_lens.data = i32(3), i32(6), i32(2)
    assert every_call() == _now(dec) and b.seq_lens.data_ptr() != keep[2].data_ptr()


@pytest.mark.parametrize("change", ["pages", "type", "batch", "bound", "keys", "page_size"])
def test_a_decoder_refuses_what_its_buffers_do_not_fit(monkeypatch, change):
    dec, cache, i32, every_call = _decoder(monkeypatch)
    every_call()
    if change == "pages":
        dec.kv.k, dec.kv.v = cache(7), cache(7)
    elif change == "type":
        dec.kv.k, dec.kv.v = cache().to(E4M3), cache().to(E4M3)
    elif change == "batch":
        dec.batch.seq_lens, dec.batch.page_indptr = i32(3), i32(4)
    elif change == "bound":
        dec.batch.max_pages_per_seq = 5
    elif change == "keys":
        dec.kv.v = None
    else:
        dec.kv.k, dec.kv.v = (torch.zeros((3, 2, 32, 128), dtype=BF16) for _ in range(2))
    for call in (dec.summarize, lambda: dec.summarize(i32(2)), lambda: dec.decode(torch.zeros((2, 4, 128), dtype=BF16))):
        with pytest.raises(ValueError, match="SparseDecoder"):
            call()


def test_a_new_decoder_describes_the_cache_as_it_is(monkeypatch):
    dec, cache, i32, every_call = _decoder(monkeypatch)
    every_call()
    old = dec.kv.k
    dec.kv.k = cache()
    other = SparseDecoder(dec.kv, dec.batch, 4, vx.MEAN_DOT, 1, 1, 3, 0.1)
    rec = vx.lib()
    rec.told.clear()
    other.select(torch.zeros((2, 4, 128), dtype=BF16), i32(2))
    assert rec.told[0][1] == dec.kv.k.data_ptr() != old.data_ptr()


@pytest.mark.parametrize("dtype,good,bad", [
    (torch.uint8, (BF16,), (torch.uint8, torch.float16, torch.float32)),      # mxfp4: rows are quantised by the append
    (BF16, (BF16, torch.int16), (torch.float32, E4M3, torch.uint8)),
    (E4M3, (E4M3, torch.uint8), (BF16, torch.float32)),                       # codes, or their bytes
])
def test_a_decoder_checks_the_type_of_new_rows(monkeypatch, dtype, good, bad):
    dec, _, i32, _ = _decoder(monkeypatch, dtype)
    q, budget = torch.zeros((2, 4, 128), dtype=BF16), i32(2)
    row = lambda t: torch.zeros((2, 2, 128), dtype=t)  # noqa: E731
    for t in good:
        dec.append(row(t), row(t))
        dec.append_select(row(t), row(t), q, budget)
    for t in bad:
        for rows in ((row(t), row(good[0])), (row(good[0]), row(t))):
            for call in (lambda: dec.append(*rows), lambda: dec.append_select(*rows, q, budget),
                         lambda: dec.step(q, budget, None, kv_new=rows)):
                with pytest.raises(TypeError, match="new rows"):
                    call()


def test_a_pool_whose_tensor_takes_other_memory(monkeypatch):
    pool = vx.PagePool.empty(6, 3, 4, 16, device="cpu")
    old = [_pool_told(monkeypatch, pool), pool.table.data]
    pool.table.data = torch.zeros((3, 9), dtype=torch.int32)
    for told in _pool_told(monkeypatch, pool):
        assert (told["table"], told["table_stride"]) == (pool.table.data_ptr(), 9) and told != old[0][0]


def test_counts_past_31_bits(monkeypatch):
    """Entries past what a call's 32-bit count holds: a capacity is the largest count, rows are refused."""
    told = {}

    class Lib:
        @staticmethod
        def vx_page_extend(*a):
            told["caps"] = a[7], a[10]
            return 0

        @staticmethod
        def vx_kv_write(*a):
            raise AssertionError("called with a cut count")

        vx_kv_read = vx_kv_write

    monkeypatch.setattr(vx, "lib", lambda: Lib)
    monkeypatch.setattr(vx, "_gpu_of", lambda t: t.get_device())
    monkeypatch.setattr(vx, "_stream", lambda *a: None)
    monkeypatch.setattr(vx, "_ptr", lambda t: None if t is None else t.data_ptr())
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    wide = lambda n, t: torch.zeros(1, dtype=t).expand(n)  # noqa: E731
    big = 2 ** 32 + 5
    vx.page_extend(vx.PagePool.empty(6, 3, 4, 16, device="cpu"), i32(2), i32(2),
                   vx.BatchSpec(i32(3), wide(big, torch.int32), i32(2), 4), i32(3), wide(big, torch.int64), i32(2), i32(64))
    assert told["caps"] == (2 ** 31 - 1, 2 ** 31 - 1)
    kv = vx.PagedKV(torch.zeros((1, 1, 16, 576), dtype=BF16), None, 512)
    rows = torch.zeros((1, 1, 576), dtype=BF16).expand(big, 1, 576)
    with pytest.raises(ValueError, match="rows"):
        vx.kv_write(kv, rows, None, wide(big, torch.int64))
    with pytest.raises(ValueError, match="rows"):
        vx.kv_read(kv, wide(big, torch.int64), rows, None)
