"""Arrays of the cache's own operators that overlap or lie at odd addresses are refused before any launch
(no GPU needed: every call here is refused)."""
import ctypes

import pytest
import torch

from paper_2606_06453_amd import vx

B, ROWS, STRIDE, PHYS = 4, 6, 8, 40
SLAB = torch.zeros(1 << 16, dtype=torch.uint8)


def _place(sizes):
    """An address for every array, apart from each other."""
    at, places = SLAB.data_ptr() + (-SLAB.data_ptr()) % 256, {}
    for name, n in sizes.items():
        places[name] = at
        at += (n + 255) // 256 * 256 + 512
    assert at < SLAB.data_ptr() + SLAB.numel()
    return places


POOL = dict(free_pages=4 * PHYS, free_count=4, table=4 * ROWS * STRIDE, lens=4 * ROWS)
EXTEND = dict(POOL, rows=4 * B, new_lens=4 * B, seq_lens=4 * B, page_indptr=4 * (B + 1), page_indices=4 * 9,
              token_indptr=4 * (B + 1), slots=8 * 11, granted=4 * B, first_block=4 * B, workspace=256)
RELEASE = dict(POOL, rows=4 * B, keep_lens=4 * B, workspace=256)
READ = {"extend": {"free_pages", "rows", "new_lens"}, "release": {"table", "rows", "keep_lens"}}


def _call(op, at):
    pool = vx._Pool(at["free_pages"], at["free_count"], at["table"], at["lens"], PHYS, ROWS, STRIDE, 16, 0)
    if op == "release":
        return vx.lib().vx_page_release(ctypes.byref(pool), B, at["rows"], at["keep_lens"], at["workspace"], 256, None)
    return vx.lib().vx_page_extend(ctypes.byref(pool), B, at["rows"], at["new_lens"], at["seq_lens"], at["page_indptr"],
                                   at["page_indices"], 9, at["token_indptr"], at["slots"], 11, at["granted"],
                                   at["first_block"], at["workspace"], 256, None)


def _msg():
    return vx.lib().vx_last_error().decode()


@pytest.mark.parametrize("op", ["extend", "release"])
def test_arrays_that_overlap(op):
    """Every pair of which the call writes one: the same address, and the last bytes of one the first of the other."""
    sizes = EXTEND if op == "extend" else RELEASE
    names, seen = list(sizes), 0
    for a in names:
        for b in names:
            if a == b or {a, b} <= READ[op]:
                continue
            step = 8 if "slots" in (a, b) else 4
            for shift in {0, sizes[a] - step} if sizes[a] > step else {0}:
                at = _place(sizes)
                at[b] = at[a] + shift
                assert _call(op, at) == 1, (a, b, shift)
                assert a in _msg() and b in _msg() and "overlap" in _msg(), (a, b, _msg())
                seen += 1
    assert seen > 2 * len(names)
@pytest.mark.parametrize("op", ["extend", "release"])
def test_odd_addresses(op):
    sizes = EXTEND if op == "extend" else RELEASE
    for name in sizes:
        for off in (1, 2) + ((4,) if name == "slots" else ()):
            at = _place(sizes)
            at[name] += off
            assert _call(op, at) == 1 and name in _msg() and "aligned" in _msg(), (name, off, _msg())


def test_odd_slots_of_rows():
    at = _place(dict(k=8192, v=8192, rows=8192, slots=80))
    kv = vx._Cache(at["k"], at["v"], 2, 2, 16, 64, 64, vx.KV_BF16, 1.0, 1.0, 0)
    for fn in (vx.lib().vx_kv_write, vx.lib().vx_kv_read):
        assert fn(ctypes.byref(kv), at["rows"], 128, 64, at["rows"] + 4096, 128, 64, at["slots"] + 4, 3, None) == 1
        assert "slots" in _msg() and "aligned" in _msg()


def _first_overlap(n, heads, row, head, dim):
    """Whether two of the rows at r * row + h * head, `dim` long, share an element: by looking at all of them."""
    at = sorted(r * row + h * head for r in range(n) for h in range(heads))
    return any(b - a < dim for a, b in zip(at, at[1:]))


def test_rows_read_into_one_another():
    """vx_kv_read stores every row at the same time; rows of k_out or v_out that overlap are refused."""
    at = _place(dict(k=8192, v=8192, rows=16384, slots=800))
    L, D, seen = vx.lib(), 64, {False: 0, True: 0}
    strides = [0, 8, 56, 64, 72, 128, 136, 192, 256, 264, 320, 512, 1024, -64, -128, -192, -1024]
    for heads in (1, 2, 4):
        kv = vx._Cache(at["k"], at["v"], 2, heads, 16, D, D, vx.KV_BF16, 1.0, 1.0, 0)
        for n in (1, 2, 3, 7):
            for row in strides:
                for head in strides:
                    bad = _first_overlap(n, heads, row, head, D)
                    seen[bad] += 1
                    if not bad:
                        continue                                     # a call that would be made
                    good = (heads * D, D)
                    for a, b, name in (((row, head), good, "k_out"), (good, (row, head), "v_out")):
                        assert L.vx_kv_read(ctypes.byref(kv), at["rows"], *a, at["rows"] + 8192, *b, at["slots"], n, None) == 1
                        assert name in _msg() and "overlap" in _msg(), (heads, n, row, head, _msg())
    assert min(seen.values()) > 100


@pytest.mark.parametrize("dtype", [vx.KV_BF16, vx.KV_FP8_E4M3, vx.KV_MXFP4])
def test_an_odd_decode_workspace(dtype):
    """The split counters at its start are 32-bit atomics."""
    at = _place(dict(k=8192, v=8192, q=1024, ints=256, out=1024, ws=4096))
    kv = vx._Cache(at["k"], at["v"], 2, 2, 16, 64, 64, dtype, 1.0, 1.0, 0)
    b = vx._Batch(1, 4, at["ints"], at["ints"], at["ints"])
    for off in (1, 2, 3):
        assert vx.lib().vx_sparse_paged_decode(at["q"], 4, ctypes.byref(kv), ctypes.byref(b), at["ints"], at["ints"], 4, 0.1,
                                               at["out"], at["ws"] + off, 1 << 24, None) == 1
        assert "workspace" in _msg() and "aligned" in _msg()
