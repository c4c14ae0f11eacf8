"""Attention of a chunk's tokens over the paged cache (vx_chunk_attention) against 64 bits: head layouts, cache
types, lengths from one token on, odd sizes, windows, strided queries, masked places that hold NaN."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests._chunk import MLA_D, MLA_V, Chunk

pytestmark = pytest.mark.gpu
KINDS = ["bf16", "fp8_e4m3", "fp8_e5m2", "mxfp4"]


def _run(c, window=0, causal=True, want_lse=True, q=None, max_pages=None):
    kv, batch, qd, qi, ql = c.on_gpu()
    if max_pages:
        batch.max_pages_per_seq = max_pages
    qd = qd if q is None else q
    ws = torch.full((vx.chunk_workspace_size(vx.CHUNK_ATTENTION, kv, batch, c.rows, c.Hq),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((c.rows, c.Hq, c.Dv), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.rows, c.Hq), 7.0, dtype=torch.float32, device="cuda") if want_lse else None
    print(f"[chunk] {c.kind} H{c.H} g{c.g} D{c.D} ps{c.ps} lens {list(c.lens)[:6]} new {list(c.new)[:6]} w{window} {causal}", flush=True)
    vx.chunk_attention(qd, kv, batch, qi, c.sm_scale, out, ws, q_lens=ql, window=window, causal=causal, lse=lse)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()


def _check(c, out, lse, window=0, causal=True, **kw):
    ref, tol, rl, rt = c.attend(window, causal, **kw)
    none = np.isnan(rl)
    if lse is not None:
        assert (lse[none] == 7.0).all(), "rows of no token were written"
        empty = np.isneginf(rl)
        assert (lse[empty] == -np.inf).all()
        ok = ~none & ~empty
        assert (np.abs(lse - rl)[ok] <= rt[ok]).all(), np.max((np.abs(lse - rl) / np.maximum(rt, 1e-30))[ok])
    assert (out[none] == 7.0).all(), "rows of no token were written"
    err = np.abs(out - ref)[~none]
    assert (err <= tol[~none]).all(), (np.nanmax(err), np.nanmax(err / tol[~none]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,H,g", [(128, 8, 4), (64, 4, 1), (128, 1, 16), (64, 2, 5), (128, 2, 3), (64, 16, 2), (128, 4, 7)])
def test_layouts_and_types(kind, D, H, g):
    c = Chunk([D, H, g], [0, 37, 129, 1], [5, 1, 33, 70], H * g, H, D, kv=kind, ps=[16, 32, 64][g % 3], spare=2)
    _check(c, *_run(c))


@pytest.mark.parametrize("kind", KINDS[:3])
@pytest.mark.parametrize("before,new", [([0, 70, 200, 5], [1, 3, 20, 9]), ([400], [37])])
def test_latent(kind, before, new):
    c = Chunk([3, len(before)], before, new, 16, 1, MLA_D, ps=64, kv=kind, spare=1, sigma=0.5)
    assert c.Dv == MLA_V
    _check(c, *_run(c))


@pytest.mark.parametrize("kind", KINDS[:2])
@pytest.mark.parametrize("before,new", [([3000, 40, 1500], [3, 70, 1]), ([1100, 0, 600, 900, 300, 1050, 20, 800], [161, 160, 150, 170, 155, 165, 149, 163])])
def test_latent_in_parts(kind, before, new):
    """Long lists of few tiles, and a little more than one tile a CU, which is cut into two parts."""
    c = Chunk([13, len(before)], before, new, 16, 1, MLA_D, ps=64, kv=kind, sigma=0.5)
    _check(c, *_run(c))


@pytest.mark.parametrize("D,new", [(128, 33), (64, 65), (128, 1)])
def test_requests_that_fill_the_grid(D, new):
    """As many tiles as rows can have: every request one row past whole tiles; and the same with refused requests."""
    for n in (3, 64, 67):
        c = Chunk([n, new], [(17 * i) % 90 for i in range(n)], [new] * n, 8, 2, D)
        _check(c, *_run(c))
        c.q_lens = np.array([0 if i % 3 == 1 else new for i in range(n)], np.int32)
        _check(c, *_run(c))


@pytest.mark.parametrize("before,new", [([0], [1]), ([15], [1]), ([16], [1]), ([0], [16]), ([63], [2]), ([1000], [1]), ([2047, 5], [2, 1]),
                                        ([0], [257]), ([100], [300]), ([511], [129]), ([0] * 9, [1, 2, 3, 15, 16, 17, 31, 32, 33]),
                                        (list(range(0, 130, 2)), [1] * 65), (list(range(0, 70)), [1 + i % 3 for i in range(70)])])
@pytest.mark.parametrize("D,Hq,H", [(128, 8, 2), (64, 3, 1)])
def test_lengths(before, new, D, Hq, H):
    c = Chunk([len(before), D], before, new, Hq, H, D)
    _check(c, *_run(c))


@pytest.mark.parametrize("window", [1, 7, 16, 64, 100, 1 << 30, 2 ** 31 - 1])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(window, causal):
    c = Chunk([window % 1000], [0, 300, 33], [40, 150, 1], 8, 2, 64, ps=32)
    _check(c, *_run(c, window, causal), window=window, causal=causal)


@pytest.mark.parametrize("D,Hq,H", [(128, 8, 2), (MLA_D, 16, 1)])
def test_not_causal(D, Hq, H):
    c = Chunk([5, D], [0, 90, 200], [33, 7, 130], Hq, H, D, ps=64 if D == MLA_D else 16)
    _check(c, *_run(c, causal=False), causal=False)


def test_rows_of_no_token():
    """Rows behind the last request, rows of refused requests, requests of no rows and of no tokens."""
    c = Chunk([9], [20, 0, 33, 0, 64], [4, 0, 6, 3, 5], 8, 2, 64, extra_rows=11)
    c.q_lens = np.array([4, 0, 0, 3, 2], np.int32)
    c.lens = np.array([24, 0, 33, 3, 66], np.int32)
    _check(c, *_run(c))


def test_rows_before_the_first_token():
    """More rows than tokens: the first ones attend nothing."""
    for D, Hq, H, ps in ((64, 4, 2, 16), (MLA_D, 16, 1, 64)):
        c = Chunk([10, D], [0, 0], [12, 200], Hq, H, D, ps=ps)
        c.lens = np.array([5, 90], np.int32)
        _check(c, *_run(c))
        out, lse = _run(c, causal=False)
        _check(c, out, lse, causal=False)


def test_page_lists_that_end_early():
    c = Chunk([11], [100], [30], 4, 2, 64)
    ref = Chunk([11], [100], [30], 4, 2, 64)
    out, _ = _run(c, max_pages=4)                     # 64 tokens of the request exist
    ref_out = ref.attend()[0]
    kv, batch, q, qi, _ = c.on_gpu()
    k64, v64 = c.k64, c.v64
    page = c.indices[np.arange(64) // 16]
    for row, _, p in c.tokens():
        for h in range(2):
            k, v = k64[page, h, np.arange(64) % 16], v64[page, h, np.arange(64) % 16]
            z = c.sm_scale * (c.q.double().numpy()[row, 2 * h:2 * h + 2] @ k.T)
            w = np.exp(z - z.max(-1, keepdims=True))
            ref_out[row, 2 * h:2 * h + 2] = w / w.sum(-1, keepdims=True) @ v
    assert np.abs(out - ref_out).max() <= 3 * 2.0 ** -8 * np.abs(v64).max()


def test_strided_queries():
    """Queries of a fused projection: strides of rows and heads, an offset, heads in another order."""
    c = Chunk([12], [50, 3], [20, 9], 8, 2, 128)
    fused = torch.full((c.rows, 13, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    fused[:, 2:10] = c.q.cuda()
    ref, lse = _run(c)
    out, lse2 = _run(c, q=fused[:, 2:10])
    assert np.array_equal(out, ref) and np.array_equal(lse, lse2)
    flipped = torch.full((c.rows, 8, 192), float("nan"), dtype=torch.bfloat16, device="cuda")
    flipped[..., :128] = c.q.cuda()
    assert np.array_equal(_run(c, q=flipped[..., :128])[0], ref)
    by_head = c.q.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    assert np.array_equal(_run(c, q=by_head)[0], ref)


@pytest.mark.parametrize("D,Hq,H,new", [(128, 8, 2, 3), (64, 16, 4, 90), (MLA_D, 16, 1, 20), (128, 4, 4, 200)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_bad_values_in_masked_places(D, Hq, H, new, bad):
    """NaN and infinities behind the request's last token, in a later token of the chunk and in a token before the
    window reach no row that does not attend them."""
    ps = 64
    c = Chunk([13, D], [70], [new], Hq, H, D, ps=ps, spare=1)
    L = int(c.lens[0])
    behind = [L] if L % ps else []
    late, early = L - 1, 5
    for tok in behind + [late, early]:
        page = c.indices[tok // ps]
        for cache, c64 in ((c.k, c.k64), (c.v, c.v64)):
            if cache is not None:
                cache[page, :, tok % ps] = bad
                c64[page, :, tok % ps] = bad
    window = 60
    out, lse = _run(c, window)
    clean = [row for row, _, p in c.tokens() if p < late and p - window + 1 > early]
    assert clean or new < 3
    with np.errstate(all="ignore"):
        ref, tol, rl, rt = c.attend(window)
    assert np.isfinite(out[clean]).all()
    assert (np.abs(out - ref)[clean] <= tol[clean]).all() and (np.abs(lse - rl)[clean] <= rt[clean]).all()
    if bad != bad:
        rest = [row for row, _, p in c.tokens() if row not in clean]
        assert np.isnan(out[rest]).all()


def test_large_scores():
    """Scores far apart and far from zero."""
    c = Chunk([14], [300], [40], 8, 2, 128, sigma=12.0)
    _check(c, *_run(c))


def test_values_near_the_largest():
    """Weights are at most 1: values of V close to the type's largest do not overflow on the way."""
    c = Chunk([15], [600], [40], 8, 2, 128)
    c.v = (c.v.float().sign() * 3.0e38).to(torch.bfloat16)
    c.v64 = c.v.double().numpy()
    out, _ = _run(c)
    ref, tol, _, _ = c.attend()
    assert np.isfinite(out).all() and (np.abs(out - ref) <= tol).all()


@pytest.mark.parametrize("new,Hq", [(1, 8), (4, 8), (2, 2)])
def test_few_rows_of_long_contexts(new, Hq):
    c = Chunk([16, new], [20000, 3, 8191], [new] * 3, Hq, 2, 64, ps=64)
    _check(c, *_run(c))


def test_a_row_does_not_depend_on_the_batch():
    """The same request alone and among others: equal but for the order of its partial sums."""
    a = Chunk([17], [500], [64], 8, 2, 128)
    out, _ = _run(a)
    _, tol, _, _ = a.attend()
    b = Chunk([17], [500, 80, 0], [64, 30, 2], 8, 2, 128)
    pages = -(-564 // 16)
    b.k[b.indices[:pages]], b.v[b.indices[:pages]] = a.k[a.indices], a.v[a.indices]
    b.k64, b.v64 = b.k.double().numpy(), b.v.double().numpy()
    b.q[:64] = a.q
    out2, lse2 = _run(b)
    assert (np.abs(out2[:64] - out) <= 2 * tol).all()
    _check(b, out2, lse2)


def test_same_inputs_same_bits():
    c = Chunk([18], [5000, 100, 0], [3, 200, 50], 16, 4, 128)
    first, other = _run(c), _run(c)
    assert np.array_equal(first[0], other[0]) and np.array_equal(first[1], other[1])


def test_offsets_past_32_bits():
    """A cache of more than 2^32 elements, whose last pages are the request's."""
    P, H, ps, D = 2 ** 19 + 40, 8, 16, 64                     # 4.3e9 elements, 8.6 GB each
    k = torch.zeros((P, H, ps, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros((P, H, ps, D), dtype=torch.bfloat16, device="cuda")
    c = Chunk([19], [300], [20], 8, 8, 64)
    ids = torch.arange(P - 20, P, device="cuda")
    idx = torch.from_numpy(c.indices).long()
    k[ids], v[ids] = c.k[idx].cuda(), c.v[idx].cuda()
    kv, batch, q, qi, _ = c.on_gpu()
    kv = vx.PagedKV(k, v, 64)
    batch.page_indices = ids.int()
    ws = torch.empty(vx.chunk_workspace_size(vx.CHUNK_ATTENTION, kv, batch, c.rows, 8), dtype=torch.uint8, device="cuda")
    out = torch.empty((c.rows, 8, 64), dtype=torch.bfloat16, device="cuda")
    vx.chunk_attention(q, kv, batch, qi, c.sm_scale, out, ws)
    ref, tol, _, _ = c.attend()
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
