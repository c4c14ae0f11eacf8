"""Selection of blocks for every token of a chunk (vx_chunk_score_topk) and attention over them
(vx_sparse_chunk_attention) against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests._chunk import Chunk

pytestmark = pytest.mark.gpu
KINDS = ["bf16", "fp8_e4m3", "fp8_e5m2", "mxfp4"]


def _attend(c, sel, count, want_lse=True):
    kv, batch, q, qi, ql = c.on_gpu()
    M = sel.shape[2]
    ws = torch.full((vx.chunk_workspace_size(vx.CHUNK_SPARSE, kv, batch, c.rows, c.Hq, M),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((c.rows, c.Hq, c.Dv), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.rows, c.Hq), 7.0, dtype=torch.float32, device="cuda") if want_lse else None
    print(f"[sparse] {c.kind} H{c.H} g{c.g} D{c.D} ps{c.ps}/{c.block} rows {c.rows} M{M}", flush=True)
    vx.sparse_chunk_attention(q, kv, batch, qi, torch.from_numpy(sel).cuda(), torch.from_numpy(count).cuda(), c.sm_scale, out, ws,
                              q_lens=ql, lse=lse)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()


def _check(c, out, lse, sel, count):
    ref, tol, rl, rt = c.attend(sel=lambda row, h: set(sel[row, h, : max(0, min(int(count[row]), sel.shape[2]))].tolist()))
    none, empty = np.isnan(rl), np.isneginf(rl)
    assert (out[none] == 7.0).all() and (out[empty] == 0.0).all()
    if lse is not None:
        assert (lse[none] == 7.0).all() and (lse[empty] == -np.inf).all()
        ok = ~none & ~empty
        assert (np.abs(lse - rl)[ok] <= rt[ok]).all()
    err = np.abs(out - ref)[~none]
    assert (err <= tol[~none]).all(), (np.max(err), np.max(err / tol[~none]))


def _lists(c, seed, M, share=0.7):
    """Each row's own blocks: random ones of those before it, its own among them, ascending."""
    rng = np.random.default_rng(seed)
    bs = c.block or c.ps
    sel, count = np.full((c.rows, c.H, M), -1, np.int32), np.zeros(c.rows, np.int32)
    for row, i, p in c.tokens():
        nb = p // bs + 1
        count[row] = n = min(M, max(1, int(nb * share)))
        for h in range(c.H):
            sel[row, h, :n] = np.sort(np.concatenate([[nb - 1], rng.choice(nb - 1, n - 1, replace=False)])) if n > 1 else nb - 1
    return sel, count


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,H,g,ps,block", [(128, 8, 4, 16, 0), (64, 4, 1, 64, 16), (128, 1, 16, 32, 0), (64, 2, 5, 64, 32), (128, 2, 3, 64, 0),
                                            (64, 16, 2, 32, 16), (128, 4, 7, 16, 0)])
def test_layouts_and_types(kind, D, H, g, ps, block):
    c = Chunk([D, H, g, 1], [0, 137, 430, 1], [5, 1, 23, 40], H * g, H, D, kv=kind, ps=ps, block=block, spare=2)
    sel, count = _lists(c, [D, g], 12)
    _check(c, *_attend(c, sel, count), sel, count)


@pytest.mark.parametrize("before,new", [([0], [1]), ([15], [1]), ([16], [1]), ([1000], [1]), ([2047, 5], [2, 1]), ([0], [130]), ([511], [67]),
                                        (list(range(0, 130, 2)), [1] * 65), ([8000], [4])])
@pytest.mark.parametrize("M", [1, 3, 64, 501])
def test_lengths(before, new, M):
    c = Chunk([len(before), 2], before, new, 8, 2, 64)
    sel, count = _lists(c, [M, 5], M)
    _check(c, *_attend(c, sel, count), sel, count)


@pytest.mark.parametrize("n,new", [(3, 17), (64, 17), (67, 17), (70, 1)])
def test_requests_that_fill_the_grid(n, new):
    """As many tiles as rows can have, and the same with refused requests."""
    c = Chunk([n, new, 5], [(37 * i) % 200 for i in range(n)], [new] * n, 8, 2, 64)
    sel, count = _lists(c, [n, 3], 8)
    _check(c, *_attend(c, sel, count), sel, count)
    c.q_lens = np.array([0 if i % 3 == 1 else new for i in range(n)], np.int32)
    _check(c, *_attend(c, sel, count), sel, count)


@pytest.mark.parametrize("kind", KINDS[:2] + KINDS[3:])
@pytest.mark.parametrize("new,D", [(3, 64), (70, 128)])
def test_most_blocks_of_a_request(kind, new, D):
    """16384 blocks: the lists' largest marks, in narrow and wide tiles."""
    c = Chunk([new, D, 7], [(1 << 18) - new], [new], 2, 1, D, kv=kind)
    sel, count = _lists(c, [new, 4], 40)
    _check(c, *_attend(c, sel, count), sel, count)


def test_lists_as_they_come():
    """Any order, blocks listed twice, ids outside the row's blocks, counts of zero, below zero and past the lists,
    rows of no token."""
    c = Chunk([21], [300, 64, 0], [40, 17, 9], 8, 2, 64, extra_rows=5)
    rng = np.random.default_rng(3)
    M = 24
    sel = rng.integers(-3, 40, size=(c.rows, 2, M)).astype(np.int32)
    sel[3], sel[4] = 7, -1
    sel[5, 0, 0] = 2 ** 31 - 1
    count = rng.integers(-2, M + 9, size=c.rows).astype(np.int32)
    count[:3] = 0
    c.q_lens = np.array([40, 17, 4], np.int32)
    c.lens = np.array([340, 81, 4], np.int32)
    bs = 16
    pos = dict((row, p) for row, _, p in c.tokens())
    clean = np.where((sel >= 0) & (sel <= np.array([pos.get(r, 0) // bs for r in range(c.rows)])[:, None, None]), sel, -1)
    _check(c, *_attend(c, sel, count), clean, count)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("new", [3, 40])
def test_bad_values_in_blocks_of_other_rows(bad, new):
    """A block that holds NaN reaches the rows that list it and no others of the tile."""
    c = Chunk([22, new], [300], [new], 8, 2, 128)
    sel, count = _lists(c, 4, 9)
    sel[:, :, 0] = np.where(np.arange(c.rows)[:, None] % 2 == 0, 1, 0)
    sel[:, :, 1:] = np.clip(sel[:, :, 1:], 2, None)
    for cache, c64 in ((c.k, c.k64), (c.v, c.v64)):
        cache[c.indices[1], :, 3] = bad
        c64[c.indices[1], :, 3] = bad
    out, lse = _attend(c, sel, count)
    clean = np.arange(c.rows) % 2 == 1
    ref, tol, rl, rt = c.attend(sel=lambda row, h: set(sel[row, h, : count[row]].tolist()))
    assert (np.abs(out - ref)[clean] <= tol[clean]).all() and (np.abs(lse - rl)[clean] <= rt[clean]).all()
    if bad != bad:
        assert np.isnan(out[~clean]).all()


def test_every_block_is_dense_attention():
    c = Chunk([23], [700, 3], [50, 20], 12, 4, 128)
    M = -(-750 // 16)
    sel = np.broadcast_to(np.arange(M, dtype=np.int32), (c.rows, 4, M)).copy()
    count = np.array([p // 16 + 1 for _, _, p in c.tokens()], np.int32)
    _check(c, *_attend(c, sel, count), sel, count)


# ---- selection -----------------------------------------------------------------------------------
def _select(c, mean, budget, n_sink, n_local, M, q=None):
    kv, batch, qd, qi, ql = c.on_gpu()
    md = torch.from_numpy(mean).cuda()
    ws = torch.full((vx.chunk_workspace_size(vx.CHUNK_SCORE_TOPK, kv, batch, c.rows, c.Hq, M),), 255, dtype=torch.uint8, device="cuda")
    sel = torch.full((c.rows, c.H, M), -2, dtype=torch.int32, device="cuda")
    count = torch.full((c.rows,), -2, dtype=torch.int32, device="cuda")
    print(f"[select] H{c.H} g{c.g} D{c.D} ps{c.ps}/{c.block} rows {c.rows} M{M}", flush=True)
    vx.chunk_score_topk(qd if q is None else q, kv, batch, qi, vx.MEAN_DOT, md, torch.from_numpy(budget).cuda(), n_sink, n_local, M, sel,
                        count, ws, q_lens=ql)
    torch.cuda.synchronize()
    return sel.cpu().numpy(), count.cpu().numpy()


def _mean(c, seed, sigma=0.25):
    r = c.ps // (c.block or c.ps)
    return (np.random.default_rng(seed).standard_normal((c.P * r, c.H, c.D)) * sigma).astype(np.float32)


def _same(c, mean, budget, n_sink, n_local, M):
    budget = np.asarray(budget, np.int32)
    ref = c.select(mean, budget, n_sink, n_local, M)
    got = _select(c, mean, budget, n_sink, n_local, M)
    assert np.array_equal(got[1], ref[1])
    bad = np.argwhere((got[0] != ref[0]).any(-1))
    assert len(bad) == 0, (bad[:4], [(got[0][tuple(b)], ref[0][tuple(b)]) for b in bad[:2]])


@pytest.mark.parametrize("D,H,g,ps,block", [(128, 8, 4, 16, 0), (64, 4, 1, 64, 16), (128, 1, 16, 32, 0), (64, 2, 5, 64, 32), (128, 2, 3, 64, 0),
                                            (64, 16, 2, 32, 16), (128, 4, 7, 16, 0)])
def test_select_layouts(D, H, g, ps, block):
    c = Chunk([D, H, g, 2], [0, 137, 1430, 1], [5, 1, 23, 40], H * g, H, D, ps=ps, block=block, spare=2)
    _same(c, _mean(c, [D, g]), [12, 9, 7, 1], 1, 2, 12)


@pytest.mark.parametrize("before,new", [([0], [1]), ([15], [1]), ([16], [1]), ([1000], [1]), ([2047, 5], [2, 1]), ([0], [130]), ([511], [67]),
                                        (list(range(0, 130, 2)), [1] * 65), ([40000], [19]), ([100000], [3])])
@pytest.mark.parametrize("M,n_sink,n_local", [(1, 0, 1), (5, 2, 2), (64, 0, 1), (600, 1, 2)])
def test_select_lengths(before, new, M, n_sink, n_local):
    c = Chunk([len(before), 4], before, new, 4, 2, 64)
    _same(c, _mean(c, [M, 6]), [M] * len(before), n_sink, n_local, M)


@pytest.mark.parametrize("n,new", [(3, 17), (64, 17), (67, 17), (5, 65), (70, 1)])
def test_select_requests_that_fill_the_grid(n, new):
    c = Chunk([n, new, 6], [(137 * i) % 600 for i in range(n)], [new] * n, 4, 2, 64)
    mean, budget = _mean(c, [n, 8]), [7] * n
    _same(c, mean, budget, 1, 2, 7)
    c.q_lens = np.array([0 if i % 3 == 1 else new for i in range(n)], np.int32)
    _same(c, mean, budget, 1, 2, 7)


@pytest.mark.parametrize("new", [2, 19])
def test_select_among_most_blocks(new):
    c = Chunk([new, 9], [(1 << 18) - new], [new], 4, 2, 64)
    _same(c, _mean(c, [new, 10]), [100], 1, 2, 100)


@pytest.mark.parametrize("what", ["equal", "two_values", "signed_zeros", "close", "huge", "bf16_ties", "nan", "inf"])
def test_select_ties_and_odd_scores(what):
    """Scores that are equal, differ in their last bits only, or are not finite."""
    c = Chunk([24], [3000, 900], [9, 20], 4, 2, 64)
    rng = np.random.default_rng(7)
    mean = _mean(c, 8)
    if what == "equal":
        mean[:] = mean[0]
    elif what == "two_values":
        mean[:] = np.where(rng.random(len(mean))[:, None, None] < 0.5, mean[0], mean[1])
    elif what == "signed_zeros":
        mean[:] = np.where(rng.random(mean.shape) < 0.5, 0.0, -0.0)
    elif what == "close":
        mean[:] = mean[0] * (1 + 2.0 ** -22 * rng.integers(0, 8, (len(mean), 1, 1)))
    elif what == "huge":
        mean *= 1e36
    elif what == "bf16_ties":                                     # the bf16 copies are equal, the means are not
        mean[:] = torch.from_numpy(mean[0]).to(torch.bfloat16).float().numpy() * (1 + 2.0 ** -12 * rng.random((len(mean), 1, 1)))
    elif what == "nan":
        mean[rng.integers(0, len(mean), 40), 0, 3] = np.nan
    elif what == "inf":
        mean[rng.integers(0, len(mean), 40), 1, 5] = np.inf
        mean[rng.integers(0, len(mean), 40), 0, 6] = -np.inf
    with np.errstate(all="ignore"):
        _same(c, mean.astype(np.float32), [37, 11], 1, 2, 40)


def test_select_budgets_and_rows_of_no_token():
    """Budgets of zero, below zero, of every block; refused requests; rows behind the last and before the first token."""
    c = Chunk([25], [300, 100, 64, 0, 200], [6, 5, 4, 8, 9], 8, 2, 64, extra_rows=3)
    c.q_lens = np.array([6, 5, 0, 8, 2], np.int32)
    c.lens = np.array([306, 105, 64, 3, 202], np.int32)
    _same(c, _mean(c, 9), [0, -5, 9, 100, 5], 2, 1, 30)


def test_select_is_the_decode_selection():
    """Each token by itself is a request of its own for vx_page_score_topk."""
    c = Chunk([26], [2000], [30], 8, 2, 128)
    mean = _mean(c, 10)
    sel, count = _select(c, mean, np.array([20], np.int32), 1, 2, 20)
    kv, batch, q, _, _ = c.on_gpu()
    B = c.rows
    lens = torch.arange(2001, 2031, dtype=torch.int32, device="cuda")
    pages = batch.page_indices.repeat(B)
    per = batch.page_indices.numel()
    one = vx.BatchSpec(torch.arange(0, B + 1, dtype=torch.int32, device="cuda") * per, pages, lens, per)
    ws = torch.empty(vx.workspace_size(vx.STAGE_SCORE_TOPK, kv, one, 8, 20), dtype=torch.uint8, device="cuda")
    s2, c2 = torch.empty((B, 2, 20), dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    vx.page_score_topk(q, kv, one, vx.MEAN_DOT, torch.from_numpy(mean).cuda(), None, None, torch.full((B,), 20, dtype=torch.int32, device="cuda"),
                       1, 2, 20, s2, c2, ws)
    torch.cuda.synchronize()
    assert np.array_equal(sel, s2.cpu().numpy()) and np.array_equal(count, c2.cpu().numpy())


def test_select_strided_queries():
    c = Chunk([27], [700], [21], 8, 2, 128)
    mean = _mean(c, 11)
    budget = np.array([9], np.int32)
    fused = torch.full((c.rows, 13, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    fused[:, 3:11] = c.q.cuda()
    a, b = _select(c, mean, budget, 1, 1, 9), _select(c, mean, budget, 1, 1, 9, q=fused[:, 3:11])
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
