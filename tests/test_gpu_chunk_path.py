"""The chunk calls as a serving program runs them: pages for a step, rotated rows into the cache, summaries, blocks
for each token, attention; then decode steps on the same cache.  Captured into a graph, and on a stream of their own."""
import math

import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from paper_2606_06453_amd.decoder import SparseDecoder
from tests._chunk import Chunk

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _reference(q, k, v, pos, scale, keep=None):
    """fp64 attention of rows q [n][Hq][D] at pos over rows k, v [L][H][D]; keep [n][H][L]: what each may attend."""
    n, Hq, D = q.shape
    g = Hq // k.shape[1]
    out, absv = np.zeros((n, Hq, v.shape[2])), np.zeros((n, Hq, v.shape[2]))
    for r in range(n):
        for x in range(Hq):
            m = np.arange(len(k)) <= pos[r]
            if keep is not None:
                m &= keep[r, x // g]
            z = scale * (k[m, x // g] @ q[r, x])
            w = np.exp(z - z.max())
            w /= w.sum()
            out[r, x], absv[r, x] = w @ v[m, x // g], w @ np.abs(v[m, x // g])
    return out, 2.0 ** -8 * np.abs(out) + 2.2 * 2.0 ** -8 * absv + 1e-6


@pytest.mark.parametrize("kind", ["bf16", "mxfp4", "fp8_e4m3"])
def test_prompts_drafts_and_decode_steps(kind):
    H, Hq, D, ps, P = 2, 8, 64, 16, 40
    g = Hq // H
    rng = np.random.default_rng([5, len(kind)])
    if kind == "mxfp4":
        K, V = vx.mxfp4_cache(P, H, ps, D), vx.mxfp4_cache(P, H, ps, D)
    else:
        t = {"bf16": torch.bfloat16, "fp8_e4m3": torch.float8_e4m3fn}[kind]
        K, V = (torch.zeros((P, H, ps, D), device=DEV).to(t) for _ in range(2))
    scale = 1.0 if kind != "fp8_e4m3" else 0.015625
    kv = vx.PagedKV(K, V, D, k_scale=scale, v_scale=scale)
    pool = vx.PagePool.empty(P, 4, 32, ps)
    rope = vx.Rope(torch.tensor([1e4 ** (-c / 32) for c in range(32)], device=DEV))
    rows = _i32(2, 0, 3)
    batch = vx.BatchSpec(torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(128, dtype=torch.int32, device=DEV),
                         torch.zeros(3, dtype=torch.int32, device=DEV), 32)
    token_indptr, granted, first = torch.zeros(4, dtype=torch.int32, device=DEV), _i32(0, 0, 0), _i32(0, 0, 0)
    page_ws = torch.zeros(vx.page_workspace_size(3), dtype=torch.uint8, device=DEV)
    mean = torch.full((P, H, D), float("nan"), device=DEV)
    sm = 1.0 / math.sqrt(D)
    written = [[np.zeros((0, H, D))] * 2 for _ in range(3)]       # what each request's cache rows read back as
    kept = [0, 0, 0]
    # two chunks of prompts (the last request's second one is refused: no pages left), drafts, a step of single tokens
    for new in ([200, 37, 5], [90, 60, 500], [4, 3, 2], [1, 1, 1]):
        n = sum(new)
        slots = torch.zeros(n + 3, dtype=torch.int64, device=DEV)
        vx.page_extend(pool, rows, _i32(*new), batch, token_indptr, slots, granted, page_ws, first_block=first)
        got = granted.tolist()
        assert got == [x if x != 500 else 0 for x in new]
        lens = batch.seq_lens.tolist()
        fused = torch.from_numpy(rng.standard_normal((n + 3, Hq + 2 * H, D)).astype(np.float32)).to(torch.bfloat16).to(DEV)
        positions = torch.zeros(n + 3, dtype=torch.int64)
        for i in range(3):
            a = sum(new[:i])
            positions[a:a + new[i]] = torch.arange(kept[i], kept[i] + new[i])
        q = torch.full((n + 3, Hq, D), 3.0, dtype=torch.bfloat16, device=DEV)
        vx.rope_kv_write(kv, rope, fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:], positions.to(DEV), slots, q)
        vx.page_summarize(kv, batch, first, mean, None, None)
        ws = torch.empty(vx.chunk_workspace_size(vx.CHUNK_ATTENTION, kv, batch, n + 3, Hq), dtype=torch.uint8, device=DEV)
        out = torch.full((n + 3, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
        vx.chunk_attention(q, kv, batch, token_indptr, sm, out, ws, q_lens=granted)
        M = 6
        budget = _i32(6, 6, 6)
        sel, count = torch.full((n + 3, H, M), -9, dtype=torch.int32, device=DEV), torch.full((n + 3,), -9, dtype=torch.int32, device=DEV)
        ws1 = torch.empty(vx.chunk_workspace_size(vx.CHUNK_SCORE_TOPK, kv, batch, n + 3, Hq, M), dtype=torch.uint8, device=DEV)
        vx.chunk_score_topk(q, kv, batch, token_indptr, vx.MEAN_DOT, mean, budget, 1, 2, M, sel, count, ws1, q_lens=granted)
        ws2 = torch.empty(vx.chunk_workspace_size(vx.CHUNK_SPARSE, kv, batch, n + 3, Hq, M), dtype=torch.uint8, device=DEV)
        sparse = torch.full_like(out, 7.0)
        vx.sparse_chunk_attention(q, kv, batch, token_indptr, sel, count, sm, sparse, ws2, q_lens=granted)
        back = [torch.empty((n + 3, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        vx.kv_read(kv, slots, *back)
        torch.cuda.synchronize()
        k_rows, v_rows = (x.double().cpu().numpy() for x in back)
        qd, od, sd = (x.double().cpu().numpy() for x in (q, out, sparse))
        pages, means = pool.table.cpu().numpy(), mean.cpu().numpy()
        for i in range(3):
            a, b = sum(new[:i]), sum(new[:i]) + got[i]
            written[i] = [np.concatenate([w, x[a:b]]) for w, x in zip(written[i], (k_rows, v_rows))]
            assert lens[i] == kept[i] + got[i] == len(written[i][0])
            if b > a:
                pos = np.arange(kept[i], lens[i])
                ref, tol = _reference(qd[a:b], *written[i], pos, sm)
                assert (np.abs(od[a:b] - ref) <= tol).all()
                phys = pages[[2, 0, 3][i]]
                keep = np.zeros((b - a, H, lens[i]), bool)
                for r in range(b - a):
                    nb = pos[r] // ps + 1
                    assert count[a + r] == min(nb, M)
                    for h in range(H):
                        z = (means[phys[:nb], h].astype(np.float64) @ qd[a + r, h * g:(h + 1) * g].mean(0)).astype(np.float32)
                        z[[0] + list(range(max(0, nb - 2), nb))] = np.inf
                        best = np.sort(np.lexsort((np.arange(nb), -z.astype(np.float64)))[:M])
                        assert np.array_equal(sel[a + r, h, : len(best)].cpu().numpy(), best)
                        keep[r, h] = np.isin(np.arange(lens[i]) // ps, best)
                ref, tol = _reference(qd[a:b], *written[i], pos, sm, keep)
                assert (np.abs(sd[a:b] - ref) <= tol).all()
            assert (od[b:sum(new[:i + 1])] == 7.0).all() and (sd[b:sum(new[:i + 1])] == 7.0).all()   # refused rows
            kept[i] = lens[i]
        assert (od[n:] == 7.0).all() and (sd[n:] == 7.0).all() and (sel[n:] == -9).all() and (count[n:] == -9).all()
    # the last step again as a decode step over the blocks that the chunk call chose
    dec = SparseDecoder(kv, batch, Hq, vx.MEAN_DOT, 1, 2, M, sm)
    dec.summarize()
    dec.select(q[:3].contiguous(), budget)
    assert torch.equal(dec.sel_pages, sel[:3]) and torch.equal(dec.sel_count, count[:3])
    one = dec.decode(q[:3].contiguous()).double().cpu().numpy()
    absv = np.max([np.abs(w[1]).max() for w in written])
    assert np.abs(one - sd[:3]).max() <= 4 * 2.0 ** -8 * absv


def _calls(c, ws, sel, count, q_in, q, out, lse, sparse, kv, batch, qi, rope, rows, pos, slots, mean, budget, M, stream=None):
    vx.rope_kv_write(kv, rope, q_in, rows[0], rows[1], pos, slots, q, stream=stream)
    vx.page_summarize(kv, batch, None, mean, None, None, stream=stream)
    vx.chunk_attention(q, kv, batch, qi, c.sm_scale, out, ws[0], lse=lse, stream=stream)
    vx.chunk_score_topk(q, kv, batch, qi, vx.MEAN_DOT, mean, budget, 1, 1, M, sel, count, ws[1], stream=stream)
    vx.sparse_chunk_attention(q, kv, batch, qi, sel, count, c.sm_scale, sparse, ws[2], stream=stream)


def _setup(new, before):
    c = Chunk([31, len(new)], before, new, 8, 2, 64)
    kv, batch, q_in, qi, _ = c.on_gpu()
    n, M = c.rows, 8
    state = dict(
        ws=[torch.empty(vx.chunk_workspace_size(s, kv, batch, n, 8, M), dtype=torch.uint8, device=DEV) for s in (0, 1, 2)],
        sel=torch.empty((n, 2, M), dtype=torch.int32, device=DEV), count=torch.empty(n, dtype=torch.int32, device=DEV),
        q_in=q_in, q=torch.empty_like(q_in), out=torch.empty_like(q_in), lse=torch.empty((n, 8), device=DEV),
        sparse=torch.empty_like(q_in), kv=kv, batch=batch, qi=qi, rope=vx.Rope(torch.full((32,), 0.01, device=DEV)),
        rows=[torch.randn((n, 2, 64), device=DEV).to(torch.bfloat16) for _ in range(2)],
        pos=torch.zeros(n, dtype=torch.int64, device=DEV), slots=torch.zeros(n, dtype=torch.int64, device=DEV),
        mean=torch.zeros((c.P, 2, 64), device=DEV), budget=torch.full((len(new),), M, dtype=torch.int32, device=DEV), M=M)
    for row, i, p in c.tokens():
        state["pos"][row] = p
        state["slots"][row] = int(c.indices[c.indptr[i] + p // 16]) * 16 + p % 16
    return c, state


RESULTS = ("q", "out", "lse", "sparse", "sel", "count")


@pytest.mark.parametrize("new,before", [([1, 3], [2000, 30]), ([100, 1, 40], [3000, 500, 0])])
def test_captured_and_replayed(new, before):
    """Every replay equals the eager calls on the same inputs, with eager work and synchronizations between."""
    c, s = _setup(new, before)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _calls(c, **s)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _calls(c, **s)
    lens = s["batch"].seq_lens.clone()
    gen = torch.Generator(device=DEV).manual_seed(1)
    for turn in range(4):
        s["q_in"].copy_(torch.randn(s["q_in"].shape, generator=gen, device=DEV))
        s["rows"][0].copy_(torch.randn(s["rows"][0].shape, generator=gen, device=DEV))
        if turn == 2:                                              # the batch as it is at replay, not at capture
            s["batch"].seq_lens.copy_(lens - 1)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: s[n].clone() for n in RESULTS}
        for n in RESULTS:
            s[n].zero_()
        _calls(c, **s)
        torch.cuda.synchronize()
        for n in RESULTS:
            assert torch.equal(got[n], s[n]), (turn, n)


def test_on_a_stream_of_its_own():
    c, s = _setup([60, 2], [700, 4000])
    _calls(c, **s)
    torch.cuda.synchronize()
    want = {n: s[n].clone() for n in RESULTS}
    for n in RESULTS:
        s[n].zero_()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    _calls(c, **s, stream=stream)
    stream.synchronize()
    for n in RESULTS:
        assert torch.equal(want[n], s[n]), n


def test_two_batches_at_once():
    """Calls of two batches on two streams, each with its own workspaces."""
    a, b = _setup([3, 1], [5000, 8000]), _setup([90], [3000])
    want = []
    for c, s in (a, b):
        _calls(c, **s)
        torch.cuda.synchronize()
        want.append({n: s[n].clone() for n in RESULTS})
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for (c, s), stream in zip((a, b), streams):
            _calls(c, **s, stream=stream)
    torch.cuda.synchronize()
    for (c, s), w in zip((a, b), want):
        for n in RESULTS:
            assert torch.equal(w[n], s[n]), n


def test_arguments_of_other_types_devices_and_shapes():
    c, s = _setup([5], [40])
    kv, batch, q, qi = s["kv"], s["batch"], s["q_in"], s["qi"]
    out, ws = s["out"], s["ws"]
    ok = lambda **kw: vx.chunk_attention(**{**dict(q=q, kv=kv, batch=batch, q_indptr=qi, sm_scale=0.1, out=out, workspace=ws[0]), **kw})  # noqa: E731
    ok()
    for kw in (dict(q=q.float()), dict(q=q.cpu()), dict(q=q[0]), dict(q=q[..., ::2]), dict(out=out.float()), dict(out=out[:, :4]), dict(out=out.cpu()),
               dict(q_indptr=qi.long()), dict(q_indptr=qi[:1]), dict(q_indptr=qi.cpu()), dict(q_lens=qi), dict(workspace=ws[0].cpu()),
               dict(lse=out), dict(lse=s["lse"][:, :3])):
        with pytest.raises((TypeError, ValueError)):
            ok(**kw)
    with pytest.raises(vx.VxError):
        ok(workspace=ws[0][:0])
    sp = lambda **kw: vx.sparse_chunk_attention(**{**dict(q=q, kv=kv, batch=batch, q_indptr=qi, sel_pages=s["sel"], sel_count=s["count"], sm_scale=0.1,  # noqa: E731
                                                            out=out, workspace=ws[2]), **kw})
    for kw in (dict(sel_pages=s["sel"].long()), dict(sel_pages=s["sel"][:, :1]), dict(sel_pages=s["sel"][0]), dict(sel_count=s["count"][:2])):
        with pytest.raises((TypeError, ValueError)):
            sp(**kw)
    sc = lambda **kw: vx.chunk_score_topk(**{**dict(q=q, kv=kv, batch=batch, q_indptr=qi, kind=vx.MEAN_DOT, mean=s["mean"], pages_budget=s["budget"],  # noqa: E731
                                                      n_sink=1, n_local=1, max_sel=8, sel_pages=s["sel"], sel_count=s["count"], workspace=ws[1]), **kw})
    for kw in (dict(mean=s["mean"].to(torch.bfloat16)), dict(mean=s["mean"][:-1]), dict(pages_budget=s["budget"].long()), dict(max_sel=7)):
        with pytest.raises((TypeError, ValueError)):
            sc(**kw)
    rw = lambda **kw: vx.rope_kv_write(**{**dict(kv=kv, rope=s["rope"], q=q, k_new=s["rows"][0], v_new=s["rows"][1], positions=s["pos"],  # noqa: E731
                                                   slots=s["slots"], q_out=s["q"]), **kw})
    for kw in (dict(positions=s["pos"].int()), dict(positions=s["pos"][:2]), dict(slots=s["slots"].int()), dict(q=None), dict(q_out=None), dict(k_new=s["rows"][0][:2]),
               dict(rope=vx.Rope(torch.zeros(32))), dict(rope=vx.Rope(torch.zeros(32, device=DEV, dtype=torch.float64))),
               dict(rope=vx.Rope(torch.zeros(32, device=DEV), torch.zeros(31, dtype=torch.int32, device=DEV), 2)), dict(q=q.float())):
        with pytest.raises((TypeError, ValueError)):
            rw(**kw)
    torch.cuda.synchronize()
