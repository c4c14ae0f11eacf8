"""What lies in the cache behind a request's last token: it reaches no row, and the rows take the same way as over
zeros (the same bits: a tile done again row by row rounds otherwise)."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests._chunk import MLA_D, Chunk

pytestmark = pytest.mark.gpu
KINDS = ["bf16", "fp8_e4m3", "fp8_e5m2", "mxfp4"]
CODES = {"fp8_e4m3": {"nan": 0x7f, "large": 0x7e}, "fp8_e5m2": {"nan": 0x7f, "inf": 0x7c}}


def _behind(c, what):
    """The caches with `what` in every place of the last pages that no token has: slots of bytes or values."""
    k, v = c.k.clone(), None if c.v is None else c.v.clone()
    for x in (k, v):
        if x is None:
            continue
        for i, L in enumerate(c.lens):
            page, at = c.indices[c.indptr[i + 1] - 1], (int(L) - 1) % c.ps + 1
            if c.kind == "bf16":
                x[page, :, at:] = what
            elif c.kind != "mxfp4":
                x.view(torch.uint8)[page, :, at:] = what
            else:
                D, ps = c.D, c.ps                               # the scales of those places
                scales = x[page].reshape(c.H, -1)[:, ps * D // 2:]
                if x is k:
                    scales.view(c.H, ps, D // 32)[:, at:] = what
                else:
                    for t in range(at, ps):
                        scales.view(c.H, ps // 4, D // 32, 4)[:, t // 4, :, t % 4] = what
    return k, v


def _run(c, k, v, sel=None, count=None, window=0, causal=True):
    kv, batch, q, qi, ql = c.on_gpu()
    kv = vx.PagedKV(k.cuda(), None if v is None else v.cuda(), c.Dv, k_scale=c.scale, v_scale=c.scale, block_size=c.block)
    stage, M = (vx.CHUNK_ATTENTION, 1) if sel is None else (vx.CHUNK_SPARSE, sel.shape[2])
    ws = torch.full((vx.chunk_workspace_size(stage, kv, batch, c.rows, c.Hq, M),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((c.rows, c.Hq, c.Dv), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.rows, c.Hq), 7.0, dtype=torch.float32, device="cuda")
    print(f"[stale] {c.kind} H{c.H} g{c.g} D{c.D} ps{c.ps}/{c.block} lens {list(c.lens)[:4]} new {list(c.new)[:4]} M{M}", flush=True)
    if sel is None:
        vx.chunk_attention(q, kv, batch, qi, c.sm_scale, out, ws, lse=lse, window=window, causal=causal)
    else:
        vx.sparse_chunk_attention(q, kv, batch, qi, torch.from_numpy(sel).cuda(), torch.from_numpy(count).cuda(), c.sm_scale, out, ws, lse=lse)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu()


def _values(kind):
    if kind == "bf16":
        return [float("nan"), float("inf"), float("-inf")]
    return list(CODES[kind].values()) if kind in CODES else [255, 254]


def _same_as_zeros(c, *args, **kw):
    want = _run(c, *_behind(c, 0), *args, **kw)
    assert bool(torch.isfinite(want[0]).all())
    for what in _values(c.kind):
        got = _run(c, *_behind(c, what), *args, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), what


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("ps,block", [(64, 0), (64, 32), (32, 0), (16, 0)])
@pytest.mark.parametrize("new,D", [(3, 64), (40, 128)])
@pytest.mark.parametrize("rest", [1, 7, 15, 17, 33])
def test_listed_blocks(kind, ps, block, new, D, rest):
    """The last block holds whole runs of 16 places without a token."""
    L = [3 * 64 + rest, 64 + rest]
    c = Chunk([51, ps, new, rest], [x - new for x in L], [new, new], 8, 2, D, kv=kind, ps=ps, block=block)
    bs, M = block or ps, 20
    sel, count = np.full((c.rows, 2, M), -1, np.int32), np.zeros(c.rows, np.int32)
    for row, _, p in c.tokens():
        count[row] = n = p // bs + 1
        sel[row, :, :n] = np.arange(n)
    _same_as_zeros(c, sel, count)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("ps", [64, 16])
@pytest.mark.parametrize("new,D", [(3, 64), (40, 128), (150, 128)])
@pytest.mark.parametrize("rest", [1, 15])
def test_dense(kind, ps, new, D, rest):
    c = Chunk([52, ps, new, rest], [192 + rest, 64 + rest], [new, new], 8, 2, D, kv=kind, ps=ps)
    _same_as_zeros(c)
    _same_as_zeros(c, window=37)
    _same_as_zeros(c, causal=False)


@pytest.mark.parametrize("kind", KINDS[:3])
@pytest.mark.parametrize("new", [3, 70])
def test_latent(kind, new):
    c = Chunk([53, new], [130, 64], [new, new + 5], 16, 1, MLA_D, ps=64, kv=kind, sigma=0.5)
    _same_as_zeros(c)
    _same_as_zeros(c, causal=False)
