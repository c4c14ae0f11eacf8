"""The weights of the chunk calls' second product, against 64 bits: as exact as those of the decode step."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests._chunk import MLA_D, Chunk

pytestmark = pytest.mark.gpu


def _bounds(c, **kw):
    """Chunk.attend's result and a bound for weights of two bf16 parts.

    A weight's first part leaves at most half a step 2^-8 of it, and the second half a step of that: 2^-16 where
    Chunk.attend allows 2^-8.  Its other terms stand: the scores' error in the numerator and in the sum (from its bound of the
    log-sum-exp), n additions of 2^-23, and the result's rounding to bf16, half a step 2^-8."""
    ref, tol, lse, ltol = c.attend(**kw)
    err = (ltol - 2.0 ** -21 * (1 + np.abs(lse)))[..., None]
    wide = 2 * err + 2.0 ** -8
    absv = (tol - 1e-30 - 2.0 ** -8 * np.abs(ref)) / (wide * (1 + 2.0 ** -8))   # sum of |w v|
    delta = 2 * err + 2.0 ** -16
    return ref, 2.0 ** -8 * (np.abs(ref) + delta * absv) + delta * absv + 1e-30


def _run(c, sel=None, count=None):
    kv, batch, q, qi, ql = c.on_gpu()
    stage, M = (vx.CHUNK_ATTENTION, 1) if sel is None else (vx.CHUNK_SPARSE, sel.shape[2])
    ws = torch.full((vx.chunk_workspace_size(stage, kv, batch, c.rows, c.Hq, M),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((c.rows, c.Hq, c.Dv), 7.0, dtype=torch.bfloat16, device="cuda")
    print(f"[weights] {c.kind} H{c.H} g{c.g} D{c.D} lens {list(c.lens)[:4]} new {list(c.new)[:4]} M{M}", flush=True)
    if sel is None:
        vx.chunk_attention(q, kv, batch, qi, c.sm_scale, out, ws)
    else:
        vx.sparse_chunk_attention(q, kv, batch, qi, torch.from_numpy(sel).cuda(), torch.from_numpy(count).cuda(), c.sm_scale, out, ws)
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


def _within(got, bounds):
    ref, tol = bounds
    over = np.abs(got - ref) / tol
    assert (over <= 1).all(), (over.max(), (over > 1).mean())


# few rows (narrow tiles, or wide ones of one operand), prompts (two operands), lists in parts
CASES = [([300, 40], [2, 3], 8, 2), ([0, 77], [200, 90], 8, 2), ([5000], [2], 8, 2), ([600], [9], 16, 1)]


@pytest.mark.parametrize("kind", ["bf16", "fp8_e4m3", "fp8_e5m2", "mxfp4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("before,new,Hq,H", CASES)
def test_dense(kind, D, before, new, Hq, H):
    c = Chunk([31, D, len(before)], before, new, Hq, H, D, kv=kind)
    _within(_run(c), _bounds(c))


@pytest.mark.parametrize("kind", ["bf16", "fp8_e4m3", "fp8_e5m2"])
@pytest.mark.parametrize("before,new", [([300, 40], [2, 33]), ([3000], [3])])
def test_latent(kind, before, new):
    c = Chunk([32, len(before)], before, new, 16, 1, MLA_D, ps=64, kv=kind, sigma=0.5)
    _within(_run(c), _bounds(c))


@pytest.mark.parametrize("kind", ["bf16", "fp8_e4m3", "fp8_e5m2", "mxfp4"])
@pytest.mark.parametrize("before,new", [([700], [3]), ([500, 30], [40, 21])])
def test_listed_blocks(kind, before, new):
    c = Chunk([33, len(before)], before, new, 8, 2, 128, kv=kind)
    rng = np.random.default_rng(5)
    M = 12
    sel, count = np.full((c.rows, 2, M), -1, np.int32), np.zeros(c.rows, np.int32)
    for row, _, p in c.tokens():
        nb = p // 16 + 1
        count[row] = n = min(M, nb)
        for h in range(2):
            sel[row, h, :n] = np.sort(rng.permutation(nb)[:n])
    _within(_run(c, sel, count), _bounds(c, sel=lambda row, h: set(sel[row, h, : count[row]].tolist())))


def test_a_chunk_of_one_is_as_exact_as_a_decode_step():
    """The same token by the chunk call and by the decode call over every page: errors of the same size."""
    c = Chunk([34], [1500], [1], 32, 8, 128)
    chunk = _run(c)
    kv, batch, q, _, _ = c.on_gpu()
    M = int(c.max_pages)
    sel = torch.arange(M, dtype=torch.int32, device="cuda").repeat(1, 8, 1).contiguous()
    count = torch.full((1,), M, dtype=torch.int32, device="cuda")
    ws = torch.zeros(vx.workspace_size(vx.STAGE_DECODE, kv, batch, 32, M), dtype=torch.uint8, device="cuda")   # its counters start at zero
    out = torch.empty((1, 32, 128), dtype=torch.bfloat16, device="cuda")
    vx.sparse_paged_decode(q, kv, batch, sel, count, M, c.sm_scale, out, ws)
    torch.cuda.synchronize()
    ref, tol = _bounds(c)
    _within(chunk, (ref, tol))
    _within(out.double().cpu().numpy(), (ref, tol))
