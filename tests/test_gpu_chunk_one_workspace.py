"""One workspace for all the chunks of a prompt and the drafted tokens behind it, sized once for the largest."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests._chunk import MLA_D, Chunk

pytestmark = pytest.mark.gpu
SHORT = [150, 37, 4, 1]                                        # chunks behind the first one, whose lists are cut into parts


def _prompt(kind, latent, first):
    """A prompt whose first chunk needs no parts; every 16th of its rows is compared, and all later ones."""
    lengths = [first] + SHORT
    c = Chunk([71, latent], [600], [sum(lengths)], 16 if latent else 32, 1 if latent else 8, MLA_D if latent else 128, ps=64 if latent else 16,
              kv=kind, sigma=0.5)
    every = list(c.tokens())
    c.tokens = lambda: [t for t in every if t[0] >= first or t[0] % 16 == 0]
    kv, batch, q, _, _ = c.on_gpu()
    return c, lengths, kv, batch, q


def _close(c, out, ref, tol):
    there = ~np.isnan(ref[:, 0, 0])
    return (np.abs(out.double().cpu().numpy() - ref)[there] <= tol[there]).all()


@pytest.mark.parametrize("kind,latent", [("bf16", False), ("mxfp4", False), ("bf16", True), ("fp8_e4m3", True)])
def test_attention(kind, latent):
    c, lengths, kv, batch, q = _prompt(kind, latent, 1600 if latent else 1100)
    ref, tol, _, _ = c.attend()
    ws = torch.full((vx.chunk_workspace_size(vx.CHUNK_ATTENTION, kv, batch, lengths[0], c.Hq),), 255, dtype=torch.uint8, device="cuda")
    at, L = 0, int(c.before[0])
    for n in lengths:
        L += n
        batch.seq_lens.fill_(L)
        out = torch.empty((n, c.Hq, c.Dv), dtype=torch.bfloat16, device="cuda")
        print(f"[one workspace] {kind} {n} of {L}", flush=True)
        vx.chunk_attention(q[at:at + n], kv, batch, torch.tensor([0, n], dtype=torch.int32, device="cuda"), c.sm_scale, out, ws)
        assert _close(c, out, ref[at:at + n], tol[at:at + n]), n
        at += n


def test_selection_and_its_attention():
    c, lengths, kv, batch, q = _prompt("bf16", False, 1100)
    M = 40
    mean = (np.random.default_rng(3).standard_normal((c.P, 8, 128)) * 0.25).astype(np.float32)
    pages, count = c.select(mean, [M], 1, 2, M)
    ref, tol, _, _ = c.attend(sel=lambda row, h: set(pages[row, h, : count[row]].tolist()))
    md, budget = torch.from_numpy(mean).cuda(), torch.tensor([M], dtype=torch.int32, device="cuda")
    ws = torch.full((max(vx.chunk_workspace_size(s, kv, batch, lengths[0], c.Hq, M) for s in (vx.CHUNK_SCORE_TOPK, vx.CHUNK_SPARSE)),), 255,
                    dtype=torch.uint8, device="cuda")
    at, L = 0, int(c.before[0])
    for n in lengths:
        L += n
        batch.seq_lens.fill_(L)
        qi = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        sel, cnt = torch.empty((n, 8, M), dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
        out = torch.empty((n, c.Hq, c.Dv), dtype=torch.bfloat16, device="cuda")
        print(f"[one workspace] lists {n} of {L}", flush=True)
        vx.chunk_score_topk(q[at:at + n], kv, batch, qi, vx.MEAN_DOT, md, budget, 1, 2, M, sel, cnt, ws)
        vx.sparse_chunk_attention(q[at:at + n], kv, batch, qi, sel, cnt, c.sm_scale, out, ws)
        there = count[at:at + n] >= 0
        assert np.array_equal(sel.cpu().numpy()[there], pages[at:at + n][there]) and np.array_equal(cnt.cpu().numpy()[there], count[at:at + n][there])
        assert _close(c, out, ref[at:at + n], tol[at:at + n]), n
        at += n
