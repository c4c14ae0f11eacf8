"""Block selection of chunks where the queries of a group cancel: what is left of them selects, as in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests._chunk import Chunk

pytestmark = pytest.mark.gpu


def _select(c, mean, budget, n_sink, n_local, M):
    kv, batch, q, qi, ql = c.on_gpu()
    ws = torch.full((vx.chunk_workspace_size(vx.CHUNK_SCORE_TOPK, kv, batch, c.rows, c.Hq, M),), 255, dtype=torch.uint8, device="cuda")
    sel = torch.full((c.rows, c.H, M), -2, dtype=torch.int32, device="cuda")
    count = torch.full((c.rows,), -2, dtype=torch.int32, device="cuda")
    print(f"[select] H{c.H} g{c.g} D{c.D} rows {c.rows} M{M}", flush=True)
    vx.chunk_score_topk(q, kv, batch, qi, vx.MEAN_DOT, torch.from_numpy(mean).cuda(), torch.from_numpy(budget).cuda(), n_sink, n_local, M,
                        sel, count, ws, q_lens=ql)
    torch.cuda.synchronize()
    return sel.cpu().numpy(), count.cpu().numpy()


@pytest.mark.parametrize("new", [3, 40])
@pytest.mark.parametrize("D,g", [(128, 3), (64, 3), (128, 8)])
@pytest.mark.parametrize("large", [2 ** 8, 2 ** 12, 2 ** 16, 2 ** 22, 2 ** 26, 2 ** 30])
def test_heads_that_cancel(large, D, g, new):
    """Heads x, y, -x with x much larger than y; of eight, x, y1, x', y2, -x, y3, -x', y4."""
    c = Chunk([41, D, g, new], [8000, 2500], [new, new], 2 * g, 2, D)
    rng = np.random.default_rng([6, D, g, new])
    q = c.q.float().numpy().reshape(c.rows, 2, g, D)
    far = torch.from_numpy((rng.standard_normal((2,) + q[:, :, 0].shape) * large).astype(np.float32)).to(torch.bfloat16).float().numpy()
    if g == 3:
        q[:, :, 0], q[:, :, 2] = far[0], -far[0]
    else:
        q[:, :, 0], q[:, :, 4], q[:, :, 2], q[:, :, 6] = far[0], -far[0], far[1], -far[1]
    c.q = torch.from_numpy(q.reshape(c.rows, 2 * g, D)).to(torch.bfloat16)
    mean = (rng.standard_normal((c.P, 2, D)) * 0.25).astype(np.float32)
    budget = np.array([128, 60], np.int32)
    ref = c.select(mean, budget, 1, 2, 128)
    got = _select(c, mean, budget, 1, 2, 128)
    assert np.array_equal(got[1], ref[1])
    assert np.array_equal(got[0], ref[0]), int((got[0] != ref[0]).any(-1).sum())


def test_heads_that_cancel_select_as_a_decode_step():
    """Each token by itself as a request of its own for vx_page_score_topk."""
    c = Chunk([42], [8000], [20], 6, 2, 128)
    q = c.q.float().reshape(c.rows, 2, 3, 128)
    q[:, :, 2] = -65536.0 * q[:, :, 0]
    q[:, :, 0] *= 65536.0
    c.q = q.reshape(c.rows, 6, 128).to(torch.bfloat16)
    mean = (np.random.default_rng(12).standard_normal((c.P, 2, 128)) * 0.25).astype(np.float32)
    sel, count = _select(c, mean, np.array([64], np.int32), 1, 2, 64)
    kv, batch, qd, _, _ = c.on_gpu()
    B, per = c.rows, batch.page_indices.numel()
    one = vx.BatchSpec(torch.arange(0, B + 1, dtype=torch.int32, device="cuda") * per, batch.page_indices.repeat(B),
                       torch.arange(8001, 8001 + B, dtype=torch.int32, device="cuda"), per)
    ws = torch.empty(vx.workspace_size(vx.STAGE_SCORE_TOPK, kv, one, 6, 64), dtype=torch.uint8, device="cuda")
    s2, c2 = torch.empty((B, 2, 64), dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    vx.page_score_topk(qd, kv, one, vx.MEAN_DOT, torch.from_numpy(mean).cuda(), None, None,
                       torch.full((B,), 64, dtype=torch.int32, device="cuda"), 1, 2, 64, s2, c2, ws)
    torch.cuda.synchronize()
    assert np.array_equal(sel, s2.cpu().numpy()) and np.array_equal(count, c2.cpu().numpy())
