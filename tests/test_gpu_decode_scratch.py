"""One decode scratch buffer used by batches of other sizes and geometries in turn (the caller's
workspace, and the static one of the allocation-free entry point): the split counters keep their place,
so no batch's partials are taken for another's counters."""
import numpy as np
import pytest
import torch

from oracle import oracle as O
from paper_2606_06453_amd import vx
from tests._compare import OUT_ATOL, max_abs_err
from tests._problems import random_problem

pytestmark = pytest.mark.gpu


def _call(seed, lens, H, D, ps, cnt):
    mla = D == 576
    pb = random_problem(seed, lens, Hq=16 if mla else 2 * H, H=H, D=D, ps=ps, Dv=512 if mla else None, alias_v=mla)
    P, M = -(-np.asarray(lens) // ps), int(max(cnt))
    rng = np.random.default_rng(seed)
    sel = np.full((len(lens), H, M), -1, np.int32)
    for i in range(len(lens)):
        for h in range(H):
            sel[i, h, : cnt[i]] = np.sort(rng.choice(int(P[i]), size=int(cnt[i]), replace=False))
    return pb, P, sel, np.asarray(cnt, np.int32), M


def _run(call, ws):
    pb, P, sel, cnt, M = call
    gpu = lambda x: torch.from_numpy(np.asarray(x)).cuda()  # noqa: E731
    kv = vx.PagedKV(pb.k.cuda(), None if pb.v is None else pb.v.cuda(), pb.head_dim_v)
    batch = vx.BatchSpec(gpu(pb.page_indptr), gpu(pb.page_indices), gpu(pb.seq_lens), int(P.max()))
    out = torch.full((pb.batch, pb.q.shape[1], pb.head_dim_v), float("nan"), dtype=torch.bfloat16, device="cuda")
    args = (pb.q.cuda(), kv, batch, gpu(sel), gpu(cnt), M, 0.1, out)
    if ws is None:
        vx.sparse_paged_decode_noalloc(*args)
    else:
        assert vx.workspace_size(vx.STAGE_DECODE, kv, batch, pb.q.shape[1], M) <= ws.numel()
        vx.sparse_paged_decode(*args, ws)
    torch.cuda.synchronize()
    ref = O.attend(pb.q, pb.k, pb.v, pb.page_size, pb.page_indptr, pb.page_indices, pb.seq_lens, sel, cnt, 0.1,
                   pb.head_dim_v)
    assert max_abs_err(out, ref) <= OUT_ATOL


@pytest.mark.parametrize("workspace", [True, False])
def test_batches_take_turns_on_one_buffer(workspace):
    ws = torch.zeros(12 << 20, dtype=torch.uint8, device="cuda") if workspace else None
    one = _call(1, [16 * 300], 1, 128, 16, [290])                          # one pair, many splits
    many = _call(2, [16 * 30 + n for n in range(60)], 8, 128, 16, [12 + n % 19 for n in range(60)])
    latent = _call(3, [64 * 20] * 5, 1, 576, 64, [16] * 5)
    full = _call(4, [16 * 5] * 300, 2, 64, 16, [5] * 300)                  # not split
    for c in (one, many, latent, many, full, one, many):
        _run(c, ws)
