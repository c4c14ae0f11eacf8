"""Every attended token counts once in the chunk calls: equal scores and values that mark a few tokens a channel, so that
a token left out, taken twice or taken from beyond a row's range changes an output by more than its rounding."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests._chunk import MLA_D, Chunk

pytestmark = pytest.mark.gpu
KINDS = ["bf16", "fp8_e4m3", "fp8_e5m2", "mxfp4"]
MARK = 61                                                      # tokens of a channel: odd, so that marks and runs drift apart


def _marked(c, rnd):
    """A cache whose token t has `one` in channel t // MARK - rnd * Dv and zeros in the others.  The value of `one`."""
    one = 64 * c.scale if c.kind.startswith("fp8") else 1.0
    x = torch.zeros((c.P, c.H, c.ps, c.D), dtype=torch.float32)
    for i, L in enumerate(c.lens):
        t = np.arange(int(L))
        ch = t // MARK - rnd * c.Dv
        t, ch = t[(ch >= 0) & (ch < c.Dv)], ch[(ch >= 0) & (ch < c.Dv)]
        x[torch.from_numpy(c.indices[c.indptr[i] + t // c.ps]).long(), :, torch.from_numpy(t % c.ps).long(), torch.from_numpy(ch).long()] = one
    x = x.to(torch.bfloat16) if not c.kind.startswith("fp8") else x     # codes of 64 exactly
    cache, c64 = c._cache(x, "k" if c.D == MLA_D else "v")
    if c.D == MLA_D:
        c.k = cache
    else:
        c.v = cache
    assert set(np.unique(c64[..., : c.Dv])) <= {0.0, one}
    return one


def _run(c, sel, count, window, causal):
    kv, batch, q, qi, ql = c.on_gpu()
    stage, M = (vx.CHUNK_ATTENTION, 1) if sel is None else (vx.CHUNK_SPARSE, sel.shape[2])
    ws = torch.full((vx.chunk_workspace_size(stage, kv, batch, c.rows, c.Hq, M),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((c.rows, c.Hq, c.Dv), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.rows, c.Hq), 7.0, dtype=torch.float32, device="cuda")
    if sel is None:
        vx.chunk_attention(q, kv, batch, qi, c.sm_scale, out, ws, lse=lse, window=window, causal=causal)
    else:
        vx.sparse_chunk_attention(q, kv, batch, qi, torch.from_numpy(sel).cuda(), torch.from_numpy(count).cuda(), c.sm_scale, out, ws, lse=lse)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def _check(c, sel=None, count=None, window=0, causal=True):
    """Weights are all 2^-8 (the first score sets the reference 2^8 past it) and sums of them exact: an output is its channel's
    count times `one` over the number of tokens, rounded to bf16 (half a step 2^-8) after a product and a quotient in fp32
    (2^-21).  A token of MARK is 1 / 61 of it.  The log-sum-exp is the number's logarithm within 2^-21."""
    c.q.zero_()
    bs = c.block or c.ps
    print(f"[counts] {c.kind} H{c.H} g{c.g} D{c.D} ps{c.ps}/{c.block} lens {list(c.lens)[:4]} new {list(c.new)[:4]} w{window} {causal}", flush=True)
    for rnd in range(-(-int(c.lens.max()) // (MARK * c.Dv))):
        one = _marked(c, rnd)
        out, lse = _run(c, sel, count, window, causal)
        for row, i, p in c.tokens():
            L = int(c.lens[i])
            t = np.arange(max(0, p - window + 1) if window else 0, p + 1 if causal else L)
            for h in range(c.H):
                mine = t if sel is None else t[np.isin(t // bs, sel[row, h, : count[row]])]
                ch = mine // MARK - rnd * c.Dv
                want = np.bincount(ch[(ch >= 0) & (ch < c.Dv)], minlength=c.Dv) * one / len(mine)
                got = out[row, h * c.g:(h + 1) * c.g]
                assert (np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -21) * want).all(), (row, h, np.argwhere(np.abs(got - want) > 2.0 ** -8 * want)[:4])
                n = np.log(len(mine))
                assert (np.abs(lse[row, h * c.g:(h + 1) * c.g] - n) <= 2.0 ** -21 * (1 + n)).all(), (row, h)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,new,Hq", [(64, 1, 8), (128, 4, 8), (128, 2, 2), (64, 40, 4)])
def test_long_lists_in_parts(kind, D, new, Hq):
    c = Chunk([81, D, new], [20000, 3, 8191], [new] * 3, Hq, 2, D, ps=64, kv=kind)
    _check(c)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("window,causal", [(1000, True), (4099, True), (700, False), (0, False)])
def test_windows(kind, window, causal):
    c = Chunk([82, window], [6000, 900], [3, 70], 8, 2, 128, kv=kind)
    _check(c, window=window, causal=causal)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,before,new", [(128, [4000, 0, 17], [150, 65, 128]), (64, [2500], [300])])
def test_prompts(kind, D, before, new):
    c = Chunk([83, D], before, new, 8, 2, D, ps=32, kv=kind)
    _check(c)


@pytest.mark.parametrize("kind", KINDS[:3])
@pytest.mark.parametrize("before,new", [([20000, 1300], [3, 1]), ([3000, 70], [40, 130])])
def test_latent(kind, before, new):
    c = Chunk([84, len(before)], before, new, 16, 1, MLA_D, ps=64, kv=kind)
    _check(c)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("ps,block", [(16, 0), (64, 32), (64, 0)])
@pytest.mark.parametrize("new", [2, 30])
def test_listed_blocks_in_parts(kind, ps, block, new):
    c = Chunk([85, ps, new], [12000, 777], [new] * 2, 8, 2, 128, ps=ps, kv=kind, block=block)
    bs = block or ps
    rng = np.random.default_rng(9)
    M = 12100 // bs
    sel, count = np.full((c.rows, 2, M), -1, np.int32), np.zeros(c.rows, np.int32)
    for row, _, p in c.tokens():
        nb = p // bs + 1
        count[row] = n = max(1, int(nb * (0.2 + 0.8 * rng.random())))
        for h in range(2):
            sel[row, h, :n] = rng.permutation(nb)[:n]
    _check(c, sel, count)
