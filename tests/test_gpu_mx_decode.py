"""Attention over the selected blocks of an mxfp4 cache against fp64: head layouts, block sizes, lengths
from one token on, partial last blocks, empty selections, splits, poisoned masked places, repeated and
unordered pages.  Tolerances are derived in tests/_mx.py (attend_tolerance)."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests import _mx

pytestmark = pytest.mark.gpu


def _problem(B, H, g, D, ps, bs, lens, budget, seed, spread=1.0, poison=True, shared=False):
    """A ragged batch on scattered pages; every byte that no valid token owns is NaN-scaled garbage."""
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens)
    pages = -(-lens // ps)
    total = int(pages.sum())
    indptr = np.concatenate([[0], np.cumsum(pages)])
    perm = rng.permutation(total + 2)[:total]
    k, v = rng.normal(size=(total + 2, H, ps, D)) * spread, rng.normal(size=(total + 2, H, ps, D))
    k, v = (torch.from_numpy(x).to(torch.bfloat16).double().numpy() for x in (k, v))
    kc, vc = _mx.pack(k, "k"), _mx.pack(v, "v")
    if poison:
        owned = np.zeros((total + 2, ps), bool)
        for i in range(B):
            for j in range(pages[i]):
                owned[perm[indptr[i] + j], : max(0, min(ps, lens[i] - j * ps))] = True
        for cache, which in ((kc, "k"), (vc, "v")):
            at, _, sc = _mx.places(ps, D, which)
            flat = cache.reshape(total + 2, H, -1)
            for p, t in zip(*np.nonzero(~owned)):
                flat[p][:, at[t]] = 0x7F
                flat[p][:, sc[t]] = 255
    r = ps // bs
    blocks = -(-lens // bs)
    count = np.minimum(blocks, budget)
    M = max(1, int(count.max()))
    sel = np.full((B, H, M), -1, np.int32)
    for i in range(B):
        for h in range(H):
            if count[i]:
                pick = rng.choice(blocks[i], size=count[i], replace=False)
                if blocks[i] - 1 not in pick:
                    pick[0] = blocks[i] - 1                       # the partial one
                sel[i, h, : count[i]] = np.sort(pick)
    q = torch.from_numpy(rng.normal(size=(B, H * g, D))).to(torch.bfloat16)
    return dict(B=B, H=H, g=g, D=D, ps=ps, bs=bs, r=r, lens=lens, indptr=indptr, perm=perm, kc=kc, vc=vc, sel=sel,
                count=count, M=M, q=q, scale=D ** -0.5)


def _launch(p, noalloc=False, ws=None, stream=None):
    gpu = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()  # noqa: E731
    kv = vx.PagedKV(torch.from_numpy(p["kc"]).cuda(), torch.from_numpy(p["vc"]).cuda(),
                    block_size=p["bs"] if p["bs"] != p["ps"] else 0)
    batch = vx.BatchSpec(gpu(p["indptr"]), gpu(p["perm"] if len(p["perm"]) else [0]), gpu(p["lens"]),
                         max(1, int((-(-p["lens"] // p["ps"])).max())))
    out = torch.full((p["B"], p["H"] * p["g"], p["D"]), 7.0, dtype=torch.bfloat16, device="cuda")
    args = (p["q"].cuda(), kv, batch, gpu(p["sel"]), gpu(p["count"]), p["M"], p["scale"], out)
    if noalloc:
        vx.sparse_paged_decode_noalloc(*args)
    else:
        n = vx.workspace_size(vx.STAGE_DECODE, kv, batch, p["H"] * p["g"], p["M"])
        ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
        vx.sparse_paged_decode(*args, ws)
        first = out.clone()
        vx.sparse_paged_decode(*args, ws)                          # the counters are back at zero
        torch.cuda.synchronize()
        assert torch.equal(first.view(torch.int16), out.view(torch.int16))
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


def _check(p, got):
    k, v = _mx.unpack(p["kc"], "k"), _mx.unpack(p["vc"], "v")
    q = p["q"].double().numpy()
    for i in range(p["B"]):
        for h in range(p["H"]):
            heads = slice(h * p["g"], (h + 1) * p["g"])
            js = [j for j in p["sel"][i, h, : p["count"][i]] if 0 <= j < -(-p["lens"][i] // p["bs"])]
            pos = np.concatenate([np.arange(j * p["bs"], min((j + 1) * p["bs"], p["lens"][i])) for j in js] or [[]])
            pos = pos.astype(int)
            if not len(pos):
                assert (got[i, heads] == 0).all()
                continue
            pg = p["perm"][p["indptr"][i] + pos // p["ps"]]
            kk, vv = k[pg, h, pos % p["ps"]], v[pg, h, pos % p["ps"]]
            ref, absv, qk = _mx.attend(q[i, heads], kk, vv, p["scale"])
            tol = _mx.attend_tolerance(ref, absv, qk, p["scale"], p["D"], len(pos))
            err = np.abs(got[i, heads] - ref)
            assert (err <= tol).all(), (i, h, float((err - tol).max()), float(err.max()))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,g", [(1, 1), (8, 4), (2, 16), (4, 3), (16, 8), (1, 9)])
@pytest.mark.parametrize("ps,bs", [(16, 16), (32, 16), (64, 32), (64, 64), (32, 32)])
def test_head_layouts_and_blocks(D, H, g, ps, bs):
    lens = [1, 15, 16, 17, 5 * ps + 3, 0, 12 * ps]
    p = _problem(len(lens), H, g, D, ps, bs, lens, 7, [D, H, g, ps, bs])
    _check(p, _launch(p))


@pytest.mark.parametrize("n", list(range(1, 36)) + [47, 63, 64, 65])
def test_every_short_length(n):
    p = _problem(2, 2, 4, 128, 64, 64, [n, n + 1], 9, n)
    _check(p, _launch(p))


@pytest.mark.parametrize("B,budget,lens", [(1, 4000, 16001), (2, 700, 16001), (40, 60, 2000), (100, 33, 900), (300, 17, 400)])
@pytest.mark.parametrize("noalloc", [False, True])
def test_splits_and_full_grids(B, budget, lens, noalloc):
    """One request over many workgroups, and grids with one workgroup per pair (ordered by count)."""
    rng = np.random.default_rng(B)
    n = rng.integers(1, lens + 1, size=B) if B > 2 else [lens] * B
    p = _problem(B, 8 if B > 2 else 1, 2, 64 if B > 100 else 128, 16, 16, n, budget, B, poison=B < 3)
    _check(p, _launch(p, noalloc))


def test_large_scores_and_one_dominant_key():
    """Scores of a few hundred: the running maximum moves, weights underflow."""
    for spread in (30.0, 1e-20, 300.0):
        p = _problem(3, 2, 4, 128, 16, 16, [500, 77, 33], 40, int(spread) + 1, spread=spread)
        _check(p, _launch(p))


def test_scales_far_apart():
    """Groups whose scales span the format: tiny and huge values of V beside each other."""
    p = _problem(2, 1, 4, 128, 16, 16, [200, 90], 20, 77, poison=False)
    x = _mx.unpack(p["vc"], "v") * np.exp2(np.random.default_rng(1).integers(-100, 60, size=p["vc"].shape[:3] + (1,)))
    p["vc"] = _mx.pack(x, "v")
    _check(p, _launch(p))


def test_a_nan_group_reaches_only_its_readers():
    p = _problem(2, 2, 2, 128, 16, 16, [40, 40], 3, 5)
    page = p["perm"][p["indptr"][0] + 1]
    _, _, sc = _mx.places(16, 128, "v")
    p["vc"].reshape(len(p["vc"]), 2, -1)[page, 1, sc[3, 64]] = 255    # request 0, KV head 1, token 19, channels 64..95
    got = _launch(p)
    assert np.isnan(got[0, 2:, 64:96]).all()
    got[0, 2:, 64:96] = 0
    assert np.isfinite(got).all()


def test_selections_out_of_order_repeated_and_foreign():
    p = _problem(2, 2, 2, 64, 16, 16, [300, 100], 6, 9)
    p["sel"][0, 0, :6] = [18, 2, 2, 9, 0, 5]
    p["sel"][1, 1, :6] = [99, 3, -1, 6, 0, 2 ** 31 - 1]
    p["count"][:] = [6, 6]
    got = _launch(p)
    _check(p, got)


def test_empty_selections():
    p = _problem(3, 2, 2, 128, 16, 16, [30, 40, 50], 2, 4)
    p["count"][1] = 0
    _check(p, _launch(p))


def test_caches_past_four_gigabytes():
    """Pages whose byte offsets pass 32 bits, against the same pages in a small cache."""
    H, D, ps = 8, 128, 64
    p = _problem(2, H, 4, D, ps, ps, [400, 130], 6, 3)
    P = (1 << 32) // (H * ps * D * 17 // 32) + 50
    small = _launch(p)
    gpu = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()  # noqa: E731
    k, v = vx.mxfp4_cache(P, H, ps, D), vx.mxfp4_cache(P, H, ps, D)
    n = len(p["kc"])
    far = np.where(np.arange(n) % 2 == 0, P - 1 - np.arange(n), np.arange(n))
    k[torch.from_numpy(far).cuda()], v[torch.from_numpy(far).cuda()] = (torch.from_numpy(p[x]).cuda() for x in ("kc", "vc"))
    kv = vx.PagedKV(k, v)
    batch = vx.BatchSpec(gpu(p["indptr"]), gpu(far[p["perm"]]), gpu(p["lens"]), 7)
    out = torch.zeros((2, H * 4, D), dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(vx.workspace_size(vx.STAGE_DECODE, kv, batch, H * 4, p["M"]), dtype=torch.uint8, device="cuda")
    vx.sparse_paged_decode(p["q"].cuda(), kv, batch, gpu(p["sel"]), gpu(p["count"]), p["M"], p["scale"], out, ws)
    torch.cuda.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), small)


def test_scores_far_below_zero():
    """Every score -1e34: the weights are equal, and the output is the mean of V."""
    p = _problem(1, 1, 4, 128, 16, 16, [75], 9, 6)
    p["q"][:] = 1.0
    p["kc"] = _mx.pack(np.full(p["kc"].shape[:3] + (128,), -(2.0 ** 106)), "k")
    got = _launch(p)
    v = _mx.unpack(p["vc"], "v")[p["perm"]].reshape(-1, 128)[:75]
    want = v.mean(0)
    # equal scores leave weights of exactly 1; 75 additions in fp32, a division, bf16
    tol = 2.0 ** -8 * np.abs(want) + 80 * 2.0 ** -23 * np.abs(v).mean(0)
    assert (np.abs(got[0] - want) <= tol).all()
