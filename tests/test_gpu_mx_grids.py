"""mxfp4 attention where its grids and its scratch are at their limits: the allocation-free call at batches
whose splits would pass its buffer, and requests ordered by count at every head layout."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests.test_gpu_mx_decode import _check, _launch, _problem

pytestmark = pytest.mark.gpu


def _shared(B, H, g, D, tokens, seed):
    """B requests on the same pages, every token of them selected."""
    p = _problem(1, H, g, D, 16, 16, [tokens], tokens // 16 + 1, seed, poison=False)
    n = len(p["perm"])
    q = torch.randn((B, H * g, D), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
    rep = lambda x: np.repeat(np.asarray(x), B, axis=0)  # noqa: E731
    return dict(p, B=B, lens=rep(p["lens"]), indptr=np.arange(B + 1) * n, perm=np.tile(p["perm"], B), sel=rep(p["sel"]),
                count=rep(p["count"]), q=q)


def _workspace(p):
    meta = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    cache = torch.from_numpy(p["kc"])
    return vx.workspace_size(vx.STAGE_DECODE, vx.PagedKV(cache, cache), vx.BatchSpec(meta(p["B"] + 1), meta(1), meta(p["B"]),
                                                                                    p["M"]), p["H"] * p["g"], p["M"])


@pytest.mark.parametrize("B,H,g,tokens", [(64, 8, 16, 8192), (32, 4, 16, 32761), (32, 8, 12, 32768)])
def test_without_allocation_at_many_heads(B, H, g, tokens):
    p = _shared(B, H, g, 128, tokens, B + g)
    assert _workspace(p) > 12 << 20                                # more than the static buffer
    got = _launch(p, noalloc=True)
    assert np.array_equal(got, _launch(p, noalloc=True))           # its counters are back at zero
    _check(dict(p, B=2), got)
    last = {n: p[n][-1:] for n in ("lens", "sel", "count", "q")}
    _check(dict(p, B=1, indptr=p["indptr"][-2:], **last), got[-1:])


@pytest.mark.parametrize("D,g", [(128, 2), (128, 9), (64, 16), (128, 16)])
def test_requests_ordered_by_count(D, g):
    """One workgroup per pair, more of them than three a CU, ragged counts."""
    lens = np.random.default_rng([D, g]).integers(1, 900, size=100)
    p = _problem(100, 8, g, D, 16, 16, lens, 33, [D, g, 1], poison=False)
    _check(p, _launch(p))
    _check(p, _launch(p, noalloc=True))
