"""One workspace for calls of any number of rows up to the one that it is made for (no GPU needed)."""
import ctypes
import re

import pytest

from paper_2606_06453_amd import vx
from tests.test_chunk_refusals import _at, _batch, _kv, _msg

MLA = dict(D=576, Dv=512, H=1, v=None)


def _size(stage, kv, batch, pages, n, Hq, M):
    out, b = ctypes.c_size_t(), _batch(batch=batch, pages=pages)
    assert vx.lib().vx_chunk_workspace_size(stage, ctypes.byref(kv), ctypes.byref(b), n, Hq, M, ctypes.byref(out)) == 0, _msg()
    return out.value


def _need(stage, kv, batch, pages, n, Hq, M):
    """What a call asks for when it gets none."""
    L, b = vx.lib(), _batch(batch=batch, pages=pages)
    D = kv.head_dim_qk
    head = (_at(7), Hq * D, D, Hq, ctypes.byref(kv), ctypes.byref(b), ctypes.byref(vx._Chunk(_at(6), None, n)))
    if stage == vx.CHUNK_ATTENTION:
        st = L.vx_chunk_attention(*head, 0, 1, 0.1, _at(8), None, None, 0, None)
    elif stage == vx.CHUNK_SCORE_TOPK:
        st = L.vx_chunk_score_topk(*head, 0, _at(10), _at(12), 0, 1, M, _at(13), _at(14), None, 0, None)
    else:
        st = L.vx_sparse_chunk_attention(*head, _at(13), _at(14), M, 0.1, _at(8), None, None, 0, None)
    assert st == 3, _msg()
    return int(re.search(r"needs a workspace of (\d+) bytes", _msg()).group(1))


GEOMETRIES = [(vx.KV_BF16, dict(), 32), (vx.KV_BF16, dict(H=16, D=64), 16), (vx.KV_FP8_E4M3, dict(H=2), 10), (vx.KV_MXFP4, dict(H=1), 16),
              (vx.KV_MXFP4, dict(H=4, D=64, ps=64, block=16), 28), (vx.KV_BF16, MLA, 16), (vx.KV_FP8_E5M2, MLA, 16)]
ROWS = sorted({1, 2, 3, 5, 16, 17, 33} | {x + d for x in (64, 96, 128, 256, 384, 512, 1024, 1536, 2048, 4096, 8192) for d in (-1, 0, 1)})


@pytest.mark.parametrize("stage", [vx.CHUNK_ATTENTION, vx.CHUNK_SCORE_TOPK, vx.CHUNK_SPARSE])
@pytest.mark.parametrize("dtype,geo,Hq", GEOMETRIES)
@pytest.mark.parametrize("pages", [1, 40, 2048])
def test_enough_for_fewer(stage, dtype, geo, Hq, pages):
    """Fewer rows, fewer requests, shorter lists and shorter page lists need no more; more rows are told no less."""
    if stage != vx.CHUNK_ATTENTION and geo is MLA:
        pytest.skip("selections need the GQA geometry")
    kv = _kv(dtype, **geo)
    for batch in (1, 3, 48, 200):
        told = [_size(stage, kv, batch, pages, n, Hq, 64) for n in ROWS]
        assert told == sorted(told)
        for k in range(len(ROWS)):
            for b in {1, max(1, batch // 3), batch}:
                for M, p in ((64, pages), (1, pages), (64, max(1, pages // 3))):
                    need = _need(stage, kv, b, p, ROWS[k], Hq, M)
                    assert need <= told[k], (batch, ROWS[k], b, M, p, need, told[k])


def test_of_one_long_request():
    """The sizes that a prompt's last rows and drafted tokens behind it need."""
    kv = _kv()
    told = _size(vx.CHUNK_ATTENTION, kv, 1, 2048, 8192, 32, 1)
    needs = [_need(vx.CHUNK_ATTENTION, kv, 1, 2048, n, 32, 1) for n in range(1, 8193)]
    assert max(needs) <= told <= 2 * max(needs)
