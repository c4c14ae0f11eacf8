"""Rows by slot where a dimension of the rows has one entry, whose stride says nothing (a single row of a
projection of odd width; one KV head)."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests import _mx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,H,strides", [(1, 8, (8 * 64 + 3, 64, 1)), (1, 1, (1, 5, 1)), (9, 1, (72, 3, 1)), (1, 4, (-7, 64, 1))])
@pytest.mark.parametrize("mx", [True, False])
def test_the_stride_of_a_single_entry(mx, n, H, strides):
    D, ps = 64, 16
    if mx:
        k, v = vx.mxfp4_cache(3, H, ps, D), vx.mxfp4_cache(3, H, ps, D)
    else:
        k, v = (torch.zeros((3, H, ps, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kv = vx.PagedKV(k, v)
    x = torch.randn((2, n, H, D), generator=torch.Generator().manual_seed(n + H)).to(torch.bfloat16)
    slots = torch.arange(5, 5 + n, device="cuda")

    def strided(fill=None):
        buf = torch.full((n * 600,), 7.0, dtype=torch.bfloat16, device="cuda")
        rows = buf.as_strided((n, H, D), [s if d > 1 else max(s, 0) for s, d in zip(strides, (n, H, D))])
        if fill is not None:
            rows.copy_(fill)
        return buf, rows

    (_, kr), (_, vr) = strided(x[0]), strided(x[1])
    s = torch.cuda.current_stream().cuda_stream
    args = (strides[0], strides[1])
    assert vx.lib().vx_kv_write(kv.ref(), kr.data_ptr(), *args, vr.data_ptr(), *args, slots.data_ptr(), n, s) == 0
    (kb, ko), (vb, vo) = strided(), strided()
    assert vx.lib().vx_kv_read(kv.ref(), ko.data_ptr(), *args, vo.data_ptr(), *args, slots.data_ptr(), n, s) == 0
    torch.cuda.synchronize()
    want = x if not mx else torch.from_numpy(_mx.values(*_mx.quantize(x.double().numpy()))).to(torch.bfloat16)
    assert torch.equal(ko.cpu(), want[0]) and torch.equal(vo.cpu(), want[1])
    if n == 1:
        assert (kb[H * D:] == 7.0).all() and (vb[H * D:] == 7.0).all()
    if strides[0] > 0:                                             # through the binding as well
        vx.kv_write(kv, kr, vr, slots)
        vx.kv_read(kv, slots, ko, vo)
        torch.cuda.synchronize()
        assert torch.equal(ko.cpu(), want[0]) and torch.equal(vo.cpu(), want[1])


@pytest.mark.parametrize("row,head", [(192, 128), (-192, 128), (64, 640), (136, 1224)])
def test_rows_between_rows(row, head):
    """Layouts whose rows and heads lie between each other without meeting are read into."""
    H, n, D, ps = 2, 9, 64, 16
    kv = vx.PagedKV(vx.mxfp4_cache(2, H, ps, D), vx.mxfp4_cache(2, H, ps, D))
    x = torch.randn((2, n, H, D), generator=torch.Generator().manual_seed(row + head)).to(torch.bfloat16).cuda()
    slots = torch.randperm(2 * ps, generator=torch.Generator().manual_seed(2))[:n].cuda()
    vx.kv_write(kv, x[0], x[1], slots)
    want = torch.zeros_like(x)
    vx.kv_read(kv, slots, want[0], want[1])
    buf = torch.full((2, 4096), 7.0, dtype=torch.bfloat16, device="cuda")
    first = 8 * -row if row < 0 else 0
    s = torch.cuda.current_stream().cuda_stream
    assert vx.lib().vx_kv_read(kv.ref(), buf[0, first:].data_ptr(), row, head, buf[1, first:].data_ptr(), row, head,
                               slots.data_ptr(), n, s) == 0
    torch.cuda.synchronize()
    taken = torch.zeros(4096, dtype=torch.bool)
    for r in range(n):
        for h in range(H):
            at = first + r * row + h * head
            taken[at:at + D] = True
            assert torch.equal(buf[:, at:at + D], want[:, r, h])
    assert (buf.cpu()[:, ~taken] == 7.0).all()
