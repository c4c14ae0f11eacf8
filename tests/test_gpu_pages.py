"""vx_page_extend and vx_page_release against a plain pool (tests/_pool.py), every output equal: batches of
one to thousands, prompts and single tokens, empty requests, pools that run short, full rows, foreign
rows, cut page lists, long rows, captured graphs."""
import numpy as np
import pytest
import torch

from paper_2606_06453_amd import vx
from tests._pool import Pool

pytestmark = pytest.mark.gpu


class Rig:
    """A pool on the GPU and its plain twin."""

    def __init__(self, B, P, stride, ps, rng, lens, rows=None, block=0, table_rows=None, page_cap=None, slot_cap=64):
        R = table_rows or B
        self.rows = np.asarray(rng.permutation(R)[:B] if rows is None else rows, np.int32)
        ids, table, all_lens = rng.permutation(P).astype(np.int32), np.full((R, stride), -5, np.int32), np.zeros(R, np.int32)
        at = 0
        for row, L in zip(self.rows, lens):
            n = -(-int(L) // ps)
            if 0 <= row < R:
                table[row, :n], all_lens[row] = ids[at:at + n], L
                at += n
        free = np.full(P, -9, np.int32)
        free[: P - at] = ids[at:]
        gpu = lambda x: torch.from_numpy(np.array(x, np.int32)).cuda()  # noqa: E731
        self.pool = vx.PagePool(gpu(free), gpu([P - at]), gpu(table), gpu(all_lens), ps, block)
        self.plain = Pool(free, P - at, table, all_lens, ps, block or ps)
        self.B, self.page_cap, self.slot_cap = B, page_cap if page_cap is not None else max(1, P), slot_cap
        new = lambda n, t=torch.int32: torch.full((n,), -77, dtype=t, device="cuda")  # noqa: E731
        self.batch = vx.BatchSpec(new(B + 1), new(self.page_cap), new(B), stride)
        self.tokens, self.slots, self.granted, self.first = new(B + 1), new(slot_cap, torch.int64), new(B), new(B)
        self.ws = torch.zeros(vx.page_workspace_size(B), dtype=torch.uint8, device="cuda")
        self.gpu_rows = gpu(self.rows)

    def extend(self, new):
        self.launch_extend(torch.from_numpy(np.array(new, np.int32)).cuda())
        self.check_extend(new)

    def launch_extend(self, new):
        vx.page_extend(self.pool, self.gpu_rows, new, self.batch, self.tokens, self.slots, self.granted, self.ws, self.first)

    def check_extend(self, new):
        want = self.plain.extend(self.rows, new, self.page_cap, self.slot_cap)
        torch.cuda.synchronize()
        get = lambda t: t.cpu().numpy().tolist()  # noqa: E731
        assert get(self.batch.seq_lens) == want["seq_lens"]
        assert get(self.granted) == want["granted"]
        assert get(self.batch.page_indptr) == want["page_indptr"]
        assert get(self.tokens) == want["token_indptr"]
        assert get(self.first) == want["first_block"]
        assert get(self.slots) == want["slots"]
        n = len(want["pages"])
        assert get(self.batch.page_indices[:n]) == want["pages"]
        assert (self.batch.page_indices[n:] == -77).all() or self.again
        self.again = True
        self.check_state()

    again = False

    def release(self, keep):
        self.launch_release(None if keep is None else torch.from_numpy(np.array(keep, np.int32)).cuda())
        self.plain.release(self.rows, keep)
        torch.cuda.synchronize()
        self.check_state()

    def launch_release(self, keep):
        vx.page_release(self.pool, self.gpu_rows, keep, self.ws)

    def check_state(self):
        c = int(self.pool.free_count)
        assert c == len(self.plain.stack)
        assert self.pool.free_pages[:c].cpu().numpy().tolist() == self.plain.stack
        assert np.array_equal(self.pool.lens.cpu().numpy(), self.plain.lens)
        assert np.array_equal(self.pool.table.cpu().numpy(), self.plain.table)


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 1000, 1024, 1025, 4099])
@pytest.mark.parametrize("ps,block", [(16, 0), (32, 16), (64, 32)])
def test_steps_of_growing_requests(B, ps, block):
    rng = np.random.default_rng([B, ps])
    lens = rng.integers(0, 9 * ps, size=B) * (rng.random(B) < 0.9)
    new = [rng.integers(0, 4, size=B), rng.integers(0, 5 * ps, size=B) * (rng.random(B) < 0.3), np.ones(B, np.int64)]
    stride = 9 + 8
    rig = Rig(B, B * 16, stride, ps, rng, lens, block=block, slot_cap=int(sum(n.sum() for n in new)) + 3)
    for n in new:
        rig.extend(n)
    keep = np.where(rng.random(B) < 0.5, rng.integers(-2, 12 * ps, size=B), 0)
    rig.release(keep)
    rig.extend(new[0])
    rig.release(None)
    assert int(rig.pool.free_count) == B * 16


@pytest.mark.parametrize("free", [0, 1, 7, 40, 200])
def test_a_pool_that_runs_short(free):
    """Requests behind the shortage that need no page are still granted; one that needs fewer pages than
    are left but stands behind a refused one is not."""
    rng = np.random.default_rng(free)
    B, ps = 1500, 16
    lens = rng.integers(1, 100, size=B)
    held = int((-(-lens // ps)).sum())
    rig = Rig(B, held + free, 12, ps, rng, lens, slot_cap=4000)
    for n in (rng.integers(0, 3, size=B), rng.integers(0, 40, size=B) * (rng.random(B) < 0.05), np.ones(B, np.int64)):
        rig.extend(n)
    rig.release(lens // 2)
    rig.extend(rng.integers(0, 3, size=B))


def test_full_rows_foreign_rows_and_broken_counts():
    rng = np.random.default_rng(5)
    rows = [3, -1, 0, 9, 2, 2 ** 31 - 1, 4]
    rig = Rig(7, 100, 4, 16, rng, [64, 5, 63, 10, 1, 3, 0], rows=rows, table_rows=5, slot_cap=300)
    rig.extend([1, 4, 1, 3, -6, 2, 64])            # a full row; foreign rows; the last free token; a negative count
    rig.extend([0, 0, 1, 0, 70, 1, 1])
    rig.release([16, 3, 17, 0, -4, 1, 100])
    rig.extend([48, 1, 20, 1, 64, 1, 0])
    rig.release(None)
    rig.pool.free_count.fill_(10 ** 9)             # a broken stack: nothing out of bounds, counts held to the pool
    rig.launch_extend(torch.ones(7, dtype=torch.int32, device="cuda"))
    rig.launch_release(None)
    torch.cuda.synchronize()
    assert 0 <= int(rig.pool.free_count) <= 100


@pytest.mark.parametrize("cap", [0, 1, 17, 30])
def test_page_lists_past_the_capacity_are_cut(cap):
    rng = np.random.default_rng(cap)
    rig = Rig(5, 60, 20, 16, rng, [100, 0, 90, 40, 33], page_cap=max(cap, 1), slot_cap=max(cap, 1))
    rig.extend([30, 20, 1, 0, 50])
    assert int(rig.batch.page_indptr[-1]) <= max(cap, 1)


def test_huge_token_counts_are_refused():
    rig = Rig(3, 50, 10, 16, np.random.default_rng(1), [5, 5, 5], slot_cap=8)
    new = torch.tensor([2 ** 31 - 1, 2 ** 31 - 3, 3], dtype=torch.int32, device="cuda")
    rig.launch_extend(new)
    torch.cuda.synchronize()
    assert rig.granted.tolist() == [0, 0, 3] and rig.batch.seq_lens.tolist() == [5, 5, 8]
    assert rig.tokens.tolist() == [0, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1]
    assert rig.slots.tolist() == [-1] * 8


def test_long_rows():
    """Rows of many pages, one prompt beside single tokens."""
    rng = np.random.default_rng(8)
    rig = Rig(3, 40000, 20000, 16, rng, [300001, 0, 7], slot_cap=300010)
    rig.extend([1, 299999, 1])
    rig.release([300001, 5, 8])
    rig.extend([16, 16, 16])
    rig.release(None)


def test_an_extend_is_taken_back_exactly():
    rng = np.random.default_rng(2)
    lens = rng.integers(0, 500, size=300)
    rig = Rig(300, 20000, 64, 16, rng, lens, slot_cap=9000)
    before = rig.pool.free_pages.clone()
    rig.extend(rng.integers(0, 60, size=300))
    rig.release(lens)
    assert torch.equal(rig.pool.free_pages, before)


def test_a_captured_step_replays():
    rng = np.random.default_rng(3)
    B, lens = 70, rng.integers(0, 300, size=70)
    rig = Rig(B, 4000, 60, 16, rng, lens, slot_cap=400)
    new = torch.from_numpy(rng.integers(0, 5, size=B).astype(np.int32)).cuda()
    keep = torch.zeros(B, dtype=torch.int32, device="cuda")
    rig.extend(new.cpu().numpy())                  # once before the capture
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            rig.launch_extend(new)
    back = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(back, stream=stream):
            rig.launch_release(keep)
    torch.cuda.synchronize()
    for step in range(4):
        new.copy_(torch.from_numpy(rng.integers(0, 5, size=B).astype(np.int32)))
        g.replay()
        rig.check_extend(new.cpu().numpy())
        if step == 1:
            keep.copy_(torch.from_numpy(rng.integers(0, 300, size=B).astype(np.int32)))
            back.replay()
            rig.plain.release(rig.rows, keep.cpu().numpy())
            torch.cuda.synchronize()
            rig.check_state()


def test_on_a_stream_of_its_own():
    rng = np.random.default_rng(4)
    rig = Rig(20, 900, 40, 16, rng, rng.integers(0, 200, size=20), slot_cap=100)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        rig.extend(np.full(20, 3))
        rig.release(np.zeros(20, np.int64))


def test_the_largest_batch():
    """65535 requests (256 a workgroup), with and without a shortage."""
    rng = np.random.default_rng(6)
    B, lens = 65535, rng.integers(0, 40, size=65535)
    held = int((-(-lens // 16)).sum())
    rig = Rig(B, held + 30000, 4, 16, rng, lens, slot_cap=200000)
    rig.extend(rng.integers(0, 5, size=B))
    rig.extend(rng.integers(0, 30, size=B) * (rng.random(B) < 0.2))
    rig.extend(np.full(B, 3))                      # the pool runs short on the way
    assert 0 < int((rig.granted == 0).sum()) < B
    rig.release(lens)
