"""A page pool in plain Python: what vx_page_extend and vx_page_release do, request by request and page
by page."""
import numpy as np


class Pool:
    def __init__(self, free_pages, free_count, table, lens, ps, unit):
        self.stack, self.cap = [int(p) for p in free_pages[:free_count]], len(free_pages)
        self.table, self.lens, self.ps, self.unit = table.copy(), lens.copy(), ps, unit

    def extend(self, rows, new, page_cap, slot_cap):
        rows_n, stride = self.table.shape
        free, used = len(self.stack), 0
        r = {"seq_lens": [], "granted": [], "first_block": [], "page_indptr": [0], "token_indptr": [0], "pages": [],
             "slots": []}
        for row, n in zip(rows, new):
            n, inside = max(int(n), 0), 0 <= row < rows_n
            L = int(self.lens[row]) if inside else 0
            held, want = -(-L // self.ps), -(-(L + n) // self.ps)
            ok = inside and want <= stride
            if ok:
                used += want - held
                ok = want == held or used <= free
            if ok:
                for x in range(held, want):
                    self.table[row, x] = self.stack.pop()
                self.lens[row] = L + n
            pos = np.arange(L, L + n)
            r["slots"] += [int(self.table[row, p // self.ps]) * self.ps + int(p % self.ps) for p in pos] if ok else [-1] * n
            now = L + n if ok else L
            r["pages"] += [int(p) for p in self.table[row, : -(-now // self.ps)]] if inside else []
            r["seq_lens"].append(now)
            r["granted"].append(n if ok else 0)
            r["first_block"].append(L // self.unit)
            r["page_indptr"].append(min(len(r["pages"]), page_cap))
            r["token_indptr"].append(r["token_indptr"][-1] + n)
        r["pages"] = r["pages"][:page_cap]
        r["slots"] = (r["slots"] + [-1] * slot_cap)[:slot_cap]
        return r

    def release(self, rows, keep):
        back = []
        for i, row in enumerate(rows):
            if not 0 <= row < self.table.shape[0]:
                continue
            L = int(self.lens[row])
            k = min(max(int(keep[i]), 0), L) if keep is not None else 0
            back += [int(p) for p in self.table[row, -(-k // self.ps): -(-L // self.ps)]]
            self.lens[row] = k
        self.stack = (self.stack + back[::-1])[: self.cap]
