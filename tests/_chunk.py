"""Ragged chunks over a paged cache in 64 bits: inputs of every cache type, and what the chunk calls compute,
row by row from their definitions."""
import math

import numpy as np
import torch

from paper_2606_06453_amd import vx
from tests import _mx

FP8 = {"fp8_e4m3": (torch.float8_e4m3fn, 448.0), "fp8_e5m2": (torch.float8_e5m2, 57344.0)}
MLA_D, MLA_V = 576, 512


class Chunk:
    """A batch of requests with `before` tokens ahead of `new` ones, on scattered pages of a cache of normal rows."""

    def __init__(self, seed, before, new, Hq, H, D, ps=16, kv="bf16", block=0, spare=0, sigma=1.0, extra_rows=0):
        rng = np.random.default_rng(seed)
        self.kind, self.H, self.Hq, self.D, self.ps, self.g = kv, H, Hq, D, ps, Hq // H
        self.Dv = MLA_V if D == MLA_D else D
        self.block = block
        self.before, self.new = np.asarray(before), np.asarray(new)
        self.lens = (self.before + self.new).astype(np.int32)
        pages = -(-self.lens // ps)
        self.indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
        self.P = max(1, int(self.indptr[-1])) + spare
        self.indices = rng.permutation(self.P)[: int(self.indptr[-1])].astype(np.int32)
        self.max_pages = max(1, int(pages.max(initial=1)))
        self.q_indptr = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.rows = int(self.q_indptr[-1]) + extra_rows
        self.q_lens = None
        self.scale = float(np.float32(6.6 / FP8[kv][1])) if kv in FP8 else 1.0
        bf = lambda *s: torch.from_numpy((rng.standard_normal(s) * sigma).astype(np.float32)).to(torch.bfloat16)  # noqa: E731
        self.q = bf(self.rows, Hq, D)
        self.k, self.k64 = self._cache(bf(self.P, H, ps, D), "k")
        self.v, self.v64 = (None, self.k64[..., :MLA_V]) if D == MLA_D else self._cache(bf(self.P, H, ps, D), "v")
        self.sm_scale = 1.0 / math.sqrt(D)

    def _cache(self, x, which):
        if self.kind == "bf16":
            return x, x.double().numpy()
        if self.kind == "mxfp4":
            packed = _mx.pack(x.double().numpy(), which)
            return torch.from_numpy(packed), _mx.unpack(packed, which)
        dtype, top = FP8[self.kind]
        codes = (x.float() / self.scale).clamp(-top, top).to(dtype)
        return codes, codes.double().numpy() * self.scale

    def on_gpu(self):
        dev = "cuda"
        d = lambda x: None if x is None else torch.as_tensor(x).to(dev)  # noqa: E731
        kv = vx.PagedKV(d(self.k), d(self.v), self.Dv, k_scale=self.scale, v_scale=self.scale, block_size=self.block)
        batch = vx.BatchSpec(d(self.indptr), d(self.indices) if self.indices.size else torch.zeros(1, dtype=torch.int32, device=dev),
                             d(self.lens), self.max_pages)
        return kv, batch, d(self.q), d(self.q_indptr), d(self.q_lens)

    def tokens(self):
        """(row, request, position) of every row that belongs to a token."""
        for i in range(len(self.lens)):
            a, b = int(self.q_indptr[i]), int(self.q_indptr[i + 1])
            n = b - a if self.q_lens is None else min(max(int(self.q_lens[i]), 0), b - a)
            for t in range(n):
                yield a + t, i, int(self.lens[i]) - n + t

    def attend(self, window=0, causal=True, sel=None):
        """out [rows][Hq][Dv], its tolerance, lse [rows][Hq] and its tolerance (fp64; NaN where no token is), by row.
        sel: a set of block ids for every (row, KV head).

        Scores: D exact products added in fp32, each within 2^-23 of the sum of magnitudes qk; the score's error is
        a weight's relative error, in the numerator and in the sum.  The weights round to bf16, half a step 2^-8 of
        them; n additions 2^-23 each, exponentials and rescales a few 2^-22.  The result rounds to bf16, 2^-8."""
        out = np.full((self.rows, self.Hq, self.Dv), np.nan)
        tol, lse, ltol = np.zeros_like(out), np.full((self.rows, self.Hq), np.nan), np.zeros((self.rows, self.Hq))
        q = self.q.double().numpy()
        bs = self.block or self.ps
        for row, i, p in self.tokens():
            L = int(self.lens[i])
            tok = np.arange(max(0, p - window + 1) if window else 0, 0 if p < 0 else min(p + 1, L) if causal else L)
            page = self.indices[self.indptr[i] + tok // self.ps]
            for h in range(self.H):
                keep = slice(None) if sel is None else np.isin(tok // bs, sorted(sel(row, h)))
                k, v = self.k64[page[keep], h, tok[keep] % self.ps], self.v64[page[keep], h, tok[keep] % self.ps]
                hs = slice(h * self.g, (h + 1) * self.g)
                if len(k) == 0:
                    out[row, hs], lse[row, hs] = 0.0, -np.inf
                    continue
                z = self.sm_scale * (q[row, hs] @ k.T)
                m = z.max(-1, keepdims=True)
                w = np.exp(z - m)
                s = w.sum(-1, keepdims=True)
                out[row, hs], absv = w / s @ v, w / s @ np.abs(v)
                qk = (np.abs(q[row, hs]) @ np.abs(k).T).max(-1, keepdims=True)
                err = self.sm_scale * (self.D + 4) * 2.0 ** -23 * qk + (len(k) + 64) * 2.0 ** -23
                delta = 2 * err + 2.0 ** -8
                tol[row, hs] = 2.0 ** -8 * (np.abs(out[row, hs]) + delta * absv) + delta * absv + 1e-30
                lse[row, hs] = (m + np.log(s))[:, 0]
                ltol[row, hs] = err[:, 0] + 2.0 ** -21 * (1 + np.abs(lse[row, hs]))
        return out, tol, lse, ltol

    def select(self, mean, budget, n_sink, n_local, max_sel):
        """sel_pages and sel_count: scores in fp64 rounded to fp32, ties to the lower block; -2 where no token is."""
        bs = self.block or self.ps
        r = self.ps // bs
        pages, count = np.full((self.rows, self.H, max_sel), -2, np.int32), np.full(self.rows, -2, np.int32)
        q = self.q.double().numpy()
        for row, i, p in self.tokens():
            nb = 0 if p < 0 else p // bs + 1
            j = np.arange(nb)
            phys = self.indices[self.indptr[i] + j // r].astype(np.int64) * r + j % r
            forced = (j < n_sink) | (j >= nb - n_local)
            total = min(max(int(budget[i]), 0), max_sel)
            want = nb if total >= nb else max(total, int(forced.sum()))
            for h in range(self.H):
                z = (mean[phys, h].astype(np.float64) @ q[row, h * self.g:(h + 1) * self.g].mean(0)).astype(np.float32) + 0.0
                nan = np.isnan(z)                               # below every score, -inf too
                best = np.lexsort((j, -np.where(nan, 0.0, z).astype(np.float64), nan, ~forced))
                pages[row, h] = -1
                pages[row, h, :want] = np.sort(best[:want])
            count[row] = want
        return pages, count
