"""Performance cases of the paged cache's own operators: the calls that a serving program makes
around and on a KV cache that grows on the GPU and may be held in 4 bits.

A case is a dict of plain values; ``op`` names the call:

* ``plan``       a step's tokens get their pages, block table and slot map (``vx.page_extend``), and the
                 step is taken back (``vx.page_release``), as after drafted tokens that were refused;
* ``rows``       new K/V rows go into the cache by slot (``vx.kv_write``) and rows of the context come
                 back as values (``vx.kv_read``), as in a chunked prefill;
* ``summarize``  block summaries of an mxfp4 cache (``vx.page_summarize``);
* ``decode``     attention over the selected blocks of an mxfp4 cache (``vx.sparse_paged_decode``).

An mxfp4 cache holds E2M1 codes with one E8M0 scale per 32 channels of a token.  The slice of one
(page, KV head) is ``page * D * 17 / 32`` bytes: its codes, then its scales.

* K codes [token][D / 2], the even channel in the low nibble; K scales [token][D / 32].
* V codes [token / 4][16][token % 4][D / 32]: D / 16 channels of four tokens side by side; V scales
  [token / 4][D / 32][token % 4].
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
FP8 = {"fp8_e4m3": (torch.float8_e4m3fn, 448.0), "fp8_e5m2": (torch.float8_e5m2, 57344.0)}


# ---- cases -----------------------------------------------------------------------------------
def listed():
    return [
        # a step of four interactive users with long prompts: launches and host latency are all there is
        dict(op="plan", name="plan_few_users", batch=4, page=16, ctx_lo=24000, ctx_hi=32768, new_lo=1, new_hi=1),
        # a serving batch with up to eight drafted tokens per request
        dict(op="plan", name="plan_drafts", batch=64, page=16, ctx_lo=8192, ctx_hi=32768, new_lo=1, new_hi=8),
        # a few thousand short requests of which some begin with a prompt: 2 million page entries
        dict(op="plan", name="plan_many_requests", batch=4096, page=16, ctx_lo=0, ctx_hi=16000, new_lo=0, new_hi=600),
        # a decode step's rows of a serving batch, quantised to 4 bits, read back for the host's prefix cache
        dict(op="rows", name="rows_step_mxfp4", kv="mxfp4", tokens=64, read=64, kv_heads=8, q_heads=32, dim=128, page=16,
             padded=0.0),
        # a prompt chunk behind a long context that attention over the chunk reads as values
        dict(op="rows", name="rows_chunk_mxfp4", kv="mxfp4", tokens=8192, read=40001, kv_heads=8, q_heads=32, dim=128,
             page=32, padded=0.02),
        # whole prompts into an fp8 cache of few heads, odd count, half of them read
        dict(op="rows", name="rows_prompts_e4m3", kv="fp8_e4m3", tokens=100003, read=50001, kv_heads=4, q_heads=28,
             dim=128, page=64, padded=0.1),
        # the block means of new prompts, with the bf16 copy that selection reads first
        dict(op="summarize", name="summarize_prompts", batch=16, kv_heads=8, dim=128, page=16, block=0, ctx_lo=16384,
             ctx_hi=32768, kind="mean"),
        # envelopes over blocks of 16 on pages of 32, narrow heads, ragged short prompts
        dict(op="summarize", name="summarize_envelope", batch=48, kv_heads=4, dim=64, page=32, block=16, ctx_lo=200,
             ctx_hi=9000, kind="envelope"),
        # one user: a 128-page budget of a long context
        dict(op="decode", name="decode_one_user", batch=1, q_heads=32, kv_heads=8, dim=128, page=16, block=0,
             ctx_lo=32001, ctx_hi=32001, budget=128),
        # a decode step of a serving batch on a Llama-3-8B-shaped layer
        dict(op="decode", name="decode_serving", batch=64, q_heads=32, kv_heads=8, dim=128, page=16, block=0,
             ctx_lo=8192, ctx_hi=32768, budget=128),
        # every block of ragged contexts: the dense call, narrow heads, one query head per KV head
        dict(op="decode", name="decode_dense_narrow", batch=24, q_heads=8, kv_heads=8, dim=64, page=64, block=0,
             ctx_lo=1, ctx_hi=20000, budget=320),
        # a large batch with groups of six heads and wide budgets of 32-token blocks
        dict(op="decode", name="decode_large", batch=128, q_heads=48, kv_heads=8, dim=128, page=64, block=32,
             ctx_lo=4096, ctx_hi=24000, budget=256),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_LARGEST = {}


def draw(rng):
    if not _LARGEST:
        for c in listed():
            _LARGEST[c["op"]] = max(_LARGEST.get(c["op"], 0), work(c)["bytes"])
    while True:
        c = _draw(rng)
        if work(c)["bytes"] <= _LARGEST[c["op"]]:
            return c


def _draw(rng):
    op = rng.choice(["plan", "rows", "rows", "summarize", "decode", "decode", "decode"])
    page = rng.choice([16, 32, 64])
    if op == "plan":
        hi = _log_uniform(rng, 100, 40000)
        new = rng.choice([1, 1, 8, _log_uniform(rng, 1, 600)])
        return dict(op=op, batch=_log_uniform(rng, 1, 4096), page=page, ctx_lo=int(hi * rng.choice([0.0, 0.3, 1.0])),
                    ctx_hi=hi, new_lo=min(new, rng.choice([0, 1])), new_hi=new)
    heads, dim = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([64, 128, 128])
    if op == "rows":
        n = _log_uniform(rng, 1, 100000)
        return dict(op=op, kv=rng.choice(["mxfp4", "mxfp4", "bf16", "fp8_e4m3", "fp8_e5m2"]), tokens=n,
                    read=max(1, int(n * rng.uniform(0.3, 3.0))), kv_heads=heads, q_heads=heads * rng.randint(1, 8),
                    dim=dim, page=page, padded=rng.choice([0.0, 0.02, 0.3]))
    block = rng.choice([0, 0] + [b for b in (16, 32) if b < page])
    hi = _log_uniform(rng, 40, 65536)
    lo = max(1, int(hi * rng.choice([0.0, 0.2, 0.7, 1.0])))
    if op == "summarize":
        return dict(op=op, batch=_log_uniform(rng, 1, 96), kv_heads=heads, dim=dim, page=page, block=block, ctx_lo=lo,
                    ctx_hi=hi, kind=rng.choice(["mean", "envelope"]))
    blocks = -(-hi // (block or page))
    return dict(op=op, batch=_log_uniform(rng, 1, 160), q_heads=heads * rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 16]),
                kv_heads=heads, dim=dim, page=page, block=block, ctx_lo=lo, ctx_hi=hi,
                budget=rng.choice([blocks, max(1, int(blocks * rng.uniform(0.02, 0.5)))]))


# ---- sizes -----------------------------------------------------------------------------------
def _between(c, lo, hi, salt):
    return np.random.default_rng([salt, c["batch"], c[lo], c[hi]]).integers(c[lo], c[hi] + 1, size=c["batch"])


def _ceil(a, b):
    return -(-a // b)


def work(case):
    c = case
    if c["op"] == "plan":
        old, new, ps = _between(c, "ctx_lo", "ctx_hi", 1), _between(c, "new_lo", "new_hi", 2), c["page"]
        pages, fresh = int(_ceil(old + new, ps).sum()), int((_ceil(old + new, ps) - _ceil(old, ps)).sum())
        # per request: row, length (read, written twice), new and kept tokens, five outputs; per page: its id read and
        # listed; per new page also its table entry, and its way off and back on the free stack
        return {"bytes": c["batch"] * 4 * 11 + pages * 8 + fresh * 12 + int(new.sum()) * 8, "flops": 0}
    H, D = c["kv_heads"], c["dim"]
    if c["op"] == "rows":
        e = {"mxfp4": 17 / 32, "bf16": 2}.get(c["kv"], 1)
        return {"bytes": (c["tokens"] + c["read"]) * (2 * H * D * (2 + e) + 8), "flops": 0}
    lens = _between(c, "ctx_lo", "ctx_hi", 1)
    bs = c["block"] or c["page"]
    if c["op"] == "summarize":
        total, blocks = int(lens.sum()), int(_ceil(lens, bs).sum())
        return {"bytes": total * H * D * 17 / 32 + blocks * H * D * (6 if c["kind"] == "mean" else 4),
                "flops": 2 * total * H * D}
    count = np.minimum(_ceil(lens, bs), c["budget"])
    tokens = int(np.minimum(count * bs, lens).sum())
    return {"bytes": tokens * H * 2 * D * 17 / 32 + c["batch"] * c["q_heads"] * D * 4 + 4 * H * int(count.sum()),
            "flops": 4 * tokens * c["q_heads"] * D}


# ---- the 4-bit format in elementary operations -----------------------------------------------
def _mx_views(cache, ps, D, which):
    """Codes and scales of uint8 slices [P][H][ps][17 D / 32] as [P][H][ps][D / 2] and
    [P][H][ps][D / 32] views of the cache, V's in its quad-interleaved order."""
    P, H = cache.shape[:2]
    flat = cache.view(P, H, ps * D * 17 // 32)
    codes, scales = flat[:, :, : ps * D // 2], flat[:, :, ps * D // 2:]
    if which == "k":
        return codes.view(P, H, ps, D // 2), scales.view(P, H, ps, D // 32)
    return (codes.view(P, H, ps // 4, 16, 4, D // 32).permute(0, 1, 2, 4, 3, 5),      # [P][H][quad][token][16][bytes]
            scales.view(P, H, ps // 4, D // 32, 4).permute(0, 1, 2, 4, 3))            # [P][H][quad][token][group]


def _mx_quantize(x):
    """Rows [...][D] (any float type) -> codes [...][D / 2], scales [...][D / 32], both uint8."""
    g = x.float().unflatten(-1, (-1, 32))
    bits = g.abs().amax(-1).view(torch.int32)
    e = (((bits + 0x200000) >> 23) - 2).clamp(8, 252)        # the largest value rounds to at most 6
    scale = (e << 23).view(torch.float32)
    a = (g.abs() / scale.unsqueeze(-1)).clamp(max=6.0)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.round(a / step) * step                         # to nearest, ties to the even code
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = code + 8 * torch.signbit(g).to(torch.uint8)
    bad = bits >= 0x7F800000                                 # an infinity or NaN marks its group
    code = code.masked_fill(bad.unsqueeze(-1), 0).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], e.masked_fill(bad, 255).to(torch.uint8)


def _mx_values(codes, scales, table):
    """fp32 values [...][D] of codes [...][D / 2] and scales [...][D / 32]."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    e = scales.int()
    scale = torch.where(e < 255, (e << 23).view(torch.float32), float("nan"))
    return (table[c].unflatten(-1, (-1, 32)) * scale.unsqueeze(-1)).flatten(-2)


def _table(dtype=torch.float32):
    t = torch.tensor(E2M1, dtype=dtype, device=DEV)
    return torch.cat([t, -t])


def _mx_cache(gen, P, H, ps, D, which):
    """A cache of normal rows, quantised, a few thousand pages at a time."""
    cache = torch.empty((P, H, ps, D * 17 // 32), dtype=torch.uint8, device=DEV)
    cv, sv = _mx_views(cache, ps, D, which)
    for p in range(0, P, 4096):
        n = min(4096, P - p)
        codes, scales = _mx_quantize(torch.randn((n, H, ps, D), generator=gen, device=DEV).to(torch.bfloat16))
        cv[p:p + n] = codes.view(cv[p:p + n].shape)
        sv[p:p + n] = scales.view(sv[p:p + n].shape)
    return cache


# ---- inputs ----------------------------------------------------------------------------------
def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=DEV, dtype=dtype)


def prepare(case, seed):
    c, rng = case, np.random.default_rng(seed)
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    s = dict(c)
    if c["op"] == "plan":
        B, ps = c["batch"], c["page"]
        order = rng.permutation(B)
        old, new = _between(c, "ctx_lo", "ctx_hi", 1)[order], _between(c, "new_lo", "new_hi", 2)[order]
        held, most = _ceil(old, ps), int(_ceil(old + new, ps).max())
        total = int(_ceil(old + new, ps).sum())
        P = total + 64                                        # the pool: what is held, what is needed, a few more
        ids, rows, stride = rng.permutation(P).astype(np.int32), rng.permutation(B), max(1, most)
        table = np.full((B, stride), -1, dtype=np.int32)
        at = np.repeat(np.cumsum(held) - held, held)
        col = np.arange(int(held.sum())) - at
        table[np.repeat(rows, held), col] = ids[: int(held.sum())]
        lens, free = np.zeros(B, dtype=np.int32), np.full(P, -1, dtype=np.int32)
        lens[rows] = old
        left = ids[int(held.sum()):]
        free[: left.size] = left
        s.update(free_pages=_dev(free), free_count=_dev(np.array([left.size])), table=_dev(table), lens=_dev(lens),
                 rows=_dev(rows), new_lens=_dev(new), keep=_dev(old), seq_lens=torch.zeros(B, dtype=torch.int32, device=DEV),
                 page_indptr=torch.zeros(B + 1, dtype=torch.int32, device=DEV),
                 page_indices=torch.zeros(max(1, total), dtype=torch.int32, device=DEV),
                 token_indptr=torch.zeros(B + 1, dtype=torch.int32, device=DEV),
                 slots=torch.zeros(max(1, int(new.sum())) + 8, dtype=torch.int64, device=DEV),
                 granted=torch.zeros(B, dtype=torch.int32, device=DEV),
                 first_block=torch.zeros(B, dtype=torch.int32, device=DEV), max_pages=stride)
        return s
    H, D, ps = c["kv_heads"], c["dim"], c["page"]
    if c["op"] == "rows":
        T, R, Hq = c["tokens"], c["read"], c["q_heads"]
        P = _ceil(max(T, R) + 5 * ps, ps)
        free = rng.permutation(P * ps)                        # slots of scattered pages, in any order
        slots = free[:T].copy()
        slots[rng.random(T) < c["padded"]] = -1
        read = np.concatenate([free[:min(T, R)], free[T:T + max(0, R - T)]])
        read[rng.random(R) < c["padded"]] = -1
        # the projection's output: query, key and value heads of a token side by side
        qkv = torch.randn((T, Hq + 2 * H, D), generator=gen, device=DEV).to(torch.bfloat16)
        s.update(k_rows=qkv[:, Hq:Hq + H], v_rows=qkv[:, Hq + H:], slots=_dev(slots, torch.int64),
                 read_slots=_dev(read, torch.int64), scale_k=1.0, scale_v=1.0,
                 k_out=torch.empty((R, H, D), dtype=torch.bfloat16, device=DEV),
                 v_out=torch.empty((R, H, D), dtype=torch.bfloat16, device=DEV))
        if c["kv"] == "mxfp4":
            s.update(k=_mx_cache(gen, P, H, ps, D, "k"), v=_mx_cache(gen, P, H, ps, D, "v"), table=_table())
            return s
        if c["kv"] != "bf16":
            s["scale_k"] = s["scale_v"] = float(np.float32(6.6 / FP8[c["kv"]][1]))
        for x in ("k", "v"):
            v = torch.randn((P, H, ps, D), generator=gen, device=DEV).to(torch.bfloat16)
            s[x] = v if c["kv"] == "bf16" else _fp8(v, c["kv"], s["scale_k"])
        return s
    # a paged batch on an mxfp4 cache
    lens = rng.permutation(_between(c, "ctx_lo", "ctx_hi", 1)).astype(np.int32)
    pages, bs = _ceil(lens, ps), c["block"] or ps
    indptr = np.concatenate([[0], np.cumsum(pages)])
    P = int(indptr[-1])
    perm = rng.permutation(P)
    s.update(page_indptr=_dev(indptr), page_indices=_dev(perm), seq_lens=_dev(lens), max_pages=int(pages.max()), table=_table(),
             host_lens=lens, k=_mx_cache(gen, P, H, ps, D, "k"), v=_mx_cache(gen, P, H, ps, D, "v"))
    if c["op"] == "summarize":
        R = P * (ps // bs)
        names = (("mean", torch.float32), ("mean_bf16", torch.bfloat16)) if c["kind"] == "mean" else (
            ("max", torch.bfloat16), ("min", torch.bfloat16))
        s.update({n: torch.zeros((R, H, D), dtype=t, device=DEV) for n, t in names})
        return s
    B, Hq = c["batch"], c["q_heads"]
    blocks = _ceil(lens, bs)
    count = np.minimum(blocks, c["budget"])
    M = int(count.max())
    # each head's own blocks: the last one and others drawn from the context, ascending
    key = torch.rand((B, H, int(blocks.max())), generator=gen, device=DEV)
    j, nb = torch.arange(key.shape[2], device=DEV), _dev(blocks, torch.int64)[:, None, None]
    key = torch.where(j < nb, key, 2.0).masked_fill(j == nb - 1, -1.0)
    pick = key.argsort(-1)[..., :M]
    inside = torch.arange(M, device=DEV) < _dev(count, torch.int64)[:, None, None]
    sel = torch.where(inside, pick, 1 << 30).sort(-1)[0]
    s.update(q=torch.randn((B, Hq, D), generator=gen, device=DEV).to(torch.bfloat16),
             sel_pages=torch.where(inside, sel, -1).int().contiguous(), sel_count=_dev(count), max_sel=M,
             sm_scale=1.0 / math.sqrt(D), out=torch.empty((B, Hq, D), dtype=torch.bfloat16, device=DEV))
    return s


def _fp8(x, kind, scale):
    dtype, top = FP8[kind]
    return (x.float() / scale).clamp(-top, top).to(dtype)


# ---- one pass --------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    return {"plan": _plan, "rows": _rows, "summarize": _summarize, "decode": _decode}[s["op"]](s)


def _run_own(s):
    from paper_2606_06453_amd import vx
    if "handles" not in s:                                   # what a user's program makes once and keeps
        s["handles"] = _handles(s, vx)
    h = s["handles"]
    if s["op"] == "plan":
        vx.page_extend(h["pool"], s["rows"], s["new_lens"], h["batch"], s["token_indptr"], s["slots"], s["granted"],
                       h["ws"], first_block=s["first_block"])
        vx.page_release(h["pool"], s["rows"], s["keep"], h["ws"])
        return _plan_outputs(s)
    if s["op"] == "rows":
        vx.kv_write(h["kv"], s["k_rows"], s["v_rows"], s["slots"])
        vx.kv_read(h["kv"], s["read_slots"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if s["op"] == "summarize":
        vx.page_summarize(h["kv"], h["batch"], None, s.get("mean"), s.get("max"), s.get("min"), mean_bf16=s.get("mean_bf16"))
        return {n: s[n] for n in ("mean", "mean_bf16", "max", "min") if n in s}
    vx.sparse_paged_decode(s["q"], h["kv"], h["batch"], s["sel_pages"], s["sel_count"], s["max_sel"], s["sm_scale"],
                           s["out"], h["ws"])
    return s["out"]


def _handles(s, vx):
    h = {}
    if s["op"] != "rows":
        h["batch"] = vx.BatchSpec(s["page_indptr"], s["page_indices"], s["seq_lens"], s["max_pages"])
    if s["op"] == "plan":
        h["pool"] = vx.PagePool(s["free_pages"], s["free_count"], s["table"], s["lens"], s["page"])
        h["ws"] = torch.zeros(vx.page_workspace_size(s["batch"]), dtype=torch.uint8, device=DEV)
        return h
    h["kv"] = vx.PagedKV(s["k"], s["v"], s["dim"], k_scale=s.get("scale_k", 1.0), v_scale=s.get("scale_v", 1.0),
                         block_size=s.get("block", 0))
    if s["op"] == "decode":
        h["ws"] = torch.zeros(vx.workspace_size(vx.STAGE_DECODE, h["kv"], h["batch"], s["q_heads"], s["max_sel"]),
                              dtype=torch.uint8, device=DEV)
    return h


_PLAN = ("page_indptr", "page_indices", "seq_lens", "token_indptr", "slots", "granted", "first_block", "table", "lens",
         "free_pages", "free_count")


def _plan_outputs(s):
    return {n: s[n] for n in _PLAN}


def _plan(s):
    ps, rows = s["page"], s["rows"].long()
    old, new = s["lens"][rows].long(), s["new_lens"].long()
    stride, c = s["table"].shape[1], s["free_count"].long()
    held = (old + ps - 1) // ps
    fits = (old + new + ps - 1) // ps <= stride
    need = torch.where(fits, (old + new + ps - 1) // ps - held, 0)
    behind = need.cumsum(0)
    ok = fits & ((need == 0) | (behind <= c))
    got = torch.where(ok, new, 0)
    pages = (old + got + ps - 1) // ps
    zero = torch.zeros(1, dtype=torch.int64, device=DEV)
    indptr, tokens = torch.cat([zero, pages.cumsum(0)]), torch.cat([zero, new.cumsum(0)])

    def page_of(i, x):                                       # page x of request i: held, or from the top of the stack
        taken = c - 1 - (behind[i] - need[i] + x - held[i])
        return torch.where(x < held[i], s["table"][rows[i], x.clamp(0, stride - 1)], s["free_pages"][taken.clamp(min=0)])

    e = torch.arange(s["page_indices"].numel(), device=DEV)
    i = torch.searchsorted(indptr[1:], e, right=True).clamp(max=old.numel() - 1)
    x, inside = e - indptr[i], e < indptr[-1]
    page = page_of(i, x)
    fresh = inside & (x >= held[i])
    s["page_indices"].copy_(torch.where(inside, page, s["page_indices"]))
    t = torch.arange(s["slots"].numel(), device=DEV)
    it = torch.searchsorted(tokens[1:], t, right=True).clamp(max=old.numel() - 1)
    pos = old[it] + t - tokens[it]
    s["slots"].copy_(torch.where((t < tokens[-1]) & ok[it], page_of(it, pos // ps).long() * ps + pos % ps, -1))
    s["table"].view(-1)[(rows[i] * stride + x)[fresh]] = page[fresh]
    s["page_indptr"].copy_(indptr)
    s["token_indptr"].copy_(tokens)
    s["seq_lens"].copy_(old + got)
    s["granted"].copy_(got)
    s["first_block"].copy_(old // ps)
    s["lens"][rows] = s["seq_lens"]
    s["free_count"].copy_(c - torch.where(ok, need, 0).sum())
    # the step taken back: every page past the kept tokens returns, the first one listed on top
    now, c = s["lens"][rows].long(), s["free_count"].long()
    keep = torch.minimum(s["keep"].long(), now)
    first = (keep + ps - 1) // ps
    back = (now + ps - 1) // ps - first
    ends = back.cumsum(0)
    r = torch.arange(s["free_pages"].numel(), device=DEV)
    ir = torch.searchsorted(ends, r, right=True).clamp(max=old.numel() - 1)
    m = r < ends[-1]
    page = s["table"][rows[ir], (first[ir] + r - ends[ir] + back[ir]).clamp(0, stride - 1)]
    s["free_pages"][(c + ends[-1] - 1 - r)[m]] = page[m]
    s["free_count"].copy_(c + ends[-1])
    s["lens"][rows] = keep.int()
    return _plan_outputs(s)


def _rows(s):
    ps, D, keep = s["page"], s["dim"], s["slots"] >= 0
    slots, read = s["slots"][keep], s["read_slots"]
    p, t, rp, rt = slots // ps, slots % ps, read.clamp(min=0) // ps, read.clamp(min=0) % ps
    got = {}
    for x in ("k", "v"):
        rows, cache, scale = s[x + "_rows"][keep], s[x], s["scale_" + x]
        if s["kv"] == "mxfp4":
            codes, scales = _mx_quantize(rows)
            cv, sv = _mx_views(cache, ps, D, x)
            if x == "k":
                cv[p, :, t], sv[p, :, t] = codes, scales
                y = _mx_values(cv[rp, :, rt], sv[rp, :, rt], s["table"])
            else:
                cv[p, :, t // 4, t % 4], sv[p, :, t // 4, t % 4] = codes.unflatten(-1, (16, -1)), scales
                y = _mx_values(cv[rp, :, rt // 4, rt % 4].flatten(-2), sv[rp, :, rt // 4, rt % 4], s["table"])
        elif s["kv"] == "bf16":
            cache[p, :, t] = rows
            y = cache[rp, :, rt].float()
        else:
            raw = cache.view(torch.uint8)
            raw[p, :, t] = _fp8(rows, s["kv"], scale).view(torch.uint8)
            y = raw[rp, :, rt].view(cache.dtype).float() * scale
        got[x] = torch.where((read >= 0)[:, None, None], y, 0.0).to(torch.bfloat16)
    return got


def _request_pages(s):
    """Request of every listed page, and its place in the request's list."""
    e = torch.arange(s["page_indices"].numel(), device=DEV)
    i = torch.searchsorted(s["page_indptr"][1:].long(), e, right=True)
    return i, e - s["page_indptr"].long()[i]


def _summarize(s):
    ps, D, H = s["page"], s["dim"], s["kv_heads"]
    bs = s["block"] or ps
    cv, sv = _mx_views(s["k"], ps, D, "k")
    i, j = _request_pages(s)
    phys = s["page_indices"].long()
    x = _mx_values(cv[phys], sv[phys], s["table"]).unflatten(2, (ps // bs, bs))          # [page][H][block][token][D]
    at = (j[:, None] * ps + torch.arange(ps, device=DEV)).view(-1, 1, ps // bs, bs, 1)
    valid = at < s["seq_lens"].long()[i].view(-1, 1, 1, 1, 1)
    n = valid.sum(3)                                                                      # [page][1][block][1]
    rows = (phys[:, None] * (ps // bs) + torch.arange(ps // bs, device=DEV)).view(-1)
    any_row = (n > 0).view(-1)
    got = {}
    if s["kind"] == "mean":
        m = torch.where(valid, x, 0.0).sum(3) / n
        got["mean"], got["mean_bf16"] = m, m.to(torch.bfloat16)
    else:
        got["max"] = torch.where(valid, x, -math.inf).amax(3).to(torch.bfloat16)
        got["min"] = torch.where(valid, x, math.inf).amin(3).to(torch.bfloat16)
    for name, y in got.items():
        s[name][rows[any_row]] = y.transpose(1, 2).reshape(-1, H, D)[any_row]
    return {name: s[name] for name in got}


def _selected(s, b):
    """Physical page, first token in it, and valid tokens of every selected block of requests b."""
    ps, bs = s["page"], s["block"] or s["page"]
    r, j = ps // bs, s["sel_pages"][b].long()                                             # [b][H][M]
    ok = (torch.arange(j.shape[2], device=DEV) < s["sel_count"][b].long()[:, None, None]) & (j >= 0)
    j = j.clamp(min=0)
    phys = s["page_indices"].long()[s["page_indptr"][:-1].long()[b][:, None, None] + j // r]
    left = (s["seq_lens"].long()[b][:, None, None] - j * bs).clamp(0, bs)
    return phys, (j % r) * bs, torch.where(ok, left, 0)


def _decode(s):
    ps, D, H, Hq = s["page"], s["dim"], s["kv_heads"], s["q_heads"]
    bs, M, B = s["block"] or ps, s["max_sel"], s["batch"]
    kc, ks = _mx_views(s["k"], ps, D, "k")
    vc, vs = _mx_views(s["v"], ps, D, "v")
    h, u = torch.arange(H, device=DEV)[None, :, None, None], torch.arange(bs, device=DEV)
    out = torch.empty_like(s["out"])
    step = max(1, int(3e8 // (H * M * bs * D)))               # requests at a time, for the card's memory
    for b0 in range(0, B, step):
        b = slice(b0, min(B, b0 + step))
        phys, t0, left = _selected(s, b)
        p, t = phys[..., None], t0[..., None] + u
        k = _mx_values(kc[p, h, t], ks[p, h, t], s["table"]).flatten(2, 3)                # [b][H][tokens][D]
        v = _mx_values(vc[p, h, t // 4, t % 4].flatten(-2), vs[p, h, t // 4, t % 4], s["table"]).flatten(2, 3)
        valid = (u < left[..., None]).flatten(2)[:, :, None]
        q = s["q"][b].float().unflatten(1, (H, Hq // H))
        z = torch.where(valid, torch.matmul(q, k.transpose(2, 3)) * s["sm_scale"], -math.inf)
        w = torch.where(valid, torch.exp(z - z.amax(-1, keepdim=True)), 0.0)
        total = w.sum(-1, keepdim=True)
        o = torch.matmul(w, torch.where(valid.transpose(2, 3), v, 0.0)) / torch.where(total > 0, total, 1.0)
        out[b] = o.flatten(1, 2).to(torch.bfloat16)
    s["out"].copy_(out)
    return s["out"]


# ---- the definitions in 64 bits, written apart -------------------------------------------------
def _bytes_to_rows(cache, page, head, token, ps, D, which):
    """fp64 values [n][D] of rows (page, head, token), by the byte address of every channel."""
    flat = cache.view(cache.shape[0], cache.shape[1], -1)
    ch = torch.arange(D, device=DEV)
    page, head, token = page[:, None], head[:, None], token[:, None]
    if which == "k":
        at, sc = token * (D // 2) + ch // 2, token * (D // 32) + ch // 32
    else:
        piece, inner = ch // (D // 16), ch % (D // 16)
        at = (((token // 4) * 16 + piece) * 4 + token % 4) * (D // 32) + inner // 2
        sc = ((token // 4) * (D // 32) + ch // 32) * 4 + token % 4
    byte = flat[page, head, at].int()
    e = flat[page, head, ps * D // 2 + sc].double() - 127
    return _table(torch.float64)[(byte >> (4 * (ch % 2)).int()) & 15] * torch.exp2(e)


def _nearest_e2m1(x):
    """fp64 rows [n][D] to the format's values: the nearest of the 8 magnitudes times the group's scale,
    of two equally near ones the one with the even code."""
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140)))
    e = torch.where(top >= 1.75 * torch.exp2(e), e + 1, e) - 2
    scale = torch.exp2(e.clamp(8 - 127, 252 - 127))
    a = g.abs() / scale
    values = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
    mid = (values[1:] + values[:-1]) / 2
    up = torch.zeros_like(a, dtype=torch.int64)
    for n in range(7):                                       # a tie goes up where the upper code is even
        up += (a > mid[n]) if n % 2 == 0 else (a >= mid[n])
    return (torch.sign(g) * values[up] * scale).flatten(-2)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "plan":
        return _exact_plan(c, s)
    ps, D, H = c["page"], c["dim"], c["kv_heads"]
    if c["op"] == "rows":
        got, R = {}, c["read"]
        read, slots = s["read_slots"], s["slots"]
        source = torch.full((s["k"].shape[0] * ps,), -1, dtype=torch.int64, device=DEV)
        n = torch.arange(slots.numel(), device=DEV)
        source[slots[slots >= 0]] = n[slots >= 0]
        src = torch.where(read >= 0, source[read.clamp(min=0)], -1)
        for x in ("k", "v"):
            new = s[x + "_rows"][src.clamp(min=0)].double()
            page, token = (read.clamp(min=0) // ps), read.clamp(min=0) % ps
            if c["kv"] == "mxfp4":
                new = _nearest_e2m1(new)
                heads = torch.arange(H, device=DEV)
                old = _bytes_to_rows(s[x], page.repeat_interleave(H), heads.repeat(R), token.repeat_interleave(H), ps, D,
                                     x).view(R, H, D)
            else:
                old = s[x][page, :, token].double() if c["kv"] == "bf16" else (
                    s[x].view(torch.uint8)[page, :, token].view(s[x].dtype).double() * s["scale_" + x])
                if c["kv"] != "bf16":                        # the code nearest to the fp32 quotient
                    top, code = FP8[c["kv"]][1], torch.arange(256, dtype=torch.uint8, device=DEV).view(FP8[c["kv"]][0])
                    vals = code.double()[:128]
                    vals = vals[torch.isfinite(vals)].sort()[0]
                    q = (new / s["scale_" + x]).float().double().abs().clamp(max=top)
                    hi = torch.searchsorted(vals, q).clamp(1, vals.numel() - 1)
                    lower, upper = vals[hi - 1], vals[hi]
                    even = hi % 2 == 0                       # of positive codes in order, the even ones
                    mag = torch.where((q - lower < upper - q) | ((q - lower == upper - q) & ~even), lower, upper)
                    new = torch.sign(new) * mag * s["scale_" + x]
            y = torch.where((src >= 0)[:, None, None], new, old)
            got[x] = torch.where((read >= 0)[:, None, None], y, 0.0)
        return got
    bs = c["block"] or ps
    indptr, lens = s["page_indptr"].tolist(), s["seq_lens"].tolist()
    if c["op"] == "summarize":
        if work(c)["flops"] > 2.5e9:
            return None
        names = ("mean", "mean_bf16") if c["kind"] == "mean" else ("max", "min")
        got = {n: s[n].double() for n in names}
        heads = torch.arange(H, device=DEV)
        for i, L in enumerate(lens):                         # blocks of one request at a time
            n = -(-L // bs)
            phys = s["page_indices"][indptr[i]: indptr[i + 1]].long()
            tok = torch.arange(L, device=DEV)
            page = phys[tok // ps]
            rows = _bytes_to_rows(s["k"], page.repeat_interleave(H), heads.repeat(L), (tok % ps).repeat_interleave(H), ps, D,
                                  "k").view(L, H, D)
            blk = torch.arange(n, device=DEV)
            at = phys[blk * bs // ps] * (ps // bs) + blk % (ps // bs)
            short = n * bs - L
            if c["kind"] == "mean":
                full = torch.cat([rows, rows.new_zeros((short, H, D))]).view(n, bs, H, D).sum(1)
                count = torch.full((n, 1, 1), float(bs), dtype=torch.float64, device=DEV)
                count[-1] = bs - short
                for name in names:
                    got[name][at] = full / count
            else:
                got["max"][at] = torch.cat([rows, rows.new_full((short, H, D), -math.inf)]).view(n, bs, H, D).amax(1)
                got["min"][at] = torch.cat([rows, rows.new_full((short, H, D), math.inf)]).view(n, bs, H, D).amin(1)
        return got
    if c["batch"] * H > 1100 or work(c)["flops"] > 2e11:
        return None
    g = c["q_heads"] // H
    out = torch.zeros((c["batch"], c["q_heads"], D), dtype=torch.float64, device=DEV)
    sel, count = s["sel_pages"].cpu().numpy(), s["sel_count"].tolist()
    for i in range(c["batch"]):
        phys = s["page_indices"][indptr[i]: indptr[i + 1]].long()
        for h in range(H):                                   # the tokens of one head's selected blocks
            pos = (sel[i, h, : count[i]].astype(np.int64)[:, None] * bs + np.arange(bs)).reshape(-1)
            pos = torch.from_numpy(pos[pos < lens[i]]).to(DEV)
            page, head = phys[pos // ps], torch.full_like(pos, h)
            k = _bytes_to_rows(s["k"], page, head, pos % ps, ps, D, "k")
            v = _bytes_to_rows(s["v"], page, head, pos % ps, ps, D, "v")
            z = s["q"][i, h * g:(h + 1) * g].double() @ k.t() * s["sm_scale"]
            out[i, h * g:(h + 1) * g] = torch.softmax(z, -1) @ v
    return out


def _exact_plan(c, s):
    """The step request by request and page by page."""
    ps, n = c["page"], {k: s[k].cpu().numpy().astype(np.int64) for k in _PLAN + ("rows", "new_lens", "keep")}
    stack, table, lens = list(n["free_pages"][: int(n["free_count"][0])]), n["table"], n["lens"]
    full, indptr, tokens, indices, slots = len(stack), [0], [0], [], []
    seq, granted, first, used = [], [], [], 0
    for row, new in zip(n["rows"], n["new_lens"]):
        old = int(lens[row])
        held, want = -(-old // ps), -(-(old + int(new)) // ps)
        ok = want <= table.shape[1]
        if ok:
            used += want - held
            ok = want == held or used <= full
        if ok:
            for x in range(held, want):
                table[row, x] = stack.pop()
        got = int(new) if ok else 0
        pos = np.arange(old, old + int(new))
        slots.append(table[row, pos // ps] * ps + pos % ps if ok else np.full(int(new), -1))
        lens[row] = old + got
        seq.append(old + got)
        granted.append(got)
        first.append(old // ps)
        indices.append(table[row, : -(-(old + got) // ps)].copy())
        indptr.append(indptr[-1] + len(indices[-1]))
        tokens.append(tokens[-1] + int(new))
    flat, where = np.concatenate(indices), np.concatenate(slots)
    n["page_indices"][: flat.size] = flat
    n["slots"][:] = -1
    n["slots"][: where.size] = where
    back = []
    for row, keep in zip(n["rows"], n["keep"]):
        keep = min(int(keep), int(lens[row]))
        back += list(table[row, -(-keep // ps): -(-int(lens[row]) // ps)])
        lens[row] = keep
    stack += back[::-1]
    n["free_pages"][: len(stack)] = stack
    n.update(page_indptr=np.array(indptr), token_indptr=np.array(tokens), seq_lens=np.array(seq), granted=np.array(granted),
             first_block=np.array(first), free_count=np.array([len(stack)]))
    return {k: n[k].astype(np.int64 if k == "slots" else np.int32).reshape(tuple(s[k].shape)) for k in _PLAN}
