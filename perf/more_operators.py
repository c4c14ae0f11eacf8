"""Performance cases of the operators that take a chunk of new tokens over the paged cache: a prompt, a
part of one, or the drafted tokens of a decode step.

A case is a dict of plain values; ``op`` names the call:

* ``rope``    the rows of a fused projection: keys are rotated by their positions, rounded to the cache's
              type and stored by slot with the values, queries are rotated (``vx.rope_kv_write``);
* ``chunk``   attention of the chunk's tokens over everything before them (``vx.chunk_attention``);
* ``select``  the blocks that each token of the chunk attends, by the block-mean score
              (``vx.chunk_score_topk``);
* ``sparse``  attention of the chunk's tokens over such a selection (``vx.sparse_chunk_attention``).

A batch is ragged: request i has ``L_i`` tokens, of which the last ``n_i`` are the chunk's; their rows lie
behind each other.  An mxfp4 cache holds E2M1 codes with one E8M0 scale per 32 channels of a token; the
slice of one (page, KV head) is ``page * D * 17 / 32`` bytes: its codes, then its scales.

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
MLA, MLA_V = 576, 512


# ---- cases -----------------------------------------------------------------------------------
def listed():
    return [
        # a decode step of a serving batch, its rows straight from the projection
        dict(op="rope", name="rope_step", kv="bf16", tokens=64, q_heads=32, kv_heads=8, dim=128, page=16, rot=128, first=0,
             interleaved=False, axes=1, far=32768, padded=0.0),
        # a chunk of image and video tokens (time, height, width) into a 4-bit cache, whose rows are read back as values
        dict(op="rope", name="rope_axes_mxfp4", kv="mxfp4", tokens=8192, q_heads=32, kv_heads=8, dim=128, page=32, rot=128,
             first=0, interleaved=False, axes=3, far=20000, padded=0.02),
        # whole prompts into an fp8 cache: odd count, half of the channels rotated, in neighbouring pairs, far positions
        dict(op="rope", name="rope_prompts_e4m3", kv="fp8_e4m3", tokens=100003, q_heads=28, kv_heads=4, dim=128, page=64,
             rot=64, first=0, interleaved=True, axes=1, far=1000000, padded=0.1),
        # four drafted tokens of a few interactive users behind long contexts: latency and the cache's bandwidth
        dict(op="chunk", name="chunk_drafts", kv="bf16", batch=4, q_heads=32, kv_heads=8, dim=128, page=16, ctx_lo=24000,
             ctx_hi=32768, new_lo=4, new_hi=4, single=0.0, window=0, causal=True, lse=False),
        # a serving batch of decoding requests among which prompts arrive, on a 4-bit cache
        dict(op="chunk", name="chunk_mixed_mxfp4", kv="mxfp4", batch=48, q_heads=32, kv_heads=8, dim=128, page=16, ctx_lo=0,
             ctx_hi=12000, new_lo=100, new_hi=700, single=0.75, window=0, causal=True, lse=False),
        # a long prompt's chunk behind its first part: matrix work alone
        dict(op="chunk", name="chunk_prompt", kv="bf16", batch=1, q_heads=32, kv_heads=8, dim=128, page=16, ctx_lo=24576,
             ctx_hi=24576, new_lo=8192, new_hi=8192, single=0.0, window=0, causal=True, lse=True),
        # odd prompts on an fp8 cache of narrow heads, each token attending a window
        dict(op="chunk", name="chunk_window_e4m3", kv="fp8_e4m3", batch=12, q_heads=20, kv_heads=4, dim=64, page=64, ctx_lo=0,
             ctx_hi=6000, new_lo=333, new_hi=1777, single=0.0, window=1000, causal=True, lse=False),
        # chunks over an absorbed-weight latent
        dict(op="chunk", name="chunk_latent", kv="bf16", batch=8, q_heads=16, kv_heads=1, dim=MLA, page=64, ctx_lo=2048,
             ctx_hi=8192, new_lo=65, new_hi=300, single=0.0, window=0, causal=True, lse=False),
        # the blocks of a few users' drafted tokens
        dict(op="select", name="select_drafts", batch=8, q_heads=32, kv_heads=8, dim=128, page=16, block=0, ctx_lo=16000,
             ctx_hi=32000, new_lo=4, new_hi=4, single=0.0, budget=128, sink=1, local=2),
        # the blocks of every token of a prompt's chunk
        dict(op="select", name="select_prompt", batch=1, q_heads=32, kv_heads=8, dim=128, page=16, block=0, ctx_lo=28672,
             ctx_hi=28672, new_lo=4096, new_hi=4096, single=0.0, budget=128, sink=1, local=2),
        # drafted tokens of a serving batch over their selected blocks, fp8
        dict(op="sparse", name="sparse_drafts_e4m3", kv="fp8_e4m3", batch=32, q_heads=48, kv_heads=8, dim=128, page=64,
             block=32, ctx_lo=4096, ctx_hi=24000, new_lo=1, new_hi=5, single=0.3, budget=64, lse=False),
        # a prompt's chunk over its selected blocks
        dict(op="sparse", name="sparse_prompt", kv="bf16", batch=1, q_heads=32, kv_heads=8, dim=128, page=16, block=0,
             ctx_lo=28672, ctx_hi=28672, new_lo=4096, new_hi=4096, single=0.0, budget=128, lse=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_LARGEST = {}


def _cost(c):
    """What a pass costs, in bytes: the larger of its traffic and its work, and what the plain form gathers."""
    w = work(c)
    gathered = 0 if c["op"] == "rope" else c["batch"] * (c["ctx_hi"] + c["new_hi"]) * c["kv_heads"] * c["dim"] * 8
    return max(w["bytes"], w["flops"] / 200, gathered / 8)


def draw(rng):
    if not _LARGEST:
        for c in listed():
            _LARGEST[c["op"]] = max(_LARGEST.get(c["op"], 0), _cost(c))
    while True:
        c = _draw(rng)
        if _cost(c) <= _LARGEST[c["op"]]:
            return c


def _draw(rng):
    op = rng.choice(["rope", "chunk", "chunk", "select", "sparse"])
    kv, page = rng.choice(["bf16", "bf16", "fp8_e4m3", "fp8_e5m2", "mxfp4"]), rng.choice([16, 32, 64])
    heads, dim = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([64, 128, 128])
    q_heads = heads * rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 16])
    if op in ("rope", "chunk") and rng.random() < 0.15:
        heads, q_heads, dim = 1, 16, MLA
        kv = "bf16" if kv == "mxfp4" else kv
    if op == "rope":
        rot = 64 if dim == MLA else rng.choice([dim, dim, dim // 2, 16])
        return dict(op=op, kv=kv, tokens=_log_uniform(rng, 1, 100000), q_heads=q_heads, kv_heads=heads, dim=dim, page=page,
                    rot=rot, first=rng.choice([0, dim - rot]) if dim != MLA else MLA_V, interleaved=rng.random() < 0.5,
                    axes=rng.choice([1, 1, 3]), far=_log_uniform(rng, 100, 4000000), padded=rng.choice([0.0, 0.02, 0.3]))
    new = _log_uniform(rng, 1, 8192)
    ctx = rng.choice([0, _log_uniform(rng, 40, 65536)])
    c = dict(op=op, batch=_log_uniform(rng, 1, 64), q_heads=q_heads, kv_heads=heads, dim=dim, page=page,
             ctx_lo=int(ctx * rng.choice([0.0, 0.3, 1.0])), ctx_hi=ctx, new_lo=max(1, int(new * rng.choice([0.1, 0.5, 1.0]))),
             new_hi=new, single=rng.choice([0.0, 0.0, 0.3, 0.8]))
    if op == "chunk":
        return dict(c, kv=kv, window=rng.choice([0, 0, _log_uniform(rng, 16, 8192)]), causal=rng.random() < 0.85,
                    lse=rng.random() < 0.5)
    block = rng.choice([0, 0] + [b for b in (16, 32) if b < page])
    blocks = -(-(ctx + new) // (block or page))
    budget = max(1, min(512, int(blocks * rng.uniform(0.02, 0.6))))
    if op == "select":
        return dict(c, block=block, budget=budget + 3, sink=rng.choice([0, 1, 2]), local=rng.choice([1, 2]))
    return dict(c, kv=kv, block=block, budget=budget, lse=rng.random() < 0.3)


# ---- sizes -----------------------------------------------------------------------------------
def _ceil(a, b):
    return -(-a // b)


def _lens(c):
    """Tokens before the chunk and in it, of every request."""
    r = np.random.default_rng([7, c["batch"], c["ctx_hi"], c["new_hi"]])
    before = r.integers(c["ctx_lo"], c["ctx_hi"] + 1, size=c["batch"])
    new = r.integers(c["new_lo"], c["new_hi"] + 1, size=c["batch"])
    return before, np.where(r.random(c["batch"]) < c["single"], 1, new)


def _element(kv):
    return {"mxfp4": 17 / 32, "bf16": 2}.get(kv, 1)


def _positions(before, new):
    """Position of every row of the chunk in its request."""
    at = np.arange(int(new.sum())) - np.repeat(np.cumsum(new) - new, new)
    return np.repeat(before, new) + at


def work(case):
    c = case
    H, Hq, D = c["kv_heads"], c["q_heads"], c["dim"]
    if c["op"] == "rope":
        kv = (1 if D == MLA else 2) * H * D
        row = 2 * 2 * Hq * D + kv * (2 + _element(c["kv"])) + 8 + 8 * c["axes"]
        if c["kv"] == "mxfp4":
            row += kv * (2 + _element(c["kv"])) + 8          # the rows read back
        return {"bytes": c["tokens"] * row, "flops": c["tokens"] * (Hq + H) * c["rot"] * 3}
    before, new = _lens(c)
    n, p, total = int(new.sum()), _positions(before, new), before + new
    if c["op"] == "chunk":
        Dv = MLA_V if D == MLA else D
        end = p + 1 if c["causal"] else np.repeat(total, new)
        first = np.maximum(0, p - c["window"] + 1) if c["window"] else 0
        start = np.maximum(0, before - c["window"] + 1) if c["window"] else 0
        return {"bytes": int((total - start).sum()) * H * (D if D == MLA else 2 * D) * _element(c["kv"])
                + n * Hq * (D + Dv) * 2 + (n * Hq * 4 if c["lse"] else 0),
                "flops": int((end - first).sum()) * Hq * 2 * (D + Dv)}
    bs = c["block"] or c["page"]
    blocks = _ceil(p + 1, bs)
    if c["op"] == "select":
        return {"bytes": n * Hq * D * 2 + int(_ceil(total, bs).sum()) * H * D * 4 + n * H * c["budget"] * 4 + n * 4,
                "flops": int(blocks.sum()) * H * 2 * D}
    count = np.minimum(blocks, c["budget"])
    tokens = int(np.minimum(count * bs, p + 1).sum())
    return {"bytes": min(int(total.sum()), tokens) * H * 2 * D * _element(c["kv"]) + n * Hq * D * 4
            + n * H * int(count.max()) * 4 + (n * Hq * 4 if c["lse"] else 0),
            "flops": tokens * Hq * 4 * D}


# ---- the cache's types in elementary operations -----------------------------------------------
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


def _fp8(x, kind, scale):
    dtype, top = FP8[kind]
    return (x.float() / scale).clamp(-top, top).to(dtype)


def _cache(gen, P, H, ps, D, which, kv, scale):
    """A cache of normal rows in its type, a few thousand pages at a time."""
    if kv == "mxfp4":
        cache = torch.empty((P, H, ps, D * 17 // 32), dtype=torch.uint8, device=DEV)
        cv, sv = _mx_views(cache, ps, D, which)
    else:
        cache = torch.empty((P, H, ps, D), dtype=FP8[kv][0] if kv in FP8 else torch.bfloat16, device=DEV)
    for p in range(0, P, 4096):
        n = min(4096, P - p)
        rows = torch.randn((n, H, ps, D), generator=gen, device=DEV).to(torch.bfloat16)
        if kv == "mxfp4":
            codes, scales = _mx_quantize(rows)
            cv[p:p + n] = codes.view(cv[p:p + n].shape)
            sv[p:p + n] = scales.view(sv[p:p + n].shape)
        else:
            cache[p:p + n] = rows if kv == "bf16" else _fp8(rows, kv, scale)
    return cache


def _page_values(s, which, pages):
    """fp32 values [...][H][ps][D] of the pages [...]."""
    ps, D, cache = s["page"], s["dim"], s[which]
    if s["kv"] == "mxfp4":
        codes, scales = _mx_views(cache, ps, D, which)
        codes, scales = codes[pages], scales[pages]
        if which == "v":                                     # [...][H][quad][token][..] -> [...][H][ps][..]
            codes, scales = codes.flatten(-2).flatten(-3, -2), scales.flatten(-3, -2)
        return _mx_values(codes, scales, s["table"])
    if s["kv"] == "bf16":
        return cache[pages].float()
    return cache.view(torch.uint8)[pages].view(cache.dtype).float() * s["scale"]


# ---- inputs ----------------------------------------------------------------------------------
def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=DEV, dtype=dtype)


def prepare(case, seed):
    c, rng = case, np.random.default_rng(seed)
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    s = dict(c)
    H, Hq, D, ps = c["kv_heads"], c["q_heads"], c["dim"], c["page"]
    s["scale"] = float(np.float32(6.6 / FP8[c["kv"]][1])) if c.get("kv") in FP8 else 1.0
    s["table"] = _table()
    if c["op"] == "rope":
        T, rot = c["tokens"], c["rot"]
        P = _ceil(T + 5 * ps, ps)
        slots = rng.permutation(P * ps)[:T]                   # scattered pages, in any order
        slots[rng.random(T) < c["padded"]] = -1
        # the projection's output: query, key and value heads of a token side by side
        heads = Hq + (H if D == MLA else 2 * H)
        qkv = torch.randn((T, heads, D), generator=gen, device=DEV).to(torch.bfloat16)
        pos = rng.integers(0, c["far"], size=(c["axes"], T))
        # of three axes the first has the slowest pairs' share of all frequencies, the others lie between them
        pairs = np.arange(rot // 2)
        s.update(q_rows=qkv[:, :Hq], k_rows=qkv[:, Hq:Hq + H], v_rows=None if D == MLA else qkv[:, Hq + H:],
                 slots=_dev(slots, torch.int64), positions=_dev(pos, torch.int64),
                 inv_freq=_dev(1e6 ** (-pairs / (rot // 2)), torch.float32), axis=_dev(pairs % c["axes"]),
                 q_out=torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV),
                 k=_cache(gen, P, H, ps, D, "k", c["kv"], s["scale"]),
                 v=None if D == MLA else _cache(gen, P, H, ps, D, "v", c["kv"], s["scale"]))
        if c["kv"] == "mxfp4":
            s.update({x: torch.empty((T, H, D), dtype=torch.bfloat16, device=DEV) for x in ("k_back", "v_back")})
        return s
    before, new = _lens(c)
    order = rng.permutation(c["batch"])
    before, new = before[order], new[order]
    total, n, bs = before + new, int(new.sum()), c.get("block") or ps
    pages = _ceil(total, ps)
    indptr = np.concatenate([[0], np.cumsum(pages)])
    P = int(indptr[-1])
    s.update(page_indptr=_dev(indptr), page_indices=_dev(rng.permutation(P)), seq_lens=_dev(total), max_pages=int(pages.max()),
             q_indptr=_dev(np.concatenate([[0], np.cumsum(new)])), rows=n, pages=P,
             q=torch.randn((n, Hq, D), generator=gen, device=DEV).to(torch.bfloat16), sm_scale=1.0 / math.sqrt(D))
    if c["op"] == "select":
        # block means of normal keys, on a persistent summary of every physical block
        mean = torch.randn((P * (ps // bs), H, D), generator=gen, device=DEV) / math.sqrt(bs)
        s.update(mean=mean, mean_bf16=mean.to(torch.bfloat16), kv="bf16", max_sel=c["budget"],
                 pages_budget=_dev(np.full(c["batch"], c["budget"])),
                 sel_pages=torch.empty((n, H, c["budget"]), dtype=torch.int32, device=DEV),
                 sel_count=torch.empty(n, dtype=torch.int32, device=DEV),
                 k=torch.zeros((P, H, ps, D), dtype=torch.bfloat16, device=DEV))
        s["v"] = s["k"]
        return s
    s["k"] = _cache(gen, P, H, ps, D, "k", c["kv"], s["scale"])
    s["v"] = None if D == MLA else _cache(gen, P, H, ps, D, "v", c["kv"], s["scale"])
    s["out"] = torch.empty((n, Hq, MLA_V if D == MLA else D), dtype=torch.bfloat16, device=DEV)
    s["lse_out"] = torch.empty((n, Hq), dtype=torch.float32, device=DEV) if c["lse"] else None
    if c["op"] == "sparse":
        blocks = _dev(_ceil(_positions(before, new) + 1, bs), torch.int64)
        count = blocks.clamp(max=c["budget"])
        M = int(count.max())
        sel = torch.empty((n, H, M), dtype=torch.int32, device=DEV)
        most, step = int(blocks.max()), max(1, int(2e8 // (H * int(blocks.max()))))
        # each token keeps its own block and others by a score that neighbouring tokens share in part
        run_of = torch.arange(n, device=DEV) // 64
        shared = torch.randn((int(run_of[-1]) + 1, H, most), generator=gen, device=DEV)
        j = torch.arange(most, device=DEV)
        for a in range(0, n, step):
            b, nb = min(n, a + step), blocks[a:a + step, None, None]
            z = shared[run_of[a:b]] + 0.7 * torch.randn((b - a, H, most), generator=gen, device=DEV)
            z = torch.where(j < nb, z, -math.inf).masked_fill(j == nb - 1, math.inf)
            pick = z.topk(M, -1)[1]
            inside = torch.arange(M, device=DEV) < count[a:b, None, None]
            sel[a:b] = torch.where(inside, torch.where(inside, pick, 1 << 30).sort(-1)[0], -1)
        s.update(sel_pages=sel, sel_count=count.int(), max_sel=M)
    return s


# ---- one pass --------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    return {"rope": _rope, "chunk": _chunk, "select": _select, "sparse": _sparse}[s["op"]](s)


def _run_own(s):
    from paper_2606_06453_amd import vx
    if "handles" not in s:                                   # what a user's program makes once and keeps
        s["handles"] = _handles(s, vx)
    h = s["handles"]
    if s["op"] == "rope":
        vx.rope_kv_write(h["kv"], h["rope"], s["q_rows"], s["k_rows"], s["v_rows"], s["positions"], s["slots"], s["q_out"])
        if s["kv"] == "mxfp4":
            vx.kv_read(h["kv"], s["slots"], s["k_back"], s["v_back"])
        return _rope_outputs(s)
    if s["op"] == "chunk":
        vx.chunk_attention(s["q"], h["kv"], h["batch"], s["q_indptr"], s["sm_scale"], s["out"], h["ws"],
                           window=s["window"], causal=s["causal"], lse=s["lse_out"])
        return {"out": s["out"], "lse": s["lse_out"]}
    if s["op"] == "select":
        vx.chunk_score_topk(s["q"], h["kv"], h["batch"], s["q_indptr"], vx.MEAN_DOT, s["mean"], s["pages_budget"],
                            s["sink"], s["local"], s["max_sel"], s["sel_pages"], s["sel_count"], h["ws"])
        return {"pages": s["sel_pages"], "count": s["sel_count"]}
    vx.sparse_chunk_attention(s["q"], h["kv"], h["batch"], s["q_indptr"], s["sel_pages"], s["sel_count"], s["sm_scale"],
                              s["out"], h["ws"], lse=s["lse_out"])
    return {"out": s["out"], "lse": s["lse_out"]}


def _handles(s, vx):
    h = {"kv": vx.PagedKV(s["k"], s["v"], MLA_V if s["dim"] == MLA else s["dim"], k_scale=s["scale"], v_scale=s["scale"],
                          block_size=s.get("block", 0))}
    if s["op"] == "rope":
        h["rope"] = vx.Rope(s["inv_freq"], axis=s["axis"] if s["axes"] > 1 else None, num_axes=s["axes"], first=s["first"],
                            interleaved=s["interleaved"])
        return h
    h["batch"] = vx.BatchSpec(s["page_indptr"], s["page_indices"], s["seq_lens"], s["max_pages"])
    stage = {"chunk": vx.CHUNK_ATTENTION, "select": vx.CHUNK_SCORE_TOPK, "sparse": vx.CHUNK_SPARSE}[s["op"]]
    h["ws"] = torch.empty(vx.chunk_workspace_size(stage, h["kv"], h["batch"], s["rows"], s["q_heads"],
                                                  s.get("max_sel", 1)), dtype=torch.uint8, device=DEV)
    return h


def _rope_outputs(s):
    if s["kv"] == "mxfp4":
        return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _rotate(s, x):
    """fp32 rows [n][heads][D] with their channels first .. first + rot rotated, angles and products in 64 bits."""
    rot, first = s["rot"], s["first"]
    angle = s["positions"][s["axis"].long()].t().double() * s["inv_freq"].double()       # [n][rot / 2]
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    y = x.float()
    part = x[..., first:first + rot].double()
    if s["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        y[..., first:first + rot] = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2).float()
    else:
        a, b = part[..., : rot // 2], part[..., rot // 2:]
        y[..., first:first + rot] = torch.cat([a * cos - b * sin, b * cos + a * sin], -1).float()
    return y


def _rope(s):
    ps, D, keep = s["page"], s["dim"], s["slots"] >= 0
    s["q_out"].copy_(_rotate(s, s["q_rows"]))
    slots = s["slots"][keep]
    p, t = slots // ps, slots % ps
    for x in ("k", "v"):
        if s[x] is None:
            continue
        rows = (_rotate(s, s["k_rows"]) if x == "k" else s["v_rows"].float())[keep]
        cache = s[x]
        if s["kv"] == "mxfp4":
            codes, scales = _mx_quantize(rows)
            cv, sv = _mx_views(cache, ps, D, x)
            if x == "k":
                cv[p, :, t], sv[p, :, t] = codes, scales
            else:
                cv[p, :, t // 4, t % 4], sv[p, :, t // 4, t % 4] = codes.unflatten(-1, (16, -1)), scales
            s[x + "_back"].zero_()
            if x == "k":
                s["k_back"][keep] = _mx_values(cv[p, :, t], sv[p, :, t], s["table"]).to(torch.bfloat16)
            else:
                s["v_back"][keep] = _mx_values(cv[p, :, t // 4, t % 4].flatten(-2), sv[p, :, t // 4, t % 4],
                                               s["table"]).to(torch.bfloat16)
        elif s["kv"] == "bf16":
            cache[p, :, t] = rows.to(torch.bfloat16)
        else:
            cache.view(torch.uint8)[p, :, t] = _fp8(rows, s["kv"], s["scale"]).view(torch.uint8)
    return _rope_outputs(s)


def _row_blocks(s):
    """The chunk's rows in blocks of R rows of one request: the request and the rows [blocks][R] of each, the
    rows' positions, and which of them exist."""
    R = min(256, _ceil(s["rows"], s["batch"]))
    first, new = s["q_indptr"][:-1].long(), s["q_indptr"].long().diff()
    count = (new + R - 1) // R
    ends = count.cumsum(0)
    x = torch.arange(int(ends[-1]), device=DEV)
    req = torch.searchsorted(ends, x, right=True)
    at = ((x - ends[req] + count[req]) * R)[:, None] + torch.arange(R, device=DEV)
    there = at < new[req, None]
    pos = (s["seq_lens"].long() - new)[req, None] + at
    return req, torch.where(there, first[req, None] + at, 0), pos, there


def _request_blocks(s, req, r):
    """Summary rows [requests][most blocks] of requests, by their page lists (entries past a list: any page)."""
    j = torch.arange(s["max_pages"], device=DEV)
    at = (s["page_indptr"][:-1].long()[req, None] + j).clamp(max=s["pages"] - 1)
    phys = s["page_indices"].long()[at]
    return (phys[..., None] * r + torch.arange(r, device=DEV)).flatten(1)


def _chunk(s):
    ps, D, H, Hq = s["page"], s["dim"], s["kv_heads"], s["q_heads"]
    req, rows, pos, there = _row_blocks(s)
    L, R = s["max_pages"] * ps, rows.shape[1]
    token = torch.arange(L, device=DEV)
    step = max(1, int(1e9 // (L * max(Hq * R, 2 * H * D))))  # blocks at a time, for the card's memory
    for a in range(0, req.numel(), step):
        b = slice(a, a + step)
        pages = _request_blocks(s, req[b], 1)
        k = _page_values(s, "k", pages).transpose(1, 2).flatten(2, 3)                    # [b][H][L][D]
        v = k[..., :MLA_V] if s["v"] is None else _page_values(s, "v", pages).transpose(1, 2).flatten(2, 3)
        end = pos[b] + 1 if s["causal"] else s["seq_lens"].long()[req[b], None].expand(-1, R)
        valid = token < end[..., None]                                                    # [b][R][L]
        if s["window"]:
            valid &= token > (pos[b] - s["window"])[..., None]
        valid = valid[:, None].repeat_interleave(Hq // H, 1).flatten(1, 2)[:, None]       # [b][1][g R][L]
        q = s["q"][rows[b]].float().transpose(1, 2).unflatten(1, (H, Hq // H)).flatten(2, 3)
        z = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["sm_scale"]).masked_fill_(~valid, -math.inf)
        top = z.amax(-1, keepdim=True)
        w = z.sub_(top).exp_()
        total = w.sum(-1, keepdim=True)
        o = (torch.matmul(w, v) / total).unflatten(2, (Hq // H, R)).flatten(1, 2).transpose(1, 2)
        s["out"][rows[b][there[b]]] = o[there[b]].to(torch.bfloat16)
        if s["lse"]:
            e = (top + total.log()).squeeze(-1).unflatten(2, (Hq // H, R)).flatten(1, 2).transpose(1, 2)
            s["lse_out"][rows[b][there[b]]] = e[there[b]]
    return {"out": s["out"], "lse": s["lse_out"]}


def _select(s):
    ps, D, H, Hq, M = s["page"], s["dim"], s["kv_heads"], s["q_heads"], s["max_sel"]
    bs = s["block"] or ps
    req, rows, pos, there = _row_blocks(s)
    N, R = s["max_pages"] * (ps // bs), rows.shape[1]
    j = torch.arange(N, device=DEV)
    step = max(1, int(3e8 // (N * H * max(R, D))))
    for a in range(0, req.numel(), step):
        b = slice(a, a + step)
        mean = s["mean"][_request_blocks(s, req[b], ps // bs)].double().permute(0, 2, 3, 1).contiguous()   # [b][H][D][N]
        q = s["q"][rows[b]].double().unflatten(2, (H, Hq // H)).sum(3).transpose(1, 2)    # [b][H][R][D]
        z = (torch.matmul(q, mean) / (Hq // H)).float() + 0.0                             # -0.0 ranks as 0.0
        nb = (pos[b] // bs + 1)[:, None, :, None]
        keep = (j < s["sink"]) | (j >= nb - s["local"])
        z = z.masked_fill_(keep, math.inf).masked_fill_(j >= nb, -math.inf)
        forced = torch.minimum(nb, torch.full_like(nb, s["sink"] + s["local"]))
        count = torch.minimum(nb, torch.maximum(forced, s["pages_budget"].long()[req[b]].clamp(max=M)[:, None, None, None]))
        best = z.sort(dim=-1, descending=True, stable=True)[1][..., :M]                       # of equal scores the first
        if best.shape[-1] < M:
            best = torch.cat([best, best.new_zeros((*best.shape[:-1], M - best.shape[-1]))], -1)
        inside = torch.arange(M, device=DEV) < count
        best = torch.where(inside, torch.where(inside, best, 1 << 30).sort(-1)[0], -1).transpose(1, 2)
        s["sel_pages"][rows[b][there[b]]] = best[there[b]].int()
        s["sel_count"][rows[b][there[b]]] = count[:, 0, :, 0][there[b]].int()
    return {"pages": s["sel_pages"], "count": s["sel_count"]}


def _row_places(s):
    """Request and position of every row."""
    i = torch.searchsorted(s["q_indptr"][1:].long(), torch.arange(s["rows"], device=DEV), right=True)
    return i, s["seq_lens"].long()[i] - s["q_indptr"].long()[i + 1] + torch.arange(s["rows"], device=DEV)


def _sparse(s):
    ps, D, H, Hq, M = s["page"], s["dim"], s["kv_heads"], s["q_heads"], s["max_sel"]
    bs, g = s["block"] or ps, Hq // H
    r = ps // bs
    req, pos = _row_places(s)
    u, h = torch.arange(bs, device=DEV), torch.arange(H, device=DEV)[:, None, None]
    step = max(1, int(4e8 // (H * M * bs * D)))               # rows at a time, for the card's memory
    for a in range(0, s["rows"], step):
        b = slice(a, a + step)
        j = s["sel_pages"][b].long()
        inside = (torch.arange(M, device=DEV) < s["sel_count"][b].long()[:, None, None]) & (j >= 0)
        j = torch.where(inside, j, 0)
        page = s["page_indices"].long()[s["page_indptr"].long()[req[b]][:, None, None] + j // r][..., None]
        t = (j % r * bs)[..., None] + u                                                   # [n][H][M][bs]
        valid = ((j * bs)[..., None] + u <= pos[b, None, None, None]) & inside[..., None]
        k, v = (_token_values(s, x, page, h, t).flatten(2, 3) for x in ("k", "v"))        # [n][H][tokens][D]
        valid = valid.flatten(2)[:, :, None]
        q = s["q"][b].float().unflatten(1, (H, g))
        z = torch.where(valid, torch.matmul(q, k.transpose(2, 3)) * s["sm_scale"], -math.inf)
        top = z.amax(-1, keepdim=True)
        w = torch.exp(z - top)
        total = w.sum(-1, keepdim=True)
        s["out"][b] = (torch.matmul(w, v) / total).flatten(1, 2).to(torch.bfloat16)
        if s["lse"]:
            s["lse_out"][b] = (top + total.log()).squeeze(-1).flatten(1, 2)
    return {"out": s["out"], "lse": s["lse_out"]}


def _token_values(s, which, p, h, t):
    """fp32 values [...][D] of tokens t of pages p, heads h."""
    ps, D, cache = s["page"], s["dim"], s[which]
    if s["kv"] == "mxfp4":
        codes, scales = _mx_views(cache, ps, D, which)
        if which == "k":
            return _mx_values(codes[p, h, t], scales[p, h, t], s["table"])
        return _mx_values(codes[p, h, t // 4, t % 4].flatten(-2), scales[p, h, t // 4, t % 4], s["table"])
    if s["kv"] == "bf16":
        return cache[p, h, t].float()
    return cache.view(torch.uint8)[p, h, t].view(cache.dtype).float() * s["scale"]


# ---- the definitions in 64 bits, written apart -------------------------------------------------
def _rows_by_slot(s, which, slots, head):
    """fp64 values [n][D] of one head's rows at slots (page * page_size + token), by the byte address of every channel."""
    ps, D, cache = s["page"], s["dim"], s[which]
    page, token = (slots // ps)[:, None], (slots % ps)[:, None]
    if s["kv"] != "mxfp4":
        wide = cache[:, head].reshape(-1, D)
        if s["kv"] == "bf16":
            return wide[slots].double()
        return wide.view(torch.uint8)[slots].view(cache.dtype).double() * s["scale"]
    flat = cache.view(cache.shape[0], cache.shape[1], -1)
    ch = torch.arange(D, device=DEV)
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


def _turned(s, x):
    """The rotation as a product of complex numbers."""
    n, rot = x.shape[0], s["rot"]
    pair = torch.arange(rot // 2, device=DEV)
    lo = s["first"] + (2 * pair if s["interleaved"] else pair)
    hi = lo + (1 if s["interleaved"] else rot // 2)
    turn = torch.zeros((n, rot // 2), dtype=torch.float64, device=DEV)
    for axis in range(s["axes"]):
        mine = s["axis"].long() == axis
        turn[:, mine] = s["positions"][axis].double()[:, None] * s["inv_freq"].double()[mine]
    y = x.double()
    z = torch.complex(y[..., lo], y[..., hi]) * torch.polar(torch.ones_like(turn), turn)[:, None]
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


def _exact_rope(s):
    ps, keep = s["page"], s["slots"] >= 0
    got = {"q": _turned(s, s["q_rows"])}
    slots = s["slots"][keep]
    for x, rows in (("k", _turned(s, s["k_rows"])), ("v", None if s["v_rows"] is None else s["v_rows"].double())):
        if rows is None:
            got[x] = None
        elif s["kv"] == "mxfp4":
            got[x] = torch.where(keep[:, None, None], _nearest_e2m1(rows), 0.0)
        else:
            P, H, _, D = s[x].shape
            wide = (s[x].float() if s["kv"] in FP8 else s[x]).double().transpose(1, 2).reshape(P * ps, H, D)
            if s["kv"] in FP8:                               # the nearest code's value, in steps of the value's binade
                top, least, bits = (448.0, -6, 3) if s["kv"] == "fp8_e4m3" else (57344.0, -14, 2)
                a = (rows / s["scale"]).clamp(-top, top)
                step = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** least))) - bits)
                rows = (torch.round(a / step) * step).clamp(-top, top)
            wide[slots] = rows[keep]
            got[x] = wide.view(P, ps, H, D).transpose(1, 2)
    return got


def exact(case, seed):
    c = case
    if c["op"] == "rope":
        return _exact_rope(prepare(c, seed)) if c["tokens"] * c["q_heads"] * c["dim"] < 5e8 else None
    w = work(c)
    if w["flops"] > 8e12 or c["batch"] * c["kv_heads"] * _log_steps(c) > 20000:
        return None
    if c["op"] == "sparse" and w["flops"] > 6e11:
        return None
    s = prepare(c, seed)
    ps, D, H, Hq = c["page"], c["dim"], c["kv_heads"], c["q_heads"]
    bs, g = c.get("block") or ps, c["q_heads"] // c["kv_heads"]
    pi, qi, lens = s["page_indptr"].tolist(), s["q_indptr"].tolist(), s["seq_lens"].tolist()
    if c["op"] == "select":
        got = {"pages": s["sel_pages"].fill_(-1), "count": s["sel_count"].fill_(0)}
    else:
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
        lse = torch.zeros((s["rows"], Hq), dtype=torch.float64, device=DEV)
        got = {"out": out, "lse": lse if c["lse"] else None}
    for i, L in enumerate(lens):
        phys, n = s["page_indices"][pi[i]:pi[i + 1]].long(), qi[i + 1] - qi[i]
        pos, token = torch.arange(L - n, L, device=DEV), torch.arange(L, device=DEV)
        slots = phys[token // ps] * ps + token % ps
        for h in range(H):
            q = s["q"][qi[i]:qi[i + 1], h * g:(h + 1) * g].double()                       # [n][g][D]
            if c["op"] == "select":
                _exact_select(c, s, got, q, phys, pos, qi[i], h, bs)
                continue
            k = _rows_by_slot(s, "k", slots, h)
            v = k[:, :MLA_V].contiguous() if s["v"] is None else _rows_by_slot(s, "v", slots, h)
            kt = k.t().contiguous()
            step = max(1, int(4e8 // (L * g)))
            for a in range(0, n, step):
                p = pos[a:a + step, None]
                if c["op"] == "sparse":
                    blocks = -(-L // bs)                     # one more takes what pads the lists
                    chosen = torch.zeros((p.shape[0], blocks + 1), dtype=torch.bool, device=DEV)
                    sel = s["sel_pages"][qi[i] + a:qi[i] + a + p.shape[0], h].long()
                    chosen.scatter_(1, torch.where(sel < 0, blocks, sel), True)
                    seen = chosen[:, token // bs] & (token <= p)
                else:
                    seen = (token <= p) if c["causal"] else torch.ones((p.shape[0], L), dtype=torch.bool, device=DEV)
                    if c["window"]:
                        seen = seen & (token > p - c["window"])
                z = (q[a:a + step].reshape(-1, D) @ kt * s["sm_scale"]).view(-1, g, L)
                z = torch.where(seen[:, None], z, -math.inf)
                at = slice(qi[i] + a, qi[i] + a + p.shape[0])
                out[at, h * g:(h + 1) * g] = (torch.softmax(z, -1).view(-1, L) @ v).view(-1, g, v.shape[1])
                lse[at, h * g:(h + 1) * g] = torch.logsumexp(z, -1)
    return got


def _log_steps(c):
    """Row groups that a request's heads are taken in."""
    g = c["q_heads"] // c["kv_heads"]
    return max(1, (c["ctx_hi"] + c["new_hi"]) * c["new_hi"] * g // 400000000)


def _exact_select(c, s, got, q, phys, pos, row, h, bs):
    """The blocks of one head of one request: those with fewer than the wanted number of better ones."""
    r, M = c["page"] // bs, s["max_sel"]
    rows = (phys[:, None] * r + torch.arange(r, device=DEV)).reshape(-1)
    z = (q.mean(1) @ s["mean"][rows, h].double().t().contiguous()).float()                # [n][blocks]
    j = torch.arange(z.shape[1], device=DEV)
    for a in range(0, z.shape[0], 1024):
        y, nb = z[a:a + 1024].double(), (pos[a:a + 1024] // bs + 1)[:, None]
        forced = ((j < c["sink"]) | (j >= nb - c["local"])) & (j < nb)
        y = torch.where(forced, math.inf, torch.where(j < nb, y, -math.inf))
        rank = torch.argsort(torch.argsort(-y, dim=-1, stable=True), dim=-1)
        want = torch.maximum(forced.sum(1), torch.minimum(nb[:, 0], torch.full_like(nb[:, 0], min(c["budget"], M))))
        take = (rank < want[:, None]) & (j < nb)
        place = take.cumsum(1) - 1
        x, y = torch.nonzero(take, as_tuple=True)
        got["pages"][row + a + x, h, place[x, y]] = y.int()
        got["count"][row + a: row + a + take.shape[0]] = want.int()
