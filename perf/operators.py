"""Timed cases of the key/value operators: a paged cache of keys and values in
16, 8 or 4 bits, and the attention that reads it through the page directory.

Operators (``op`` of a case):

* ``round_trip`` -- new tokens' keys and values are quantised into their pages
  (mem_kv_write) and read back (mem_kv_read): what a turn stores is what later
  turns see.
* ``read``       -- tokens of selected chunks read back as dense rows
  (mem_kv_read).
* ``attend``     -- attention of each request's new tokens over its chunks
  (mem_attend): one token a request (serving), a few (drafted tokens), or a
  whole turn; causal, window, prefix and document masks, scores capped by a
  tanh, distance bias.

The cache (one layer).  A page holds ``page_tokens`` tokens of every head; a
head's part of a page is [K codes][V codes][K scales][V scales], each with one
row per token.  A row of ``d`` elements is cut into blocks of 32 that share
the scale 2^e, held as the byte e + 127:

* ``fp4``: 0, .5, 1, 1.5, 2, 3, 4, 6 and a sign, two to a byte, the even
  element in the low half; e is the smallest with max|x| <= 7 * 2^e;
* ``fp8``: 4 exponent and 3 mantissa bits, largest 448; e is the smallest
  with max|x| <= 464 * 2^e;
* ``bf16``: the values themselves, no scales.

Values are rounded to nearest, ties to the even code, and saturate.  With a
power of two as scale the division is exact, so codes have one right value.
Chunk c is the pages table[c, :]; its first tok_len[c] tokens are written.
A request's context is its chunks' tokens in the order of its list.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
PIECE = 1 << 25         # elements quantised at a time
SCORES = 1 << 28        # scores held at a time by the plain attention
FP4_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------- cases

def listed():
    return [
        # 64 sessions each store the token that they have just produced
        dict(name="turn_round_trip", op="round_trip", fmt="fp4", dtype="bf16", n=64, run=1, hq=32, hkv=8, d=128,
             page_tokens=64, ppc=8),
        # ingestion of 128 chunks of 512 tokens, from an encoder that gives fp32
        dict(name="ingest_round_trip", op="round_trip", fmt="fp8", dtype="f32", n=65536, run=512, hq=8, hkv=8, d=128,
             page_tokens=256, ppc=2),
        # one request's top-5 chunks as dense rows
        dict(name="read_top5", op="read", fmt="fp8", dtype="bf16", n=2560, run=512, hq=32, hkv=8, d=128,
             page_tokens=64, ppc=8),
        # the memory of a batch of requests as dense rows, a ragged number of tokens
        dict(name="read_batch", op="read", fmt="fp4", dtype="bf16", n=131071, run=509, hq=32, hkv=8, d=128,
             page_tokens=64, ppc=8),
        # one request, one new token, over its top-5 chunks
        dict(name="decode_top5", op="attend", fmt="fp4", m=1, k=5, fill="full", q=1, hq=32, hkv=8, d=128,
             page_tokens=64, ppc=8, causal=False, window=0, prefix=0, docs=0, cap=0.0, bias=False),
        # a batch of requests with their ragged memories, scores capped
        dict(name="decode_batch", op="attend", fmt="fp4", m=64, k=8, fill="ragged", q=1, hq=64, hkv=8, d=128,
             page_tokens=64, ppc=8, causal=False, window=0, prefix=0, docs=0, cap=30.0, bias=False),
        # few requests over long histories (131,072 tokens)
        dict(name="decode_long", op="attend", fmt="fp4", m=4, k=256, fill="full", q=1, hq=32, hkv=8, d=128,
             page_tokens=64, ppc=8, causal=False, window=0, prefix=0, docs=0, cap=0.0, bias=False),
        # a full batch over 32,768 tokens each
        dict(name="decode_full", op="attend", fmt="fp4", m=128, k=64, fill="full", q=1, hq=32, hkv=8, d=128,
             page_tokens=64, ppc=8, causal=False, window=0, prefix=0, docs=0, cap=0.0, bias=False),
        # five drafted tokens a request, wide heads, a window with the first tokens kept
        dict(name="draft_window", op="attend", fmt="fp8", m=32, k=16, fill="ragged", q=5, hq=16, hkv=2, d=256,
             page_tokens=128, ppc=4, causal=True, window=4096, prefix=64, docs=0, cap=50.0, bias=False),
        # a turn of 2,048 tokens behind 6,144 tokens of memory
        dict(name="prefill_turn", op="attend", fmt="fp4", m=4, k=16, fill="full", q=2048, hq=32, hkv=8, d=128,
             page_tokens=64, ppc=8, causal=True, window=0, prefix=0, docs=0, cap=50.0, bias=False),
        # a long turn over an unquantised cache, distance bias, a prefix seen by all
        dict(name="prefill_long", op="attend", fmt="bf16", m=1, k=64, fill="full", q=8192, hq=32, hkv=8, d=128,
             page_tokens=64, ppc=8, causal=True, window=0, prefix=1024, docs=0, cap=0.0, bias=True),
        # ragged turns packed with several documents, one head a group, small heads and pages
        dict(name="prefill_docs", op="attend", fmt="fp8", m=7, k=9, fill="ragged", q=1531, hq=12, hkv=12, d=64,
             page_tokens=32, ppc=16, causal=True, window=0, prefix=0, docs=3, cap=0.0, bias=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    fmt = rng.choice(["fp4", "fp4", "fp8", "bf16"])
    d = rng.choice([64, 128, 128, 256])
    page_tokens = rng.choice([32, 64, 128, 256])
    ppc = max(1, rng.choice([256, 512, 512, 1024]) // page_tokens)
    hkv = rng.choice([1, 2, 4, 8, 8, 12])
    group = rng.choice([1, 2, 4, 5, 8, 16])
    base = dict(fmt=fmt, hkv=hkv, hq=hkv * group, d=d, page_tokens=page_tokens, ppc=ppc)
    kind = rng.choice(["round_trip", "read", "decode", "decode", "draft", "prefill"])
    if kind in ("round_trip", "read"):
        n = min(_log(rng, 1, 131072), (1 << 27) // (hkv * d))
        pool = n * page_tokens * ppc * hkv * d              # elements, were every token in a chunk of its own
        run = max(rng.choice([1, 7, 64, 200]), -(-pool // (1 << 32)))
        return dict(base, op=kind, dtype=rng.choice(["bf16", "f32"]), n=n, run=run)
    mask = dict(cap=rng.choice([0.0, 0.0, 30.0, 50.0]), bias=rng.random() < 0.25, fill=rng.choice(["full", "ragged"]),
                window=0, prefix=0, docs=0, causal=False)
    chunk = page_tokens * ppc
    if kind == "decode":
        ctx = _log(rng, 64, 131072)
        m = min(_log(rng, 1, 256), max(1, (1 << 32) // (ctx * hkv * d)))
        q = 1
    else:
        ctx = _log(rng, 256, 32768)
        q = _log(rng, 2, 16) if kind == "draft" else min(_log(rng, 17, 8192), ctx)
        m = _log(rng, 1, 64)
        m = max(1, min(m, (1 << 32) // (ctx * hkv * d), (1 << 34) // (ctx * q * hkv * group * d // 64)))
        mask["causal"] = rng.random() < 0.8
        mask["docs"] = rng.choice([0, 0, 3])
    if rng.random() < 0.3:
        mask["window"] = _log(rng, 16, 8192)
    if rng.random() < 0.3:
        mask["prefix"] = _log(rng, 1, 1024)
    return dict(base, op="attend", m=m, k=min(4096, -(-ctx // chunk)), q=q, **mask)


# ------------------------------------------- what a case's lengths and lists are (host)

def _row_bytes(case):
    """Bytes of codes and of scales of one head's row."""
    d = case["d"]
    return {"bf16": (2 * d, 0), "fp8": (d, d // 32), "fp4": (d // 2, d // 32)}[case["fmt"]]


def _sizes(case):
    """Lengths of the case, the same for every seed: context chunk lengths, new tokens and document labels."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    cap = case["page_tokens"] * case["ppc"]
    reqs = []
    for i in range(case["m"]):
        if case["fill"] == "full":
            lens, nq = [cap] * case["k"], case["q"]
        else:
            nc = case["k"] if i == 0 else rng.randint(0 if i % 8 == 3 else 1, case["k"])
            lens = [cap if rng.random() < 0.6 else rng.randint(1, cap) for _ in range(nc)]
            nq = case["q"] if i == 0 or case["q"] == 1 else rng.randint(0, case["q"])
        ctx = sum(lens)
        if case["causal"]:
            nq = min(nq, ctx)
        doc = [min(case["docs"] - 1, j * case["docs"] // max(1, len(lens))) for j in range(len(lens))] \
            if case["docs"] else [0] * len(lens)
        if case["docs"] and len(doc) > 2 and i % 3 == 1:
            doc[1] = -1                                     # a chunk that was deleted
        reqs.append(dict(lens=lens, ctx=ctx, nq=nq, doc=doc, no_doc=i % 4 == 2))
    return reqs


def _query_doc(case, r):
    """Document label of each new token of a request: that of the chunk that holds its position."""
    lab = np.repeat(np.asarray(r["doc"], np.int32), r["lens"]) if r["lens"] else np.zeros(0, np.int32)
    pos = np.arange(r["nq"]) + r["ctx"] - r["nq"]
    out = np.zeros(r["nq"], np.int32)
    ok = pos >= 0
    if r["ctx"]:
        out[ok] = lab[pos[ok]]
    if r["no_doc"] and r["nq"]:
        out[r["nq"] // 2] = -1                              # a token that may see nothing
    return out


def _visible_pairs(case, r):
    """(query, key) pairs that the masks leave, and the keys that any query sees."""
    ctx, nq = r["ctx"], r["nq"]
    if ctx == 0 or nq == 0:
        return 0, 0
    pos = np.arange(nq, dtype=np.int64) + ctx - nq
    hi = np.minimum(pos + 1, ctx) if case["causal"] else np.full(nq, ctx)
    lo = np.maximum(pos - case["window"] + 1, 0) if case["window"] else np.zeros(nq, np.int64)
    lo, hi = np.minimum(lo, ctx), np.maximum(hi, 0)
    pre = np.full(nq, min(case["prefix"], ctx))
    labels = np.repeat(np.asarray(r["doc"]), r["lens"]) if case["docs"] else np.zeros(ctx, np.int64)
    qdoc = _query_doc(case, r) if case["docs"] else np.zeros(nq, np.int64)
    pairs, keys = 0, 0
    for lab in sorted(set(int(x) for x in qdoc if x >= 0)):
        before = np.concatenate([[0], np.cumsum(labels == lab)])
        sel = qdoc == lab
        l, h, p = lo[sel], np.maximum(hi[sel], lo[sel]), pre[sel]
        pairs += int((before[h] - before[l] + before[np.minimum(p, l)]
                      + before[np.maximum(p, h)] - before[h]).sum())
        seen = np.zeros(ctx + 1, np.int64)
        np.add.at(seen, l, 1)
        np.add.at(seen, h, -1)
        cover = np.cumsum(seen)[:ctx] > 0
        cover[:int(p.max())] = True
        keys += int((cover & (labels == lab)).sum())
    return pairs, keys


def work(case):
    rb, sb = _row_bytes(case)
    h, d = case["hkv"], case["d"]
    if case["op"] in ("round_trip", "read"):
        n, e = case["n"], 2 if case["dtype"] == "bf16" else 4
        dense, packed = 2 * n * h * d * e, 2 * n * h * (rb + sb)
        elems = 2 * n * h * d
        if case["op"] == "read":
            return {"bytes": dense + packed + 8 * n, "flops": elems}
        return {"bytes": 2 * dense + 2 * packed + 8 * n, "flops": 4 * elems}
    pairs = keys = new = 0
    for r in _sizes(case):
        p, s = _visible_pairs(case, r)
        pairs, keys, new = pairs + p, keys + s, new + r["nq"]
    return {"bytes": keys * h * 2 * (rb + sb) + new * case["hq"] * (4 * d + 4) + 4 * case["m"] * case["k"],
            "flops": 4 * d * case["hq"] * pairs}


# ------------------------------------------- the cache in plain torch

def _views(case, pool):
    """(K codes, V codes, K scales, V scales) of every page: uint8 [pages, heads, page_tokens, bytes] views."""
    rb, sb = _row_bytes(case)
    t, h = case["page_tokens"], case["hkv"]
    slab = 2 * t * (rb + sb)
    pages = pool.shape[0]

    def view(offset, width):
        return torch.as_strided(pool, (pages, h, t, width), (pool.stride(0), slab, width, 1),
                                pool.storage_offset() + offset)

    return (view(0, rb), view(t * rb, rb), view(2 * t * rb, sb), view(2 * t * rb + t * sb, sb))


def _encode(case, x):
    """Codes and scale bytes of float32 rows [..., d]."""
    if case["fmt"] == "bf16":
        return x.to(torch.bfloat16).contiguous().view(torch.uint8), None
    fp4 = case["fmt"] == "fp4"
    b = x.unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1)
    frac, ex = torch.frexp(amax)                            # amax = frac * 2^ex, frac in [0.5, 1)
    top, limit = (3, 0.875) if fp4 else (9, 0.90625)        # 7 = 0.875 * 2^3, 464 = 0.90625 * 2^9
    e = torch.clamp(ex - top + (frac > limit).int(), -110, 125 if fp4 else 119)
    e = torch.where(amax == 0, torch.full_like(e, -110), e)
    y = torch.ldexp(b, -e.unsqueeze(-1)).flatten(-2)
    scale = (e + 127).to(torch.uint8)
    if not fp4:
        return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), scale
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    code = code + 8 * (y < 0).to(torch.uint8)
    return code[..., 0::2] + 16 * code[..., 1::2], scale


def _decode(case, codes, scale):
    """float32 rows of codes [..., bytes] and scale bytes [..., d / 32]."""
    if case["fmt"] == "bf16":
        return codes.contiguous().view(torch.bfloat16).float()
    if case["fmt"] == "fp8":
        y = codes.contiguous().view(torch.float8_e4m3fn).float()
    else:
        lut = torch.tensor(FP4_VALUES + tuple(-v for v in FP4_VALUES), device=codes.device)
        y = lut[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    p = torch.exp2(scale.float() - 127)
    return (y.unflatten(-1, (-1, 32)) * p.unsqueeze(-1)).flatten(-2)


def _store(case, pool, k, v, page, slot):
    views = _views(case, pool)
    for x, codes, scales in ((k, views[0], views[2]), (v, views[1], views[3])):
        c, s = _encode(case, x.float())
        codes[page, :, slot] = c
        if s is not None:
            scales[page, :, slot] = s


def _load(case, pool, page, slot):
    kc, vc, ks, vs = _views(case, pool)
    return (_decode(case, kc[page, :, slot], ks[page, :, slot]),
            _decode(case, vc[page, :, slot], vs[page, :, slot]))


# ------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) % (1 << 62))


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(n, heads, d, g, outlier):
    """Keys (a few strong channels, as keys have) or values of n tokens, float32."""
    x = torch.randn((n, heads, d), device=DEV, generator=g)
    return x * outlier


def _channels(heads, d, g):
    c = 0.5 + torch.rand((heads, d), device=DEV, generator=g)
    return torch.where(torch.rand((heads, d), device=DEV, generator=g) < 0.03, 4 * c, c)


def _new_pool(case, n_chunks, g):
    rb, sb = _row_bytes(case)
    n_pages = n_chunks * case["ppc"]
    page_bytes = case["hkv"] * 2 * case["page_tokens"] * (rb + sb)
    pool = torch.zeros((n_pages, page_bytes), dtype=torch.uint8, device=DEV)
    table = torch.randperm(n_pages, device=DEV, generator=g).to(torch.int32).view(n_chunks, case["ppc"])
    return pool, table


def _fill(case, pool, g):
    """Every page of the pool holds keys and values."""
    h, t, d = case["hkv"], case["page_tokens"], case["d"]
    out_k, out_v = _channels(h, d, g), _channels(h, d, g)
    step = max(1, PIECE // (h * t * d))
    slot = torch.arange(t, device=DEV)
    for p0 in range(0, pool.shape[0], step):
        page = torch.arange(p0, min(p0 + step, pool.shape[0]), device=DEV)
        n = page.numel() * t
        _store(case, pool, _rows(n, h, d, g, out_k), _rows(n, h, d, g, out_v), page.repeat_interleave(t),
               slot.repeat(page.numel()))


def _runs(case):
    """Chunk and position of each token: runs of ``run`` consecutive tokens, one run to a chunk."""
    n, cap = case["n"], case["page_tokens"] * case["ppc"]
    run = min(case["run"], cap)
    i = np.arange(n)
    chunk = i // run
    start = (chunk * 37) % (cap - run + 1)
    return chunk.astype(np.int32), (start + i % run).astype(np.int32)


def prepare(case, seed):
    g = _gen(seed)
    st = {"case": case}
    h, hq, d = case["hkv"], case["hq"], case["d"]
    if case["op"] in ("round_trip", "read"):
        chunk, pos = _runs(case)
        n_chunks = int(chunk.max()) + 1
        pool, table = _new_pool(case, n_chunks, g)
        order = torch.randperm(n_chunks, device=DEV, generator=g).to(torch.int32)
        st.update(pool=pool, table=table, chunk=order[torch.from_numpy(chunk).to(DEV).long()],
                  pos=torch.from_numpy(pos).to(DEV))
        if case["op"] == "read":
            _fill(case, pool, g)
        else:                                               # keys and values as a fused projection leaves them
            n = case["n"]
            qkv = torch.empty((n, hq + 2 * h, d), dtype=_dtype(case), device=DEV)
            qkv[:, :hq] = 0
            qkv[:, hq:hq + h] = _rows(n, h, d, g, _channels(h, d, g)).to(qkv.dtype)
            qkv[:, hq + h:] = _rows(n, h, d, g, _channels(h, d, g)).to(qkv.dtype)
            st.update(k=qkv[:, hq:hq + h], v=qkv[:, hq + h:])
    else:
        reqs = _sizes(case)
        lens = [x for r in reqs for x in r["lens"]]
        n_chunks = max(1, len(lens))
        pool, table = _new_pool(case, n_chunks, g)
        _fill(case, pool, g)
        order = torch.randperm(n_chunks, generator=torch.Generator().manual_seed(int(seed) % (1 << 62))).numpy()
        tok_len, chunk_ns = np.zeros(n_chunks, np.int32), np.zeros(n_chunks, np.int32)
        ids = np.full((case["m"], case["k"]), -1, np.int32)
        at, new = 0, [0]
        for i, r in enumerate(reqs):
            mine = order[at:at + len(r["lens"])]
            ids[i, :len(mine)] = mine
            tok_len[mine] = r["lens"]
            chunk_ns[mine] = r["doc"]
            at += len(mine)
            new.append(new[-1] + r["nq"])
        q = torch.randn((new[-1], hq, d), device=DEV, generator=g)
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
        st.update(pool=pool, table=table, ids=up(ids), tok_len=up(tok_len), q=q.to(torch.bfloat16), reqs=reqs,
                  scale=1.0 / math.sqrt(d), q_offsets=None, prefix=None, chunk_ns=None, query_ns=None, slopes=None,
                  ids_host=ids)
        if case["q"] != 1:
            st["q_offsets"] = up(np.asarray(new, np.int32))
        if case["prefix"]:
            st["prefix"] = torch.full((case["m"],), case["prefix"], dtype=torch.int32, device=DEV)
        if case["docs"]:
            st["chunk_ns"] = up(chunk_ns)
            st["query_ns"] = up(np.concatenate([_query_doc(case, r) for r in reqs]).astype(np.int32))
        if case["bias"]:
            st["slopes"] = torch.exp2(-8.0 * (torch.arange(hq, device=DEV) + 1) / hq)
    if own:
        import paper_2607_05708_amd as pm
        fmt = {"bf16": pm.MEM_KV_BF16, "fp8": pm.MEM_KV_FP8, "fp4": pm.MEM_KV_FP4}[case["fmt"]]
        st["cache"] = pm.KvCache(st["pool"], st["table"], case["page_tokens"], h, d, fmt)
        if case["op"] == "attend":
            st["ws"] = torch.empty(max(1, pm.mem_attend_workspace_bytes(st["cache"], case["m"], case["k"],
                                                                       st["q"].shape[0], hq)),
                                   dtype=torch.uint8, device=DEV)
    return st


# ------------------------------------------- one pass

def run(st):
    case = st["case"]
    if own:
        import paper_2607_05708_amd as pm
        if case["op"] == "round_trip":
            pm.mem_kv_write(st["cache"], st["k"], st["v"], st["chunk"], st["pos"])
        if case["op"] in ("round_trip", "read"):
            return pm.mem_kv_read(st["cache"], st["chunk"], st["pos"], dtype=_dtype(case))
        return pm.mem_attend(st["cache"], st["tok_len"], st["ids"], st["q"], st["scale"], q_offsets=st["q_offsets"],
                             causal=case["causal"], window=case["window"], prefix_len=st["prefix"],
                             chunk_ns=st["chunk_ns"], query_ns=st["query_ns"], softcap=case["cap"],
                             slopes=st["slopes"], workspace=st["ws"])
    if case["op"] in ("round_trip", "read"):
        t = case["page_tokens"]
        chunk, pos = st["chunk"].long(), st["pos"].long()
        page, slot = st["table"].long()[chunk, pos // t], pos % t
        if case["op"] == "round_trip":
            _store(case, st["pool"], st["k"], st["v"], page, slot)
        k, v = _load(case, st["pool"], page, slot)
        return k.to(_dtype(case)), v.to(_dtype(case))
    return _plain_attend(st)


def _plain_attend(st):
    case = st["case"]
    t, h, d = case["page_tokens"], case["hkv"], case["d"]
    grp = case["hq"] // h
    q = st["q"].float()
    out = torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, device=DEV)
    table, slot_of = st["table"].long(), torch.arange(t * case["ppc"], device=DEV)
    q0 = 0
    for i, r in enumerate(st["reqs"]):
        nq, ctx = r["nq"], r["ctx"]
        if nq and ctx:
            ids = st["ids"][i, :len(r["lens"])].long()
            page = table[ids][:, slot_of // t].flatten()
            slot = (slot_of % t).repeat(len(r["lens"]))
            if ctx != page.numel():
                used = (slot_of < st["tok_len"][ids].unsqueeze(1)).flatten().nonzero().flatten()
                page, slot = page[used], slot[used]
            k, v = _load(case, st["pool"], page, slot)
            kt, vh = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()
            kpos = torch.arange(ctx, device=DEV)
            if case["docs"]:
                kdoc = st["chunk_ns"][ids].repeat_interleave(torch.tensor(r["lens"], device=DEV), output_size=ctx)
            step = max(1, SCORES // (case["hq"] * ctx))
            for a in range(0, nq, step):
                b = min(a + step, nq)
                rows = q[q0 + a:q0 + b].view(b - a, h, grp, d).permute(1, 2, 0, 3).reshape(h, grp * (b - a), d)
                s = torch.matmul(rows, kt).view(h, grp, b - a, ctx) * st["scale"]
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                dist = (torch.arange(a, b, device=DEV) + ctx - nq).unsqueeze(1) - kpos
                if case["bias"]:
                    s = s - st["slopes"].view(h, grp, 1, 1) * dist.abs()
                see = torch.ones_like(dist, dtype=torch.bool)
                if case["causal"]:
                    see &= dist >= 0
                if case["window"]:
                    see &= dist < case["window"]
                if case["prefix"]:
                    see |= kpos < case["prefix"]
                if case["docs"]:
                    see &= (st["query_ns"][q0 + a:q0 + b].unsqueeze(1) == kdoc) & (kdoc >= 0)
                s = s.masked_fill(~see, -math.inf)
                top = s.amax(-1, keepdim=True)
                p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
                tot = p.sum(-1, keepdim=True)
                o = torch.matmul(p.view(h, grp * (b - a), ctx), vh).view(h, grp, b - a, d)
                o = torch.where(tot > 0, o / tot, torch.zeros_like(o))
                out[q0 + a:q0 + b] = o.permute(2, 0, 1, 3).reshape(b - a, h * grp, d)
                lse[q0 + a:q0 + b] = (top + torch.log(tot)).squeeze(-1).permute(2, 0, 1).reshape(b - a, h * grp)
        q0 += nq
    return out.to(torch.bfloat16), lse


# ------------------------------------------- the definition in 64 bits

def _nearest(case, x):
    """The value that a block of 32 stands for once it is held in the case's format, in 64 bits."""
    x = x.double()
    if case["fmt"] == "bf16":
        _, ex = torch.frexp(x)
        step = torch.ldexp(torch.ones_like(x), ex - 8)
        return torch.where(x == 0, x, torch.round(x / step) * step)
    fp4 = case["fmt"] == "fp4"
    top, low, bits, largest = (7.0, 0, 1, 6.0) if fp4 else (464.0, -6, 3, 448.0)
    b = x.unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp(amax, min=2.0 ** -140) / top))
    e = torch.where(amax > top * torch.exp2(e), e + 1, e)
    e = torch.where(amax <= top * torch.exp2(e - 1), e - 1, e)
    e = torch.clamp(e, -110, 125 if fp4 else 119)
    y = b / torch.exp2(e)
    _, ex = torch.frexp(y)
    step = torch.exp2(torch.clamp(ex - 1, min=low).double() - bits)
    return (torch.clamp(torch.round(y / step) * step, -largest, largest) * torch.exp2(e)).flatten(-2)


def _values(case, codes, scale):
    """64-bit values of codes, from each byte's fields."""
    if case["fmt"] == "bf16":
        w = codes.contiguous().view(torch.int16).long() & 0xFFFF
        man, ex = (w & 127).double(), (w >> 7) & 255
        mag = torch.where(ex == 0, man / 128 * 2.0 ** -126, (1 + man / 128) * torch.exp2(ex.double() - 127))
        return torch.where(w >= 32768, -mag, mag)
    table = []
    for c in range(256 if case["fmt"] == "fp8" else 16):
        bits, bias, sign = (3, 7, c >> 7) if case["fmt"] == "fp8" else (1, 1, c >> 3)
        man, ex = c & ((1 << bits) - 1), (c >> bits) & (15 if case["fmt"] == "fp8" else 3)
        mag = man / (1 << bits) * 2.0 ** (1 - bias) if ex == 0 else (1 + man / (1 << bits)) * 2.0 ** (ex - bias)
        table.append(-mag if sign else mag)
    lut = torch.tensor(table, dtype=torch.float64, device=codes.device)
    c = codes.int()
    if case["fmt"] == "fp4":
        c = torch.stack([c % 16, c // 16], -1).flatten(-2)
    power = torch.exp2(torch.arange(256, device=codes.device, dtype=torch.float64) - 127)
    return lut[c] * power[scale.int()].repeat_interleave(32, -1)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "round_trip":
        return _nearest(case, st["k"]), _nearest(case, st["v"])
    kc, vc, ks, vs = _views(case, st["pool"])
    t = case["page_tokens"]
    if case["op"] == "read":
        page = st["table"][st["chunk"].long(), torch.div(st["pos"], t, rounding_mode="floor").long()].long()
        slot = torch.remainder(st["pos"], t).long()
        return (_values(case, kc[page, :, slot], ks[page, :, slot]),
                _values(case, vc[page, :, slot], vs[page, :, slot]))
    h, hq, d = case["hkv"], case["hq"], case["d"]
    out = torch.zeros((st["q"].shape[0], hq, d), dtype=torch.float64, device=DEV)
    lse = torch.full((st["q"].shape[0], hq), -math.inf, dtype=torch.float64, device=DEV)
    q0 = 0
    for i, r in enumerate(st["reqs"]):
        nq, ctx = r["nq"], r["ctx"]
        if nq == 0 or ctx == 0:
            q0 += nq
            continue
        where = [(int(c), p) for c, n in zip(st["ids_host"][i], r["lens"]) for p in range(0, n, t)]
        counts = [min(t, n - p) for n in r["lens"] for p in range(0, n, t)]
        pages = st["table"][[c for c, _ in where], [p // t for _, p in where]].long()
        keep = torch.cat([torch.arange(c) + j * t for j, c in enumerate(counts)]).to(DEV)
        label = np.repeat(np.asarray(r["doc"]), r["lens"])
        label, qdoc = torch.from_numpy(label).to(DEV), torch.from_numpy(_query_doc(case, r)).to(DEV)
        kpos = torch.arange(ctx, device=DEV, dtype=torch.float64)
        for head in range(h):
            k = _values(case, kc[pages, head], ks[pages, head]).flatten(0, 1)[keep]
            v = _values(case, vc[pages, head], vs[pages, head]).flatten(0, 1)[keep]
            for j in range(head * (hq // h), (head + 1) * (hq // h)):
                step = max(1, SCORES // (4 * ctx))
                for a in range(0, nq, step):
                    b = min(a + step, nq)
                    s = (st["q"][q0 + a:q0 + b, j].double() @ k.T) / math.sqrt(d)
                    if case["cap"]:
                        s = torch.tanh(s / case["cap"]) * case["cap"]
                    qpos = torch.arange(ctx - nq + a, ctx - nq + b, device=DEV, dtype=torch.float64)[:, None]
                    if case["bias"]:
                        s = s - 2.0 ** (-8.0 * (j + 1) / hq) * torch.abs(qpos - kpos)
                    hide = torch.zeros_like(s, dtype=torch.bool)
                    if case["causal"]:
                        hide |= kpos > qpos
                    if case["window"]:
                        hide |= kpos <= qpos - case["window"]
                    if case["prefix"]:
                        hide &= kpos >= case["prefix"]
                    if case["docs"]:
                        hide |= (label < 0) | (label != qdoc[a:b, None])
                    s[hide] = -math.inf
                    z = torch.logsumexp(s, -1)
                    lse[q0 + a:q0 + b, j] = z
                    w = torch.exp(s - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None])
                    out[q0 + a:q0 + b, j] = w @ v
        q0 += nq
    return out, lse
