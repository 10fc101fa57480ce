"""Timed cases of the rotating cache writes and of latent attention.

Operators (``op`` of a case):

* ``append``  -- new tokens' keys are rotated by their positions and stored with
  their values in the paged cache, their queries are rotated (mem_kv_append);
  the stored rows are read back (mem_kv_read): what a turn stores is what later
  turns see.
* ``latent_append`` -- the same for a latent cache: one latent vector and one
  rotated key part a token, shared by all heads (mem_latent_append,
  mem_latent_read).
* ``latent``  -- attention of each request's new tokens over its chunks in a
  latent cache (mem_latent_attend): one token a request (serving), a few
  (drafted tokens), or a whole turn; causal, window, prefix and document masks.

Rotation.  ``dim`` elements of a row are rotated in pairs (i, i + dim / 2), or
(2 i, 2 i + 1) with ``pairs``: pair i of a token at position p by the angle
p * freq[i]; the rest of the row stays.  Rotated elements are computed in 64 bits
and rounded once, to what they are held in.

Attention.  With c the latent vector and r the rotated key part of a token, head
h's key is [W_h c, r], its value is V_h c; W_h and V_h are rows 0 .. d - 1 and
d .. 2 d - 1 of w[h].  A query is its d elements and its rotated part:
    s(p) = scale * (<q_h, W_h c_p> + <t_h, r_p>),   out_h = V_h sum_p softmax(s)(p) c_p
over the tokens that the masks leave.  (W_h can as well be taken to the query's
side, and V_h behind the sum: what the forms are about.)

A page of the key/value cache holds, head by head, [K codes][V codes][K scales]
[V scales], each with a row per token; a page of the latent cache [latent codes]
[key parts in bf16][latent scales].  Rows are cut into blocks of 32 elements that
share the scale 2^e, held as the byte e + 127:

* ``fp4``: 0, .5, 1, 1.5, 2, 3, 4, 6 and a sign, two to a byte, the even
  element in the low half; e is the smallest with max|x| <= 7 * 2^e;
* ``fp8``: 4 exponent and 3 mantissa bits, largest 448; e is the smallest
  with max|x| <= 464 * 2^e;
* ``bf16``: the values themselves, no scales.

Chunk c is the pages table[c, :]; its first tok_len[c] tokens are written.  A
request's context is its chunks' tokens in the order of its list.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
PIECE = 1 << 25         # elements quantised at a time
SCORES = 1 << 28        # scores held at a time by the plain attention
ROPE = 64               # elements of the rotated key part of a latent cache
FP4_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------- cases

def listed():
    none = dict(causal=False, window=0, prefix=0, docs=0)
    turn = dict(causal=True, window=0, prefix=0, docs=0)
    return [
        # 64 sessions each store the token that they have just produced, and rotate its queries
        dict(name="append_tokens", op="append", fmt="fp4", dtype="bf16", n=64, run=1, hq=32, hkv=8, d=128, dim=128,
             pairs=False, far=32768, page_tokens=64, ppc=8),
        # ingestion of 64 chunks of 512 tokens, half of each head rotated, at far positions
        dict(name="append_chunks", op="append", fmt="fp8", dtype="bf16", n=32768, run=512, hq=32, hkv=8, d=128, dim=64,
             pairs=True, far=1000000, page_tokens=256, ppc=2),
        # a batch of requests each store a token's latent vector
        dict(name="latent_append_tokens", op="latent_append", fmt="fp8", dtype="bf16", n=128, run=1, hq=16, lat=512,
             pairs=True, far=32768, page_tokens=64, ppc=8),
        # ingestion of 256 chunks from a projection that gives fp32, a ragged number of tokens
        dict(name="latent_append_chunks", op="latent_append", fmt="bf16", dtype="f32", n=131071, run=509, hq=0, lat=512,
             pairs=False, far=1000000, page_tokens=64, ppc=8),
        # one request, one new token, over its top-5 chunks
        dict(name="latent_top5", op="latent", fmt="fp4", m=1, k=5, fill="full", q=1, hq=16, lat=512, d=128,
             page_tokens=64, ppc=8, **none),
        # a batch of requests with their ragged memories
        dict(name="latent_batch", op="latent", fmt="fp8", m=64, k=8, fill="ragged", q=1, hq=32, lat=512, d=128,
             page_tokens=64, ppc=8, **none),
        # few requests over long histories (131,072 tokens), unquantised
        dict(name="latent_long", op="latent", fmt="bf16", m=4, k=256, fill="full", q=1, hq=16, lat=512, d=128,
             page_tokens=64, ppc=8, **none),
        # a full batch over 32,768 tokens each, all heads of a wide model on one GPU
        dict(name="latent_full", op="latent", fmt="fp8", m=64, k=64, fill="full", q=1, hq=128, lat=512, d=128,
             page_tokens=64, ppc=8, **none),
        # five drafted tokens a request, a window with the first tokens kept, small latent vectors
        dict(name="latent_draft", op="latent", fmt="fp4", m=32, k=16, fill="ragged", q=5, hq=20, lat=256, d=64,
             page_tokens=128, ppc=4, causal=True, window=4096, prefix=64, docs=0),
        # a turn of 2,048 tokens behind 6,144 tokens of memory
        dict(name="latent_turn", op="latent", fmt="fp8", m=4, k=16, fill="full", q=2048, hq=16, lat=512, d=128,
             page_tokens=64, ppc=8, **turn),
        # a long turn over an unquantised cache, a prefix seen by all
        dict(name="latent_prompt", op="latent", fmt="bf16", m=1, k=64, fill="full", q=8192, hq=32, lat=512, d=128,
             page_tokens=64, ppc=8, causal=True, window=0, prefix=1024, docs=0),
        # ragged turns packed with several documents, small heads and pages
        dict(name="latent_docs", op="latent", fmt="fp4", m=7, k=9, fill="ragged", q=1531, hq=12, lat=256, d=64,
             page_tokens=32, ppc=16, causal=True, window=0, prefix=0, docs=3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    fmt = rng.choice(["fp4", "fp8", "fp8", "bf16"])
    page_tokens = rng.choice([32, 64, 128, 256])
    ppc = max(1, rng.choice([256, 512, 512, 1024]) // page_tokens)
    base = dict(fmt=fmt, page_tokens=page_tokens, ppc=ppc)
    kind = rng.choice(["append", "latent_append", "decode", "decode", "draft", "prefill", "prefill"])
    if kind in ("append", "latent_append"):
        store = dict(base, op=kind, dtype=rng.choice(["bf16", "f32"]), pairs=rng.random() < 0.5,
                     far=_log(rng, 4096, 1000000))
        if kind == "append":
            d, hkv = rng.choice([64, 128, 128, 256]), rng.choice([1, 2, 4, 8, 8, 12])
            hq = hkv * rng.choice([0, 1, 2, 4, 5, 8])
            row, kept = (hq + 2 * hkv) * d, 2 * hkv * d
            store.update(hq=hq, hkv=hkv, d=d, dim=rng.choice([d, d, d // 2, 16, 48]))
        else:
            hq, lat = rng.choice([0, 5, 16, 32, 128]), rng.choice([256, 512, 512])
            row, kept = hq * ROPE + lat + ROPE, lat + ROPE
            store.update(hq=hq, lat=lat)
        n = min(_log(rng, 1, 65536), (1 << 26) // row)
        pool = n * page_tokens * ppc * kept                 # elements, were every token in a chunk of its own
        return dict(store, n=n, run=max(rng.choice([1, 7, 64, 200]), -(-pool // (1 << 32))))
    lat, hq, d = rng.choice([256, 512, 512]), rng.choice([1, 5, 16, 16, 20, 32, 64, 128]), rng.choice([64, 128, 128])
    mask = dict(causal=False, window=0, prefix=0, docs=0, fill=rng.choice(["full", "ragged"]))
    chunk = page_tokens * ppc
    if kind == "decode":
        ctx = _log(rng, 64, 131072)
        m = max(1, min(_log(rng, 1, 256), (1 << 20) // ctx, (1 << 26) // (ctx * hq)))
        q = 1
    else:
        ctx = _log(rng, 256, 24576)
        q = _log(rng, 2, 16) if kind == "draft" else min(_log(rng, 17, 8192), ctx)
        m = max(1, min(_log(rng, 1, 64), (1 << 20) // ctx, (1 << 32) // (ctx * q * hq)))
        mask["causal"] = rng.random() < 0.8
        mask["docs"] = rng.choice([0, 0, 3])
    if rng.random() < 0.3:
        mask["window"] = _log(rng, 16, 8192)
    if rng.random() < 0.3:
        mask["prefix"] = _log(rng, 1, 1024)
    return dict(base, op="latent", m=m, k=min(4096, -(-ctx // chunk)), q=q, hq=hq, lat=lat, d=d, **mask)


# ------------------------------------------- what a case's lengths and lists are (host)

def _code_bytes(case, d):
    """Bytes of codes and of scales of a row of d elements."""
    return {"bf16": (2 * d, 0), "fp8": (d, d // 32), "fp4": (d // 2, d // 32)}[case["fmt"]]


def _token_bytes(case):
    """Bytes of a token in its page."""
    if case["op"] == "append":
        return 2 * case["hkv"] * sum(_code_bytes(case, case["d"]))
    return sum(_code_bytes(case, case["lat"])) + 2 * ROPE


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


def _query_doc(r):
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
    qdoc = _query_doc(r) if case["docs"] else np.zeros(nq, np.int64)
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
    if case["op"] != "latent":
        n, e = case["n"], 2 if case["dtype"] == "bf16" else 4
        if case["op"] == "append":
            kept, turned = 2 * case["hkv"] * case["d"], (case["hkv"] + case["hq"]) * case["dim"]
            queries = case["hq"] * case["d"]
        else:
            kept, turned = case["lat"] + ROPE, (1 + case["hq"]) * ROPE
            queries = case["hq"] * ROPE
        # rows in, codes out and in again, rows out; queries in and out
        return {"bytes": n * (2 * kept * e + 2 * _token_bytes(case) + queries * (e + 2) + 12),
                "flops": n * (3 * turned + 4 * kept)}
    pairs = keys = new = 0
    for r in _sizes(case):
        p, s = _visible_pairs(case, r)
        pairs, keys, new = pairs + p, keys + s, new + r["nq"]
    h, d, lat = case["hq"], case["d"], case["lat"]
    absorbed = h * (2 * pairs * (2 * lat + ROPE) + 4 * new * d * lat)
    expanded = h * (2 * pairs * (2 * d + ROPE) + 4 * keys * d * lat)
    return {"bytes": keys * _token_bytes(case) + 2 * new * h * (2 * d + ROPE) + 4 * h * d * lat
            + 4 * case["m"] * case["k"], "flops": min(absorbed, expanded)}


# ------------------------------------------- the caches in plain torch

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


def _page_view(pool, shape, strides, offset):
    return torch.as_strided(pool, (pool.shape[0], *shape), (pool.stride(0), *strides), pool.storage_offset() + offset)


def _kv_views(case, pool):
    """(K codes, V codes, K scales, V scales) of every page: uint8 [pages, heads, page_tokens, bytes] views."""
    rb, sb = _code_bytes(case, case["d"])
    t, h = case["page_tokens"], case["hkv"]
    slab = 2 * t * (rb + sb)
    return [_page_view(pool, (h, t, w), (slab, w, 1), at)
            for at, w in ((0, rb), (t * rb, rb), (2 * t * rb, sb), (2 * t * rb + t * sb, sb))]


def _latent_views(case, pool):
    """(latent codes, key parts, latent scales) of every page: uint8 [pages, page_tokens, bytes] views."""
    rb, sb = _code_bytes(case, case["lat"])
    t = case["page_tokens"]
    return [_page_view(pool, (t, w), (w, 1), at)
            for at, w in ((0, rb), (t * rb, 2 * ROPE), (t * (rb + 2 * ROPE), sb))]


def _store_kv(case, pool, k, v, page, slot):
    kc, vc, ks, vs = _kv_views(case, pool)
    for x, codes, scales in ((k, kc, ks), (v, vc, vs)):
        c, s = _encode(case, x)
        codes[page, :, slot] = c
        if s is not None:
            scales[page, :, slot] = s


def _load_kv(case, pool, page, slot):
    kc, vc, ks, vs = _kv_views(case, pool)
    return (_decode(case, kc[page, :, slot], ks[page, :, slot]), _decode(case, vc[page, :, slot], vs[page, :, slot]))


def _store_latent(case, pool, c, r, page, slot):
    codes, parts, scales = _latent_views(case, pool)
    x, s = _encode(case, c)
    codes[page, slot] = x
    parts[page, slot] = r.to(torch.bfloat16).contiguous().view(torch.uint8)
    if s is not None:
        scales[page, slot] = s


def _load_latent(case, pool, page, slot):
    codes, parts, scales = _latent_views(case, pool)
    return (_decode(case, codes[page, slot], scales[page, slot]),
            parts[page, slot].contiguous().view(torch.bfloat16).float())


def _to_odd(x):
    """64-bit numbers as float32, rounded to the neighbour with an odd last bit where they are none: what rounds that to
    fewer bits gives what one rounding gives."""
    f = x.float()
    bits = f.view(torch.int32)
    bits = bits - (f.double().abs() > x.abs()).int()        # towards zero
    return torch.where(f.double() != x, bits | 1, bits).view(torch.float32)


def _rotate(case, x, at, freq):
    """Rows [n, ..., d] rotated by the positions at [n], the first 2 len(freq) elements of each: as _to_odd gives them."""
    half = freq.numel()
    angle = at.double().unsqueeze(-1) * freq.double()
    shape = (x.shape[0], *[1] * (x.dim() - 2), half)
    cos, sin = angle.cos().view(shape), angle.sin().view(shape)
    part = x[..., :2 * half].double()
    a, b = (part[..., 0::2], part[..., 1::2]) if case["pairs"] else (part[..., :half], part[..., half:])
    turned = _to_odd(a * cos - b * sin), _to_odd(a * sin + b * cos)
    turned = torch.stack(turned, -1).flatten(-2) if case["pairs"] else torch.cat(turned, -1)
    return torch.cat([turned, x[..., 2 * half:].float()], -1)


# ------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) % (1 << 62))


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _channels(shape, g):
    """Sizes of channels, a few of them strong, as keys and latent vectors have them."""
    c = 0.5 + torch.rand(shape, device=DEV, generator=g)
    return torch.where(torch.rand(shape, device=DEV, generator=g) < 0.03, 4 * c, c)


def _new_pool(case, n_chunks, g):
    n_pages = n_chunks * case["ppc"]
    pool = torch.zeros((n_pages, case["page_tokens"] * _token_bytes(case)), dtype=torch.uint8, device=DEV)
    table = torch.randperm(n_pages, device=DEV, generator=g).to(torch.int32).view(n_chunks, case["ppc"])
    return pool, table


def _fill(case, pool, g):
    """Every page of the pool holds latent vectors and key parts."""
    t = case["page_tokens"]
    sizes = _channels((case["lat"],), g)
    sizes = sizes / sizes.square().mean().sqrt()            # latent vectors are normalised
    step = max(1, PIECE // (t * case["lat"]))
    slot = torch.arange(t, device=DEV)
    for p0 in range(0, pool.shape[0], step):
        page = torch.arange(p0, min(p0 + step, pool.shape[0]), device=DEV)
        n = page.numel() * t
        c = torch.randn((n, case["lat"]), device=DEV, generator=g) * sizes
        r = torch.randn((n, ROPE), device=DEV, generator=g)
        _store_latent(case, pool, c, r, page.repeat_interleave(t), slot.repeat(page.numel()))


def _runs(case):
    """Chunk and position of each token: runs of ``run`` consecutive tokens, one run to a chunk."""
    n, cap = case["n"], case["page_tokens"] * case["ppc"]
    run = min(case["run"], cap)
    i = np.arange(n)
    chunk = i // run
    start = (chunk * 37) % (cap - run + 1)
    return chunk.astype(np.int32), (start + i % run).astype(np.int32)


def _prepare_append(case, seed, st):
    g = _gen(seed)
    n, hq = case["n"], case["hq"]
    chunk, pos = _runs(case)
    n_chunks = int(chunk.max()) + 1
    pool, table = _new_pool(case, n_chunks, g)
    order = torch.randperm(n_chunks, device=DEV, generator=g).to(torch.int32)
    chunk_t, pos_t = torch.from_numpy(chunk).to(DEV), torch.from_numpy(pos).to(DEV)
    # a chunk's tokens stand one after the other in the conversation
    at = torch.randint(0, case["far"], (n_chunks,), device=DEV, generator=g)[chunk_t.long()].to(torch.int32) + pos_t
    if case["op"] == "append":                              # as a fused projection leaves them
        h, d = case["hkv"], case["d"]
        qkv = torch.randn((n, hq + 2 * h, d), device=DEV, generator=g)
        qkv[:, hq:] *= _channels((2 * h, d), g)
        qkv = qkv.to(_dtype(case))
        st.update(q=qkv[:, :hq], k=qkv[:, hq:hq + h], v=qkv[:, hq + h:])
        dim = case["dim"]
    else:                                                   # latent vector and key part from one projection
        lat = case["lat"]
        x = torch.randn((n, lat + ROPE), device=DEV, generator=g)
        x[:, :lat] *= _channels((lat,), g)
        x = x.to(_dtype(case))
        q = torch.randn((n, hq, 128 + ROPE), device=DEV, generator=g).to(_dtype(case))
        st.update(q=q[..., 128:], c=x[:, :lat], r=x[:, lat:])
        dim = ROPE
    freq = torch.pow(10000.0, -torch.arange(dim // 2, device=DEV, dtype=torch.float64) / (dim // 2)).float()
    st.update(pool=pool, table=table, chunk=order[chunk_t.long()], pos=pos_t, at=at, freq=freq)


def _prepare_latent(case, seed, st):
    g = _gen(seed)
    reqs = _sizes(case)
    n_chunks = max(1, sum(len(r["lens"]) for r in reqs))
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
    h, d, lat = case["hq"], case["d"], case["lat"]
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    q = torch.randn((new[-1], h, d + ROPE), device=DEV, generator=g).to(torch.bfloat16)
    w = (torch.randn((h, 2 * d, lat), device=DEV, generator=g) / math.sqrt(lat)).to(torch.bfloat16)
    st.update(pool=pool, table=table, ids=up(ids), tok_len=up(tok_len), q=q[..., :d], t=q[..., d:], w=w, reqs=reqs,
              scale=1.0 / math.sqrt(d + ROPE), q_offsets=None, prefix=None, chunk_ns=None, query_ns=None, ids_host=ids)
    if case["q"] != 1:
        st["q_offsets"] = up(np.asarray(new, np.int32))
    if case["prefix"]:
        st["prefix"] = torch.full((case["m"],), case["prefix"], dtype=torch.int32, device=DEV)
    if case["docs"]:
        st["chunk_ns"] = up(chunk_ns)
        st["query_ns"] = up(np.concatenate([_query_doc(r) for r in reqs]).astype(np.int32))


def prepare(case, seed):
    st = {"case": case}
    (_prepare_latent if case["op"] == "latent" else _prepare_append)(case, seed, st)
    if own:
        import paper_2607_05708_amd as pm
        fmt = {"bf16": pm.MEM_KV_BF16, "fp8": pm.MEM_KV_FP8, "fp4": pm.MEM_KV_FP4}[case["fmt"]]
        if case["op"] == "append":
            st["cache"] = pm.KvCache(st["pool"], st["table"], case["page_tokens"], case["hkv"], case["d"], fmt)
        else:
            st["cache"] = pm.LatentCache(st["pool"], st["table"], case["page_tokens"], case["lat"], ROPE, fmt)
        if case["op"] == "latent":
            need = pm.mem_latent_attend_workspace_bytes(st["cache"], case["m"], case["k"], st["q"].shape[0],
                                                        case["hq"], case["d"])
            st["ws"] = torch.empty(max(1, need), dtype=torch.uint8, device=DEV)
    return st


# ------------------------------------------- one pass

def run(st):
    case = st["case"]
    if own:
        import paper_2607_05708_amd as pm
        if case["op"] == "latent":
            return pm.mem_latent_attend(st["cache"], st["tok_len"], st["ids"], st["q"], st["t"], st["w"], st["scale"],
                                        q_offsets=st["q_offsets"], causal=case["causal"], window=case["window"],
                                        prefix_len=st["prefix"], chunk_ns=st["chunk_ns"], query_ns=st["query_ns"],
                                        workspace=st["ws"])
        queries = st["q"] if case["hq"] else None
        if case["op"] == "append":
            q = pm.mem_kv_append(st["cache"], st["k"], st["v"], st["chunk"], st["pos"], st["at"], st["freq"],
                                 q=queries, pairs=case["pairs"])
            return q, pm.mem_kv_read(st["cache"], st["chunk"], st["pos"], dtype=_dtype(case))
        q = pm.mem_latent_append(st["cache"], st["c"], st["r"], st["chunk"], st["pos"], st["at"], st["freq"],
                                 q=queries, pairs=case["pairs"])
        return q, pm.mem_latent_read(st["cache"], st["chunk"], st["pos"], dtype=_dtype(case))
    if case["op"] == "latent":
        return _plain_latent(st)
    t = case["page_tokens"]
    chunk, pos = st["chunk"].long(), st["pos"].long()
    page, slot = st["table"].long()[chunk, pos // t], pos % t
    turned = lambda x: _rotate(case, x, st["at"], st["freq"])  # noqa: E731
    q = turned(st["q"]).to(torch.bfloat16) if case["hq"] else None
    if case["op"] == "append":
        _store_kv(case, st["pool"], turned(st["k"]), st["v"].float(), page, slot)
        kept = _load_kv(case, st["pool"], page, slot)
    else:
        _store_latent(case, st["pool"], st["c"].float(), turned(st["r"]), page, slot)
        kept = _load_latent(case, st["pool"], page, slot)
    return q, tuple(x.to(_dtype(case)) for x in kept)


def _plain_latent(st):
    case = st["case"]
    t, h, d = case["page_tokens"], case["hq"], case["d"]
    q, tq, w = st["q"].float(), st["t"].float(), st["w"].float()
    out = torch.zeros((q.shape[0], h, d), device=DEV)
    table, slot_of = st["table"].long(), torch.arange(t * case["ppc"], device=DEV)
    few = case["q"] <= 16                                   # W goes to the queries' side
    if few:
        q = torch.matmul(q.transpose(0, 1), w[:, :d]).transpose(0, 1)
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
            c, kr = _load_latent(case, st["pool"], page, slot)
            kpos = torch.arange(ctx, device=DEV)
            if case["docs"]:
                kdoc = st["chunk_ns"][ids].repeat_interleave(torch.tensor(r["lens"], device=DEV), output_size=ctx)
            step = max(1, SCORES // (h * ctx))
            keys = c.T if few else torch.matmul(w[:, :d], c.T)      # [lat, ctx], or [h, d, ctx]
            for a in range(0, nq, step):
                b = min(a + step, nq)
                s = torch.matmul(q[q0 + a:q0 + b].transpose(0, 1), keys)
                s = (s + torch.matmul(tq[q0 + a:q0 + b].transpose(0, 1), kr.T)) * st["scale"]  # [h, b - a, ctx]
                dist = (torch.arange(a, b, device=DEV) + ctx - nq).unsqueeze(1) - kpos
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
                o = torch.matmul(torch.matmul(p, c), w[:, d:].transpose(1, 2))
                out[q0 + a:q0 + b] = torch.where(tot > 0, o / tot, torch.zeros_like(o)).transpose(0, 1)
        q0 += nq
    return out.to(torch.bfloat16)


# ------------------------------------------- the definition in 64 bits

def _nearest(case, x):
    """The value that a block of 32 stands for once it is held in the case's format, in 64 bits."""
    x = x.double()
    if case["fmt"] == "bf16":
        return _nearest_bf16(x)
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


def _nearest_bf16(x):
    _, ex = torch.frexp(x)
    step = ((ex.long() - 8 + 1023) << 52).view(torch.float64)       # 2^(ex - 8)
    return torch.where(x == 0, x, torch.round(x / step) * step)


def _turned(case, x, at, freq):
    """x [n, d] or [n, heads, d] rotated in 64 bits, as complex numbers."""
    n, half = x.shape[0], freq.numel()
    x = x.double()
    part = x[..., :2 * half]
    z = torch.complex(part[..., 0::2], part[..., 1::2]) if case["pairs"] else \
        torch.complex(part[..., :half], part[..., half:])
    phase = torch.outer(at.double(), freq.double()).view(n, *[1] * (x.dim() - 2), half)
    z = z * torch.polar(torch.ones_like(phase), phase)
    back = torch.view_as_real(z).flatten(-2) if case["pairs"] else torch.cat([z.real, z.imag], -1)
    return torch.cat([back, x[..., 2 * half:]], -1)


def _values(case, codes, scale):
    """64-bit values of codes, from each byte's fields."""
    if case["fmt"] == "bf16":
        return _bf16_values(codes)
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


def _bf16_values(codes):
    w = codes.contiguous().view(torch.int16).long() & 0xFFFF
    man, ex = (w & 127).double(), (w >> 7) & 255
    mag = torch.where(ex == 0, man / 128 * 2.0 ** -126, (1 + man / 128) * torch.exp2(ex.double() - 127))
    return torch.where(w >= 32768, -mag, mag)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] != "latent":
        turned = lambda x: _turned(case, x, st["at"], st["freq"])  # noqa: E731
        q = turned(st["q"]) if case["hq"] else None
        if case["op"] == "append":
            return q, (_nearest(case, turned(st["k"])), _nearest(case, st["v"]))
        return q, (_nearest(case, st["c"]), _nearest_bf16(turned(st["r"])))
    codes, parts, scales = _latent_views(case, st["pool"])
    t, h, d = case["page_tokens"], case["hq"], case["d"]
    out = torch.zeros((st["q"].shape[0], h, d), dtype=torch.float64, device=DEV)
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
        lat = _values(case, codes[pages], scales[pages]).flatten(0, 1)[keep]
        part = _bf16_values(parts[pages]).flatten(0, 1)[keep]
        label = np.repeat(np.asarray(r["doc"]), r["lens"])
        label, qdoc = torch.from_numpy(label).to(DEV), torch.from_numpy(_query_doc(r)).to(DEV)
        kpos = torch.arange(ctx, device=DEV, dtype=torch.float64)
        step = max(1, SCORES // (4 * ctx))
        for a in range(0, nq, step):
            b = min(a + step, nq)
            qpos = torch.arange(ctx - nq + a, ctx - nq + b, device=DEV, dtype=torch.float64)[:, None]
            hide = torch.zeros((b - a, ctx), dtype=torch.bool, device=DEV)
            if case["causal"]:
                hide |= kpos > qpos
            if case["window"]:
                hide |= kpos <= qpos - case["window"]
            if case["prefix"]:
                hide &= kpos >= case["prefix"]
            if case["docs"]:
                hide |= (label < 0) | (label != qdoc[a:b, None])
            for head in range(h):
                wk, wv = st["w"][head, :d].double(), st["w"][head, d:].double()
                mine = st["q"][q0 + a:q0 + b, head].double()
                s = (mine @ wk) @ lat.T if b - a < d else mine @ (lat @ wk.T).T
                s = (s + st["t"][q0 + a:q0 + b, head].double() @ part.T) / math.sqrt(d + ROPE)
                s[hide] = -math.inf
                z = torch.logsumexp(s, -1, keepdim=True)
                p = torch.exp(s - torch.where(torch.isinf(z), torch.zeros_like(z), z))
                out[q0 + a:q0 + b, head] = (p @ lat) @ wv.T
        q0 += nq
    return out
