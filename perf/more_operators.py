"""A paged cache of keys and values and the attention that reads it, as measurable cases.

Three operators, each in a plain form (elementary torch operations in 32 bits, rounded once at the end) and, with
``own`` set, as the calls a user makes of this package:

* ``put``     rows of keys and values into the pages of their tokens
* ``back``    the same into a cache of 8- or 4-bit integers with a scale for each token and head, and the whole cache
  read back:  scale = max|x| / L,  q = rint(x * L / max|x|),  value = q * scale,  L = 127 or 7
* ``get``     rows of tokens out of the pages
* ``attend``  attention of new (or kept) tokens over the cache:
      out[r, h] = sum_j p_j v_j,   p = softmax over the visible j of q[r, h] . k_j / sqrt(D)
  Visible to a query at position p are the keys before the sequence's length whose unit (a frame of `unit` tokens, or a
  token) is at most `back` units before the query's own and at most `ahead` after it (-1: any number).

Token t of a sequence lies in page table[sequence, t // page], row t % page, of a [pages, heads, page, D] pool.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LEVELS = {"i8": 127.0, "i4": 7.0}


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one conditioning token of a 72-wide-head model: nothing but latency
        dict(name="put one token", kind="put", B=1, rows=1, keys=256, heads=16, D=72, dtype="bf16", cache="bf16", page=32),
        # SD3-shaped Token Cache step: keys and values of the kept tokens replace those of the step before
        dict(name="put sd3 kept tokens", kind="put", B=2, rows=2560, keys=4096, heads=24, D=64, dtype="bf16", cache="bf16", page=64),
        # an odd number of kept tokens of a small 32-bit model into 4 bits, everything read back
        dict(name="back latte 4 bits fp32", kind="back", B=3, rows=333, keys=1001, heads=16, D=72, dtype="f32", cache="i4", page=48),
        # SVD-XT level 1: 25 frames written whole in 8 bits and read back
        dict(name="back svd video 8 bits", kind="back", B=25, rows=9216, keys=9216, heads=5, D=64, dtype="bf16", cache="i8", page=128),
        # some tokens of a 4-bit cache, in 32 bits
        dict(name="get latte odd rows", kind="get", B=2, rows=777, keys=4096, heads=16, D=72, dtype="f32", cache="i4", page=16),
        # one conditioning token over a text-sized cache: latency
        dict(name="attend one token", kind="attend", B=1, rows=1, keys=256, heads=16, kv=16, D=72, dtype="bf16", cache="bf16",
             page=32, unit=0, back=-1, ahead=-1, ragged=False, at="last"),
        # the 16x16 frame with one 64-wide head in fp32
        dict(name="attend tiny fp32", kind="attend", B=1, rows=256, keys=256, heads=1, kv=1, D=64, dtype="f32", cache="f32",
             page=64, unit=0, back=-1, ahead=-1, ragged=False, at="last"),
        # single tokens of many requests over long caches of 8 bits, keys shared by four heads
        dict(name="attend single long 8 bits", kind="attend", B=16, rows=1, keys=32768, heads=32, kv=8, D=128, dtype="bf16",
             cache="i8", page=64, unit=0, back=-1, ahead=-1, ragged=True, at="last"),
        # chunks of very different lengths behind one another, each token seeing those before it, odd pages
        dict(name="attend ragged chunks", kind="attend", B=6, rows=1500, keys=5000, heads=8, kv=2, D=128, dtype="bf16",
             cache="bf16", page=48, unit=1, back=-1, ahead=0, ragged=True, at="last"),
        # Latte-shaped video (16 frames of 16x16), frames seeing themselves and earlier ones, half of the tokens kept
        dict(name="attend latte frames 8 bits", kind="attend", B=2, rows=2048, keys=4096, heads=16, kv=16, D=72, dtype="bf16",
             cache="i8", page=64, unit=256, back=-1, ahead=0, ragged=False, at="kept"),
        # SD3-shaped attention block under Token Cache: the kept tokens over all tokens
        dict(name="attend sd3 kept tokens", kind="attend", B=2, rows=2560, keys=4096, heads=24, kv=24, D=64, dtype="bf16",
             cache="bf16", page=64, unit=0, back=-1, ahead=-1, ragged=False, at="kept"),
        # SVD-XT level 1: half of the tokens of each of 25 frames over all tokens of the frame
        dict(name="attend svd frames", kind="attend", B=25, rows=4608, keys=9216, heads=5, kv=5, D=64, dtype="bf16",
             cache="bf16", page=128, unit=0, back=-1, ahead=-1, ragged=False, at="kept"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["put", "back", "get", "attend", "attend", "attend"])
    D, dtype, page = 8 * rng.choice([4, 5, 8, 8, 9, 10, 16]), rng.choice(["bf16", "bf16", "f32"]), 16 * rng.randint(1, 9)
    while True:
        B, keys, heads = _log(rng, 1, 32), _log(rng, 1, 32768), rng.choice([1, 2, 5, 8, 16, 24])
        rows = min(keys, _log(rng, 1, 9216))
        if kind != "attend":
            if B * keys * heads * D > 25 * 9216 * 5 * 64:
                continue
            cache = {"put": dtype, "back": rng.choice(["i8", "i4"]), "get": rng.choice([dtype, "i8", "i4"])}[kind]
            return dict(kind=kind, B=B, rows=rows, keys=keys, heads=heads, D=D, dtype=dtype, cache=cache, page=page)
        group = rng.choice([1, 1, 2, 4, 8])
        flops = 4.0 * B * rows * keys * heads * group * D
        if flops > (1 if dtype == "bf16" else 0.02) * 4.0 * 25 * 4608 * 9216 * 5 * 64 or B * keys * heads * D > 16 * 32768 * 8 * 128:
            continue
        unit = rng.choice([0, 1, _log(rng, 2, 1024)])
        ahead = rng.choice([0, 0, 1, -1]) if unit else -1
        back = rng.choice([-1, -1, 0, 3]) if unit else -1
        return dict(kind=kind, B=B, rows=rows, keys=keys, heads=heads * group, kv=heads, D=D, dtype=dtype,
                    cache=rng.choice([dtype, dtype, "i8", "i4"]), page=page, unit=unit, back=back, ahead=ahead,
                    ragged=rng.random() < 0.4, at=rng.choice(["last", "kept"]))


def _lengths(c):
    """(new rows, keys) of each sequence: all alike, or from one to the most, spread by the golden ratio."""
    out = []
    for s in range(c["B"]):
        rows, keys = c["rows"], c["keys"]
        if c.get("ragged"):
            f = (0.5 + 0.6180339887 * s) % 1.0
            rows, keys = (rows, keys) if s == c["B"] // 2 else (max(1, int(rows * f * f)), max(1, int(keys * f)))
            rows = min(rows, keys)
        out.append((rows, keys))
    return out


# ---- inputs --------------------------------------------------------------------------------------------------------
def _normal(gen, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _levels(x, L):
    """(whole numbers, scales) of the last axis; in 64 bits, for values next to a rounding border"""
    x = x.double()
    most = x.abs().amax(-1, keepdim=True)
    return (x * L / most).round().to(torch.int8), (most / L).squeeze(-1).float()


def _pack(q, cache):
    """4-bit numbers two to a byte, the first one low"""
    if cache == "i8":
        return q
    q = q.to(torch.uint8) & 15
    return q[..., 0::2] | (q[..., 1::2] << 4)


def _unpack(q, cache):
    if cache == "i8":
        return q
    q = torch.stack([q & 15, q >> 4], -1).flatten(-2).to(torch.int8)
    return torch.where(q > 7, q - 16, q)


def _pool(gen, c, heads, pages):
    """(pool, scales or None) with values a program wrote earlier"""
    shape = (pages, heads, c["page"], c["D"])
    if c["cache"] not in LEVELS:
        return torch.randn(shape, generator=gen, device="cuda", dtype=DTYPES[c["cache"]]), None
    L = LEVELS[c["cache"]]
    q = torch.randint(-int(L), int(L) + 1, shape, generator=gen, device="cuda", dtype=torch.int8)
    # (rows of that many levels spread evenly have an rms of L / sqrt(3): values of about 1)
    scale = (torch.rand(shape[:-1], generator=gen, device="cuda") + 0.5) * (math.sqrt(3.0) / L)
    return _pack(q, c["cache"]), scale


def _kept(gen, B, keys, rows):
    order = torch.rand(B, keys, generator=gen, device="cuda").argsort(1)[:, :rows].sort(1).values
    return (order + torch.arange(B, device="cuda")[:, None] * keys).reshape(-1).to(torch.int32)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, per_seq, dt, D = c["B"], -(-c["keys"] // c["page"]), DTYPES[c["dtype"]], c["D"]
    heads = c["kv"] if c["kind"] == "attend" else c["heads"]
    pages = B * per_seq
    s = {"case": c, "idx": None, "kv_len": None, "q_start": None}
    s["table"] = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32).view(B, per_seq)
    s["k_pool"], s["k_scale"] = _pool(gen, c, heads, pages)
    s["v_pool"], s["v_scale"] = _pool(gen, c, heads, pages)
    if c["kind"] != "attend":
        n = B * c["rows"]
        s["idx"] = _kept(gen, B, c["keys"], c["rows"])
        # keys as oc_rope leaves them, [batch, heads, rows, D]; values where the projection wrote them
        s["k"] = _normal(gen, B, heads, c["rows"], D, dtype=dt)
        s["v"] = _normal(gen, n, 3 * heads, D, dtype=dt)[:, 2 * heads:]
        if c["kind"] == "back":
            s["k_out"], s["v_out"] = (torch.empty(B * c["keys"], heads, D, dtype=dt, device="cuda") for _ in range(2))
        if c["kind"] == "get":
            s["k_out"], s["v_out"] = (torch.empty(n, heads, D, dtype=dt, device="cuda") for _ in range(2))
        return s
    s["lengths"] = _lengths(c)
    if c["ragged"]:
        starts = [0]
        for rows, _ in s["lengths"]:
            starts.append(starts[-1] + rows)
        n = starts[-1]
        s["q_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["q"] = _normal(gen, n, c["heads"], D, dtype=dt)
    else:
        n = B * c["rows"]
        s["q"] = _normal(gen, B, c["heads"], c["rows"], D, dtype=dt)
    s["kv_len"] = torch.tensor([k for _, k in s["lengths"]], dtype=torch.int32, device="cuda")
    if c["at"] == "kept":
        s["idx"] = torch.cat([_kept(gen, 1, keys, rows) + i * c["keys"] for i, (rows, keys) in enumerate(s["lengths"])])
    s["out"] = torch.empty(n, c["heads"], D, dtype=dt, device="cuda")
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _place(c, s, idx):
    """(page, row of the page) of tokens"""
    seq, at = idx.long() // c["keys"], idx.long() % c["keys"]
    return s["table"].long()[seq, at // c["page"]], at % c["page"]


def _read(c, pool, scale, page, row):
    """rows [tokens, heads, D] in 32 bits"""
    x = pool[page, :, row]
    if scale is None:
        return x.float()
    return _unpack(x, c["cache"]).float() * scale[page, :, row].unsqueeze(-1)


def _write(c, pool, scale, page, row, x):
    if scale is None:
        pool[page, :, row] = x
        return
    q, sc = _levels(x, LEVELS[c["cache"]])
    pool[page, :, row] = _pack(q, c["cache"])
    scale[page, :, row] = sc


def _plain_rows(c, s):
    page, row = _place(c, s, s["idx"])
    if c["kind"] == "get":
        return {"k": _read(c, s["k_pool"], s["k_scale"], page, row).to(DTYPES[c["dtype"]]),
                "v": _read(c, s["v_pool"], s["v_scale"], page, row).to(DTYPES[c["dtype"]])}
    _write(c, s["k_pool"], s["k_scale"], page, row, s["k"].transpose(1, 2).flatten(0, 1))
    _write(c, s["v_pool"], s["v_scale"], page, row, s["v"])
    if c["kind"] == "put":
        return {"k": s["k_pool"], "v": s["v_pool"]}
    page, row = _place(c, s, torch.arange(c["B"] * c["keys"], device="cuda"))
    return {"k": _read(c, s["k_pool"], s["k_scale"], page, row).to(DTYPES[c["dtype"]]),
            "v": _read(c, s["v_pool"], s["v_scale"], page, row).to(DTYPES[c["dtype"]])}


def _plain_attend(c, s):
    D, group, outs, at = c["D"], c["heads"] // c["kv"], [], 0
    for i, (rows, keys) in enumerate(s["lengths"]):
        page, row = _place(c, s, torch.arange(keys, device="cuda") + i * c["keys"])
        k = _read(c, s["k_pool"], s["k_scale"], page, row).permute(1, 2, 0)                     # [kv, D, keys]
        v = _read(c, s["v_pool"], s["v_scale"], page, row).transpose(0, 1)                      # [kv, keys, D]
        q = s["q"][at:at + rows].transpose(0, 1) if c["ragged"] else s["q"][i]                  # [heads, rows, D]
        pos = (s["idx"][at:at + rows].long() - i * c["keys"] if s["idx"] is not None
               else torch.arange(rows, device="cuda") + keys - rows)
        hidden = None
        if c["unit"]:
            apart = torch.arange(keys, device="cuda")[None] // c["unit"] - pos[:, None] // c["unit"]
            hidden = torch.zeros_like(apart, dtype=torch.bool)
            if c["ahead"] >= 0:
                hidden |= apart > c["ahead"]
            if c["back"] >= 0:
                hidden |= apart < -c["back"]
        got = []
        for h in range(c["kv"]):                                     # the heads that share a key-value head at a time
            x = (q[h * group:(h + 1) * group].float() @ k[h]) * (1.0 / math.sqrt(D))
            if hidden is not None:
                x = x.masked_fill(hidden, -math.inf)
            most = x.amax(-1, keepdim=True)
            x = torch.exp(x - torch.where(most == -math.inf, torch.zeros_like(most), most))
            total = x.sum(-1, keepdim=True)
            o = x @ v[h]
            got.append(torch.where(total > 0, o / total, torch.zeros_like(o)).to(DTYPES[c["dtype"]]))
        outs.append(torch.cat(got).transpose(0, 1))
        at += rows
    return torch.cat(outs)


# ---- this package's calls ------------------------------------------------------------------------------------------
_handle = None


def _package():
    """The package's binding and a context on the current device, made once for the process."""
    global _handle
    if _handle is None:
        from paper_2607_23844_b200 import omnicache as oc
        _handle = oc, oc.Context(torch.cuda.current_device())
    return _handle


def _cache_desc(c, oc, heads):
    types = {"bf16": oc.DTYPE_BF16, "f32": oc.DTYPE_F32, "i8": oc.DTYPE_I8, "i4": oc.DTYPE_I4}
    return oc.kv_desc(types[c["cache"]], heads, c["D"], c["B"], c["keys"], page_rows=c["page"])


def _own_rows(c, s, oc, ctx):
    dt = {"bf16": oc.DTYPE_BF16, "f32": oc.DTYPE_F32}[c["dtype"]]
    if "cache_desc" not in s:
        s["cache_desc"] = _cache_desc(c, oc, c["heads"])
        s["in_desc"] = oc.kv_rows(s["cache_desc"], c["B"] * c["rows"], dt, k=s["k"], v=s["v"])
        if "k_out" in s:
            s["out_desc"] = oc.kv_rows(s["cache_desc"], s["k_out"].shape[0], dt, k=s["k_out"], v=s["v_out"])
    pools = dict(k_scale=s["k_scale"], v_scale=s["v_scale"], page_table=s["table"])
    if c["kind"] != "get":
        ctx.kv_put(s["cache_desc"], s["in_desc"], s["k"], s["k_pool"], s["v"], s["v_pool"], idx=s["idx"], **pools)
        if c["kind"] == "put":
            return {"k": s["k_pool"], "v": s["v_pool"]}
    ctx.kv_get(s["cache_desc"], s["out_desc"], s["k_pool"], s["k_out"], s["v_pool"], s["v_out"],
               idx=s["idx"] if c["kind"] == "get" else None, **pools)
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attend(c, s, oc, ctx):
    if "desc" not in s:
        s["cache_desc"] = _cache_desc(c, oc, c["kv"])
        s["desc"] = oc.attention_desc(s["cache_desc"], s["out"].shape[0], {"bf16": oc.DTYPE_BF16, "f32": oc.DTYPE_F32}[c["dtype"]],
                                      c["heads"], 1.0 / math.sqrt(c["D"]), rows_per_batch=c["rows"], unit=c["unit"],
                                      back=c["back"], ahead=c["ahead"], q=s["q"], out=s["out"])
    ctx.attention(s["cache_desc"], s["desc"], s["q"], s["k_pool"], s["v_pool"], s["out"], k_scale=s["k_scale"],
                  v_scale=s["v_scale"], page_table=s["table"], kv_len=s["kv_len"], q_start=s["q_start"], idx=s["idx"])
    return s["out"]


def run(state):
    c = state["case"]
    if own:
        return (_own_attend if c["kind"] == "attend" else _own_rows)(c, state, *_package())
    return (_plain_attend if c["kind"] == "attend" else _plain_rows)(c, state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def _row_bytes(c):
    """bytes of a cached row of one head"""
    return {"f32": 4 * c["D"], "bf16": 2 * c["D"], "i8": c["D"] + 4, "i4": c["D"] // 2 + 4}[c["cache"]]


def _visible(c, rows, keys):
    """(pairs of query and visible key, keys that some query sees); kept tokens taken as evenly spread"""
    if not c["unit"]:
        return rows * keys, keys
    pairs, first, last = 0, keys, 0
    for i in range(rows):
        u = (keys - rows + i if c["at"] == "last" else int((i + 0.5) * keys / rows)) // c["unit"]
        lo = 0 if c["back"] < 0 else max(0, (u - c["back"]) * c["unit"])
        hi = keys if c["ahead"] < 0 else min(keys, (u + c["ahead"] + 1) * c["unit"])
        pairs, first, last = pairs + max(0, hi - lo), min(first, lo), max(last, hi)
    return pairs, max(0, last - first)


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "attend":
        got = [(rows,) + _visible(c, rows, keys) for rows, keys in _lengths(c)]
        rows, pairs, seen = (sum(g[i] for g in got) for i in range(3))
        return {"bytes": 2 * rows * c["heads"] * c["D"] * e + 2 * seen * c["kv"] * _row_bytes(c) + (4 * rows if c["at"] == "kept" else 0),
                "flops": 4 * pairs * c["heads"] * c["D"]}
    heads, n = 2 * c["heads"], c["B"] * c["rows"]                     # of keys and of values
    moved = n * heads * (c["D"] * e + _row_bytes(c)) + 4 * n
    flops = 0
    if c["kind"] == "back":
        moved += c["B"] * c["keys"] * heads * (c["D"] * e + _row_bytes(c))
        flops = heads * c["D"] * (3 * n + c["B"] * c["keys"])
    elif c["kind"] == "get" and c["cache"] in LEVELS:
        flops = heads * c["D"] * n
    return {"bytes": moved, "flops": flops}


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------
def _exact_cache(c, s, m):
    """The whole cache as [sequences, tokens, heads, D] of the values that it holds"""
    pool, scale = s[m + "_pool"], s[m + "_scale"]
    if scale is None:
        x = pool.double()
    else:
        if c["cache"] == "i4":
            low, high = (pool.int() << 28) >> 28, (pool.int() << 24) >> 28
            pool = torch.empty(pool.shape[:-1] + (c["D"],), dtype=torch.int32, device="cuda")
            pool[..., ::2], pool[..., 1::2] = low, high
        x = pool.double() * scale.double()[..., None]
    x = torch.index_select(x, 0, s["table"].reshape(-1).long()).permute(0, 2, 1, 3)             # pages in order
    return x.reshape(c["B"], -1, x.shape[2], c["D"])[:, : c["keys"]]


def _exact_rows(c, s):
    got = {}
    for m in "kv":
        cache = _exact_cache(c, s, m).reshape(-1, c["heads"], c["D"])
        if c["kind"] == "get":
            got[m] = cache.index_select(0, s["idx"].long())
            continue
        x = s[m].double()
        if m == "k":
            x = x.permute(0, 2, 1, 3).reshape(-1, c["heads"], c["D"])
        if c["cache"] in LEVELS:
            step = x.abs().max(-1, keepdim=True).values / LEVELS[c["cache"]]
            x = torch.round(x / step) * step
        cache = cache.index_copy(0, s["idx"].long(), x)
        if c["kind"] == "put":                                       # the pool's own order, rows behind a sequence kept
            whole = s[m + "_pool"].double().permute(0, 2, 1, 3).contiguous()
            seq = torch.arange(c["B"] * c["keys"], device="cuda")
            seq, at = torch.div(seq, c["keys"], rounding_mode="floor"), seq % c["keys"]
            whole[s["table"].long()[seq, torch.div(at, c["page"], rounding_mode="floor")], at % c["page"]] = cache
            cache = whole.permute(0, 2, 1, 3)
        got[m] = cache
    return got


def _exact_attend(c, s):
    k_all, v_all = _exact_cache(c, s, "k"), _exact_cache(c, s, "v")
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for i, (rows, keys) in enumerate(s["lengths"]):
        where = torch.arange(keys - rows, keys, device="cuda") if s["idx"] is None else s["idx"][at:at + rows].long() % c["keys"]
        j = torch.arange(keys, device="cuda")
        seen = None
        if c["unit"]:
            mine, theirs = (where // c["unit"]).unsqueeze(1), (j // c["unit"]).unsqueeze(0)
            seen = (theirs <= (mine + c["ahead"] if c["ahead"] >= 0 else keys)) & (theirs >= (mine - c["back"] if c["back"] >= 0 else 0))
        for h in range(c["heads"]):
            q = (s["q"][at:at + rows, h] if c["ragged"] else s["q"][i, h]).double()
            hk = h * c["kv"] // c["heads"]
            score = torch.mm(q, k_all[i, :keys, hk].t()).div_(math.sqrt(c["D"]))
            if seen is not None:
                score = torch.where(seen, score, torch.full_like(score, -torch.inf))
            p = (score - torch.logsumexp(score, 1, keepdim=True)).exp_()
            if seen is not None:
                p = torch.where(seen, p, torch.zeros_like(p))
            out[at:at + rows, h] = torch.mm(p, v_all[i, :keys, hk])
        at += rows
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_attend(case, s) if case["kind"] == "attend" else _exact_rows(case, s)
