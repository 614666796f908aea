"""The operators around and inside a transformer block whose tokens are partly cached, as measurable cases.

Three operators, each in a plain form (elementary torch operations in 32 bits, rounded once at the end) and, with
``own`` set, as the calls a user makes of this package:

* ``block``  restore of the cached rows, norm after a block, gate and residual scale, norm before the next block and
  its modulation, with the rows of the next block written in their dense order.  For row i of unit u, s = slot_of[u]:
      v = z[s] if s >= 0 else cache[i];  cache[i] = v;  r = a * x[i] + gate * post(v);  out[i] = r
      h[s] = pre(r) * (1 + scale) + shift                                   (only where s >= 0)
* ``rope``   rotary positions with up to three axes (time, height, width) on queries and keys read out of one packed
  projection, the position of a dense row being that of the token it was gathered from, after an optional RMS norm of
  each head.
* ``int8``   matrix product in 8-bit integers, one scale for each token and one for each output channel:
      out[m, n] = a_scale[m] * w_scale[n] * sum_k a[m, k] * w[n, k] + bias[n]
  with the 8-bit rows at hand ("q"), made from 16-bit rows in the call ("rows"), or made by the norm and modulation
  of a residual stream in the call ("norm").
"""
import math

import torch

own = False

EPS = 1e-6
THETA = 10000.0
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one conditioning token of the Latte width in front of its first block: nothing but latency
        dict(name="block one token", kind="block", B=1, T=1, H=1, W=1, C=1152, dtype="bf16", param="f32", post="none",
             pre="layer", z=False, mod=True, gate=False, res=1.0, reuse=0.0, unit="token"),
        # SD3-shaped attention block under Token Cache: half of the candidates come from the cache
        dict(name="block sd3 token cache", kind="block", B=2, T=1, H=64, W=64, C=1536, dtype="bf16", param="bf16",
             post="rms", pre="layer", z=True, mod=True, gate=True, res=1.0, reuse=0.5, unit="token"),
        # an odd number of fp32 rows of an odd width, no cache: a block of a small 32-bit model
        dict(name="block odd fp32", kind="block", B=1, T=1, H=13, W=77, C=644, dtype="f32", param="f32", post="layer",
             pre="rms", z=True, mod=False, gate=True, res=0.5, reuse=0.0, unit="token"),
        # SVD-XT level 1 under Frame Cache: whole frames come from the cache, one modulation for each frame
        dict(name="block svd frame cache", kind="block", B=1, T=25, H=72, W=128, C=320, dtype="bf16", param="f32",
             post="rms", pre="layer", z=True, mod=True, gate=True, res=1.0, reuse=0.5, unit="frame"),
        # the tiny 16x16 frame with one 64-wide head in fp32
        dict(name="rope tiny fp32", kind="rope", B=1, T=1, H=16, W=16, heads=1, kv=1, D=64, axes="0,32,32", pairs="adjacent",
             dtype="f32", norm=False, keep=1.0, at="grid", inverse=False),
        # SD3-shaped kept tokens, head norm and rotation of q and k in one pass
        dict(name="rope sd3 kept tokens", kind="rope", B=2, T=1, H=64, W=64, heads=24, kv=24, D=64, axes="0,32,32",
             pairs="adjacent", dtype="bf16", norm=True, keep=0.625, at="kept", inverse=False),
        # Latte-shaped video with 72-wide heads (36 pairs: not a whole number of 16-byte words), rotated back, positions
        # given row by row, keys shared by four heads
        dict(name="rope latte 72 wide", kind="rope", B=1, T=16, H=16, W=16, heads=16, kv=4, D=72, axes="24,24,24",
             pairs="halves", dtype="bf16", norm=False, keep=1.0, at="rows", inverse=True),
        # SVD-XT level 1 video: every token of 25 frames, three axes
        dict(name="rope svd video", kind="rope", B=1, T=25, H=72, W=128, heads=5, kv=5, D=64, axes="16,24,24",
             pairs="halves", dtype="bf16", norm=True, keep=1.0, at="grid", inverse=False),
        # the modulation projection of a classifier-free-guidance pair: two rows against the whole weight matrix
        dict(name="int8 modulation pair", kind="int8", form="rows", M=2, K=1536, N=9216, bias=True, out="bf16"),
        # text-sized odd rows and widths, 32-bit outputs
        dict(name="int8 odd fp32 out", kind="int8", form="q", M=333, K=1168, N=1159, bias=True, out="f32"),
        # q, k, v of the kept tokens of an SD3-shaped layer, from the residual stream
        dict(name="int8 sd3 qkv from norm", kind="int8", form="norm", M=5120, K=1536, N=4608, bias=True, out="bf16"),
        # feed-forward expansion of SVD-XT level 2 (gated: twice four times the width) over 25 frames
        dict(name="int8 svd feed-forward", kind="int8", form="q", M=57600, K=640, N=5120, bias=False, out="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["block", "rope", "int8"])
    if kind == "int8":
        while True:
            M, N, K = _log(rng, 1, 60000), _log(rng, 16, 10000), 16 * _log(rng, 2, 400)
            if M * N * K <= 57600 * 5120 * 640 and M * N <= 57600 * 5120 and 3072 not in (M, N, K):
                break
        form = rng.choice(["q", "rows", "norm"])
        return dict(kind=kind, form=form, M=M, K=K, N=N, bias=rng.random() < 0.5,
                    out=rng.choice(["bf16", "f32"]) if form == "q" else "bf16")
    while True:
        B, T, H, W = rng.choice([1, 2, 3]), _log(rng, 1, 25), _log(rng, 1, 72), _log(rng, 1, 128)
        n = B * T * H * W
        if kind == "block":
            dtype = rng.choice(["bf16", "f32"])
            C = (8 if dtype == "bf16" else 4) * _log(rng, 4, 512)
            if n * C * (2 if dtype == "bf16" else 4) > 25 * 72 * 128 * 320 * 2 or 3072 in (n, C, H, W):
                continue
            z = rng.random() < 0.8
            return dict(kind=kind, B=B, T=T, H=H, W=W, C=C, dtype=dtype, param=rng.choice(["bf16", "f32"]),
                        post=rng.choice(["none", "rms", "layer"]) if z else "none", pre=rng.choice(["rms", "layer"]),
                        z=z, mod=rng.random() < 0.7, gate=z and rng.random() < 0.7, res=rng.choice([1.0, 0.5]),
                        reuse=rng.choice([0.0, 0.25, 0.5, 0.75]), unit=rng.choice(["token", "frame"]))
        D = 8 * rng.choice([4, 5, 8, 9, 10, 16])
        kv = rng.choice([1, 2, 4, 5])
        heads = kv * rng.choice([1, 2, 4])
        dtype = rng.choice(["bf16", "f32"])
        if n * (heads + 2 * kv) * D * (2 if dtype == "bf16" else 4) > 25 * 72 * 128 * 15 * 64 * 2 or n == 3072:
            continue
        a = 2 * rng.randint(1, D // 8)
        axes = rng.choice([(0, D // 2 // 2 * 2, D - D // 2 // 2 * 2), (D - 4 * (a // 2), 2 * (a // 2), 2 * (a // 2)), (a, a, a)])
        at = rng.choice(["grid", "kept", "rows"])
        return dict(kind=kind, B=B, T=T, H=H, W=W, heads=heads, kv=kv, D=D, axes="%d,%d,%d" % axes,
                    pairs=rng.choice(["adjacent", "halves"]), dtype=dtype, norm=rng.random() < 0.5,
                    keep=rng.choice([0.25, 0.5, 0.625]) if at == "kept" else 1.0, at=at, inverse=rng.random() < 0.25)


# ---- inputs --------------------------------------------------------------------------------------------------------
def _selection(groups, units, n_keep, gen):
    """A selection of n_keep units in each group: (kept units in ascending order, slot of each unit or -1)."""
    order = torch.rand(groups, units, generator=gen, device="cuda").argsort(1)[:, :n_keep].sort(1).values
    kept = (order + torch.arange(groups, device="cuda")[:, None] * units).reshape(-1)
    slot = torch.full((groups * units,), -1, dtype=torch.int32, device="cuda")
    slot[kept] = torch.arange(kept.numel(), dtype=torch.int32, device="cuda")
    return kept.to(torch.int32), slot


def _normal(gen, *shape, std=1.0, mean=0.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)


def _block_plan(c):
    """(groups of the selection, units in each, rows of a unit, kept units in each)"""
    frames, rows = c["B"] * c["T"], c["H"] * c["W"]
    groups, units, unit_rows = (frames, rows, 1) if c["unit"] == "token" else (c["B"], c["T"], rows)
    reps = -(-units // (4 if c["unit"] == "token" else 2))
    return groups, units, unit_rows, units - int(c["reuse"] * (units - reps))


def _prepare_block(c, gen):
    groups, units, unit_rows, keep = _block_plan(c)
    n, C, dt, pt = groups * units * unit_rows, c["C"], DTYPES[c["dtype"]], DTYPES[c["param"]]
    s = {"kept": None, "slot_of": None, "z": None, "cache": None, "out": None}
    x = torch.randn(n, C, generator=gen, device="cuda").mul_(2.0)
    x += torch.randn(n, 1, generator=gen, device="cuda")                 # residual streams are not centred
    s["x"] = x.to(dt)
    del x
    n_dense = groups * keep * unit_rows
    if c["reuse"] > 0:
        s["kept"], s["slot_of"] = _selection(groups, units, keep, gen)
    if c["z"]:
        s["z"] = _normal(gen, n_dense, C, dtype=dt)
        s["out"] = torch.empty_like(s["x"])
        if c["reuse"] > 0:
            s["cache"] = _normal(gen, n, C, dtype=dt)
    s["h"] = torch.empty(n_dense, C, dtype=dt, device="cuda")
    # one vector of shift, scale and gate for each frame, as the modulation projection leaves them
    mod = _normal(gen, c["B"] * c["T"], 3 * C, std=0.3, dtype=pt)
    s["mod"] = mod
    s["shift"], s["scale"] = (mod[:, :C], mod[:, C:2 * C]) if c["mod"] else (None, None)
    s["gate"] = mod[:, 2 * C:] if c["gate"] else None
    s["post_w"] = _normal(gen, C, std=0.1, mean=1.0, dtype=pt) if c["post"] != "none" else None
    s["pre_w"] = _normal(gen, C, std=0.1, mean=1.0, dtype=pt) if c["pre"] == "rms" else None
    return s


def _axes(c):
    return [int(v) for v in c["axes"].split(",")]


def _rope_rows(c):
    per = c["T"] * c["H"] * c["W"]
    return c["B"], max(1, int(c["keep"] * per))


def _prepare_rope(c, gen):
    B, n = _rope_rows(c)
    dt, D, wide = DTYPES[c["dtype"]], c["D"], (c["heads"] + 2 * c["kv"]) * c["D"]
    s = {"qkv": _normal(gen, B * n, wide, dtype=dt), "idx": None, "pos": None, "q_w": None, "k_w": None}
    s["q"] = s["qkv"][:, : c["heads"] * D].view(B * n, c["heads"], D)
    s["k"] = s["qkv"][:, c["heads"] * D: (c["heads"] + c["kv"]) * D].view(B * n, c["kv"], D)
    if c["at"] == "kept":
        s["idx"] = _selection(B, c["T"] * c["H"] * c["W"], n, gen)[0]
    if c["at"] == "rows":
        s["pos"] = torch.stack([torch.randint(0, m, (B * n,), generator=gen, device="cuda") for m in (c["T"], c["H"], c["W"])], 1).to(torch.int32)
    if c["norm"]:
        s["q_w"], s["k_w"] = _normal(gen, D, std=0.1, mean=1.0), _normal(gen, D, std=0.1, mean=1.0)
    # cos, sin of every position of every axis: [positions of the axis][its pairs][2], the axes one after the other
    s["table"] = torch.cat([torch.stack([f(_angles(m, d)) for f in (torch.cos, torch.sin)], -1).reshape(-1)
                            for m, d in zip((c["T"], c["H"], c["W"]), _axes(c))]).float().cuda()
    s["q_out"] = torch.empty(B, c["heads"], n, D, dtype=dt, device="cuda")
    s["k_out"] = torch.empty(B, c["kv"], n, D, dtype=dt, device="cuda")
    return s


def _angles(positions, dims):
    return torch.arange(positions, dtype=torch.float64)[:, None] * THETA ** (-torch.arange(0, dims, 2, dtype=torch.float64) / max(dims, 1))


def _prepare_int8(c, gen):
    M, K, N = c["M"], c["K"], c["N"]
    s = {"bias": _normal(gen, N, std=0.5) if c["bias"] else None}
    s["w"] = torch.randn(N, K, generator=gen, device="cuda").mul_(36.0).round_().clamp_(-127, 127).to(torch.int8)
    s["w_scale"] = (torch.rand(N, generator=gen, device="cuda") + 0.5) / (36.0 * math.sqrt(K))
    if c["form"] == "q":
        s["a"] = torch.randn(M, K, generator=gen, device="cuda").mul_(36.0).round_().clamp_(-127, 127).to(torch.int8)
        s["a_scale"] = (torch.rand(M, generator=gen, device="cuda") + 0.5) / 36.0
    else:
        s["x"] = _normal(gen, M, K, std=2.0, dtype=torch.bfloat16)
        s["a"] = torch.empty(M, K, dtype=torch.int8, device="cuda")
        s["a_scale"] = torch.empty(M, device="cuda")
    if c["form"] == "norm":
        s["mod"] = _normal(gen, 1, 2 * K, std=0.3, dtype=torch.bfloat16)
        s["shift"], s["scale"] = s["mod"][:, :K], s["mod"][:, K:]
    s["out"] = torch.empty(M, N, dtype=DTYPES[c["out"]], device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"block": _prepare_block, "rope": _prepare_rope, "int8": _prepare_int8}[case["kind"]](case, gen)
    s["case"] = case
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _norm(v, how, w):
    if how == "none":
        return v
    if how == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v if w is None else v * w.float()


def _rows_of_units(units, unit_rows):
    """Row numbers of whole units."""
    return (units.long()[:, None] * unit_rows + torch.arange(unit_rows, device=units.device)).reshape(-1)


def _plain_block(c, s):
    unit_rows = _block_plan(c)[2]
    r, new_cache, out = s["x"].float(), None, None
    frames, n, C = c["B"] * c["T"], r.shape[0], c["C"]
    if s["z"] is not None:
        v = s["z"]
        if s["cache"] is not None:
            v = s["cache"].index_copy(0, _rows_of_units(s["kept"], unit_rows), v)
            new_cache = v
        t = _norm(v.float(), c["post"], s["post_w"])
        if s["gate"] is not None:
            t = (t.view(frames, -1, C) * s["gate"].float()[:, None]).view(n, C)
        r = c["res"] * r + t
        out = r.to(s["x"].dtype)
    h = _norm(r, c["pre"], s["pre_w"])
    if c["mod"]:
        h = (h.view(frames, -1, C) * (1 + s["scale"].float()[:, None]) + s["shift"].float()[:, None]).view(n, C)
    if s["kept"] is not None:
        h = h[_rows_of_units(s["kept"], unit_rows)]
    return {"out": out, "cache": new_cache, "h": h.to(s["x"].dtype)}


def _plain_positions(c, s, n_rows):
    if s["pos"] is not None:
        return s["pos"].long().unbind(1)
    i = s["idx"].long() if s["idx"] is not None else torch.arange(n_rows, device="cuda")
    i = i % (c["T"] * c["H"] * c["W"])
    return i // (c["H"] * c["W"]), i // c["W"] % c["H"], i % c["W"]


def _plain_rotate(v, w, cos, sin, c):
    v, P = v.float(), cos.shape[-1]
    if w is not None:
        v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * w
    first, second = (v[..., 0:2 * P:2], v[..., 1:2 * P:2]) if c["pairs"] == "adjacent" else (v[..., :P], v[..., P:2 * P])
    turned = first * cos - second * sin, second * cos + first * sin
    turned = torch.stack(turned, -1).flatten(-2) if c["pairs"] == "adjacent" else torch.cat(turned, -1)
    return torch.cat([turned, v[..., 2 * P:]], -1)


def _plain_rope(c, s):
    B, n = _rope_rows(c)
    sizes = [m * d // 2 for m, d in zip((c["T"], c["H"], c["W"]), _axes(c))]
    parts = [t.view(m, d // 2, 2)[p] for t, m, d, p in zip((s["table"].view(-1, 2)).split(sizes), (c["T"], c["H"], c["W"]), _axes(c),
                                                          _plain_positions(c, s, B * n))]
    cos, sin = torch.cat(parts, 1).unsqueeze(1).unbind(-1)
    sin = -sin if c["inverse"] else sin
    q, k = (_plain_rotate(s[m], s[m + "_w"], cos, sin, c).to(s[m].dtype).view(B, n, -1, c["D"]).transpose(1, 2).contiguous() for m in "qk")
    return {"q": q, "k": k}


def _plain_int8(c, s):
    a, a_scale = s["a"].float(), s["a_scale"]
    if c["form"] != "q":
        x = s["x"].float()
        if c["form"] == "norm":
            x = _norm(x, "layer", None) * (1 + s["scale"].float()) + s["shift"].float()
        a_scale = x.abs().amax(1) / 127
        a = (x / a_scale[:, None]).round()
    out = (a @ s["w"].float().t()) * a_scale[:, None] * s["w_scale"]
    if s["bias"] is not None:
        out = out + s["bias"]
    return out.to(s["out"].dtype)


# ---- this package's calls ------------------------------------------------------------------------------------------
_handle = None


def _package():
    """The package's binding and a context on the current device, made once for the process."""
    global _handle
    if _handle is None:
        from paper_2607_23844_b200 import omnicache as oc
        _handle = oc, oc.Context(torch.cuda.current_device())
    return _handle


def _own_block(c, s, oc, ctx):
    if "desc" not in s:
        kinds = {"none": oc.NORM_NONE, "rms": oc.NORM_RMS, "layer": oc.NORM_LAYER}
        types = {"bf16": oc.DTYPE_BF16, "f32": oc.DTYPE_F32}
        s["desc"] = oc.block_norm_desc(s["x"].shape[0], c["C"], types[c["dtype"]], types[c["dtype"]], types[c["param"]],
                                       post_norm=kinds[c["post"]], pre_norm=kinds[c["pre"]], post_eps=EPS, pre_eps=EPS,
                                       res_scale=c["res"], rows_per_group=c["H"] * c["W"], mod_stride=3 * c["C"],
                                       unit_rows=_block_plan(c)[2], dense_rows=s["h"].shape[0])
    ctx.block_norm(s["desc"], s["x"], z=s["z"], slot_of=s["slot_of"], cache=s["cache"], cache_out=s["cache"], out=s["out"],
                   post_w=s["post_w"], gate=s["gate"], pre_w=s["pre_w"], scale=s["scale"], shift=s["shift"], h=s["h"])
    return {"out": s["out"], "cache": s["cache"], "h": s["h"]}


def _own_rope(c, s, oc, ctx):
    if "desc" not in s:
        B, n = _rope_rows(c)
        s["desc"] = oc.rope_desc(B * n, {"bf16": oc.DTYPE_BF16, "f32": oc.DTYPE_F32}[c["dtype"]], c["D"], _axes(c),
                                 (c["T"], c["H"], c["W"]), q_heads=c["heads"], k_heads=c["kv"], rows_per_batch=n,
                                 pairing=oc.ROPE_ADJACENT if c["pairs"] == "adjacent" else oc.ROPE_HALVES,
                                 inverse=c["inverse"], eps=EPS, q=s["q"], q_out=s["q_out"], k=s["k"], k_out=s["k_out"])
    ctx.rope(s["desc"], s["table"], s["q"], s["q_out"], k=s["k"], k_out=s["k_out"], idx=s["idx"], pos=s["pos"],
             q_w=s["q_w"], k_w=s["k_w"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_int8(c, s, oc, ctx):
    M, K, N = c["M"], c["K"], c["N"]
    if c["form"] == "rows":
        ctx.quantize_rows(s["x"], oc.DTYPE_BF16, M, K, s["a"], s["a_scale"])
    elif c["form"] == "norm":
        if "desc" not in s:
            s["desc"] = oc.block_norm_desc(M, K, oc.DTYPE_BF16, oc.DTYPE_I8, oc.DTYPE_BF16, pre_norm=oc.NORM_LAYER,
                                           pre_eps=EPS, rows_per_group=M, mod_stride=2 * K)
        ctx.block_norm(s["desc"], s["x"], scale=s["scale"], shift=s["shift"], h=s["a"], h_scale=s["a_scale"])
    ctx.linear_int8(s["a"], s["a_scale"], M, K, s["w"], s["w_scale"], N, s["out"],
                    oc.DTYPE_BF16 if c["out"] == "bf16" else oc.DTYPE_F32, bias=s["bias"])
    return s["out"]


def run(state):
    c = state["case"]
    if own:
        return {"block": _own_block, "rope": _own_rope, "int8": _own_int8}[c["kind"]](c, state, *_package())
    return {"block": _plain_block, "rope": _plain_rope, "int8": _plain_int8}[c["kind"]](c, state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "int8":
        M, K, N = c["M"], c["K"], c["N"]
        a = M * K + 4 * M if c["form"] == "q" else 2 * M * K + (4 * K if c["form"] == "norm" else 0)
        return {"bytes": a + N * K + 4 * N * (2 if c["bias"] else 1) + M * N * (2 if c["out"] == "bf16" else 4),
                "flops": 2 * M * N * K}
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rope":
        B, n = _rope_rows(c)
        values = B * n * (c["heads"] + c["kv"]) * c["D"]
        table = 4 * sum(m * d for m, d in zip((c["T"], c["H"], c["W"]), _axes(c)))
        index = B * n * {"grid": 0, "kept": 4, "rows": 12}[c["at"]]
        return {"bytes": 2 * values * e + table + index, "flops": 3 * values + (4 * values if c["norm"] else 0)}
    groups, units, unit_rows, keep = _block_plan(c)
    rows, dense = groups * units * unit_rows, groups * keep * unit_rows
    cached = c["z"] and c["reuse"] > 0
    moved = dense + (2 * rows + dense if c["z"] else dense)               # h; x, out and z (or the kept rows of x)
    moved += (rows - dense) + dense if cached else 0                      # reused rows read, computed rows written
    vectors = c["B"] * c["T"] * ((2 if c["mod"] else 0) + (1 if c["gate"] else 0)) + (c["post"] != "none") + (c["pre"] == "rms")
    return {"bytes": moved * c["C"] * e + vectors * c["C"] * (2 if c["param"] == "bf16" else 4) + (4 * groups * units if c["reuse"] > 0 else 0),
            "flops": c["C"] * (10 * rows + 10 * dense)}


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------
def _exact_block(c, s):
    unit_rows = _block_plan(c)[2]
    x = s["x"].double()
    n, C = x.shape
    frame = torch.arange(n, device="cuda") // (c["H"] * c["W"])
    unit = torch.arange(n, device="cuda") // unit_rows
    slot = s["slot_of"].long()[unit] if s["slot_of"] is not None else unit
    dense = torch.where(slot >= 0, slot * unit_rows + torch.arange(n, device="cuda") % unit_rows, -1)
    if s["z"] is not None:
        v = s["z"].double()[dense.clamp(min=0)]
        if s["cache"] is not None:
            v = torch.where(dense[:, None] >= 0, v, s["cache"].double())
        t = v
        if c["post"] != "none":
            if c["post"] == "layer":
                t = t - t.sum(1, keepdim=True) / C
            t = t / ((t ** 2).sum(1, keepdim=True) / C + EPS).sqrt() * s["post_w"].double()
        x = x * c["res"] + (t * s["gate"].double()[frame] if s["gate"] is not None else t)
    h = x
    if c["pre"] == "layer":
        h = h - h.sum(1, keepdim=True) / C
    h = h / ((h ** 2).sum(1, keepdim=True) / C + EPS).sqrt()
    if s["pre_w"] is not None:
        h = h * s["pre_w"].double()
    if c["mod"]:
        h = h * (s["scale"].double()[frame] + 1) + s["shift"].double()[frame]
    kept = torch.nonzero(dense >= 0).reshape(-1)
    placed = torch.empty(s["h"].shape, dtype=torch.float64, device="cuda")
    placed[dense[kept]] = h[kept]
    return {"out": x if s["z"] is not None else None, "cache": v if s["cache"] is not None else None, "h": placed}


def _exact_rope(c, s):
    B, n = _rope_rows(c)
    T, H, W = c["T"], c["H"], c["W"]
    if s["pos"] is not None:
        where = s["pos"].double()
    else:
        i = s["idx"].long() if s["idx"] is not None else torch.arange(B * n, device="cuda")
        where = torch.stack([i // (W * H) % T, i // W % H, i % W], 1).double()
    turn = []
    for a, d in enumerate(_axes(c)):
        turn += [where[:, a] / THETA ** (2 * j / d) for j in range(d // 2)]
    z = torch.polar(torch.ones(len(turn), B * n, dtype=torch.float64, device="cuda"), torch.stack(turn) * (-1 if c["inverse"] else 1)).t()[:, None]
    P, got = len(turn), {}
    for m in "qk":
        v = s[m].double()
        if s[m + "_w"] is not None:
            v = v / ((v ** 2).sum(-1, keepdim=True) / c["D"] + EPS).sqrt() * s[m + "_w"].double()
        first = torch.arange(P, device="cuda") * (2 if c["pairs"] == "adjacent" else 1)
        second = first + (1 if c["pairs"] == "adjacent" else P)
        t = torch.complex(v[..., first], v[..., second]) * z
        v[..., first], v[..., second] = t.real, t.imag
        got[m] = v.view(B, n, -1, c["D"]).transpose(1, 2).contiguous()
    return got


def _exact_int8(c, s):
    if c["form"] == "q":
        a, a_scale = s["a"].double(), s["a_scale"].double()
    else:
        x = s["x"].double()
        if c["form"] == "norm":
            x = x - x.sum(1, keepdim=True) / c["K"]
            x = x / ((x ** 2).sum(1, keepdim=True) / c["K"] + EPS).sqrt() * (s["scale"].double() + 1) + s["shift"].double()
        a_scale = x.abs().max(1).values / 127
        a = torch.round(x / a_scale[:, None])
    out = torch.mm(a, s["w"].double().t())
    out *= a_scale[:, None]
    out *= s["w_scale"].double()
    return out if s["bias"] is None else out + s["bias"].double()


def exact(case, seed):
    return {"block": _exact_block, "rope": _exact_rope, "int8": _exact_int8}[case["kind"]](case, prepare(case, seed))
