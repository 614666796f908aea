"""The operators of the wrapped block on kept tokens -- oc_block_norm, oc_rope, oc_quantize_rows, oc_linear_int8 --
against plain restatements in 64 bits.

Tolerances.  u = 2^-24 is the unit roundoff of fp32.  Every result is a short chain of fp32 operations on sums of at
most 48 terms per thread and ten tree levels, so its error is bounded by a small multiple of u times the sum of the
magnitudes that went into it; the references return that sum beside the value, and 128 u of it is allowed.  A bf16
result adds one rounding, at most 2^-9 of the value (2^-8 allowed).  8-bit values may be one step from the exact
quotient only where that lies within the same error of a rounding boundary, which the bound on q * scale covers.  The
integer product itself is exact: four roundings (conversion, two scales, bias) are allowed, 4 u.
"""
import math

import pytest
import torch

U = 2.0 ** -24
BF16, F32, I8 = torch.bfloat16, torch.float32, torch.int8


@pytest.fixture(scope="module")
def oc():
    from paper_2607_23844_b200 import build
    build.build()
    from paper_2607_23844_b200 import omnicache
    return omnicache


@pytest.fixture(scope="module")
def ctx(oc):
    with oc.Context(0) as c:
        yield c


def tag(oc, dt):
    return {F32: oc.DTYPE_F32, BF16: oc.DTYPE_BF16, I8: oc.DTYPE_I8}[dt]


def rand(seed, *shape, dtype=F32, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=torch.float64) * std + mean).to(dtype)


def cu(t):
    return None if t is None else t.cuda()


def d64(t):
    return None if t is None else t.cpu().double()


def assert_close(got, want, mag, factor=128.0):
    """|got - want| within `factor` u of the magnitudes, plus the rounding of a bf16 result; infinities and NaN alike."""
    got_t, got = got.dtype, d64(got)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    bound = factor * U * mag + (2.0 ** -8 * want.abs() if got_t == BF16 else 0.0) + 1e-37
    worst = ((got - want).abs() - bound)[fine]
    assert worst.numel() == 0 or worst.max() <= 0, f"off by {((got - want).abs()[fine]).max()} where {bound[fine][worst.argmax()]} is allowed"


# ---- block_norm -----------------------------------------------------------------------------------------------------
def ref_norm(v, mag, how, eps, w, b):
    C = v.shape[1]
    if how == "none":
        n, m = v, mag
    else:
        mean = v.mean(1, keepdim=True) if how == "layer" else torch.zeros(v.shape[0], 1, dtype=torch.float64)
        rstd = 1.0 / ((v - mean).square().mean(1, keepdim=True) + eps).sqrt()
        n = (v - mean) * rstd
        # an error of the inputs moves the value, the mean and, through the sum of squares, the factor
        moved = mag + (mag.mean(1, keepdim=True) if how == "layer" else 0.0)
        m = moved * rstd + n.abs() * ((moved * (v - mean).abs()).sum(1, keepdim=True) / C * rstd * rstd + 1.0)
    if w is not None:
        n, m = n * w, m * w.abs()
    if b is not None:
        n, m = n + b, m + b.abs()
    return n, m


def ref_block(x, z, slot, cache, p, res, post, pre, eps, rows_per_group, unit_rows, dense_rows):
    """Values and magnitudes of (out, cache, h) in 64 bits; h rows that nothing is written to are None."""
    n, C = x.shape
    row = torch.arange(n)
    s = slot.long()[row // unit_rows] if slot is not None else row // unit_rows
    dense = torch.where((s >= 0) & (s < max(dense_rows // unit_rows, 1)), s * unit_rows + row % unit_rows, -1)
    g = row // rows_per_group
    per_group = {k: (p[k][g] if p.get(k) is not None else None) for k in ("gate", "scale", "shift")}
    r, mr, v = res * x, (res * x).abs(), None
    if z is not None:
        v = z[dense.clamp(min=0)]
        if cache is not None:
            v = torch.where(dense[:, None] >= 0, v, cache)
        t, mt = ref_norm(v, v.abs(), post, eps, p.get("post_w"), p.get("post_b"))
        if per_group["gate"] is not None:
            t, mt = t * per_group["gate"], mt * per_group["gate"].abs()
        r, mr = r + t, mr + mt
    h, mh = ref_norm(r, mr, pre, eps, p.get("pre_w"), p.get("pre_b"))
    if per_group["scale"] is not None:
        h, mh = h * (1 + per_group["scale"]), mh * (1 + per_group["scale"].abs())
    if per_group["shift"] is not None:
        h, mh = h + per_group["shift"], mh + per_group["shift"].abs()
    return r, mr, v, h, mh, dense


def run_block(oc, ctx, n, C, dtype, h_dtype=None, param=F32, post="rms", pre="layer", z=True, slot=None, dense_rows=None,
              unit_rows=1, rows_per_group=None, res=1.0, eps=1e-6, with_params=("post_w", "post_b", "pre_w", "pre_b", "gate", "scale", "shift"),
              in_place=False, own_cache=False, x=None, zz=None, seed=0, stream=None, h_out=True):
    kinds = {"none": oc.NORM_NONE, "rms": oc.NORM_RMS, "layer": oc.NORM_LAYER}
    h_dtype = h_dtype or dtype
    dense_rows = n if dense_rows is None else dense_rows
    rows_per_group = rows_per_group or max(n, 1)
    G = (n + rows_per_group - 1) // rows_per_group
    x = rand(seed + 1, n, C, dtype=dtype, std=2.0) if x is None else x
    zt = (rand(seed + 2, dense_rows, C, dtype=dtype) if zz is None else zz) if z else None
    cache = rand(seed + 3, n, C, dtype=dtype) if z and slot is not None else None
    names = [k for k in with_params if z or not (k.startswith("post") or k == "gate")]
    if not z:
        post = "none"
    mod = rand(seed + 4, G, 3 * C + 8, dtype=param, std=0.3)
    p = {k: rand(seed + 5 + i, C, dtype=param, std=0.2, mean=1.0 if k.endswith("_w") else 0.0)
         for i, k in enumerate(("post_w", "post_b", "pre_w", "pre_b")) if k in names}
    modc = mod.cuda()
    parts = {k: modc[:, i * C:(i + 1) * C] for i, k in enumerate(("gate", "scale", "shift")) if k in names}
    xd, zd, cd = cu(x), cu(zt), cu(cache)
    out = None if not z else (xd if in_place else torch.full((n + 1, C), 7.0, dtype=dtype, device="cuda")[:n])
    cache_out = (torch.full((n, C), 7.0, dtype=dtype, device="cuda") if own_cache else cd) if z and (slot is not None or own_cache) else None
    h = torch.full((dense_rows, C), 9, dtype=h_dtype, device="cuda") if h_out else None
    h_scale = torch.full((dense_rows,), 9.0, device="cuda") if h_dtype == I8 else None
    desc = oc.block_norm_desc(n, C, tag(oc, dtype), tag(oc, h_dtype), tag(oc, param), kinds[post], kinds[pre], eps, eps, res,
                              rows_per_group, 3 * C + 8, unit_rows, dense_rows)
    # (16-byte aligned column ranges of the modulation tensor, as a projection leaves them)
    ctx.block_norm(desc, xd, z=zd, slot_of=cu(slot), cache=cd, cache_out=cache_out, out=out, h=h, h_scale=h_scale, stream=stream,
                   **{k: cu(v) for k, v in p.items()}, **parts)
    torch.cuda.synchronize()
    q = {k: d64(v) for k, v in p.items()}
    q.update({k: d64(v) for k, v in parts.items()})
    r, mr, v, hh, mh, dense = ref_block(d64(x), d64(zt), slot, d64(cache), q, res, post, pre, eps, rows_per_group, unit_rows, dense_rows)
    return dict(out=out, cache=cache_out, h=h, h_scale=h_scale, r=r, mr=mr, v=v, hh=hh, mh=mh, dense=dense, x=x)


def check_block(o):
    if o["out"] is not None:
        assert_close(o["out"], o["r"], o["mr"])
    if o["cache"] is not None:
        assert torch.equal(d64(o["cache"]), o["v"])                       # a bit copy
    if o["h"] is None:
        return
    rows = torch.nonzero(o["dense"] >= 0).reshape(-1)
    written = o["dense"][rows]
    want, mag = o["hh"][rows], o["mh"][rows]
    if o["h"].dtype == I8:
        scale = d64(o["h_scale"])[written]
        top, top_mag = want.abs().max(1).values, mag.max(1).values
        assert ((scale * 127 - top).abs() <= 128 * U * (top_mag + top)).all()
        q = d64(o["h"])[written]
        assert ((q * scale[:, None] - want).abs() <= 0.5 * scale[:, None] + 256 * U * (mag + top[:, None])).all()
    else:
        assert_close(o["h"][written.cuda()], want, mag)
    rest = torch.ones(o["h"].shape[0], dtype=torch.bool)
    rest[written] = False
    assert (o["h"].cpu()[rest] == 9).all()                                # rows of no unit are left untouched


def slots(n_units, keep, seed=0, dense_units=None):
    g = torch.Generator().manual_seed(seed)
    kept = torch.randperm(n_units, generator=g)[:keep].sort().values
    s = torch.full((n_units,), -1, dtype=torch.int32)
    s[kept] = torch.arange(keep, dtype=torch.int32)
    return s


WIDTHS = {BF16: (8, 64, 72, 136, 200, 264, 320, 328, 520, 640, 720, 1000, 1152, 1536, 1544, 2056, 3080, 6152, 12296, 24576),
          F32: (4, 32, 100, 160, 164, 260, 320, 388, 512, 644, 768, 772, 1028, 3076, 6148, 12288)}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,C", [(t, c) for t in (BF16, F32) for c in WIDTHS[t]])
def test_block_norm_every_row_width(oc, ctx, dtype, C):
    n = 37
    s = slots(n, 21, seed=C)
    check_block(run_block(oc, ctx, n, C, dtype, slot=s, dense_rows=21, rows_per_group=10, post="layer", pre="rms", seed=C))
    if C % 16 == 0:
        check_block(run_block(oc, ctx, n, C, dtype, I8, param=BF16, slot=s, dense_rows=21, rows_per_group=7, seed=C + 1))
    assert ctx.device_status() == oc.OK


@pytest.mark.gpu
@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("dtype,h_dtype,param", [(BF16, BF16, F32), (BF16, F32, BF16), (F32, BF16, F32), (F32, F32, BF16), (F32, I8, F32)])
def test_block_norm_kinds_and_types(oc, ctx, post, pre, dtype, h_dtype, param):
    check_block(run_block(oc, ctx, 50, 96, dtype, h_dtype, param, post, pre, rows_per_group=16, res=0.5))
    for names in ((), ("gate",), ("scale",), ("shift", "post_w"), ("pre_b", "post_b")):
        check_block(run_block(oc, ctx, 9, 96, dtype, h_dtype, param, post, pre, with_params=names, seed=len(names)))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [0, 1, 2, 31, 33, 300])
@pytest.mark.parametrize("C", [64, 1152, 4096])
def test_block_norm_row_counts(oc, ctx, n, C):
    check_block(run_block(oc, ctx, n, C, BF16, rows_per_group=5))
    check_block(run_block(oc, ctx, n, C, BF16, z=False, rows_per_group=5))
    check_block(run_block(oc, ctx, n, C, BF16, h_out=False, in_place=True))


@pytest.mark.gpu
@pytest.mark.parametrize("keep", [0, 1, 40, 64])
@pytest.mark.parametrize("own_cache", [False, True])
def test_block_norm_selections(oc, ctx, keep, own_cache):
    s = slots(64, keep, seed=keep)
    check_block(run_block(oc, ctx, 64, 256, BF16, slot=s, dense_rows=70, own_cache=own_cache))         # dense tail unused
    check_block(run_block(oc, ctx, 64, 256, F32, slot=s, dense_rows=64, own_cache=own_cache, in_place=True))
    check_block(run_block(oc, ctx, 64, 256, BF16, slot=s, dense_rows=64, z=False))
    # units of several rows: whole frames
    check_block(run_block(oc, ctx, 64 * 6, 256, BF16, I8, slot=s, dense_rows=64 * 6, unit_rows=6, rows_per_group=6, own_cache=own_cache))


@pytest.mark.gpu
def test_block_norm_identity_step_fills_the_cache(oc, ctx):
    check_block(run_block(oc, ctx, 40, 320, BF16, own_cache=True))


@pytest.mark.gpu
def test_block_norm_slot_outside_the_dense_rows(oc, ctx):
    s = slots(20, 8)
    s[3], s[4] = 8, 2 ** 30
    check_block(run_block(oc, ctx, 20, 64, BF16, slot=s, dense_rows=8))
    assert ctx.device_status() == oc.ERR_INVALID_ARG and ctx.device_status() == oc.OK
    check_block(run_block(oc, ctx, 20, 64, BF16, slot=s, dense_rows=8, z=False))
    assert ctx.device_status() == oc.ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,C", [(F32, 320), (F32, 2048)])
def test_block_norm_large_common_offset(oc, ctx, dtype, C):
    """A mean of 1000 standard deviations: the two-pass statistics keep the digits that are there."""
    x = rand(5, 33, C, dtype=dtype, mean=1000.0)
    check_block(run_block(oc, ctx, 33, C, dtype, x=x, z=False, pre="layer"))


@pytest.mark.gpu
@pytest.mark.parametrize("C", [64, 1536, 2560])
def test_block_norm_zero_rows_and_values_that_are_not_finite(oc, ctx, C):
    x = rand(7, 12, C, dtype=BF16)
    x[0] = 0
    x[3, 5], x[6, C - 1], x[8, 0] = math.inf, -math.inf, math.nan
    o = run_block(oc, ctx, 12, C, BF16, x=x, z=False, pre="rms", with_params=())
    h = d64(o["h"])
    fine = torch.tensor([i not in (3, 6, 8) for i in range(12)])
    assert (h[0] == 0).all() and torch.isfinite(h[fine]).all()
    assert_close(o["h"][fine.cuda()], o["hh"][fine], o["mh"][fine])
    assert torch.isnan(h[8]).all() and torch.isnan(h[3, 5]) and torch.isnan(h[6, C - 1])
    o = run_block(oc, ctx, 12, C, BF16, I8, x=x, z=False, pre="none", with_params=())
    s, q = o["h_scale"].cpu(), o["h"].cpu()
    assert s[0] == 0 and (q[0] == 0).all()
    assert s[3] == math.inf and s[6] == math.inf and torch.isnan(s[8]) and (q[[3, 6, 8]] == 0).all()
    assert torch.isfinite(s[fine]).all() and (q[fine][1:].abs().max(1).values == 127).all()


@pytest.mark.gpu
def test_block_norm_offsets_past_32_bits(oc, ctx):
    """2^31 elements of x and more; only the last units have slots, so the rest is not read."""
    C, n = 8192, 2 ** 18 + 40
    x = torch.zeros(n, C, dtype=BF16, device="cuda")
    tail = rand(3, 8, C, dtype=BF16)
    x[-8:] = tail.cuda()
    slot = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    slot[-8:] = torch.arange(8, dtype=torch.int32, device="cuda")
    h = torch.empty(8, C, dtype=BF16, device="cuda")
    desc = oc.block_norm_desc(n, C, oc.DTYPE_BF16, oc.DTYPE_BF16, oc.DTYPE_F32, pre_norm=oc.NORM_LAYER, dense_rows=8)
    ctx.block_norm(desc, x, slot_of=slot, h=h)
    torch.cuda.synchronize()
    want, mag = ref_norm(d64(tail), d64(tail).abs(), "layer", 1e-6, None, None)
    assert_close(h, want, mag)


@pytest.mark.gpu
def test_block_norm_on_another_stream_and_in_a_graph(oc, ctx):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        check_block(run_block(oc, ctx, 64, 320, BF16, slot=slots(64, 30), dense_rows=30))
    x = rand(1, 100, 320, dtype=BF16).cuda()
    h = torch.zeros_like(x)
    desc = oc.block_norm_desc(100, 320, oc.DTYPE_BF16, oc.DTYPE_BF16, oc.DTYPE_F32, pre_norm=oc.NORM_RMS)
    ctx.block_norm(desc, x, h=h)
    torch.cuda.synchronize()
    want = h.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.block_norm(desc, x, h=h)
    h.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(h, want)


@pytest.mark.gpu
def test_block_norm_refusals(oc, ctx):
    n, C = 4, 64
    t = lambda dt=BF16: torch.zeros(n, C, dtype=dt, device="cuda")     # noqa: E731
    x, z, cache, out, h = t(), t(), t(), t(), t()
    h8, hs, slot, vec = t(I8), torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(C, device="cuda")

    def st(d=None, **kw):
        args = dict(rows_per_group=n, pre_norm=oc.NORM_RMS)
        args.update(d or {})
        desc = oc.block_norm_desc(args.pop("n", n), args.pop("C", C), args.pop("dtype", oc.DTYPE_BF16), args.pop("h_dtype", oc.DTYPE_BF16),
                                  args.pop("param", oc.DTYPE_F32), **args)
        return ctx.block_norm(desc, kw.pop("x", x), check=False, **kw)
    bad, align, no = oc.ERR_INVALID_ARG, oc.ERR_ALIGNMENT, oc.ERR_UNSUPPORTED
    assert st(h=h) == oc.OK
    assert st(h=h, x=None) == bad
    assert st() == bad                                                  # nothing to write
    assert st(dict(dtype=oc.DTYPE_I8), h=h) == bad
    assert st(dict(h_dtype=3), h=h) == bad
    assert st(dict(pre_norm=3), h=h) == bad
    assert st(dict(pre_eps=-1.0), h=h) == bad
    assert st(dict(pre_eps=math.nan), h=h) == bad
    assert st(dict(res_scale=math.inf), h=h) == bad
    assert st(dict(n=-1, dense_rows=0, rows_per_group=1), h=h) == bad
    assert st(dict(rows_per_group=0), h=h) == bad
    assert st(dict(unit_rows=3), h=h) == bad                            # rows not a whole number of units
    assert st(dict(dense_rows=2), h=h) == bad                           # no slots, and not enough dense rows
    assert st(h=h, cache=cache) == bad                                  # a cache without z
    assert st(dict(post_norm=oc.NORM_RMS), h=h) == bad
    assert st(z=z, slot_of=slot, out=out) == bad                        # reused rows without a cache
    assert st(dict(h_dtype=oc.DTYPE_I8), h=h8) == bad                   # 8 bits without scales
    assert st(z=z, out=z) == bad and st(h=x) == bad and st(z=z, out=out, h=out) == bad
    assert st(dict(C=60), h=h) == align
    assert st(dict(C=56, h_dtype=oc.DTYPE_I8), h=h8, h_scale=hs) == align
    assert st(h=h, x=x.data_ptr() + 2) == align
    assert st(dict(mod_stride=6), h=h, scale=vec) == align
    assert st(h=h, pre_w=vec.data_ptr() + 4) == align
    assert st(dict(param=oc.DTYPE_BF16), h=h, pre_w=vec.data_ptr() + 8) == align
    assert st(dict(C=49152), h=h) == no
    assert st(dict(n=2 ** 31, dense_rows=2 ** 31), h=h) == no
    assert oc._lib.oc_block_norm(None, *[None] * 17) == bad


# ---- rope -----------------------------------------------------------------------------------------------------------
def ref_rope(v, w, at, axes, pairs, inverse, eps, theta=10000.0):
    """v [rows, heads, D] in 64 bits, at [rows, 3] -> (value, magnitude)."""
    mag = v.abs()
    if w is not None:
        f = w / (v.square().mean(-1, keepdim=True) + eps).sqrt()
        v, mag = v * f, 2 * mag * f.abs()
    angle = torch.cat([at[:, a:a + 1].double() * theta ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / max(d, 1)) for a, d in enumerate(axes)], 1)
    c, s = angle.cos()[:, None], angle.sin()[:, None] * (-1 if inverse else 1)
    P = angle.shape[1]
    i = torch.arange(P) * (2 if pairs == "adjacent" else 1)
    j = i + (1 if pairs == "adjacent" else P)
    out, m = v.clone(), mag.clone()
    out[..., i], out[..., j] = v[..., i] * c - v[..., j] * s, v[..., j] * c + v[..., i] * s
    m[..., i] = m[..., j] = mag[..., i] + mag[..., j]
    return out, m


def run_rope(oc, ctx, n, D, axes, lens, hq, hk, dtype, pairs="adjacent", inverse=False, norm=False, idx=None, pos=None, batch=1,
             unit_rows=1, head_major=True, shift=0, pad=0, seed=0, in_place=False):
    """q and k as parts of one projection (rows `pad` elements longer, `shift` elements from an aligned start)."""
    wide = (hq + 2 * hk) * D + pad
    store = rand(seed, n * wide + shift + 8, dtype=dtype)
    dev = store.cuda()
    def part(t, first, heads):
        return t[shift + first * D:].as_strided((n, heads, D), (wide, D, 1))
    q, k = part(dev, 0, hq), part(dev, hq, hk) if hk else None
    rpb = max(n // batch, 1)
    if in_place:
        qo, ko = q, k
    elif head_major:
        qo, ko = (torch.full((batch, h, rpb, D), 5.0, dtype=dtype, device="cuda") if h else None for h in (hq, hk))
    else:
        qo, ko = (torch.full((n, h, D), 5.0, dtype=dtype, device="cuda") if h else None for h in (hq, hk))
    ws = [rand(seed + 9 + i, D, std=0.2, mean=1.0) if norm else None for i in range(2)]
    desc = oc.rope_desc(n, tag(oc, dtype), D, axes, lens, hq, hk, rows_per_batch=rpb, unit_rows=unit_rows, inverse=inverse,
                        pairing=oc.ROPE_ADJACENT if pairs == "adjacent" else oc.ROPE_HALVES, eps=1e-6, q=q, q_out=qo, k=k, k_out=ko)
    ctx.rope(desc, oc.rope_table(desc).cuda(), q, qo, k=k, k_out=ko, idx=cu(idx), pos=cu(pos), q_w=cu(ws[0]), k_w=cu(ws[1]) if hk else None)
    torch.cuda.synchronize()
    r = torch.arange(n)
    if pos is not None:
        at, live = pos, ((pos >= 0) & (pos < torch.tensor(lens)) | (torch.tensor(axes) == 0)).all(1)
    else:
        unit = idx.long()[r // unit_rows] if idx is not None else r // unit_rows
        live, token = unit >= 0, unit * unit_rows + r % unit_rows
        at = torch.stack([token // (lens[1] * lens[2]) % lens[0], token // lens[2] % lens[1], token % lens[2]], 1)
    for name, got, h, first, w in (("q", qo, hq, 0, ws[0]), ("k", ko, hk, hq, ws[1])):
        if not h or n == 0:
            continue
        src = d64(part(store, first, h))
        want, mag = ref_rope(src, d64(w), at, axes, pairs, inverse, 1e-6)
        got = got.transpose(1, 2).reshape(n, h, D) if head_major and not in_place else got
        assert_close(got[live.cuda()], want[live], mag[live], 16.0)
        untouched = src[~live] if in_place else torch.full_like(src[~live], 5.0)
        assert torch.equal(d64(got[(~live).cuda()]), untouched)


HEADS = [(64, (0, 32, 32)), (64, (16, 24, 24)), (64, (10, 10, 10)), (72, (24, 24, 24)), (80, (0, 40, 40)), (128, (32, 48, 48)),
         (40, (2, 2, 2)), (8, (2, 2, 4)), (256, (0, 0, 256)), (16, (0, 0, 2))]


@pytest.mark.gpu
@pytest.mark.parametrize("D,axes", HEADS)
@pytest.mark.parametrize("pairs", ["adjacent", "halves"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("norm", [False, True])
def test_rope_heads(oc, ctx, D, axes, pairs, dtype, norm):
    run_rope(oc, ctx, 60, D, axes, (3, 4, 5), 5, 2, dtype, pairs, norm=norm, seed=D)
    run_rope(oc, ctx, 7, D, axes, (2, 2, 5), 1, 1, dtype, pairs, norm=norm, inverse=True, head_major=False, seed=D + 1)
    assert ctx.device_status() == oc.OK


@pytest.mark.gpu
@pytest.mark.parametrize("n", [0, 1, 5, 33, 2000])
@pytest.mark.parametrize("hq,hk", [(1, 0), (1, 1), (24, 24), (9, 3)])
def test_rope_sizes(oc, ctx, n, hq, hk):
    run_rope(oc, ctx, n, 64, (16, 24, 24), (2, 30, 40), hq, hk, BF16, "halves", norm=True)


@pytest.mark.gpu
@pytest.mark.parametrize("pairs", ["adjacent", "halves"])
@pytest.mark.parametrize("shift,pad", [(1, 0), (2, 0), (4, 4), (0, 1), (0, 2), (8, 8)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rope_alignments(oc, ctx, pairs, shift, pad, dtype):
    if pairs == "adjacent" and (shift | pad) & 1:
        with pytest.raises(oc.OmniCacheError):
            run_rope(oc, ctx, 20, 64, (0, 32, 32), (1, 4, 5), 3, 2, dtype, pairs, shift=shift, pad=pad)
        return
    run_rope(oc, ctx, 20, 64, (0, 32, 32), (1, 4, 5), 3, 2, dtype, pairs, shift=shift, pad=pad, norm=True)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
def test_rope_kept_rows_keep_their_positions(oc, ctx, in_place):
    idx = torch.tensor([0, 3, 7, -1, 19, 20, 39, -1], dtype=torch.int32)      # two batch elements of 20 tokens
    run_rope(oc, ctx, 8, 64, (16, 24, 24), (1, 4, 5), 4, 2, BF16, idx=idx, batch=2, head_major=not in_place, in_place=in_place)
    frames = torch.tensor([0, 2, -1, 5], dtype=torch.int32)                   # whole frames of 20 tokens
    run_rope(oc, ctx, 80, 64, (16, 24, 24), (6, 4, 5), 2, 2, F32, "halves", idx=frames, unit_rows=20, norm=True, in_place=in_place, head_major=not in_place)
    assert ctx.device_status() == oc.OK


@pytest.mark.gpu
def test_rope_positions_row_by_row(oc, ctx):
    g = torch.Generator().manual_seed(0)
    pos = torch.stack([torch.randint(0, m, (50,), generator=g) for m in (3, 70, 90)], 1).to(torch.int32)
    run_rope(oc, ctx, 50, 72, (24, 24, 24), (3, 70, 90), 4, 1, BF16, "halves", pos=pos)
    assert ctx.device_status() == oc.OK
    pos[4, 1], pos[9, 2] = 70, -1
    run_rope(oc, ctx, 50, 72, (24, 24, 24), (3, 70, 90), 4, 1, BF16, "halves", pos=pos)
    assert ctx.device_status() == oc.ERR_INVALID_ARG
    pos[:, 0] = 99                                                            # an axis that turns nothing is not looked at
    pos[4, 1] = pos[9, 2] = 0
    run_rope(oc, ctx, 50, 72, (0, 24, 24), (3, 70, 90), 4, 1, F32, pos=pos)
    assert ctx.device_status() == oc.OK


@pytest.mark.gpu
def test_rope_inverse_undoes_it_and_is_its_gradient(oc, ctx):
    """The rotation is orthogonal: the inverse is the transpose, <R x, y> = <x, R' y>, and differences agree."""
    n, D, axes, lens = 40, 64, (16, 24, 24), (2, 4, 5)
    x, y = rand(1, n, 1, D).cuda(), rand(2, n, 1, D).cuda()
    def rot(t, inverse):
        o = torch.empty_like(t)
        d = oc.rope_desc(n, oc.DTYPE_F32, D, axes, lens, 1, inverse=inverse, q=t, q_out=o)
        ctx.rope(d, oc.rope_table(d).cuda(), t, o)
        return o
    back = rot(rot(x, False), True)
    assert (back - x).abs().max() <= 32 * U * x.abs().max() * 2
    grad = rot(y, True)                                                       # of <R x, y> with respect to x
    a, b = (rot(x, False).double() * y.double()).sum(), (x.double() * grad.double()).sum()
    assert abs(a - b) <= 64 * U * (x.double().abs() * y.double().abs()).sum() * 2
    step = torch.zeros_like(x)
    step[17, 0, 20] = 0.5
    f = [(rot(x + e * step, False).double() * y.double()).sum() for e in (1, -1)]
    assert abs((f[0] - f[1]) / 1.0 - grad[17, 0, 20].double()) <= 256 * U * (x.double().abs() * y.double().abs()).sum()


@pytest.mark.gpu
def test_rope_infinities_stay_in_their_pair(oc, ctx):
    x = rand(3, 6, 2, 72, dtype=F32)
    x[2, 0, 3], x[4, 1, 71] = math.inf, math.nan                              # the second lies past the 68 rotated elements
    xd = x.cuda()
    o = torch.empty_like(xd)
    d = oc.rope_desc(6, oc.DTYPE_F32, 72, (0, 20, 48), (1, 2, 3), 2, q=xd, q_out=o)
    ctx.rope(d, oc.rope_table(d).cuda(), xd, o)
    torch.cuda.synchronize()
    bad = ~torch.isfinite(o.cpu())
    want = torch.zeros_like(bad)
    want[2, 0, 2:4], want[4, 1, 71] = True, True
    assert torch.equal(bad, want)


@pytest.mark.gpu
def test_rope_offsets_past_32_bits(oc, ctx):
    stride, n = 2 ** 28 + 64, 10
    big = torch.empty(n * stride, dtype=BF16, device="cuda")
    rows = rand(4, n, 1, 64, dtype=BF16)
    view = big.as_strided((n, 1, 64), (stride, 64, 1))
    view.copy_(rows)
    d = oc.rope_desc(n, oc.DTYPE_BF16, 64, (0, 0, 64), (1, 1, n), 1, q=view, q_out=view)
    ctx.rope(d, oc.rope_table(d).cuda(), view, view)
    torch.cuda.synchronize()
    at = torch.stack([torch.zeros(n), torch.zeros(n), torch.arange(n)], 1)
    want, mag = ref_rope(d64(rows), None, at, (0, 0, 64), "adjacent", False, 1e-6)
    assert_close(view, want, mag, 16.0)


@pytest.mark.gpu
def test_rope_refusals(oc, ctx):
    x, o = torch.zeros(8, 2, 64, dtype=BF16, device="cuda"), torch.zeros(8, 2, 64, dtype=BF16, device="cuda")
    w, tab = torch.ones(64, device="cuda"), torch.zeros(4096, device="cuda")
    idx, pos = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(8, 3, dtype=torch.int32, device="cuda")

    def st(d=None, change=None, **kw):
        args = dict(dtype=oc.DTYPE_BF16, head_dim=64, axes=(0, 32, 32), lens=(1, 2, 4), q_heads=2, n=8)
        args.update(d or {})
        desc = oc.rope_desc(args["n"], args["dtype"], args["head_dim"], args["axes"], args["lens"], args["q_heads"], args.get("k_heads", 2),
                            rows_per_batch=args.get("rpb"), unit_rows=args.get("unit", 1), pairing=args.get("pairing", 0), eps=args.get("eps", 1e-6),
                            **{m: (512, 128, 64) for m in ("q", "q_out", "k", "k_out")})
        for f, v in (change or {}).items():
            setattr(desc, f, v)
        call = dict(table=tab, q=x, q_out=o)
        call.update(kw)
        return ctx.rope(desc, call.pop("table"), call.pop("q"), call.pop("q_out"), check=False, **call)
    bad, align, no = oc.ERR_INVALID_ARG, oc.ERR_ALIGNMENT, oc.ERR_UNSUPPORTED
    assert st() == oc.OK
    assert st(table=None) == bad and st(q=None) == bad and st(q_out=None) == bad
    assert st(dict(dtype=2)) == bad and st(dict(pairing=2)) == bad and st(dict(head_dim=0)) == bad
    assert st(dict(axes=(0, 0, 0))) == bad and st(dict(axes=(1, 32, 31))) == bad and st(dict(axes=(2, 32, 32))) == bad
    assert st(dict(axes=(-2, 32, 32))) == bad and st(dict(lens=(0, 2, 4))) == bad
    assert st(dict(q_heads=0)) == bad and st(dict(n=-1, rpb=1)) == bad and st(dict(rpb=0)) == bad and st(dict(unit=0)) == bad
    assert st(change=dict(rows_per_batch=0)) == bad
    assert st(k=x) == bad and st(k_out=o) == bad and st(idx=idx, pos=pos) == bad
    assert st(k=x, k_out=o, q_w=w) == bad and st(k_w=w) == bad and st(dict(eps=-1.0), q_w=w) == bad
    assert st(change=dict(q=oc.CRopeView(0, -128, 64))) == bad
    assert st(q=x.data_ptr() + 2) == align and st(q=x.data_ptr() + 1) == align and st(table=tab.data_ptr() + 4) == align
    assert st(change=dict(q=oc.CRopeView(512, 129, 64))) == align
    assert st(dict(lens=(2 ** 11, 2 ** 11, 2 ** 11))) == no and st(dict(head_dim=1024)) == no
    assert oc._lib.oc_rope(None, *[None] * 11) == bad


def test_rope_table_is_the_formula(oc):
    d = oc.rope_desc(4, oc.DTYPE_F32, 64, (8, 0, 20), (5, 3, 700), 1)
    got, want = oc.rope_table(d, 500.0), []
    for a, (dims, n) in enumerate(((8, 5), (0, 3), (20, 700))):
        for p in range(n):
            for j in range(dims // 2):
                want += [math.cos(p * 500.0 ** (-2 * j / dims)), math.sin(p * 500.0 ** (-2 * j / dims))]
    assert got.numel() == len(want) and (got.double() - torch.tensor(want, dtype=torch.float64)).abs().max() <= 2 * U
    assert oc._lib.oc_rope_table(None, 1.0, None) == oc.ERR_INVALID_ARG
    for theta in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(oc.OmniCacheError):
            oc.rope_table(d, theta)


# ---- quantize_rows, linear_int8 -------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,K", [(0, 64), (1, 16), (3, 1152), (40, 336), (65, 1536), (5, 4096), (2, 12288)])
def test_quantize_rows(oc, ctx, dtype, n, K):
    x = rand(n + K, n + 3, K + 16, dtype=dtype, std=3.0)
    xd = x.cuda()
    q, s = torch.full((n, K), 9, dtype=I8, device="cuda"), torch.full((n,), 9.0, device="cuda")
    ctx.quantize_rows(xd, tag(oc, dtype), n, K, q, s, x_stride=K + 16)
    want = d64(x)[:n, :K]
    top = want.abs().amax(1)
    assert ((d64(s) * 127 - top).abs() <= 4 * U * top).all()
    assert ((d64(q) * d64(s)[:, None] - want).abs() <= d64(s)[:, None] * (0.5 + 512 * U)).all()
    if n < 3:
        return
    idx = torch.tensor([n + 2, -1, 0] + [1] * (n - 3), dtype=torch.int32)
    q.fill_(9), s.fill_(9.0)
    ctx.quantize_rows(xd, tag(oc, dtype), n, K, q, s, idx=idx.cuda(), x_rows=n + 3, x_stride=K + 16)
    assert (q[1] == 9).all() and s[1] == 9
    assert ((d64(q) * d64(s)[:, None] - d64(x)[idx.long().clamp(min=0), :K]).abs()[[0, 2]] <= d64(s)[[0, 2], None] * (0.5 + 512 * U)).all()
    assert ctx.device_status() == oc.OK
    idx[1] = n + 3
    ctx.quantize_rows(xd, tag(oc, dtype), n, K, q, s, idx=idx.cuda(), x_rows=n + 3, x_stride=K + 16)
    assert ctx.device_status() == oc.ERR_INVALID_ARG and (q[1] == 9).all()


@pytest.mark.gpu
def test_quantize_rows_special_values(oc, ctx):
    x = torch.zeros(6, 32)
    x[1, 3] = 1e-38
    x[2, 31] = -math.inf
    x[3, 0] = math.nan
    x[4] = torch.linspace(-1e30, 1e30, 32)
    x[5] = torch.linspace(-1e-29, 1e-29, 32)
    q, s = torch.empty(6, 32, dtype=I8, device="cuda"), torch.empty(6, device="cuda")
    ctx.quantize_rows(x.cuda(), oc.DTYPE_F32, 6, 32, q, s)
    q, s = q.cpu(), s.cpu()
    assert (q[:4] == 0).all() and s[0] == 0 and s[1] == 0 and s[2] == math.inf and math.isnan(s[3])
    for i in (4, 5):
        assert q[i, 0] == -127 and q[i, 31] == 127 and ((q[i].double() * s[i].double() - x[i].double()).abs() <= 0.51 * s[i].double()).all()


def run_linear(oc, ctx, M, K, N, out_dtype=BF16, bias=True, out_idx=None, out_rows=None, pad=0, seed=0, a=None, w=None, a_scale=None, off=0):
    g = torch.Generator().manual_seed(seed)
    a = torch.randint(-128, 128, (M, K), generator=g).to(I8) if a is None else a
    w = torch.randint(-128, 128, (N, K), generator=g).to(I8) if w is None else w
    sa = (torch.rand(M, generator=g) + 0.1) / 50 if a_scale is None else a_scale
    sw = (torch.rand(N, generator=g) + 0.1) / 50
    b = torch.randn(N, generator=g) if bias else None
    rows = M if out_rows is None else out_rows
    store = torch.full((rows * (N + pad) + 16 + off,), 5.0, dtype=out_dtype, device="cuda")
    out = store[off:].as_strided((rows, N), (N + pad, 1))
    ctx.linear_int8(a.cuda(), sa.cuda(), M, K, w.cuda(), sw.cuda(), N, out, tag(oc, out_dtype), bias=cu(b), out_rows=rows, out_stride=N + pad, out_idx=cu(out_idx))
    torch.cuda.synchronize()
    acc = (a.cuda().double() @ w.cuda().double().t()).cpu()                   # whole numbers below 2^53: exact
    want = acc * sa.double()[:, None] * sw.double()
    mag = want.abs()
    if bias:
        want, mag = want + b.double(), mag + b.double().abs()
    dst = out_idx.long() if out_idx is not None else torch.arange(M)
    live = (dst >= 0) & (dst < rows)
    got = out.cpu()
    assert_close(got[dst[live]], want[live], mag[live], 4.0)
    full = torch.ones(store.numel(), dtype=torch.bool)
    at = off + dst[live][:, None] * (N + pad) + torch.arange(N)
    full[at.reshape(-1)] = False
    assert (store.cpu()[full] == 5).all()                                     # nothing else is written
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 2, 3, 7, 8, 9, 16, 127, 128, 129, 300])
@pytest.mark.parametrize("K,N", [(16, 1), (128, 32), (144, 100), (1168, 257), (512, 520)])
@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_linear_int8_sizes(oc, ctx, M, K, N, out_dtype):
    run_linear(oc, ctx, M, K, N, out_dtype, bias=M % 2 == 1, seed=M)
    run_linear(oc, ctx, M, K, N, out_dtype, bias=M % 2 == 0, pad=-N % 8 + 8, seed=M + 1)
    assert ctx.device_status() == oc.OK


@pytest.mark.gpu
@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("M,K,N", [(2500, 256, 2304), (2561, 640, 2309), (1000, 2048, 4104), (20000, 320, 320), (1100, 96, 1096), (700, 6400, 600),
                                   (20000, 320, 2560), (9000, 880, 2816), (2000, 64, 20000)])
def test_linear_int8_large(oc, ctx, M, K, N, out_dtype):
    run_linear(oc, ctx, M, K, N, out_dtype, seed=M)
    run_linear(oc, ctx, M, K, N, out_dtype, bias=False, pad=1, off=1, seed=N)
    assert ctx.device_status() == oc.OK


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(2, 64, 40), (5, 64, 40), (200, 320, 136), (2500, 256, 2304)])
def test_linear_int8_rows_to_named_places(oc, ctx, M, K, N):
    g = torch.Generator().manual_seed(M)
    idx = torch.randperm(M + 50, generator=g)[:M].to(torch.int32)
    idx[M // 2] = -1
    run_linear(oc, ctx, M, K, N, F32, out_idx=idx, out_rows=M + 50)
    assert ctx.device_status() == oc.OK
    idx[M // 3] = M + 50
    run_linear(oc, ctx, M, K, N, BF16, out_idx=idx, out_rows=M + 50)
    assert ctx.device_status() == oc.ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 4, 40])
def test_linear_int8_sums_are_exact(oc, ctx, M):
    """The largest sums: K = 131056 products of -128 * -128 stay just below 2^31."""
    K = 131056
    a, w = torch.full((M, K), -128, dtype=I8), torch.full((24, K), 127, dtype=I8)
    w[0] = -128
    w[1, ::2] = -128
    run_linear(oc, ctx, M, K, 24, F32, a=a, w=w)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 130])
def test_linear_int8_rows_that_are_not_finite(oc, ctx, M):
    """A row whose scale says infinity or NaN (its integers are zeros) shows it in every column, other rows do not."""
    sa = torch.full((M,), 0.01)
    a = torch.randint(-127, 128, (M, 64)).to(I8)
    sa[0], sa[2] = math.inf, math.nan
    a[0] = a[2] = 0
    out = run_linear(oc, ctx, M, 64, 48, BF16, a=a, a_scale=sa)
    assert torch.isnan(out[[0, 2]]).all() and torch.isfinite(out[1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 6, 24])
def test_linear_int8_offsets_past_32_bits(oc, ctx, M):
    K, N, stride = 64, 40, 2 ** 29 // M * 5
    g = torch.Generator().manual_seed(0)
    a, w = torch.randint(-127, 128, (M, K), generator=g).to(I8), torch.randint(-127, 128, (N, K), generator=g).to(I8)
    big = torch.empty(M * stride, dtype=F32, device="cuda")
    out = big.as_strided((M, N), (stride, 1))
    one = torch.ones(max(M, N), device="cuda")
    ctx.linear_int8(a.cuda(), one[:M], M, K, w.cuda(), one[:N], N, out, oc.DTYPE_F32, out_stride=stride)
    assert torch.equal(out.cpu().double(), a.double() @ w.double().t())


@pytest.mark.gpu
def test_int8_refusals(oc, ctx):
    a, w = torch.zeros(16, 64, dtype=I8, device="cuda"), torch.zeros(32, 64, dtype=I8, device="cuda")
    sa, sw, out = torch.ones(16, device="cuda"), torch.ones(32, device="cuda"), torch.zeros(16, 32, device="cuda")
    bad, align, no = oc.ERR_INVALID_ARG, oc.ERR_ALIGNMENT, oc.ERR_UNSUPPORTED

    def st(**kw):
        v = dict(a=a, a_scale=sa, M=16, K=64, w=w, w_scale=sw, N=32, out=out, out_dtype=oc.DTYPE_F32)
        v.update(kw)
        return ctx.linear_int8(check=False, **v)
    assert st() == oc.OK and st(M=0) == oc.OK
    for name in ("a", "a_scale", "w", "w_scale", "out"):
        assert st(**{name: None}) == bad
    assert st(out_dtype=oc.DTYPE_I8) == bad and st(M=-1) == bad and st(K=0) == bad and st(N=0) == bad
    assert st(out_stride=31) == bad and st(out_rows=15) == bad
    assert st(K=63) == align and st(a=a.data_ptr() + 1) == align and st(w=w.data_ptr() + 8) == align and st(out=out.data_ptr() + 2) == align
    assert st(a_scale=sa.data_ptr() + 1) == align
    assert st(K=131072) == no and st(M=2 ** 31, out_rows=2 ** 31) == no and st(M=2 ** 31 - 500, out_rows=2 ** 31 - 500) == no
    assert st(N=2 ** 31 - 1, out_stride=2 ** 31 - 1) == no
    x, q = torch.zeros(16, 64, device="cuda"), torch.zeros(16, 64, dtype=I8, device="cuda")

    def sq(**kw):
        v = dict(x=x, dtype=oc.DTYPE_F32, n_rows=16, K=64, q=q, scale=sa)
        v.update(kw)
        return ctx.quantize_rows(check=False, **v)
    assert sq() == oc.OK
    assert sq(x=None) == bad and sq(q=None) == bad and sq(scale=None) == bad and sq(dtype=oc.DTYPE_I8) == bad
    assert sq(n_rows=-1, x_rows=0) == bad and sq(K=0) == bad and sq(x_rows=15) == bad and sq(x_stride=48) == bad
    assert sq(K=40) == align and sq(x_stride=66) == align and sq(x=x.data_ptr() + 4) == align and sq(q=q.data_ptr() + 8) == align
    assert sq(K=16384, x_stride=16384) == no and sq(n_rows=2 ** 31) == no
    assert oc._lib.oc_linear_int8(None, None, None, 1, 16, None, None, 1, None, None, 0, 1, 16, None, None) == bad
    assert oc._lib.oc_quantize_rows(None, None, 0, 1, 16, None, 1, 16, None, None, None) == bad


@pytest.mark.gpu
@pytest.mark.parametrize("n,C", [(40, 64), (100003, 64), (20011, 640), (12003, 1536), (5003, 3200)])
def test_block_norm_no_dense_rows_at_all(oc, ctx, n, C):
    """Every unit is reused and there is no dense row: a selection like any other, however long a CTA's queue is."""
    x, cache, z = (rand(i, n, C, dtype=BF16).cuda() for i in (1, 2, 3))
    slot = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    out, h = torch.empty_like(x), torch.full((1, C), 9.0, dtype=BF16, device="cuda")
    desc = oc.block_norm_desc(n, C, oc.DTYPE_BF16, oc.DTYPE_BF16, oc.DTYPE_F32, dense_rows=0)
    ctx.block_norm(desc, x, slot_of=slot, out=out, h=h)
    assert ctx.device_status() == oc.OK
    assert torch.equal(out, x) and (h == 9).all()
    ctx.block_norm(desc, x, z=z, slot_of=slot, cache=cache, cache_out=cache, out=out, h=h)
    assert ctx.device_status() == oc.OK
    assert torch.equal(out, (x.float() + cache.float()).to(BF16)) and (h == 9).all()


@pytest.mark.gpu
def test_block_norm_empty_dense_tensors(oc, ctx):
    """A step that computes nothing: z and h are tensors of no rows, which have no address."""
    n, C = 50, 96
    x, cache = (rand(i, n, C, dtype=BF16).cuda() for i in (1, 2))
    slot = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    none, want = torch.empty(0, C, dtype=BF16, device="cuda"), cache.clone()
    out, h_scale = torch.empty_like(x), torch.empty(0, device="cuda")
    for h_dtype, h in ((BF16, none), (I8, torch.empty(0, C, dtype=I8, device="cuda"))):
        desc = oc.block_norm_desc(n, C, oc.DTYPE_BF16, tag(oc, h_dtype), oc.DTYPE_F32, post_norm=oc.NORM_RMS, dense_rows=0)
        out.zero_()
        ctx.block_norm(desc, x, z=none, slot_of=slot, cache=cache, cache_out=cache, out=out, h=h, h_scale=h_scale)
        r, mag = ref_norm(d64(want), d64(want).abs(), "rms", 1e-6, None, None)
        assert_close(out, d64(x) + r, d64(x).abs() + mag)
        assert torch.equal(cache, want)
        desc = oc.block_norm_desc(n, C, oc.DTYPE_BF16, tag(oc, h_dtype), oc.DTYPE_F32, pre_norm=oc.NORM_RMS, dense_rows=0)
        ctx.block_norm(desc, x, slot_of=slot, h=h, h_scale=h_scale)           # norm and gather of no unit
    assert ctx.device_status() == oc.OK
    # with dense rows z cannot be left out beside a cache, nor all outputs
    desc = oc.block_norm_desc(n, C, oc.DTYPE_BF16, oc.DTYPE_BF16, oc.DTYPE_F32, dense_rows=2)
    assert ctx.block_norm(desc, x, slot_of=slot, cache=cache, out=out, check=False) == oc.ERR_INVALID_ARG
    assert ctx.block_norm(desc, x, slot_of=slot, check=False) == oc.ERR_INVALID_ARG


# ---- queues of row sets: more rows than one set for every resident CTA ---------------------------------------------
def ref_rows(x, z, slot, cache, p, post, pre, rows_per_group, unit_rows, dense_rows):
    """ref_block on the GPU (its helper tensors too)."""
    with torch.device("cuda"):
        return ref_block(x, z, slot, cache, p, 1.0, post, pre, 1e-6, rows_per_group, unit_rows, dense_rows)


def assert_rows_close(got, want, mag):
    """assert_close's bound, for finite values that stay on the GPU."""
    bound = 128 * U * mag
    if got.dtype == BF16:
        bound += 2.0 ** -8 * want.abs()
    assert torch.isfinite(got).all() and ((got.double() - want).abs() <= bound + 1e-37).all()


def check_queues(oc, ctx, n_units, unit_rows, C, dtype, h_dtype, param, post, pre, rows_per_group, in_place):
    """All seven parameters, a selection of 2 in 5 units with a dense tail that stays unused, a cache in place or beside."""
    kinds = {"rms": oc.NORM_RMS, "layer": oc.NORM_LAYER}
    n = n_units * unit_rows
    gen = torch.Generator(device="cuda").manual_seed(n + C)
    def draw(*shape, dt=dtype, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dt)
    keep = max(2 * n_units // 5, 1)
    kept = torch.randperm(n_units, generator=gen, device="cuda")[:keep].sort().values
    slot = torch.full((n_units,), -1, dtype=torch.int32, device="cuda")
    slot[kept] = torch.arange(keep, dtype=torch.int32, device="cuda")
    dense = (keep + 3) * unit_rows
    G = -(-n // rows_per_group)
    x, z, cache = draw(n, C, std=2.0), draw(dense, C), draw(n, C)
    mod = draw(G, 3 * C + 8, dt=param, std=0.3)
    p = {k: draw(C, dt=param, std=0.2, mean=float(k.endswith("_w"))) for k in ("post_w", "post_b", "pre_w", "pre_b")}
    p.update({k: mod[:, i * C:(i + 1) * C] for i, k in enumerate(("gate", "scale", "shift"))})
    r, mr, v, hh, mh, at = ref_rows(x.double(), z.double(), slot, cache.double(), {k: t.double() for k, t in p.items()}, post, pre,
                                    rows_per_group, unit_rows, dense)
    del mod
    out = x if in_place else torch.empty_like(x)
    cache_out = cache if in_place else torch.empty_like(cache)
    h = torch.full((dense, C), 9, dtype=h_dtype, device="cuda")
    h_scale = torch.full((dense,), 9.0, device="cuda") if h_dtype == I8 else None
    desc = oc.block_norm_desc(n, C, tag(oc, dtype), tag(oc, h_dtype), tag(oc, param), kinds[post], kinds[pre], 1e-6, 1e-6, 1.0,
                              rows_per_group, 3 * C + 8, unit_rows, dense)
    ctx.block_norm(desc, x, z=z, slot_of=slot, cache=cache, cache_out=cache_out, out=out, h=h, h_scale=h_scale, **p)
    assert ctx.device_status() == oc.OK
    assert torch.equal(cache_out.double(), v)
    assert_rows_close(out, r, mr)
    rows = torch.nonzero(at >= 0).reshape(-1)
    written, want, mag = at[rows], hh[rows], mh[rows]
    if h_dtype == I8:
        s, q = h_scale.double()[written], h.double()[written]
        top, top_mag = want.abs().amax(1), mag.amax(1)
        assert ((s * 127 - top).abs() <= 128 * U * (top_mag + top)).all()
        assert ((q * s[:, None] - want).abs() <= 0.5 * s[:, None] + 256 * U * (mag + top[:, None])).all()
        assert (h_scale[keep * unit_rows:] == 9).all()
    else:
        assert_rows_close(h[written], want, mag)
    assert (h[keep * unit_rows:] == 9).all()


# units, rows of a unit, columns, type, type of h, of the parameters, norms, rows of a group.  8, 32, 64, 256 and 512
# threads per row; of the first four both lengths of queue, with room for twice the CTAs that fit today; groups that end
# inside a set of rows, a set's length, and whole queues apart; row counts that are no whole number of sets.
QUEUES = [(100003, 1, 64, BF16, BF16, F32, "rms", "layer", 997), (33335, 3, 64, BF16, I8, BF16, "layer", "rms", 37),
          (400003, 1, 8, BF16, F32, F32, "layer", "layer", 7), (400003, 1, 16, F32, I8, BF16, "rms", "rms", 30001),
          (20011, 1, 640, BF16, I8, F32, "layer", "layer", 1024), (6671, 3, 640, BF16, BF16, BF16, "rms", "rms", 50),
          (310001, 1, 520, BF16, BF16, F32, "rms", "layer", 9216), (103335, 3, 528, BF16, I8, F32, "rms", "layer", 13),
          (12003, 1, 1536, BF16, I8, BF16, "rms", "layer", 4096), (4001, 3, 772, F32, F32, F32, "layer", "rms", 5),
          (152003, 1, 1296, BF16, I8, F32, "layer", "rms", 1000), (5003, 1, 3200, BF16, I8, BF16, "rms", "rms", 777),
          (152003, 1, 1540, F32, BF16, BF16, "rms", "layer", 64), (2001, 3, 3088, F32, I8, F32, "layer", "layer", 11)]


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", QUEUES, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}")
def test_block_norm_queues_of_row_sets(oc, ctx, case, in_place):
    check_queues(oc, ctx, *case, in_place)


@pytest.mark.gpu
@pytest.mark.parametrize("n,C,groups", [(100003, 64, 1), (20011, 640, 5), (12003, 1536, 1)])
@pytest.mark.parametrize("h_dtype", [BF16, I8])
def test_block_norm_queues_without_a_block(oc, ctx, n, C, groups, h_dtype):
    """Norm, modulation and gather alone: the kernels that hold no block's output."""
    x = rand(n, n, C, dtype=BF16, std=2.0).cuda()
    scale, shift = (rand(i, groups, C, std=0.3).cuda() for i in (1, 2))
    slot = slots(n, 2 * n // 5, seed=C).cuda()
    rows, per = torch.nonzero(slot >= 0).reshape(-1), -(-n // groups)
    h, s = torch.full((rows.numel(), C), 9, dtype=h_dtype, device="cuda"), torch.full((rows.numel(),), 9.0, device="cuda")
    desc = oc.block_norm_desc(n, C, oc.DTYPE_BF16, tag(oc, h_dtype), oc.DTYPE_F32, pre_norm=oc.NORM_LAYER, rows_per_group=per,
                              mod_stride=C, dense_rows=rows.numel())
    ctx.block_norm(desc, x, slot_of=slot, scale=scale, shift=shift, h=h, h_scale=s if h_dtype == I8 else None)
    assert ctx.device_status() == oc.OK
    v = x[rows].double()
    want, mag = ref_norm(v, v.abs(), "layer", 1e-6, None, None)
    g = rows // per
    want, mag = want * (1 + scale.double()[g]) + shift.double()[g], mag * (1 + scale.double()[g].abs()) + shift.double()[g].abs()
    if h_dtype == I8:
        top = want.abs().amax(1)
        assert ((s.double() * 127 - top).abs() <= 128 * U * (mag.amax(1) + top)).all()
        assert ((h.double() * s.double()[:, None] - want).abs() <= 0.5 * s.double()[:, None] + 256 * U * (mag + top[:, None])).all()
    else:
        assert_rows_close(h, want, mag)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(20000, 320, 2560), (9000, 880, 2816)])
@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_linear_int8_resident_weights_to_named_places(oc, ctx, M, K, N, out_dtype):
    """Tiles enough for the form that keeps its rows of w in shared memory, and rows of out that do not keep their order."""
    idx = torch.randperm(M + 50, generator=torch.Generator().manual_seed(M))[:M].to(torch.int32)
    idx[M // 2] = -1
    run_linear(oc, ctx, M, K, N, out_dtype, out_idx=idx, out_rows=M + 50)
    run_linear(oc, ctx, M, K, N, out_dtype, out_idx=idx, out_rows=M + 50, pad=1, bias=False)
    assert ctx.device_status() == oc.OK


@pytest.mark.gpu
def test_rope_and_int8_on_another_stream_and_in_a_graph(oc, ctx):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run_rope(oc, ctx, 60, 64, (16, 24, 24), (3, 4, 5), 5, 2, BF16, "halves", norm=True)
        run_linear(oc, ctx, 2, 144, 100)
        run_linear(oc, ctx, 300, 144, 104)
        run_linear(oc, ctx, 20000, 320, 2560)
    torch.cuda.current_stream().wait_stream(side)
    M, K, N, D = 300, 128, 192, 64
    x, w = rand(1, M, K, dtype=BF16).cuda(), torch.randint(-127, 128, (N, K), generator=torch.Generator().manual_seed(2)).to(I8).cuda()
    a, s, sw = torch.empty(M, K, dtype=I8, device="cuda"), torch.empty(M, device="cuda"), torch.full((N,), 0.01, device="cuda")
    y, r = torch.empty(M, N, dtype=BF16, device="cuda"), torch.empty(M, N // D, D, dtype=BF16, device="cuda")
    q = y.view(M, N // D, D)
    d = oc.rope_desc(M, oc.DTYPE_BF16, D, (0, 32, 32), (1, 15, 20), N // D, q=q, q_out=r)
    table = oc.rope_table(d).cuda()

    def step():
        ctx.quantize_rows(x, oc.DTYPE_BF16, M, K, a, s)
        ctx.linear_int8(a, s, M, K, w, sw, N, y, oc.DTYPE_BF16)
        ctx.rope(d, table, q, r)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (a, s, y, r)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t in (a, s, y, r):
        t.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, u) for t, u in zip((a, s, y, r), want))
    assert ctx.device_status() == oc.OK


@pytest.mark.gpu
def test_quantize_rows_of_a_column_range(oc, ctx):
    """A part of a packed projection, its stride taken from the tensor."""
    x = rand(1, 40, 3 * 64, dtype=BF16).cuda()
    q, s = torch.empty(40, 64, dtype=I8, device="cuda"), torch.empty(40, device="cuda")
    want_q, want_s = torch.empty_like(q), torch.empty_like(s)
    ctx.quantize_rows(x[:, 64:128], oc.DTYPE_BF16, 40, 64, q, s)
    ctx.quantize_rows(x[:, 64:128].contiguous(), oc.DTYPE_BF16, 40, 64, want_q, want_s)
    assert torch.equal(q, want_q) and torch.equal(s, want_s)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 40, 300])
def test_linear_int8_into_a_column_range(oc, ctx, M):
    """A part of a packed tensor, its stride taken from it; the columns beside it stay."""
    K, N = 64, 40
    g = torch.Generator().manual_seed(M)
    a, w = (torch.randint(-127, 128, (n, K), generator=g).to(I8).cuda() for n in (M, N))
    one, packed = torch.ones(max(M, N), device="cuda"), torch.full((M, 3 * N), 5.0, device="cuda")
    ctx.linear_int8(a, one[:M], M, K, w, one[:N], N, packed[:, N:2 * N], oc.DTYPE_F32)
    assert torch.equal(packed[:, N:2 * N].double(), a.double() @ w.double().t())
    assert (packed[:, :N] == 5).all() and (packed[:, 2 * N:] == 5).all()


@pytest.mark.gpu
def test_rope_outputs_have_a_place_for_every_head(oc, ctx):
    """Several heads, rows or batch elements of an output at a stride of 0 would be written over one another: refused.  Of
    an input they are a broadcast."""
    n, D = 8, 64
    x, o = torch.zeros(n, 2, D, dtype=BF16, device="cuda"), torch.zeros(n, 2, D, dtype=BF16, device="cuda")
    good = (4 * 128, 128, 64)

    def st(heads=2, rows=n, rpb=4, **views):
        v = {m: good for m in ("q", "q_out", "k", "k_out")}
        v.update(views)
        d = oc.rope_desc(rows, oc.DTYPE_BF16, D, (0, 32, 32), (1, 2, 4), heads, heads, rows_per_batch=rpb, **v)
        return ctx.rope(d, oc.rope_table(d).cuda(), x, o, k=x, k_out=o.clone(), check=False)
    assert st() == oc.OK
    for m in ("q_out", "k_out"):
        assert st(**{m: (512, 128, 0)}) == oc.ERR_INVALID_ARG
        assert st(**{m: (512, 0, 64)}) == oc.ERR_INVALID_ARG
        assert st(**{m: (0, 128, 64)}) == oc.ERR_INVALID_ARG
        assert st(rpb=n, **{m: (0, 128, 64)}) == oc.OK                        # one batch element
        assert st(rpb=n + 3, **{m: (0, 128, 64)}) == oc.OK
        assert st(heads=1, **{m: (512, 128, 0)}) == oc.OK
        assert st(rpb=1, **{m: (128, 0, 64)}) == oc.OK                        # every row a batch element
        assert st(rows=1, **{m: (0, 0, 64)}) == oc.OK
    for m in ("q", "k"):
        assert st(**{m: (0, 0, 0)}) == oc.OK
    # a descriptor made without a tensor's strides (for a table) is none for a call
    full = oc.rope_desc(n, oc.DTYPE_BF16, D, (0, 32, 32), (1, 2, 4), 2, 2, q=x, q_out=o, k=x, k_out=o)
    table = oc.rope_table(full).cuda()
    for left_out in ("q", "q_out", "k", "k_out"):
        t = {m: v for m, v in dict(q=x, q_out=o, k=x, k_out=o).items() if m != left_out}
        d = oc.rope_desc(n, oc.DTYPE_BF16, D, (0, 32, 32), (1, 2, 4), 2, 2, **t)
        assert torch.equal(oc.rope_table(d), oc.rope_table(full))
        assert ctx.rope(d, table, x, o, k=x, k_out=o.clone(), check=False) == oc.ERR_INVALID_ARG
    # (a single row of a single head lies wherever its pointer says)
    one = oc.rope_desc(1, oc.DTYPE_BF16, D, (0, 32, 32), (1, 2, 4), 1)
    assert ctx.rope(one, table, x, o, check=False) == oc.OK
    assert ctx.device_status() == oc.OK
