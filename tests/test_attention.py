"""The paged cache (oc_kv_put, oc_kv_get) and attention over it (oc_attention) against plain restatements in 64 bits.

Tolerances.  u = 2^-24 is the unit roundoff of fp32, b = 2^-8 that of bf16 (half a step, relative to the value).

Cache: a copy is exact.  A whole number is rint(x L / max|x|) of the inputs as they are, so it has to be equal.  Its scale
is max|x| * fl(1 / L): 2 u.  A value q * scale read back: 3 u, plus b in bf16.

Attention.  A score is a sum of D products in fp32 (products of bf16 are exact): off by at most (D + 2) u sum_d |q_d k_d|,
and (with whole numbers) 3 u of it for the scales; times the softmax scale that is e in the exponent, where the product with
log2(e) and the subtraction of the maximum add 4 u times the largest |exponent|.  The largest e of a row bounds the
relative error of every p and of their sum, which adds at most 2^-12 for the exponential itself (a polynomial of degree 3 and
better) and one u per addition.  A probability in bf16 adds b where it meets V.  So
    |out - exact| <= (2 e + n u + 2 * 2^-12 [bf16: + b] ) * sum_j p_j |v_j| + (D + n) u sum_j p_j |v_j| + b |exact| [bf16]
with n keys; in fp32 the exponential is exp2f, good to 2 ulp: 8 u in the place of 2 * 2^-12.
"""
import math

import pytest
import torch

U, B16 = 2.0 ** -24, 2.0 ** -8
BF16, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


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


def tag(oc, t):
    return {F32: oc.DTYPE_F32, BF16: oc.DTYPE_BF16, "i8": oc.DTYPE_I8, "i4": oc.DTYPE_I4}[t]


def rand(gen, *shape, dtype=F32, std=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * std).to(dtype)


def levels(x, kind):
    """(whole numbers, scales) of the last axis, by the definition"""
    L = 127 if kind == "i8" else 7
    x = x.double()
    most = x.abs().amax(-1, keepdim=True)
    small, strange = most < 2.0 ** -100, ~torch.isfinite(most) | torch.isnan(x).any(-1, keepdim=True)
    q = torch.round(x * L / most)
    q = torch.where(small | strange, torch.zeros_like(q), q)
    scale = torch.where(strange, most, torch.where(small, torch.zeros_like(most), most / L))
    return q.to(torch.int8), scale.squeeze(-1)


def pack(q):
    q = q.to(torch.uint8) & 15
    return q[..., 0::2] | (q[..., 1::2] << 4)


def unpack(q):
    q = torch.stack([q & 15, q >> 4], -1).flatten(-2).to(torch.int8)
    return torch.where(q > 7, q - 16, q)


class Cache:
    """A cache on the CPU and on the GPU: n_seqs sequences of seq_rows tokens in shuffled pages of a larger pool, every
    place that belongs to no token of `lens` filled with NaN (or numbers with NaN scales)."""

    def __init__(self, oc, kind, heads, D, n_seqs, seq_rows, page_rows=16, lens=None, seed=0, spare=3, table=True, empty=False):
        self.oc, self.kind, self.heads, self.D, self.n_seqs, self.seq_rows, self.page_rows = oc, kind, heads, D, n_seqs, seq_rows, page_rows
        gen = torch.Generator().manual_seed(seed)
        per = -(-seq_rows // page_rows)
        self.pages = n_seqs * per + (spare if table else 0)
        order = torch.randperm(self.pages, generator=gen) if table else torch.arange(self.pages)
        self.table = order[: n_seqs * per].to(torch.int32).view(n_seqs, per)
        self.desc = oc.kv_desc(tag(oc, kind), heads, D, n_seqs, seq_rows, page_rows, n_pages=self.pages)
        lens = [seq_rows] * n_seqs if lens is None else lens
        self.lens = lens
        self.val, self.pool, self.scale = {}, {}, {}
        for m in "kv":
            x = rand(gen, n_seqs, seq_rows, heads, D)
            if not isinstance(kind, str):
                pool, scale, vals = torch.full((self.pages, heads, page_rows, D), NAN, dtype=kind), None, x.to(kind)
            else:
                q, sc = levels(x, kind)
                sc = sc.float()
                pool = torch.randint(-7, 8, (self.pages, heads, page_rows, D), generator=gen, dtype=torch.int8)
                scale = torch.full((self.pages, heads, page_rows), NAN)
                vals = q.double() * sc.double()[..., None]
            if empty:
                vals = torch.full_like(vals, NAN)
            for s in range(n_seqs):
                for t in range(0 if empty else lens[s]):
                    pg, r = self.place(s, t)
                    if scale is None:
                        pool[pg, :, r] = vals[s, t]
                    else:
                        pool[pg, :, r], scale[pg, :, r] = q[s, t], sc[s, t]
            self.val[m] = vals.double()
            self.pool[m] = (pack(pool) if kind == "i4" else pool).cuda()
            self.scale[m] = None if scale is None else scale.cuda()
        self.gpu_table = self.table.cuda() if table else None

    def place(self, s, t):
        return int(self.table[s, t // self.page_rows]), t % self.page_rows

    def args(self):
        return dict(k_scale=self.scale["k"], v_scale=self.scale["v"], page_table=self.gpu_table)

    def tokens(self, m):
        """What the GPU's pool holds: (whole numbers or values [n_seqs, seq_rows, heads, D], scales or None)"""
        pool = self.pool[m].cpu()
        pool = unpack(pool) if self.kind == "i4" else pool
        per = self.table.shape[1]
        seqs = pool[self.table.long()].permute(0, 1, 3, 2, 4).reshape(self.n_seqs, per * self.page_rows, self.heads, self.D)[:, : self.seq_rows]
        if self.scale[m] is None:
            return seqs, None
        sc = self.scale[m].cpu()[self.table.long()].permute(0, 1, 3, 2).reshape(self.n_seqs, per * self.page_rows, self.heads)[:, : self.seq_rows]
        return seqs, sc


# ---- the cache --------------------------------------------------------------------------------------------------------
KINDS = [(F32, F32), (BF16, BF16), (F32, "i8"), (BF16, "i8"), (F32, "i4"), (BF16, "i4")]


def same(a, b):
    return torch.equal(torch.nan_to_num(a.double(), nan=1234.5), torch.nan_to_num(b.double(), nan=1234.5))


def check_put(cache, m, rows, tokens):
    """rows [n, heads, D] were written as `tokens`"""
    got, scale = cache.tokens(m)
    got = got.reshape(-1, cache.heads, cache.D)[tokens]
    if scale is None:
        assert same(got, rows)
        return
    q, sc = levels(rows, cache.kind)
    assert torch.equal(got, q)
    scale = scale.reshape(-1, cache.heads)[tokens].double()
    fine = torch.isfinite(sc)
    assert torch.equal(torch.isnan(scale), torch.isnan(sc)) and torch.equal(torch.isinf(scale), torch.isinf(sc))
    assert ((scale - sc).abs()[fine] <= 2 * U * sc[fine]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("D", [8, 40, 64, 72, 128, 256])
@pytest.mark.parametrize("heads,page_rows,n", [(1, 16, 1), (5, 48, 37), (9, 64, 130)])
def test_put_and_get(oc, ctx, dtype, kind, D, heads, page_rows, n):
    cache = Cache(oc, kind, heads, D, 2, 100, page_rows, empty=True)
    before = {m: cache.pool[m].clone() for m in "kv"}
    gen = torch.Generator().manual_seed(n)
    tokens = torch.randperm(200, generator=gen)[:n].sort().values
    idx = torch.cat([tokens, torch.tensor([-1, -1, -1])]).to(torch.int32)
    k, v = (rand(gen, n + 3, heads, D, dtype=dtype, std=3.0) for _ in range(2))
    packed = torch.zeros(n + 3, 3 * heads, D, dtype=dtype)
    packed[:, heads:2 * heads] = v
    packed = packed.cuda()
    # keys [batch, heads, rows, D], values out of a packed projection
    kk = k.view(1, n + 3, heads, D).transpose(1, 2).contiguous().cuda()
    vv = packed[:, heads:2 * heads]
    d = oc.kv_rows(cache.desc, n + 3, tag(oc, dtype), k=kk, v=vv)
    ctx.kv_put(cache.desc, d, kk, cache.pool["k"], vv, cache.pool["v"], idx=idx.cuda(), **cache.args())
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.OK
    for m, rows in (("k", k), ("v", v)):
        check_put(cache, m, rows[:n], tokens)
        # nothing else was written
        touched = torch.zeros(cache.pages, heads, page_rows, dtype=torch.bool)
        for t in tokens.tolist():
            pg, r = cache.place(t // 100, t % 100)
            touched[pg, :, r] = True
        assert same(cache.pool[m].cpu()[~touched], before[m].cpu()[~touched])
    # back, in another order, with rows left alone
    back = torch.stack([idx.flip(0), idx.flip(0)], 1).reshape(-1)
    out = {m: torch.full((2 * (n + 3), heads, D), 77.0, dtype=dtype, device="cuda") for m in "kv"}
    d = oc.kv_rows(cache.desc, 2 * (n + 3), tag(oc, dtype), k=out["k"], v=out["v"])
    ctx.kv_get(cache.desc, d, cache.pool["k"], out["k"], cache.pool["v"], out["v"], idx=back.cuda(), **cache.args())
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.OK
    for m, rows in (("k", k), ("v", v)):
        got = out[m].cpu().double()
        live = back >= 0
        assert (got[~live] == 77.0).all()
        want = rows[:n].flip(0).repeat_interleave(2, 0)
        if not isinstance(kind, str):
            assert same(got[live], want)
            continue
        q, sc = levels(want, kind)
        want = q.double() * sc[..., None]
        assert ((got[live] - want).abs() <= (3 * U + (B16 if dtype == BF16 else 0)) * want.abs()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["i8", "i4"])
def test_put_rounds_as_defined(oc, ctx, dtype, kind):
    """Ties and their neighbours: the largest value makes quotients exact halves; then values of every kind."""
    L = 127 if kind == "i8" else 7
    heads, D, n = 4, 64, 64
    gen = torch.Generator().manual_seed(1)
    x = rand(gen, n, heads, D, dtype=dtype)
    x[:16] = (torch.randint(-2 * L, 2 * L + 1, (16, heads, D), generator=gen).double() / 2).to(dtype)       # halves, L the largest
    x[:16, :, 0] = L
    x[16:24] = (torch.randint(-2 * L, 2 * L + 1, (8, heads, D), generator=gen).double() / 2 * 2.0 ** -40).to(dtype)
    x[16:24, :, 0] = -L * 2.0 ** -40
    x[24:32] = (x[24:32].double() * 2.0 ** 100).to(dtype)
    x[32:36] = (torch.randint(-3, 4, (4, heads, D), generator=gen)).to(dtype)                              # few levels, a maximum of 3
    x[32:36, :, 5] = 3
    if dtype == F32:                                                                                        # a step beside a tie
        x[36:44] = (torch.randint(-2 * L + 1, 2 * L, (8, heads, D), generator=gen).double() / 2 * (1 + 2.0 ** -23)).to(dtype)
        x[36:44, :, 0] = L
    x[60], x[61] = 0.0, 2.0 ** -101
    x[62, 0, 3], x[62, 1, 4], x[63, 2, 5] = math.inf, -math.inf, NAN
    cache = Cache(oc, kind, heads, D, 1, n, 16, empty=True)
    xx = x.cuda()
    ctx.kv_put(cache.desc, oc.kv_rows(cache.desc, n, tag(oc, dtype), k=xx), xx, cache.pool["k"], k_scale=cache.scale["k"], page_table=cache.gpu_table)
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.OK
    check_put(cache, "k", x, torch.arange(n))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("shift,pad", [(1, 0), (4, 4), (0, 3), (8, 8)])
def test_put_and_get_alignments(oc, ctx, dtype, kind, shift, pad):
    n, heads, D = 33, 3, 72
    cache = Cache(oc, kind, heads, D, 1, n, 16, table=False, empty=True)
    gen = torch.Generator().manual_seed(5)
    store = rand(gen, n * heads * (D + pad) + shift, dtype=dtype)
    view = store.as_strided((n, heads, D), (heads * (D + pad), D + pad, 1), shift)
    gs = store.cuda()
    gv = gs.as_strided((n, heads, D), (heads * (D + pad), D + pad, 1), shift)
    d = oc.kv_rows(cache.desc, n, tag(oc, dtype), k=gv, v=gv)
    ctx.kv_put(cache.desc, d, gv, cache.pool["k"], gv, cache.pool["v"], **cache.args())
    check_put(cache, "v", view, torch.arange(n))
    back = torch.full_like(gs, 55.0)
    bv = back.as_strided((n, heads, D), (heads * (D + pad), D + pad, 1), shift)
    ctx.kv_get(cache.desc, oc.kv_rows(cache.desc, n, tag(oc, dtype), k=bv), cache.pool["v"], bv, k_scale=cache.scale["v"])
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.OK
    want = view.double()
    if isinstance(kind, str):
        q, sc = levels(view, kind)
        want = q.double() * sc[..., None]
    assert ((bv.cpu().double() - want).abs() <= (3 * U + (B16 if dtype == BF16 else 0)) * want.abs()).all()
    rest = torch.ones(back.numel(), dtype=torch.bool)
    rest.as_strided((n, heads, D), (heads * (D + pad), D + pad, 1), shift).fill_(False)
    assert (back.cpu()[rest] == 55.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, "i8", "i4"])
def test_pages_and_tokens_outside(oc, ctx, kind):
    """Numbers outside the pool or the cache write nothing, read zeros or leave rows as they were, and are recorded."""
    heads, D, n = 2, 64, 64
    cache = Cache(oc, kind, heads, D, 1, n, 16, empty=True)
    table = cache.table.clone()
    table[0, 1], table[0, 2] = cache.pages, -1
    gt = table.cuda()
    gen = torch.Generator().manual_seed(2)
    x = rand(gen, n + 2, heads, D, dtype=BF16)
    xx = x.cuda()
    idx = torch.cat([torch.arange(n), torch.tensor([n, 2 ** 31 - 1])]).to(torch.int32).cuda()
    before = cache.pool["k"].clone()
    d = oc.kv_rows(cache.desc, n + 2, oc.DTYPE_BF16, k=xx)
    ctx.kv_put(cache.desc, d, xx, cache.pool["k"], k_scale=cache.scale["k"], page_table=gt, idx=idx)
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.ERR_INVALID_ARG and ctx.device_status() == oc.OK
    live = torch.cat([torch.arange(16), torch.arange(48, 64)])
    check_put(cache, "k", x[live], live)
    untouched = [p for p in range(cache.pages) if p not in (int(table[0, 0]), int(table[0, 3]))]
    assert same(cache.pool["k"].cpu()[untouched], before.cpu()[untouched])
    out = torch.full((n + 2, heads, D), 9.0, dtype=BF16, device="cuda")
    ctx.kv_get(cache.desc, oc.kv_rows(cache.desc, n + 2, oc.DTYPE_BF16, k=out), cache.pool["k"], out, k_scale=cache.scale["k"], page_table=gt, idx=idx)
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.ERR_INVALID_ARG
    assert (out[16:48] == 0).all() and (out[n:] == 9.0).all() and (out[:16] != 9.0).any()


@pytest.mark.gpu
def test_cache_offsets_past_32_bits(oc, ctx):
    """Pools of over 4 GB: the last pages."""
    heads, D, page = 2, 128, 64
    pages = 70000                                                            # x 2 x 64 x 128 x 4 bytes = 4.6 GB
    desc = oc.kv_desc(oc.DTYPE_F32, heads, D, 1, 128, page, n_pages=pages)
    pool = torch.empty(pages, heads, page, D, device="cuda")
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    x = torch.randn(128, heads, D, device="cuda")
    ctx.kv_put(desc, oc.kv_rows(desc, 128, oc.DTYPE_F32, k=x), x, pool, page_table=table)
    y = torch.empty_like(x)
    ctx.kv_get(desc, oc.kv_rows(desc, 128, oc.DTYPE_F32, k=y), pool, y, page_table=table)
    torch.cuda.synchronize()
    assert torch.equal(x, y) and torch.equal(pool[pages - 1].transpose(0, 1), x[:64])
    assert ctx.device_status() == oc.OK
    q, out = torch.randn(3, heads, D, device="cuda"), torch.empty(3, heads, D, device="cuda")
    ctx.attention(desc, oc.attention_desc(desc, 3, oc.DTYPE_F32, heads, 0.1, q=q, out=out), q, pool, pool, out, page_table=table)
    p = torch.softmax(torch.einsum("rhd,jhd->hrj", q.double(), x.double()) * 0.1, -1)
    want = torch.einsum("hrj,jhd->rhd", p, x.double())
    assert (out.double() - want).abs().max() <= 400 * U * 8                   # (|v| < 8: the bound above with n = D = 128)


# ---- attention --------------------------------------------------------------------------------------------------------
def seen_by(p, length, unit, back, ahead):
    """The keys that a row at position p sees"""
    j = torch.arange(length)
    ok = torch.ones(length, dtype=torch.bool)
    if unit > 0:
        apart = torch.div(j, unit, rounding_mode="floor") - math.floor(p / unit)
        if back >= 0:
            ok &= apart >= -back
        if ahead >= 0:
            ok &= apart <= ahead
    return ok


def exact(cache, q, rows, scale, unit=0, back=-1, ahead=-1):
    """q [rows, heads, D]; rows: (sequence, position) of each, or None.  (out, its bound without the output's rounding, lse)"""
    n, H, D = q.shape
    G = H // cache.heads
    out, bound = torch.zeros(n, H, D, dtype=torch.float64), torch.zeros(n, H, D, dtype=torch.float64)
    lse = torch.full((n, H), -math.inf, dtype=torch.float64)
    lse_bound = torch.zeros(n, H, dtype=torch.float64)
    bf16 = q.dtype == BF16
    for s in sorted({r[0] for r in rows if r is not None}):
        mine = [i for i, r in enumerate(rows) if r is not None and r[0] == s]
        L = cache.lens[s]
        if L == 0:
            continue
        k, v = (cache.val[m][s, :L].repeat_interleave(G, 1).transpose(0, 1) for m in "kv")        # [H, L, D]
        ok = torch.stack([seen_by(rows[i][1], L, unit, back, ahead) for i in mine])                 # [r, L]
        qq = q[mine].double().transpose(0, 1)                                                      # [H, r, D]
        sc = qq @ k.transpose(1, 2) * scale
        mag = qq.abs() @ k.abs().transpose(1, 2) * scale
        e = (((D + 5) * U * mag + 4 * U * sc.abs()).masked_fill(~ok, 0)).amax(-1, keepdim=True)
        sc = sc.masked_fill(~ok, -math.inf)
        ls = torch.logsumexp(sc, -1, keepdim=True)
        p = torch.where(ok & (sc > -math.inf), torch.exp(sc - ls), torch.zeros_like(sc))
        e = e + 4 * U * (sc.masked_fill(~ok, 0).abs().amax(-1, keepdim=True) + ls.masked_fill(~ok.any(-1, keepdim=True), 0).abs())
        got, pv = p @ v, p @ v.abs()
        rel = 2 * e + (2 * L + D) * U + (2 * 2.0 ** -12 + B16 if bf16 else 8 * U)
        out[mine], bound[mine] = got.transpose(0, 1), (rel * pv).transpose(0, 1)
        lse[mine] = ls[..., 0].T
        lse_bound[mine] = (e + L * U + (2.0 ** -12 if bf16 else 8 * U) + 4 * U * ls.abs())[..., 0].T
    return out, bound, lse, lse_bound


def assert_attn(out, want, bound, rows, untouched=5.0):
    got = out.cpu().double()
    bound = bound + (B16 if out.dtype == BF16 else 2 * U) * want.abs() + 1e-30
    for i, r in enumerate(rows):
        if r is None:
            assert (got[i] == untouched).all(), f"row {i} was written"
    live = [i for i, r in enumerate(rows) if r is not None]
    if live:
        over = ((got - want).abs() / bound)[live]
        assert not torch.isnan(over).any(), "NaN"
        assert over.max() <= 1, f"off by {over.max():.2f} of what is allowed at row {live[int(over.amax((1, 2)).argmax())]}"


def run(oc, ctx, cache, q, n_seqs_rows, scale=None, unit=0, back=-1, ahead=-1, idx=None, ragged=False, lse=True, seed=0, check=True, stream=None):
    """q [n, heads, D] on the CPU; n_seqs_rows: rows of each sequence (all alike unless ragged).  Checks out and lse."""
    n, H, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    rows, at = [], 0
    for s, m in enumerate(n_seqs_rows):
        for i in range(m):
            p = cache.lens[s] - m + i if idx is None else int(idx[at + i]) - s * cache.seq_rows
            rows.append(None if idx is not None and idx[at + i] < 0 else (s, p))
        at += m
    rows += [None] * (n - at)
    qq = q.cuda()
    out = torch.full((n, H, D), 5.0, dtype=q.dtype, device="cuda")
    ls = torch.full((n, H), 5.0, device="cuda") if lse else None
    start = None
    if ragged:
        start = torch.tensor([sum(n_seqs_rows[:i]) for i in range(len(n_seqs_rows) + 1)], dtype=torch.int32).cuda()
    d = oc.attention_desc(cache.desc, n, tag(oc, q.dtype), H, scale, rows_per_batch=max(max(n_seqs_rows), 1), unit=unit, back=back, ahead=ahead, q=qq, out=out)
    lens = torch.tensor(cache.lens, dtype=torch.int32).cuda()
    ctx.attention(cache.desc, d, qq, cache.pool["k"], cache.pool["v"], out, kv_len=lens, q_start=start,
                  idx=None if idx is None else idx.to(torch.int32).cuda(), lse=ls, stream=stream, **cache.args())
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.OK
    if check:
        want, bound, wl, bl = exact(cache, q, rows, scale, unit, back, ahead)
        assert_attn(out, want, bound, rows)
        if lse:
            got = ls.cpu().double()
            for i, r in enumerate(rows):
                if r is None:
                    assert (got[i] == 5.0).all()
                else:
                    empty = wl[i] == -math.inf
                    assert torch.equal(got[i] == -math.inf, empty)
                    assert ((got[i] - wl[i]).abs()[~empty] <= bl[i][~empty]).all()
    return out


TYPES = [(BF16, BF16), (BF16, "i8"), (BF16, "i4"), (F32, F32), (F32, "i8"), (F32, "i4")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("keys", [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 1100])
@pytest.mark.parametrize("rows", [1, 5, 200])
def test_attention_lengths(oc, ctx, dtype, kind, keys, rows):
    cache = Cache(oc, kind, 2, 64, 1, max(keys, 1), 16 if keys < 200 else 48, lens=[keys], seed=keys)
    q = rand(torch.Generator().manual_seed(rows), rows, 2, 64, dtype=dtype)
    run(oc, ctx, cache, q, [rows])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("D", [8, 16, 24, 32, 40, 64, 72, 80, 96, 104, 120, 128])
@pytest.mark.parametrize("rows", [1, 40])
def test_attention_head_dims(oc, ctx, dtype, kind, D, rows):
    cache = Cache(oc, kind, 2, D, 1, 275, 32, seed=D)
    q = rand(torch.Generator().manual_seed(rows), rows, 2, D, dtype=dtype)
    run(oc, ctx, cache, q, [rows])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 2), (6, 2), (8, 1), (16, 2), (20, 1)])
@pytest.mark.parametrize("rows", [1, 2, 3, 37, 130])
def test_attention_shared_heads(oc, ctx, dtype, kind, heads, kv, rows):
    cache = Cache(oc, kind, kv, 72, 2, 210, 16, lens=[210, 133], seed=heads)
    q = rand(torch.Generator().manual_seed(rows), 2 * rows, heads, 72, dtype=dtype)
    run(oc, ctx, cache, q, [rows, rows], unit=1, ahead=0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 513])
def test_attention_row_counts(oc, ctx, dtype, kind, rows):
    cache = Cache(oc, kind, 1, 64, 1, 600, 64, seed=rows)
    q = rand(torch.Generator().manual_seed(rows), rows, 1, 64, dtype=dtype)
    run(oc, ctx, cache, q, [rows], unit=1, ahead=0)


MASKS = [(1, -1, 0), (1, 0, 0), (1, 3, 0), (1, 200, -1), (1, -1, 5), (64, -1, 0), (37, 0, 0), (37, 1, 1), (37, 2, 0), (128, -1, 0), (300, 0, 0),
         (2 ** 31 - 1, 0, 0), (1, 2 ** 40, 2 ** 40)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("unit,back,ahead", MASKS)
@pytest.mark.parametrize("kept", [False, True])
def test_attention_windows(oc, ctx, dtype, kind, unit, back, ahead, kept):
    keys, rows, gen = [700, 411], 180, torch.Generator().manual_seed(unit % 1000)
    cache = Cache(oc, kind, 2, 72, 2, 700, 32, lens=keys, seed=3)
    q = rand(gen, 2 * rows, 2, 72, dtype=dtype)
    idx = None
    if kept:                                                                 # ascending tokens with an unused tail; some beyond the keys
        idx = torch.cat([torch.cat([torch.randperm(700, generator=gen)[: rows - 7].sort().values + 700 * s, torch.full((7,), -1)]) for s in range(2)])
    run(oc, ctx, cache, q, [rows, rows], unit=unit, back=back, ahead=ahead, idx=idx)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("lens,rows", [([300, 0, 5, 129, 64], [70, 0, 5, 1, 64]), ([40, 40], [3, 60]), ([500] * 9, [1, 2, 0, 130, 16, 17, 257, 5, 8])])
def test_attention_packed_sequences(oc, ctx, dtype, kind, lens, rows):
    """Ragged rows behind one another; more rows than keys (positions before the first key see nothing); rows behind the last."""
    cache = Cache(oc, kind, 2, 40, len(lens), max(lens), 16, lens=lens, seed=7)
    q = rand(torch.Generator().manual_seed(8), sum(rows) + 9, 4, 40, dtype=dtype)
    run(oc, ctx, cache, q, rows, unit=1, ahead=0, ragged=True)
    run(oc, ctx, cache, q, rows, ragged=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [(BF16, BF16), (BF16, "i8"), (F32, F32)])
def test_attention_rows_behind_the_last_sequence(oc, ctx, dtype, kind):
    cache = Cache(oc, kind, 2, 64, 2, 100, 16, seed=7)
    q = rand(torch.Generator().manual_seed(8), 50, 2, 64, dtype=dtype)
    run(oc, ctx, cache, q, [20, 20])                                         # 10 rows too many
    run(oc, ctx, cache, q[:33], [20, 13], ragged=True)
    lens = cache.lens                                                        # and a last sequence with fewer rows than the others
    qq, out = q[:33].cuda(), torch.full((33, 2, 64), 5.0, dtype=dtype, device="cuda")
    d = oc.attention_desc(cache.desc, 33, tag(oc, dtype), 2, 0.125, rows_per_batch=20, q=qq, out=out)
    ctx.attention(cache.desc, d, qq, cache.pool["k"], cache.pool["v"], out, kv_len=torch.tensor(lens, dtype=torch.int32).cuda(), **cache.args())
    rows = [(i // 20, 0) for i in range(33)]
    want, bound, _, _ = exact(cache, q[:33], rows, 0.125)
    assert_attn(out, want, bound, rows)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 7, 150])
def test_attention_long_caches_few_rows(oc, ctx, dtype, kind, rows):
    """Keys split over the CTAs of a cluster, some of them without any."""
    lens = [5000, 1, 77, 2049]
    cache = Cache(oc, kind, 1, 64, 4, 5000, 64, lens=lens, seed=9)
    q = rand(torch.Generator().manual_seed(rows), 4 * rows, 2, 64, dtype=dtype, std=2.0)
    run(oc, ctx, cache, q, [rows] * 4)
    run(oc, ctx, cache, q, [rows] * 4, unit=1, back=600, ahead=0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 140])
def test_attention_large_scores(oc, ctx, dtype, kind, rows):
    """The running maximum grows by hundreds, early and late; and scores all far below zero."""
    cache = Cache(oc, kind, 1, 64, 1, 700, 32, seed=11)
    q = rand(torch.Generator().manual_seed(rows), rows, 1, 64, dtype=dtype, std=30.0)
    run(oc, ctx, cache, q, [rows], scale=1.0)
    run(oc, ctx, cache, q, [rows], scale=1e-6)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 3, 140])
@pytest.mark.parametrize("what", [NAN, math.inf, -math.inf])
@pytest.mark.parametrize("bad", [290, 256, 319])
def test_attention_values_that_are_no_numbers(oc, ctx, dtype, kind, rows, what, bad):
    """In a key or a value that rows do not see: no influence.  In one that they see: it shows there and nowhere else."""
    keys = 400
    cache = Cache(oc, kind, 1, 72, 1, keys, 16, seed=12)
    q = rand(torch.Generator().manual_seed(rows), rows, 1, 72, dtype=dtype)
    pg, r = cache.place(0, bad)
    pos = torch.arange(rows) + bad - rows // 2                               # rows before and behind it
    good = [i for i in range(rows) if pos[i] < bad]
    hit = [i for i in range(rows) if pos[i] >= bad]
    for m in "kv":
        kept = (cache.pool[m].clone(), None if cache.scale[m] is None else cache.scale[m].clone())
        if cache.scale[m] is None:
            cache.pool[m][pg, 0, r, 5] = what
        else:
            cache.scale[m][pg, 0, r] = what
        out = run(oc, ctx, cache, q, [rows], unit=1, ahead=0, idx=pos, check=False).cpu().double()
        want, bound, _, _ = exact(cache, q, [(0, int(p)) for p in pos], 72 ** -0.5, 1, -1, 0)
        bound = bound + (B16 if dtype == BF16 else 2 * U) * want.abs() + 1e-30
        if good:
            assert ((out - want).abs() <= bound)[good].all()
        if hit and m == "v":
            column = out[hit][..., 5]
            if cache.scale[m] is None:
                assert torch.isnan(column).all() if what != what else (column == what).all()
                other = [d for d in range(72) if d != 5]
                assert ((out - want).abs() <= bound)[hit][..., other].all()
            else:
                # the value is q * scale: NaN for a q of 0, otherwise the scale's own infinity or NaN with q's sign
                value = torch.tensor(float(cache.tokens(m)[0][0, bad, 0, 5])).double() * what
                assert torch.isnan(column).all() if torch.isnan(value) else (column == value).all()
        if hit and m == "k" and what != what:
            assert torch.isnan(out[hit]).all()
        cache.pool[m], cache.scale[m] = kept


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [(BF16, BF16), (BF16, "i8"), (F32, F32)])
@pytest.mark.parametrize("rows", [1, 130])
def test_attention_a_key_of_nan_shows_wherever_it_is(oc, ctx, dtype, kind, rows):
    cache = Cache(oc, kind, 1, 64, 1, 256, 16, seed=16)
    q = rand(torch.Generator().manual_seed(rows), rows, 1, 64, dtype=dtype)
    for at in list(range(128, 160)) + [0, 63, 255]:
        pg, r = cache.place(0, at)
        where = (pg, 0, r) if cache.scale["k"] is not None else (pg, 0, r, 7)
        store = cache.scale["k"] if cache.scale["k"] is not None else cache.pool["k"]
        was = store[where].clone()
        store[where] = NAN
        assert torch.isnan(run(oc, ctx, cache, q, [rows], check=False)).all(), at
        store[where] = was


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 140])
def test_attention_scores_that_grow_along_the_keys(oc, ctx, dtype, kind, rows):
    """The maximum of a row rises from tile to tile by a few powers of two, by many, and falls back."""
    keys = 1500
    cache = Cache(oc, kind, 1, 64, 1, keys, 16, seed=17)
    gen = torch.Generator().manual_seed(rows)
    q = rand(gen, rows, 1, 64, dtype=dtype, std=0.1)
    q[..., 0] = (torch.rand(rows, 1, generator=gen) + 0.5).to(dtype)
    rise = torch.cat([torch.linspace(0, 60, 700), torch.linspace(300, 400, 300), torch.linspace(400, 0, 500)])
    x = cache.val["k"][0].clone()
    x[:, 0, 0] = rise.double()
    xx = x.to(dtype)
    ctx.kv_put(cache.desc, oc.kv_rows(cache.desc, keys, tag(oc, dtype), k=xx.cuda()), xx.cuda(), cache.pool["k"], k_scale=cache.scale["k"], page_table=cache.gpu_table)
    if isinstance(kind, str):
        w, sc = levels(xx, kind)
        cache.val["k"][0] = w.double() * sc.float().double()[..., None]
    else:
        cache.val["k"][0] = xx.double()
    for scale in (0.05, 0.3, 1.0):
        run(oc, ctx, cache, q, [rows], scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [(BF16, BF16), (BF16, "i8"), (F32, F32)])
@pytest.mark.parametrize("rows", [2, 150])
@pytest.mark.parametrize("shift,pad", [(0, 0), (1, 0), (4, 4), (0, 3), (8, 8)])
def test_attention_strides(oc, ctx, dtype, kind, rows, shift, pad):
    heads, D = 4, 64
    cache = Cache(oc, kind, 2, D, 1, 200, 16, seed=13)
    q = rand(torch.Generator().manual_seed(rows), rows, heads, D, dtype=dtype)
    want = run(oc, ctx, cache, q, [rows])
    size, st = rows * heads * (D + pad) + shift, (heads * (D + pad), D + pad, 1)
    a = torch.zeros(size, dtype=dtype, device="cuda")
    qv = a.as_strided((rows, heads, D), st, shift)
    qv.copy_(q)
    b = torch.full((size,), 5.0, dtype=dtype, device="cuda")
    ov = b.as_strided((rows, heads, D), st, shift)
    lens = torch.tensor(cache.lens, dtype=torch.int32).cuda()

    def call(x, y):
        d = oc.attention_desc(cache.desc, rows, tag(oc, dtype), heads, D ** -0.5, q=x, out=y)
        ctx.attention(cache.desc, d, x, cache.pool["k"], cache.pool["v"], y, kv_len=lens, **cache.args())
        torch.cuda.synchronize()
        assert ctx.device_status() == oc.OK
    call(qv, ov)
    assert torch.equal(ov, want)
    rest = torch.ones(size, dtype=torch.bool)
    rest.as_strided((rows, heads, D), st, shift).fill_(False)
    assert (b.cpu()[rest] == 5.0).all()
    call(qv, qv)                                                             # in place
    assert torch.equal(qv, want)
    hm = q.cuda().view(1, rows, heads, D).transpose(1, 2).contiguous()       # heads first, as oc_rope leaves them
    ho = torch.empty_like(hm)
    call(hm, ho)
    assert torch.equal(ho[0].transpose(0, 1), want)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, "i8", "i4"])
@pytest.mark.parametrize("rows", [1, 150])
def test_attention_bad_pages_read_as_zeros(oc, ctx, kind, rows):
    keys = 300
    cache = Cache(oc, kind, 1, 64, 1, keys, 32, seed=14)
    q = rand(torch.Generator().manual_seed(rows), rows, 1, 64, dtype=BF16)
    table = cache.table.clone()
    table[0, 2], table[0, 5] = -7, cache.pages
    qq, out = q.cuda(), torch.empty(rows, 1, 64, dtype=BF16, device="cuda")
    d = oc.attention_desc(cache.desc, rows, oc.DTYPE_BF16, 1, 0.125, q=qq, out=out)
    ctx.attention(cache.desc, d, qq, cache.pool["k"], cache.pool["v"], out, k_scale=cache.scale["k"], v_scale=cache.scale["v"], page_table=table.cuda())
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.ERR_INVALID_ARG
    for m in "kv":
        cache.val[m][0, 64:96] = 0
        cache.val[m][0, 160:192] = 0
    want, bound, _, _ = exact(cache, q, [(0, 0)] * rows, 0.125)
    assert_attn(out, want, bound, [(0, 0)] * rows)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 150])
def test_attention_wrong_lengths_and_rows_are_recorded(oc, ctx, rows):
    cache = Cache(oc, BF16, 1, 64, 2, 128, 32, seed=15)
    q = rand(torch.Generator().manual_seed(rows), 2 * rows, 1, 64, dtype=BF16)
    qq = q.cuda()

    def call(n=2 * rows, **kw):
        out = torch.full((2 * rows, 1, 64), 5.0, dtype=BF16, device="cuda")
        d = oc.attention_desc(cache.desc, n, oc.DTYPE_BF16, 1, 0.125, rows_per_batch=rows, q=qq, out=out)
        kw = {k: torch.tensor(v, dtype=torch.int32).cuda() for k, v in kw.items()}
        ctx.attention(cache.desc, d, qq, cache.pool["k"], cache.pool["v"], out, page_table=cache.gpu_table, **kw)
        torch.cuda.synchronize()
        return ctx.device_status(), out
    st, out = call(kv_len=[-3, 129])                                         # taken as 0 and 128
    assert st == oc.ERR_INVALID_ARG and (out[:rows] == 0).all() and not (out[rows:] == 5.0).any()
    for start in ([0, rows, 2 * rows + 1], [0, -1, 2 * rows], [-1, rows, 2 * rows], [0, 2 * rows, rows], [2 ** 31 - 1, 0, 0]):
        st, out = call(q_start=start)
        assert st == oc.ERR_INVALID_ARG
    st, out = call(q_start=[0, rows, 2 * rows], idx=[128] * rows + [127] + [128] * (rows - 1))       # tokens of the other sequence
    assert st == oc.ERR_INVALID_ARG and (out[: rows + 1] == 5.0).all() and not (out[rows + 1:] == 5.0).any()
    st, out = call(kv_len=[128, 128])
    assert st == oc.OK


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [(BF16, BF16), (BF16, "i8"), (F32, F32)])
@pytest.mark.parametrize("rows", [1, 300])
def test_on_another_stream_and_in_two_graphs(oc, ctx, dtype, kind, rows):
    """put, attention and get captured; two graphs replayed at once with inputs changed in place."""
    heads, D, keys = 2, 64, 2000
    caches = [Cache(oc, kind, heads, D, 1, keys, 64, seed=20 + i) for i in range(2)]
    gen = torch.Generator().manual_seed(rows)
    state, graphs = [], []
    for c in caches:
        q, k, v = (torch.zeros(rows, heads, D, dtype=dtype, device="cuda") for _ in range(3))
        out, back = torch.zeros_like(q), torch.zeros_like(q)
        idx = torch.arange(rows, dtype=torch.int32, device="cuda") * 3
        kd, gd = oc.kv_rows(c.desc, rows, tag(oc, dtype), k=k, v=v), oc.kv_rows(c.desc, rows, tag(oc, dtype), k=back)
        ad = oc.attention_desc(c.desc, rows, tag(oc, dtype), heads, 0.125, q=q, out=out)

        def step(c=c, q=q, k=k, v=v, out=out, back=back, idx=idx, kd=kd, gd=gd, ad=ad):
            ctx.kv_put(c.desc, kd, k, c.pool["k"], v, c.pool["v"], idx=idx, **c.args())
            ctx.attention(c.desc, ad, q, c.pool["k"], c.pool["v"], out, **c.args())
            ctx.kv_get(c.desc, gd, c.pool["k"], back, idx=idx, k_scale=c.scale["k"], page_table=c.gpu_table)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        state.append((c, q, k, v, out, back, step))
        graphs.append(g)
    for _ in range(2):
        new = []
        for c, q, k, v, out, back, step in state:
            for t in (q, k, v):
                t.copy_(rand(gen, rows, heads, D, dtype=dtype))
            out.zero_()
            step()
            torch.cuda.synchronize()
            new.append((out.clone(), back.clone()))
            out.zero_(), back.zero_()
        streams = [torch.cuda.Stream() for _ in graphs]
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for (c, q, k, v, out, back, _), (wo, wb) in zip(state, new):
            assert torch.equal(out, wo) and torch.equal(back, wb)
            at = torch.arange(rows) * 3
            for m, t in (("k", k), ("v", v)):
                if isinstance(kind, str):
                    qq, sc = levels(t.cpu(), kind)
                    c.val[m][0, at] = qq.double() * sc[..., None]
                else:
                    c.val[m][0, at] = t.cpu().double()
            want, bound, _, _ = exact(c, q.cpu(), [(0, 0)] * rows, 0.125)
            assert_attn(out, want, bound * (1 + 1e-6), [(0, 0)] * rows)
    assert ctx.device_status() == oc.OK


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 3, 140])
def test_attention_over_a_cache_of_no_tokens(oc, ctx, dtype, kind, rows):
    """No tokens, no pages, no addresses: zeros, and a log of 0."""
    d = oc.kv_desc(tag(oc, kind), 2, 64, 2, 0, 16)
    q = rand(torch.Generator().manual_seed(rows), 2 * rows, 2, 64, dtype=dtype).cuda()
    out, lse = torch.full_like(q, 5.0), torch.full((2 * rows, 2), 5.0, device="cuda")
    a = oc.attention_desc(d, 2 * rows, tag(oc, dtype), 2, 0.1, rows_per_batch=rows, q=q, out=out)
    ctx.attention(d, a, q, None, None, out, lse=lse)
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.OK and (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 5, 200])
def test_attention_two_calls_at_once(oc, dtype, kind, rows):
    """Contexts of their own on streams of their own."""
    cache = Cache(oc, kind, 2, 64, 2, 900, 32, seed=30)
    q = rand(torch.Generator().manual_seed(rows), 2 * rows, 4, 64, dtype=dtype)
    with oc.Context(0) as a, oc.Context(0) as b:
        want = run(oc, a, cache, q, [rows, rows])
        streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(want) for _ in range(8)]
        qq = q.cuda()
        d = oc.attention_desc(cache.desc, 2 * rows, tag(oc, dtype), 4, 0.125, rows_per_batch=rows, q=qq, out=outs[0])
        torch.cuda.synchronize()
        for i, o in enumerate(outs):
            (a, b)[i % 2].attention(cache.desc, d, qq, cache.pool["k"], cache.pool["v"], o, stream=streams[i % 2], **cache.args())
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs) and a.device_status() == oc.OK and b.device_status() == oc.OK


@pytest.mark.gpu
def test_the_same_call_gives_the_same_bits(oc, ctx):
    for dtype, kind in TYPES:
        for rows in (1, 70):
            cache = Cache(oc, kind, 2, 72, 1, 1500, 32, seed=21)
            q = rand(torch.Generator().manual_seed(rows), rows, 4, 72, dtype=dtype)
            first = run(oc, ctx, cache, q, [rows], check=False)
            for _ in range(5):
                assert torch.equal(run(oc, ctx, cache, q, [rows], check=False), first)


# ---- refusals: decided on the host before the context is looked at, so they need no GPU --------------------------------
class HostCalls:
    """The calls with a context that holds nothing: whatever is not refused would fail on a machine without a GPU, so only
    refusals are asked for."""

    def __init__(self, oc):
        self.oc, self.ctx = oc, object.__new__(oc.Context)
        self.mem = (oc.C.c_uint8 * 65536)()
        self.ctx._h = oc.C.c_void_p(oc.C.addressof(self.mem))

    def close(self):
        self.ctx._h = None


@pytest.fixture
def host(oc):
    h = HostCalls(oc)
    yield h
    h.close()


A = 0x10000                                                                  # an address that nobody follows


def kv(oc, **kw):
    f = dict(dtype=oc.DTYPE_BF16, heads=2, head_dim=64, n_seqs=2, seq_rows=100, page_rows=16, n_pages=14, table_stride=7)
    f.update(kw)
    return oc.CKv(*f.values())


def test_cache_descriptor_refusals_and_sizes(oc):
    def status(**kw):
        d = kv(oc, **kw)
        a, b = oc.C.c_size_t(), oc.C.c_size_t()
        return oc._lib.oc_kv_bytes(oc.C.byref(d), oc.C.byref(a), oc.C.byref(b))
    assert status() == oc.OK
    for bad in (dict(dtype=4), dict(dtype=-1), dict(heads=0), dict(head_dim=0), dict(n_seqs=-1), dict(seq_rows=-1), dict(page_rows=0),
                dict(n_pages=-1), dict(table_stride=-1), dict(table_stride=6), dict(n_pages=0)):
        assert status(**bad) == oc.ERR_INVALID_ARG, bad
    for bad in (dict(head_dim=60), dict(page_rows=8), dict(page_rows=24)):
        assert status(**bad) == oc.ERR_ALIGNMENT, bad
    for bad in (dict(head_dim=264), dict(n_seqs=2 ** 16, seq_rows=2 ** 16, table_stride=2 ** 20), dict(n_pages=2 ** 28), dict(heads=70000)):
        assert status(**bad) == oc.ERR_UNSUPPORTED, bad
    n = 14 * 2 * 16
    for t, per, scales in ((oc.DTYPE_F32, 256, 0), (oc.DTYPE_BF16, 128, 0), (oc.DTYPE_I8, 64, 4), (oc.DTYPE_I4, 32, 4)):
        assert oc.kv_bytes(kv(oc, dtype=t)) == (n * per, n * scales)
        pool, scale = oc.kv_pools(kv(oc, dtype=t), device="cpu")
        assert pool.numel() * pool.element_size() == n * per and (0 if scale is None else scale.numel() * 4) == n * scales


def test_put_and_get_refusals(oc, host):
    def put(cache=None, dtype=oc.DTYPE_BF16, n=20, per=20, view=(2560, 128, 64), k=A, kp=2 * A, v=3 * A, vp=4 * A, table=A, idx=A, get=False, **kw):
        r = oc.CKvRows(dtype, n, per, oc.CRopeView(*view), oc.CRopeView(*view))
        cache = cache or kv(oc)
        if get:
            return host.ctx.kv_get(cache, r, kp, k, vp, v, page_table=table, idx=idx, stream=0, check=False, **kw)
        return host.ctx.kv_put(cache, r, k, kp, v, vp, page_table=table, idx=idx, stream=0, check=False, **kw)
    i8 = kv(oc, dtype=oc.DTYPE_I8)
    for get in (False, True):
        for bad in (dict(dtype=oc.DTYPE_I8), dict(dtype=oc.DTYPE_F32), dict(n=-1), dict(per=0), dict(k=None), dict(v=None), dict(vp=None), dict(kp=None),
                    dict(view=(2560, -128, 64)), dict(idx=None, n=201), dict(k_scale=A), dict(v_scale=A), dict(cache=i8), dict(cache=i8, k_scale=A),
                    dict(table=None, cache=kv(oc, n_pages=13)), dict(kp=A)):
            assert put(get=get, **bad) == oc.ERR_INVALID_ARG, bad
        for bad in (dict(k=A + 1), dict(kp=2 * A + 8), dict(vp=4 * A + 2), dict(idx=A + 2), dict(table=A + 1), dict(cache=i8, k_scale=A + 2, v_scale=A)):
            assert put(get=get, **bad) == oc.ERR_ALIGNMENT, bad
        assert put(get=get, n=2 ** 31, idx=A) == oc.ERR_UNSUPPORTED
        assert put(get=get, n=0, k=None, kp=None, v=None, vp=None) == oc.OK
    for view in ((2560, 0, 64), (2560, 128, 0)):
        assert put(get=True, view=view) == oc.ERR_INVALID_ARG
    assert put(get=True, per=10, view=(0, 128, 64)) == oc.ERR_INVALID_ARG
    host.ctx._h = None
    assert put() == oc.ERR_INVALID_ARG and put(get=True) == oc.ERR_INVALID_ARG


def test_attention_refusals(oc, host):
    def call(cache=None, dtype=oc.DTYPE_BF16, heads=4, scale=0.1, n=20, per=10, unit=0, view=(2560, 256, 64), oview=None, q=A, kp=2 * A, vp=3 * A, out=4 * A, table=A, **kw):
        d = oc.CAttention(dtype, heads, scale, n, per, unit, -1, -1, oc.CRopeView(*view), oc.CRopeView(*(oview or view)))
        return host.ctx.attention(cache or kv(oc), d, q, kp, vp, out, page_table=table, stream=0, check=False, **kw)
    i4 = kv(oc, dtype=oc.DTYPE_I4)
    for bad in (dict(dtype=oc.DTYPE_F32), dict(dtype=oc.DTYPE_I8), dict(heads=3), dict(heads=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=math.inf),
                dict(n=-1), dict(per=0), dict(unit=-1), dict(q=None), dict(out=None), dict(kp=None), dict(vp=None), dict(view=(2560, -1, 64)),
                dict(oview=(2560, 0, 64)), dict(oview=(2560, 256, 0)), dict(oview=(0, 256, 64)), dict(k_scale=A), dict(cache=i4), dict(cache=i4, v_scale=A),
                dict(table=None, cache=kv(oc, n_pages=13)), dict(out=2 * A), dict(out=3 * A)):
        assert call(**bad) == oc.ERR_INVALID_ARG, bad
    for bad in (dict(q=A + 1), dict(out=4 * A + 1), dict(kp=2 * A + 4), dict(kv_len=A + 1), dict(q_start=A + 2), dict(idx=A + 1), dict(lse=A + 2),
                dict(cache=kv(oc, head_dim=36))):
        assert call(**bad) == oc.ERR_ALIGNMENT, bad
    for bad in (dict(cache=kv(oc, head_dim=136)), dict(n=2 ** 31), dict(n=2 ** 30, per=2 ** 30)):
        assert call(**bad) == oc.ERR_UNSUPPORTED, bad
    assert call(n=0, q=None, out=None) == oc.OK
    assert call(cache=kv(oc, n_seqs=0)) == oc.OK


def test_two_outputs_in_one_place_are_refused(oc, host):
    def move(call, cache, k, kp, v, vp, ks=None, vs=None):
        r = oc.CKvRows(oc.DTYPE_BF16, 20, 20, oc.CRopeView(2560, 128, 64), oc.CRopeView(2560, 128, 64))
        args = (k, kp, v, vp) if call == "kv_put" else (kp, k, vp, v)
        return getattr(host.ctx, call)(cache, r, *args, k_scale=ks, v_scale=vs, page_table=A, idx=A, stream=0, check=False)
    assert move("kv_put", kv(oc), A, 2 * A, 3 * A, 2 * A) == oc.ERR_INVALID_ARG
    assert move("kv_put", kv(oc, dtype=oc.DTYPE_I8), A, 2 * A, 3 * A, 4 * A, 5 * A, 5 * A) == oc.ERR_INVALID_ARG
    assert move("kv_get", kv(oc), A, 2 * A, A, 3 * A) == oc.ERR_INVALID_ARG


def test_a_scale_whose_binary_logarithm_leaves_fp32_is_refused(oc, host):
    view = oc.CRopeView(2560, 256, 64)
    for scale in (2.0 ** 127, 3.4e38):
        d = oc.CAttention(oc.DTYPE_BF16, 4, scale, 20, 10, 0, -1, -1, view, view)
        assert host.ctx.attention(kv(oc), d, A, 2 * A, 3 * A, 4 * A, page_table=A, stream=0, check=False) == oc.ERR_INVALID_ARG


def test_descriptors_take_strides_from_tensors(oc):
    d = kv(oc)
    packed = torch.zeros(20, 6, 64)
    r = oc.kv_rows(d, 20, oc.DTYPE_F32, k=packed[:, 2:4], v=torch.zeros(2, 2, 10, 64))
    assert (r.rows_per_batch, r.k.batch_stride, r.k.row_stride, r.k.head_stride) == (10, 3840, 384, 64)
    assert (r.v.batch_stride, r.v.row_stride, r.v.head_stride) == (1280, 64, 640)
    a = oc.attention_desc(d, 20, oc.DTYPE_BF16, 4, 1.0, q=torch.zeros(2, 4, 10, 64), out=torch.zeros(20, 4, 64))
    assert a.rows_per_batch == 10 and (a.out.batch_stride, a.out.row_stride, a.out.head_stride) == (2560, 256, 64)
    for bad in (torch.zeros(20, 3, 64), torch.zeros(20, 2, 32), torch.zeros(19, 2, 64), torch.zeros(20, 128), torch.zeros(20, 2, 128)[..., ::2], torch.zeros(2, 2, 9, 64)):
        with pytest.raises(ValueError):
            oc.kv_rows(d, 20, oc.DTYPE_F32, k=bad, rows_per_batch=10)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["i8", "i4"])
def test_put_rounds_every_pair_of_bf16_values(oc, ctx, kind):
    """Every quotient of two 8-bit mantissas, at every distance of their exponents that matters."""
    L = 127 if kind == "i8" else 7
    m = torch.arange(128, 256).double()
    rows = []
    for shift in range(10 if kind == "i8" else 6):
        n = torch.arange(128, 256).double() * 2.0 ** -shift
        n = torch.where(n[None] <= m[:, None], n[None].expand(128, 128), -n[None] / 2)          # no element above the maximum
        rows.append(torch.cat([m[:, None].expand(128, 8), n], 1))                              # [128, 136]
    x = torch.stack(rows).to(BF16).reshape(-1, 1, 136)
    pad = x.shape[0]
    cache = Cache(oc, kind, 1, 136, 1, pad, 16, table=False, empty=True)
    xx = x.cuda()
    ctx.kv_put(cache.desc, oc.kv_rows(cache.desc, pad, oc.DTYPE_BF16, k=xx), xx, cache.pool["k"], k_scale=cache.scale["k"])
    torch.cuda.synchronize()
    check_put(cache, "k", x, torch.arange(pad))
