"""Attention over the paged cache at its edges: values that are no numbers, the largest numbers, cuts between the CTAs that share
a sequence's keys.  Restatement and bounds are those of test_attention."""
import os
import subprocess
import sys

import pytest
import torch

from test_attention import BF16, F32, NAN, TYPES, Cache, check_put, ctx, exact, host, oc, rand, seen_by, tag  # noqa: F401 (fixtures)


def poison(cache, m, tokens, what, column=7):
    """`what` in the tokens' keys or values of sequence 0, all heads: in their scales, or one column"""
    for t in tokens:
        pg, r = cache.place(0, t)
        if cache.scale[m] is None:
            cache.pool[m][pg, :, r, column] = what
        else:
            cache.scale[m][pg, :, r] = what


def with_lse(oc, ctx, cache, q, **kw):
    """(out, lse) of one sequence on the CPU"""
    n, H, D = q.shape
    qq, lse = q.cuda(), torch.full((n, H), 5.0, device="cuda")
    out = torch.full_like(qq, 5.0)
    idx, window = kw.pop("idx", None), {k: kw.pop(k) for k in ("unit", "back", "ahead") if k in kw}
    d = oc.attention_desc(cache.desc, n, tag(oc, q.dtype), H, kw.pop("scale", D ** -0.5), q=qq, out=out, **window)
    ctx.attention(cache.desc, d, qq, cache.pool["k"], cache.pool["v"], out, lse=lse, kv_len=torch.tensor(cache.lens, dtype=torch.int32).cuda(),
                  idx=None if idx is None else torch.as_tensor(idx, dtype=torch.int32).cuda(), **cache.args(), **kw)
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.OK
    return out.cpu(), lse.cpu()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 4, 16, 40])
def test_a_cta_that_sees_keys_of_nan_only(oc, ctx, dtype, kind, rows):
    """Where a cluster splits the keys: the last key alone in a CTA, a CTA's whole share, a window's last key."""
    q = rand(torch.Generator().manual_seed(rows), rows, 1, 64, dtype=dtype)
    for lens, bad in ((33, [32]), (17, [16]), (65, [64]), (512, range(256, 512)), (512, range(0, 256))):
        cache = Cache(oc, kind, 1, 64, 1, 512, 16, lens=[lens], seed=40)
        poison(cache, "k", bad, NAN)
        for t in with_lse(oc, ctx, cache, q):
            assert torch.isnan(t).all(), (lens, bad)
    cache = Cache(oc, kind, 1, 64, 1, 2048, 16, seed=41)
    poison(cache, "k", [1024], NAN)
    for t in with_lse(oc, ctx, cache, q, unit=1, back=32, ahead=0, idx=[1024] * rows):
        assert torch.isnan(t).all()
    assert not torch.isnan(with_lse(oc, ctx, cache, q, unit=1, back=32, ahead=0, idx=[1023] * rows)[0]).any()


def test_sequences_whose_tiles_would_pass_2_to_the_31_are_refused(oc, host):
    """A small pool may stand for as many tokens: pages of the table may be shared."""
    view = oc.CRopeView(2560, 256, 64)
    d = oc.CAttention(oc.DTYPE_BF16, 4, 0.1, 20, 20, 0, -1, -1, view, view)
    for seq_rows in (2 ** 31 - 1, 2 ** 31 - 100, 2 ** 31 - 4096):
        cache = oc.CKv(oc.DTYPE_BF16, 2, 64, 1, seq_rows, 2 ** 20, 1, 2 ** 11)
        assert host.ctx.attention(cache, d, 0x10000, 0x20000, 0x30000, 0x40000, page_table=0x50000, stream=0, check=False) == oc.ERR_UNSUPPORTED, seq_rows


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["i8", "i4"])
@pytest.mark.parametrize("most", [1.0, 3.0, 0.7, 2.0 ** -99, 2.0 ** 99, 1.1e30, 1e36, 2.6e36, 2.7e36, 4.9e37, 1e38, 3.4028234e38])
def test_put_rounds_beside_ties_as_defined(oc, ctx, kind, most):
    """Quotients at a tie and up to three steps of x beside it, also where x L leaves fp32."""
    L = 127 if kind == "i8" else 7
    top = torch.tensor(most)
    gen = torch.Generator().manual_seed(3)
    rows = []
    for _ in range(64):
        half = torch.randint(0, L, (1, 64), generator=gen).double() + 0.5
        x = (half * top.double() / L).to(F32)
        for _ in range(int(torch.randint(0, 4, (1,), generator=gen))):
            x = torch.nextafter(x, torch.zeros(()) if len(rows) % 2 else top)
        x = x * torch.where(torch.rand(1, 64, generator=gen) < 0.5, -1.0, 1.0)
        x[0, 9] = top
        rows.append(x)
    x = torch.stack(rows)                                                                # [64, 1, 64]
    cache = Cache(oc, kind, 1, 64, 1, 64, 16, empty=True)
    xx = x.cuda()
    ctx.kv_put(cache.desc, oc.kv_rows(cache.desc, 64, oc.DTYPE_F32, k=xx), xx, cache.pool["k"], k_scale=cache.scale["k"], page_table=cache.gpu_table)
    torch.cuda.synchronize()
    check_put(cache, "k", x, torch.arange(64))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["i8", "i4"])
def test_put_rounds_scales_once(oc, ctx, dtype, kind):
    """scale = max|x| / L is the nearest fp32 number, for every magnitude and where the vector is zero or no number."""
    n, heads = 512, 4
    gen = torch.Generator().manual_seed(4)
    x = rand(gen, n, heads, 64, dtype=F32) * 2.0 ** torch.randint(-98, 120, (n, heads, 1), generator=gen).float()
    x[0], x[1, 1, 5], x[2, 1, 6], x[3] = 0.0, float("inf"), NAN, 2.0 ** -101
    x = x.to(dtype)
    x[:, 0, 0] = (3.0 + torch.arange(n) * 2.0 ** (-7 if dtype == BF16 else -21)).to(dtype)          # neighbours
    cache = Cache(oc, kind, heads, 64, 1, n, 16, table=False, empty=True)
    xx = x.cuda()
    ctx.kv_put(cache.desc, oc.kv_rows(cache.desc, n, tag(oc, dtype), k=xx), xx, cache.pool["k"], k_scale=cache.scale["k"])
    torch.cuda.synchronize()
    check_put(cache, "k", x, torch.arange(n))
    most = x.float().abs().amax(-1)
    want = torch.where(most < 2.0 ** -100, torch.zeros(()), most / torch.tensor(127.0 if kind == "i8" else 7.0))
    got = cache.tokens("k")[1][0]
    assert torch.equal(got.nan_to_num(nan=-1.0), want.nan_to_num(nan=-1.0))


def test_sizes_of_a_cache_without_a_table(oc):
    d = oc.CKv(oc.DTYPE_I8, 2, 64, 2, 100, 16, 14, 0)
    assert oc.kv_bytes(d) == (14 * 2 * 16 * 64, 14 * 2 * 16 * 4)
    for bad in (oc.CKv(oc.DTYPE_I8, 2, 64, 2, 100, 16, 13, 0), oc.CKv(oc.DTYPE_I8, 2, 64, 2, 100, 16, 14, 6)):
        with pytest.raises(oc.OmniCacheError):
            oc.kv_bytes(bad)
    assert oc.kv_bytes(oc.CKv(oc.DTYPE_BF16, 2, 64, 1, 100, 16, 3, 0)) == (3 * 2 * 16 * 128, 0)      # one sequence, pages shared by a table


def check_no_numbers(oc, ctx, cache, q, pos, bad, unit=0, back=-1, ahead=-1, scale=None):
    """Rows at `pos` over values of which some are no numbers: bad = [(key, column, what)], with whole numbers what is the key's scale.
    A column of a row is the sum of those that it sees, whatever their probabilities, and as if they were zeros where it sees none."""
    n, H, D = q.shape
    held = {m: (cache.pool[m].clone(), None if cache.scale[m] is None else cache.scale[m].clone()) for m in "kv"}
    vals = cache.val["v"].clone()
    strange = torch.zeros(n, H, D, dtype=torch.float64)
    group = H // cache.heads
    for key, column, what in bad:
        poison(cache, "v", [key], what, column)
        sees = torch.tensor([bool(seen_by(p, cache.lens[0], unit, back, ahead)[key]) for p in pos])
        if cache.scale["v"] is None:
            strange[sees, :, column] += what
            cache.val["v"][0, key, :, column] = 0
        else:
            strange[sees] += (cache.tokens("v")[0][0, key].double() * what).repeat_interleave(group, 0)
            cache.val["v"][0, key] = 0
    want, bound, _, _ = exact(cache, q, [(0, p) for p in pos], D ** -0.5 if scale is None else scale, unit, back, ahead)
    idx = torch.tensor(pos)
    got = with_lse(oc, ctx, cache, q, idx=idx, unit=unit, back=back, ahead=ahead, **({} if scale is None else dict(scale=scale)))[0].double()
    bound = bound + (2.0 ** -8 if q.dtype == BF16 else 2.0 ** -23) * want.abs() + 1e-30
    plain = strange == 0
    assert ((got - want).abs() <= bound)[plain].all()
    assert torch.equal(got[~plain].nan_to_num(nan=7.0), strange[~plain].nan_to_num(nan=7.0))
    cache.val["v"] = vals
    for m in "kv":
        cache.pool[m], cache.scale[m] = held[m]


INF = float("inf")
BAD = [[(100, 3, INF)], [(1, 0, NAN), (1400, 71, -INF)], [(700, 5, INF), (710, 5, -INF), (711, 6, INF), (1200, 5, INF)], [(j, j % 72, NAN) for j in range(640, 900)]]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 5, 140])
@pytest.mark.parametrize("bad", BAD)
def test_values_that_are_no_numbers_in_several_places(oc, ctx, dtype, kind, rows, bad):
    cache = Cache(oc, kind, 1, 72, 1, 1500, 16, seed=42)
    q = rand(torch.Generator().manual_seed(rows), rows, 2, 72, dtype=dtype)
    for first in (0, 700 - rows, 705, 1500 - rows):
        check_no_numbers(oc, ctx, cache, q, list(range(first, first + rows)), bad, unit=1, ahead=0)
    check_no_numbers(oc, ctx, cache, q, list(range(640, 640 + rows)), bad, unit=50, back=1, ahead=2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 5, 140])
@pytest.mark.parametrize("bad", BAD)
def test_values_that_are_no_numbers_count_whatever_their_probability(oc, ctx, dtype, kind, rows, bad):
    """Scores hundreds apart, so that most probabilities are 0 in fp32; in tiles that every row sees, and that some do not."""
    cache = Cache(oc, kind, 1, 72, 1, 1500, 16, seed=43)
    q = rand(torch.Generator().manual_seed(rows), rows, 2, 72, dtype=dtype, std=30.0)
    check_no_numbers(oc, ctx, cache, q, list(range(rows)), bad, scale=1.0)
    check_no_numbers(oc, ctx, cache, q, list(range(1500 - rows, 1500)), bad, unit=1, ahead=0, scale=1.0)
    check_no_numbers(oc, ctx, cache, q, list(range(680, 680 + rows)), bad, unit=1, back=60, ahead=-1, scale=1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 2000])
def test_values_that_no_row_sees_take_no_time(oc, ctx, dtype, kind, rows):
    """Unwritten pages of NaN behind a causal window: within a factor of 4 of what it takes over numbers."""
    desc = oc.kv_desc(tag(oc, kind), 8, 72, 2, 4096, 64)
    (kp, ks), (vp, vs) = oc.kv_pools(desc), oc.kv_pools(desc)
    x, q = torch.randn(8192, 8, 72, device="cuda", dtype=dtype), torch.randn(2 * rows, 8, 72, device="cuda", dtype=dtype)
    ctx.kv_put(desc, oc.kv_rows(desc, 8192, tag(oc, dtype), k=x, v=x), x, kp, x, vp, k_scale=ks, v_scale=vs)
    idx = (torch.arange(2000 - rows, 2000)[None] + 4096 * torch.arange(2)[:, None]).flatten().int().cuda()
    out = torch.empty_like(q)
    d = oc.attention_desc(desc, 2 * rows, tag(oc, dtype), 8, 72 ** -0.5, rows_per_batch=rows, unit=1, ahead=0, q=q, out=out)

    def time():
        spans = []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            ctx.attention(desc, d, q, kp, vp, out, k_scale=ks, v_scale=vs, idx=idx)
            b.record()
            torch.cuda.synchronize()
            spans.append(a.elapsed_time(b))
        return min(spans)
    plain, want = time(), out.clone()
    for pool, scale in ((kp, ks), (vp, vs)):
        store = (pool if scale is None else scale).view(2, 64, 8, 64, -1)
        store[:, 31, :, 16:], store[:, 32:] = NAN, NAN                                   # tokens from 2000 on
    assert time() <= 4 * plain and torch.equal(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, "i8", "i4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [1, 16, 140])
def test_the_log_sum_exp_is_of_fp32(oc, ctx, kind, D, rows):
    """One key at a score of 0 and 127 at -x exactly (one element of the products is not 0): lse = log(1 + 127 exp(-x)).
    u = 2^-24.  The exponent x log2(e) is two roundings and the scale's two off, 4 u x; the exponential, a special function or a
    polynomial, 5 u; 128 terms in chains of at most 34 additions 34 u of the sum, whose logarithm adds 4 u."""
    u = 2.0 ** -24
    cache = Cache(oc, kind, 1, D, 1, 128, 16, seed=44)
    key = torch.zeros(128, 1, D)
    key[1:, 0, 0] = -1.0
    key = key.to(BF16).cuda()
    ctx.kv_put(cache.desc, oc.kv_rows(cache.desc, 128, oc.DTYPE_BF16, k=key), key, cache.pool["k"], k_scale=cache.scale["k"], page_table=cache.gpu_table)
    for step in range(0, 256, rows):
        x = (torch.arange(step, step + rows) % 256 / 256.0 + 0.5).to(BF16)
        q = torch.zeros(rows, 1, D, dtype=BF16)
        q[:, 0, 0] = x
        x, lse = x.double(), with_lse(oc, ctx, cache, q, scale=1.0)[1][:, 0].double()
        want = torch.log(1 + 127 * torch.exp(-x))
        level = 3 * u * x if isinstance(kind, str) else 0                                # (scale * q of a whole number)
        assert ((lse - want).abs() <= 4 * u * x + level + 43 * u + 2 * u * want).all(), float(((lse - want).abs()).max() / u)


def test_outputs_in_the_place_of_others_are_refused(oc, host):
    A = 0x10000
    view = oc.CRopeView(2560, 256, 64)

    def attend(q=A, kp=2 * A, vp=3 * A, out=4 * A, ks=5 * A, vs=6 * A, lse=7 * A, oview=view, n=20, per=10, heads=4, kind=oc.DTYPE_I8, **kw):
        d = oc.CAttention(oc.DTYPE_BF16, heads, 0.1, n, per, 0, -1, -1, view, oview)
        cache = oc.CKv(kind, 2, 64, 2, 100, 16, 14, 7)
        return host.ctx.attention(cache, d, q, kp, vp, out, k_scale=ks, v_scale=vs, page_table=8 * A, lse=lse, stream=0, check=False, **kw)
    for bad in (dict(lse=4 * A), dict(lse=A), dict(lse=2 * A), dict(lse=6 * A), dict(lse=8 * A), dict(out=5 * A), dict(out=6 * A), dict(out=8 * A), dict(out=9 * A, kv_len=9 * A),
                dict(lse=9 * A, idx=9 * A), dict(out=A, oview=oc.CRopeView(2560, 64, 640)), dict(out=A, oview=oc.CRopeView(5120, 256, 64)), dict(out=A, oview=oc.CRopeView(2560, 512, 64))):
        assert attend(**bad) == oc.ERR_INVALID_ARG, bad

    def move(put, k=A, kp=2 * A, v=3 * A, vp=4 * A, ks=5 * A, vs=6 * A, table=7 * A, idx=8 * A):
        r = oc.CKvRows(oc.DTYPE_BF16, 20, 20, oc.CRopeView(2560, 128, 64), oc.CRopeView(2560, 128, 64))
        args = (k, kp, v, vp) if put else (kp, k, vp, v)
        return getattr(host.ctx, "kv_put" if put else "kv_get")(oc.CKv(oc.DTYPE_I8, 2, 64, 2, 100, 16, 14, 7), r, *args, k_scale=ks, v_scale=vs, page_table=table, idx=idx,
                                                                stream=0, check=False)
    for bad in (dict(kp=3 * A), dict(vp=A), dict(ks=2 * A), dict(vs=2 * A), dict(ks=4 * A), dict(vs=4 * A), dict(ks=A), dict(vs=3 * A), dict(kp=7 * A), dict(vs=8 * A)):
        assert move(True, **bad) == oc.ERR_INVALID_ARG, bad
    for bad in (dict(k=4 * A), dict(v=2 * A), dict(k=5 * A), dict(v=6 * A), dict(v=7 * A), dict(k=8 * A)):
        assert move(False, **bad) == oc.ERR_INVALID_ARG, bad


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("rows", [1, 16, 200])
def test_in_place_with_strides_that_do_not_count(oc, ctx, dtype, kind, rows):
    """out is q: strides of axes of one element may differ."""
    cache = Cache(oc, kind, 1, 64, 1, 300, 16, seed=45)
    q = rand(torch.Generator().manual_seed(rows), rows, 1, 64, dtype=dtype)
    want = with_lse(oc, ctx, cache, q)[0]
    x = q.cuda()
    d = oc.attention_desc(cache.desc, rows, tag(oc, dtype), 1, 0.125, q=x, out=(7, 64, 0))
    ctx.attention(cache.desc, d, x, cache.pool["k"], cache.pool["v"], x, **cache.args())
    assert torch.equal(x.cpu(), want)


def test_tensors_of_another_type_are_refused(oc, host):
    cache = oc.CKv(oc.DTYPE_BF16, 2, 64, 2, 100, 16, 14, 7)
    x, y = torch.zeros(20, 2, 64, dtype=BF16), torch.zeros(20, 2, 64)
    for kw in (dict(k=y), dict(k=x, v=y), dict(k=y, v=x)):
        with pytest.raises(ValueError):
            oc.kv_rows(cache, 20, oc.DTYPE_BF16, **kw)
    rows, pool = oc.kv_rows(cache, 20, oc.DTYPE_BF16, k=x, v=x), torch.zeros(14, 2, 16, 64, dtype=BF16)
    desc = oc.attention_desc(cache, 20, oc.DTYPE_BF16, 2, 0.1, rows_per_batch=10, q=x, out=x)
    for bad in (torch.zeros(20, dtype=torch.int64), torch.zeros(20, dtype=torch.int16), torch.zeros(20)):
        for name in ("idx", "page_table", "kv_len", "q_start"):
            with pytest.raises(ValueError):
                host.ctx.attention(cache, desc, x, pool, pool, x, stream=0, check=False, **{name: bad})
            if name in ("idx", "page_table"):
                with pytest.raises(ValueError):
                    host.ctx.kv_put(cache, rows, x, pool, stream=0, check=False, **{name: bad})
                with pytest.raises(ValueError):
                    host.ctx.kv_get(cache, rows, pool, x, stream=0, check=False, **{name: bad})
    for q, out in ((y, x), (x, y)):
        with pytest.raises(ValueError):
            host.ctx.attention(cache, desc, q, pool, pool, out, stream=0, check=False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [(BF16, BF16), (BF16, "i8"), (F32, "i8")])
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_pools_of_more_than_2_to_the_32_bytes(oc, ctx, dtype, kind, rows):
    """The last pages of a pool, in every kernel; their values as floating-point vectors read back."""
    heads, D, page = 2, 128, 64
    pages = 140000 if kind == BF16 else 280000                                           # 4.6 GB
    desc = oc.kv_desc(tag(oc, kind), heads, D, 1, 200, page, n_pages=pages)
    shape = (pages, heads, page)
    pool = torch.empty(*shape, D, device="cuda", dtype=BF16 if kind == BF16 else torch.int8)
    scale = None if kind == BF16 else torch.empty(shape, device="cuda")
    table = torch.tensor([[pages - 1, pages - 3, pages - 2, pages - 4]], dtype=torch.int32, device="cuda")
    x = rand(torch.Generator().manual_seed(1), 200, heads, D, dtype=dtype).cuda()
    ctx.kv_put(desc, oc.kv_rows(desc, 200, tag(oc, dtype), k=x), x, pool, k_scale=scale, page_table=table)
    back, q = torch.empty_like(x), rand(torch.Generator().manual_seed(2), rows, heads, D, dtype=dtype).cuda()
    held = torch.empty(200, heads, D, device="cuda") if kind != BF16 else back
    ctx.kv_get(desc, oc.kv_rows(desc, 200, oc.DTYPE_BF16 if kind == BF16 else oc.DTYPE_F32, k=held), pool, held, k_scale=scale, page_table=table)
    out = torch.empty_like(q)
    ctx.attention(desc, oc.attention_desc(desc, rows, tag(oc, dtype), heads, 0.1, q=q, out=out), q, pool, pool, out, k_scale=scale, v_scale=scale, page_table=table)
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.OK
    assert ((held.double() - x.double()).abs() <= (0 if kind == BF16 else 0.5001 / 127) * x.double().abs().amax(-1, keepdim=True)).all()
    p = torch.softmax(torch.einsum("rhd,jhd->hrj", q.double(), held.double()) * 0.1, -1)
    want, size = torch.einsum("hrj,jhd->rhd", p, held.double()), torch.einsum("hrj,jhd->rhd", p, held.double().abs())
    # scores of up to 128 terms: 2 x 133 u times at most 128 x 25 x 0.1; p in bf16 and the output: 2 half steps
    assert ((out.double() - want).abs() <= (2 * 133 * 2.0 ** -24 * 320 + 400 * 2.0 ** -24 + (2.0 ** -7 if dtype == BF16 else 0)) * size).all()


CAPTURED = """
import torch
from paper_2607_23844_b200 import omnicache as oc
ctx = oc.Context(0)
done = []
for dtype, tag in ((torch.bfloat16, oc.DTYPE_BF16), (torch.float32, oc.DTYPE_F32)):
    for kind in (tag, oc.DTYPE_I8, oc.DTYPE_I4):
        for rows in (1, 300):
            d = oc.kv_desc(kind, 2, 64, 1, 600, 64)
            (kp, ks), (vp, vs) = oc.kv_pools(d), oc.kv_pools(d)
            x, q = torch.randn(600, 2, 64, device="cuda", dtype=dtype), torch.randn(rows, 2, 64, device="cuda", dtype=dtype)
            out = torch.zeros_like(q)
            r, a = oc.kv_rows(d, 600, tag, k=x, v=x), oc.attention_desc(d, rows, tag, 2, 0.125, q=q, out=out)
            g = torch.cuda.CUDAGraph()
            def step():
                ctx.kv_put(d, r, x, kp, x, vp, k_scale=ks, v_scale=vs)
                ctx.attention(d, a, q, kp, vp, out, k_scale=ks, v_scale=vs)
            with torch.cuda.graph(g):
                step()
            g.replay()
            torch.cuda.synchronize()
            got = out.clone()
            out.zero_()
            step()
            torch.cuda.synchronize()
            assert got.abs().sum() > 0 and torch.equal(got, out) and ctx.device_status() == oc.OK
print("captured")
"""


@pytest.mark.gpu
def test_a_process_s_first_calls_may_be_captured(oc):
    got = subprocess.run([sys.executable, "-c", CAPTURED], capture_output=True, text=True, timeout=300, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert got.returncode == 0 and "captured" in got.stdout, got.stderr[-2000:]
