"""Attention over the paged cache in the forms that large calls take: two tiles of 128 rows in a CTA, from 148 pairs of tiles
on.  The restatement in 64 bits and its bounds are those of test_attention, computed on the device: the calls are larger."""
import pytest
import torch

from test_attention import BF16, TYPES, Cache, assert_attn, ctx, exact, oc, rand, tag  # noqa: F401 (fixtures)

KINDS = [BF16, "i8", "i4"]


@pytest.fixture(scope="module")
def shared(oc):
    """Caches that several tests read"""
    made = {}

    def get(*key, **kw):
        if (key, tuple(kw.items())) not in made:
            made[key, tuple(kw.items())] = Cache(oc, *key, **kw)
        return made[key, tuple(kw.items())]
    return get


def attend(oc, ctx, cache, q, counts, unit=0, back=-1, ahead=-1, idx=None, ragged=False, check=True):
    """q [n, heads, D] on the CPU, counts: rows of each sequence.  One call, its outputs and log-sum-exps checked."""
    n, H, D = q.shape
    rows, at = [], 0
    for s, m in enumerate(counts):
        for i in range(m):
            p = cache.lens[s] - m + i if idx is None else int(idx[at + i]) - s * cache.seq_rows
            rows.append(None if idx is not None and idx[at + i] < 0 else (s, p))
        at += m
    rows += [None] * (n - at)
    qq = q.cuda()
    out, lse = torch.full((n, H, D), 5.0, dtype=q.dtype, device="cuda"), torch.full((n, H), 5.0, device="cuda")
    ints = lambda x: None if x is None else torch.as_tensor(x).to(torch.int32).cuda()  # noqa: E731
    start = [sum(counts[:i]) for i in range(len(counts) + 1)] if ragged else None
    d = oc.attention_desc(cache.desc, n, tag(oc, q.dtype), H, D ** -0.5, rows_per_batch=max(counts), unit=unit, back=back, ahead=ahead, q=qq, out=out)
    ctx.attention(cache.desc, d, qq, cache.pool["k"], cache.pool["v"], out, kv_len=ints(cache.lens), q_start=ints(start), idx=ints(idx), lse=lse, **cache.args())
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.OK
    if not check:
        return out
    held, cache.val = cache.val, {m: v.cuda() for m, v in cache.val.items()}
    with torch.device("cuda"):
        want, bound, wl, bl = (t.cpu() for t in exact(cache, qq, rows, D ** -0.5, unit, back, ahead))
    cache.val = held
    assert_attn(out, want, bound, rows)
    got, live = lse.cpu().double(), torch.tensor([r is not None for r in rows])
    assert (got[~live] == 5.0).all()
    empty = torch.isinf(wl) & live[:, None]
    assert (got[empty] == -float("inf")).all() and ((got - wl).abs() <= bl)[live[:, None] & ~empty].all()
    return out


def steps_apart(n_seqs, seq_rows, apart, gen, swap=False):
    """Kept tokens of sequences of 512 rows: of every 256 the first 128 lie in one tile of 128 keys, the others `apart` tiles behind
    it (or before it: swap), so that with a causal window one tile of rows ends that many steps before the other."""
    out = []
    for s in range(n_seqs):
        for pair in range(2):
            near = 128 * pair + torch.randint(0, 128, (128,), generator=gen)
            far = near + 128 * apart
            out += [s * seq_rows + x for x in ((far, near) if swap else (near, far))]
    return torch.cat(out)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("apart", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("swap", [False, True])
def test_one_tile_of_rows_ends_before_the_other(oc, ctx, shared, kind, D, apart, swap):
    cache = shared(kind, 20, D, 4, 1317, 64)
    gen = torch.Generator().manual_seed(apart)
    q = rand(gen, 4 * 512, 20, D, dtype=BF16)
    idx = steps_apart(4, 1317, apart, gen, swap)
    first = attend(oc, ctx, cache, q, [512] * 4, unit=1, ahead=0, idx=idx)
    for _ in range(3):
        assert torch.equal(attend(oc, ctx, cache, q, [512] * 4, unit=1, ahead=0, idx=idx, check=False), first)
    attend(oc, ctx, cache, q, [512] * 4, unit=1, back=0, ahead=-1, idx=idx)              # and one that begins before the other
    attend(oc, ctx, cache, q, [512] * 4, unit=100, back=0, ahead=0, idx=idx)             # windows with a gap between them


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [40, 64, 72, 128])
@pytest.mark.parametrize("unit,back,ahead,kept", [(0, -1, -1, False), (1, -1, 0, False), (1, 200, 0, True), (256, -1, 0, True), (256, 0, 0, True), (100, 1, 0, False)])
def test_pairs_of_tiles_under_windows(oc, ctx, shared, kind, D, unit, back, ahead, kept):
    """Rows that are no whole number of tiles; kept lists in order and with an unused tail; lengths that end inside a tile."""
    lens, rows, gen = [700, 411], 390, torch.Generator().manual_seed(D)
    cache = shared(kind, 40, D, 2, 700, 48, lens=tuple(lens), seed=3)
    q = rand(gen, 2 * rows, 40, D, dtype=BF16)
    idx = None
    if kept:
        idx = torch.cat([torch.cat([torch.randperm(700, generator=gen)[: rows - 7].sort().values + 700 * s, torch.full((7,), -1)]) for s in range(2)])
    attend(oc, ctx, cache, q, [rows, rows], unit=unit, back=back, ahead=ahead, idx=idx)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_pairs_of_tiles_of_packed_sequences_and_shared_heads(oc, ctx, kind, D):
    """Sequences of very different lengths behind one another, more rows than keys in one, none in another; four heads to a key."""
    lens, rows = [900, 0, 300, 77, 640], [300, 0, 310, 77, 5]
    cache = Cache(oc, kind, 10, D, 5, 900, 32, lens=lens, seed=4)
    q = rand(torch.Generator().manual_seed(5), sum(rows) + 3, 40, D, dtype=BF16)
    attend(oc, ctx, cache, q, rows, unit=1, ahead=0, ragged=True)
    attend(oc, ctx, cache, q, rows, ragged=True)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_pairs_of_tiles_of_unsorted_rows(oc, ctx, kind, D):
    """Kept lists in descending and in no order: every tile of rows sees every tile of keys in part."""
    gen = torch.Generator().manual_seed(6)
    cache = Cache(oc, kind, 20, D, 4, 520, 16, lens=[520, 519, 129, 1], seed=6)
    q = rand(gen, 4 * 512, 20, D, dtype=BF16)
    for order in (lambda x: x.flip(0), lambda x: x[torch.randperm(512, generator=gen)]):
        idx = torch.cat([order(torch.arange(512)) + 520 * s for s in range(4)])
        attend(oc, ctx, cache, q, [512] * 4, unit=1, ahead=0, idx=idx)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("n_seqs,heads", [(32, 8), (256, 1), (300, 1), (149, 2)])
@pytest.mark.parametrize("how", ["all alike", "ascending", "scattered"])
def test_single_tokens_of_many_sequences(oc, ctx, dtype, kind, n_seqs, heads, how):
    """More CTAs than the device holds at once, where bf16 rows of long sequences come first; equal lengths, and none at all."""
    gen = torch.Generator().manual_seed(n_seqs)
    lens = {"all alike": [100] * n_seqs, "ascending": [s * 130 // n_seqs for s in range(n_seqs)], "scattered": torch.randint(0, 131, (n_seqs,), generator=gen).tolist()}[how]
    cache = Cache(oc, kind, heads, 64, n_seqs, 130, 16, lens=lens, seed=8)
    q = rand(gen, n_seqs, 2 * heads, 64, dtype=dtype)
    attend(oc, ctx, cache, q, [1] * n_seqs)
    attend(oc, ctx, cache, q, [1] * n_seqs, unit=1, back=20, ahead=0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, "i8"])
def test_lengths_out_of_range_among_many_sequences(oc, ctx, kind):
    """Recorded, and taken as the nearer end, wherever the sequence comes in the order of lengths."""
    n = 200
    cache = Cache(oc, kind, 1, 64, n, 48, 16, seed=9)
    q = rand(torch.Generator().manual_seed(9), n, 1, 64, dtype=BF16)
    qq, out = q.cuda(), torch.full((n, 1, 64), 5.0, dtype=BF16, device="cuda")
    lens = torch.full((n,), 48, dtype=torch.int32)
    lens[3], lens[7], lens[11] = 2 ** 31 - 1, -(2 ** 31), -1
    d = oc.attention_desc(cache.desc, n, oc.DTYPE_BF16, 1, 0.125, rows_per_batch=1, q=qq, out=out)
    ctx.attention(cache.desc, d, qq, cache.pool["k"], cache.pool["v"], out, kv_len=lens.cuda(), **cache.args())
    torch.cuda.synchronize()
    assert ctx.device_status() == oc.ERR_INVALID_ARG and ctx.device_status() == oc.OK
    assert (out[7] == 0).all() and (out[11] == 0).all()
    rows = [(s, 0) for s in range(n)]
    cache.lens = [max(0, min(48, int(x))) for x in lens]
    want, bound, _, _ = exact(cache, q, rows, 0.125)
    assert_attn(out, want, bound, rows)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", TYPES)
def test_a_long_chunk_among_single_tokens(oc, ctx, dtype, kind):
    cache = Cache(oc, kind, 2, 72, 40, 700, 32, lens=[700 - 17 * s for s in range(40)], seed=10)
    rows = [1] * 20 + [300] + [1] * 19
    q = rand(torch.Generator().manual_seed(10), sum(rows), 4, 72, dtype=dtype)
    attend(oc, ctx, cache, q, rows, unit=1, ahead=0, ragged=True)
