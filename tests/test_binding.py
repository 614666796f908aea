"""What the Python binding makes of its arguments before the library sees them: addresses, strides of parts of larger
tensors.  No GPU: a recorder stands in for the library."""
import enum

import pytest
import torch


@pytest.fixture(scope="module")
def oc():
    from paper_2607_23844_b200 import build
    build.build()
    from paper_2607_23844_b200 import omnicache
    return omnicache


@pytest.fixture
def calls(oc, monkeypatch):
    """(a context, the arguments of every call that it made)"""
    made = []

    class Recorder:
        def __getattr__(self, name):
            def call(*args):
                made.append((name, args))
                return oc.OK
            return call
    monkeypatch.setattr(oc, "_lib", Recorder())
    ctx = object.__new__(oc.Context)
    ctx._h = None
    return ctx, made


class Address(enum.IntEnum):
    BUFFER = 0x7000


def test_addresses_may_be_any_int(oc):
    for p in (oc._ptr, oc._ptr_strided):
        assert p(None) is None and p(64) == 64 and p(Address.BUFFER) == 0x7000
    t = torch.zeros(4, 6)
    assert oc._ptr(t) == t.data_ptr()
    with pytest.raises(AssertionError):
        oc._ptr(t[:, :3])


def test_quantize_rows_takes_the_stride_of_a_column_range(oc, calls):
    ctx, made = calls
    packed, q, s = torch.zeros(7, 96), torch.zeros(7, 32, dtype=torch.int8), torch.zeros(7)

    def stride(x, **kw):
        ctx.quantize_rows(x, oc.DTYPE_F32, 7, 32, q, s, stream=0, **kw)
        name, args = made.pop()
        assert name == "oc_quantize_rows" and args[1] == (x if isinstance(x, int) else x.data_ptr())
        return args[4]
    assert stride(packed[:, 32:64]) == 96
    assert stride(packed[:, 32:64], x_stride=96) == 96
    assert stride(packed.as_strided((7, 32), (40, 1))) == 40
    # dense tensors, and addresses, keep the default and what is asked for
    assert stride(torch.zeros(7, 32)) == 32 and stride(torch.zeros(7, 4, 8)) == 32 and stride(torch.zeros(7 * 32)) == 32
    assert stride(0x1000) == 32 and stride(0x1000, x_stride=64) == 64 and stride(packed, x_stride=96) == 96
    for x in (packed[:, :32].t(), packed[:, 0:64:2], packed.view(7, 12, 8)[:, :4], packed[:, :16], packed[:, :48]):
        with pytest.raises(ValueError):
            stride(x)
    for x in (torch.zeros(32, 7).t(), packed[:, 0:64:2]):
        with pytest.raises(ValueError):
            stride(x, x_stride=96)
    assert not made


def test_linear_int8_takes_the_stride_of_a_column_range(oc, calls):
    ctx, made = calls
    a, s, w, sw = torch.zeros(7, 16, dtype=torch.int8), torch.zeros(7), torch.zeros(32, 16, dtype=torch.int8), torch.zeros(32)
    packed = torch.zeros(7, 96)

    def stride(out, **kw):
        ctx.linear_int8(a, s, 7, 16, w, sw, 32, out, oc.DTYPE_F32, stream=0, **kw)
        name, args = made.pop()
        assert name == "oc_linear_int8" and args[9] == (out if isinstance(out, int) else out.data_ptr())
        return args[12]
    assert stride(packed[:, 32:64]) == 96 and stride(packed[:, 32:64], out_stride=96) == 96
    assert stride(torch.zeros(7, 32)) == 32 and stride(torch.zeros(7, 4, 8)) == 32 and stride(packed, out_stride=96) == 96
    assert stride(0x1000) == 32 and stride(0x1000, out_stride=40) == 40
    for out in (packed[:, 0:64:2], packed.view(7, 12, 8)[:, :4], packed[:, :48], torch.zeros(32, 7).t()):
        with pytest.raises(ValueError):
            stride(out)
    with pytest.raises(ValueError):
        stride(packed[:, 0:64:2], out_stride=96)
    assert not made


def test_block_norm_group_vectors_lie_mod_stride_apart(oc, calls):
    ctx, made = calls
    C, G = 32, 4
    x, h = torch.zeros(20, C), torch.zeros(20, C)
    mod = torch.zeros(G, 3 * C)

    def run(t, mod_stride, rows_per_group=5, name="scale"):
        d = oc.block_norm_desc(20, C, oc.DTYPE_F32, oc.DTYPE_F32, oc.DTYPE_F32, rows_per_group=rows_per_group, mod_stride=mod_stride)
        ctx.block_norm(d, x, h=h, stream=0, **{name: t})
        got, args = made.pop()
        assert got == "oc_block_norm" and args[{"gate": 10, "scale": 13, "shift": 14}[name]] == (t if isinstance(t, int) else t.data_ptr())

    def refused(*args, **kw):
        with pytest.raises(ValueError):
            run(*args, **kw)
        assert not made
    for name in ("gate", "scale", "shift"):
        run(mod[:, C:2 * C], 3 * C, name=name)
        run(0x1000, 3 * C, name=name)
        refused(mod[:, C:2 * C], 0, name=name)                                # group 0's vector for every row
        refused(mod[:, C:2 * C], C, name=name)
        refused(mod[:, 0:2 * C:2], 3 * C, name=name)                          # every other element
    # one vector for all groups
    vector = torch.zeros(C)
    for t in (vector, vector[None], vector.expand(G, C), mod[1:2, :C], mod[1, :C]):
        run(t, 0)
    # more groups than vectors
    refused(vector, C), refused(torch.zeros(1, C)[:, None], 2 * C), refused(torch.zeros(G, 2, C)[:3], 2 * C)
    # vectors by any route that are as far apart as was said
    run(mod.view(G, 3, C)[:, 1:2], 3 * C), run(mod.view(2, 2, 3 * C)[..., :C], 3 * C), run(mod.view(G, 3, C), 3 * C)
    run(mod.view(-1)[C:], 3 * C), run(mod[0, :C], 3 * C), run(mod.view(1, -1)[:, C:2 * C], 3 * C)
    refused(mod[1, :C], 3 * C), refused(mod.view(1, -1)[:, 3 * C:4 * C], 3 * C)                # (the last one past the end)
    run(torch.zeros(G, C), C), run(torch.zeros(6, 3 * C)[:, :C], 3 * C)
    refused(torch.zeros(2, 3, 3 * C)[:, :2, :C], 3 * C)                       # (a gap after every second)
    # a single group: only the elements of its vector matter
    run(mod[:1, :C], 3 * C, 20), run(vector, 96, 20), run(mod[:, :C], 0, 20), refused(mod[:1, 0:2 * C:2], 3 * C, 20)


def views(d):
    return [[getattr(getattr(d, v), f) for f in ("batch_stride", "row_stride", "head_stride")] for v in ("q", "q_out", "k", "k_out")]


def test_rope_desc_head_major_inputs(oc):
    """Rows of q and k follow one another at one stride: a [batch, heads, rows, head_dim] tensor of several batch elements
    has none, unless its batch elements follow one another like its rows."""
    B, n, heads, D = 3, 10, 4, 8

    def desc(q, rows=B * n, **kw):
        return oc.rope_desc(rows, oc.DTYPE_F32, D, (0, 4, 4), (1, 5, 6), heads, rows_per_batch=n, q=q, **kw)
    head_major, out = torch.zeros(B, heads, n, D), torch.zeros(B, heads, n, D)
    for m in ("q", "k"):
        with pytest.raises(ValueError):
            desc(**{"q": out.transpose(1, 2).reshape(B * n, heads, D), "k_heads": heads, m: head_major})
    assert views(desc(torch.zeros(B, n, heads, D).transpose(1, 2), q_out=out))[:2] == [[n * heads * D, heads * D, D], [heads * n * D, D, n * D]]
    assert views(desc(head_major[:1], rows=n))[0][1:] == [D, n * D]
    assert views(desc(torch.zeros(B * n, heads, D)))[0][1:] == [heads * D, D]


def test_rope_desc_tensors_hold_all_rows(oc):
    """rows_per_batch is the length of a batch element of a head-major output; a tensor of fewer rows than the call's is
    no place for them."""
    B, n, heads, D = 3, 10, 4, 8
    rows, head_major = torch.zeros(B * n, heads, D), torch.zeros(B, heads, n, D)

    def desc(rows_per_batch=n, n_rows=B * n, **kw):
        return oc.rope_desc(n_rows, oc.DTYPE_F32, D, (0, 4, 4), (1, 5, 6), heads, heads, rows_per_batch=rows_per_batch, **kw)
    for m in ("q", "k"):
        desc(**{m: rows, m + "_out": head_major})
        for bad in ({m + "_out": head_major, "rows_per_batch": None},         # all rows in batch element 0
                    {m + "_out": head_major, "rows_per_batch": n + 1}, {m + "_out": head_major[:2]}, {m + "_out": rows[1:]},
                    {m: rows[1:]}, {m: torch.zeros(1, heads, B * n - 1, D)}):
            with pytest.raises(ValueError):
                desc(**bad)
        # longer ones are: a cache with room for what follows, one batch element shorter than the others could be
        desc(**{m: torch.zeros(40, heads, D), m + "_out": torch.zeros(B + 1, heads, n + 5, D)})
        desc(rows_per_batch=64, n_rows=n, **{m + "_out": head_major})
        desc(n_rows=0, rows_per_batch=None, **{m: rows[:0], m + "_out": rows[:0]})
        desc(n_rows=25, **{m + "_out": head_major})                           # the last batch element is not full


def test_rope_desc_strides_given_afterwards(oc):
    """Only strides that something is reached by are left invalid where no tensor was given."""
    def left(n_rows, heads):
        d = oc.rope_desc(n_rows, oc.DTYPE_F32, 8, (0, 4, 4), (1, 5, 6), heads, heads)
        assert len({tuple(v) for v in views(d)}) == 1
        return views(d)[0]
    assert left(10, 4) == [0, -1, -1] and left(1, 4) == [0, 0, -1] and left(10, 1) == [0, -1, 0] and left(1, 1) == [0, 0, 0]
