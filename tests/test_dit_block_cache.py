"""The example's block with attention over the paged cache (examples/dit_block.py --kv) against the same block in plain 32-bit torch
operations, the cache held as the values that it stands for.

Tolerance: as for the block that attends to the kept tokens alone, nine roundings to bf16 at the same places on both sides and
8-bit values a step apart only where those roundings differ: 0.4 % of the output's norm, 1.5 % allowed.  The
probabilities' rounding to bf16 is one more of the same size.  In 4 bits a step is a seventh of a head's largest value: a
key or value whose bf16 roundings differ (by 2^-8 of it at most, a fortieth of a step) lands a step apart once in 40 times at
most, which adds sqrt(1 / 40) / 7 = 2.3 % of the largest value to such elements: 4 % allowed.
"""
import pytest
import torch
import torch.nn.functional as F

from test_dit_block import plain_norm, q8

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def dit():
    from paper_2607_23844_b200 import build
    build.build()
    from examples import dit_block
    return dit_block


def held(x, kv):
    """The values that the cache holds of [rows, heads, D]"""
    if kv == "bf16":
        return x.float()
    L = 127 if kv == "i8" else 7
    x = x.double()
    step = x.abs().amax(-1, keepdim=True) / L
    return ((x / step).round() * step).float()


def plain_step(b, x, cond, slot_of, cache, kvs, kv):
    """The block's step on the rows that slot_of keeps; cache and kvs are updated in place."""
    C, D, per, n = b.C, b.D, b.per, b.n
    lin = lambda name, t: (q8(t.float()) @ q8(b.weights[name][0]).t() + b.weights[name][1]).to(BF16)      # noqa: E731
    mod = lin("mod", F.silu(cond)).float().repeat_interleave(per, 0).split(C, 1)
    kept = torch.arange(n, device="cuda") if slot_of is None else torch.nonzero(slot_of >= 0).reshape(-1)
    h = (plain_norm(x.float()) * (1 + mod[1]) + mod[0])[kept]
    qkv = lin("qkv", h).float().view(-1, 3, b.heads, D)
    y, xx = kept % per // b.W, kept % b.W
    ang = torch.cat([p[:, None].double() * 10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d) for p, d in ((y, b.axes[1]), (xx, b.axes[2]))], 1)
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]

    def turn(t, w):
        t = t * torch.rsqrt(t.pow(2).mean(-1, keepdim=True) + 1e-6) * w
        p, q = t[..., 0::2], t[..., 1::2]
        return torch.stack([p * cos - q * sin, q * cos + p * sin], -1).flatten(-2).to(BF16)
    kvs[0][kept], kvs[1][kept] = held(turn(qkv[:, 1], b.k_w), kv), held(qkv[:, 2].to(BF16), kv)
    q = turn(qkv[:, 0], b.q_w).float().view(b.B, -1, b.heads, D).transpose(1, 2)
    k, v = (t.view(b.B, per, b.heads, D).transpose(1, 2) for t in kvs)
    a = ((q @ k.transpose(-1, -2) / D ** 0.5).softmax(-1) @ v).to(BF16).transpose(1, 2).reshape(-1, C)
    cache[0][kept] = lin("proj", a)
    r = x.float() + mod[2] * cache[0].float()
    h = (plain_norm(r) * (1 + mod[4]) + mod[3])[kept]
    cache[1][kept] = lin("down", F.gelu(lin("up", h).float(), approximate="tanh").to(BF16))
    return (r.to(BF16).float() + mod[5] * cache[1].float()).to(BF16)


@pytest.mark.parametrize("kv,allowed", [("bf16", 0.015), ("i8", 0.015), ("i4", 0.04)])
@pytest.mark.parametrize("B,H,W,heads,D", [(2, 16, 16, 4, 64), (1, 16, 24, 3, 48)])
def test_block_steps_over_the_cache_match_the_plain_block(dit, kv, allowed, B, H, W, heads, D):
    oc = dit.oc
    C = heads * D
    layout = oc.Layout(oc.KIND_TOKEN, oc.DTYPE_BF16, B, 1, H, W, C)
    with oc.Context(0, oc.match_workspace_bytes(layout)) as ctx:
        block = dit.Block(ctx, B, H, W, heads, D, reuse=0.5, kv=kv)
        cond = torch.randn(B, C, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(BF16)
        cache = [torch.zeros(block.n, C, dtype=BF16, device="cuda") for _ in range(2)]
        kvs = [torch.zeros(block.n, heads, D, device="cuda") for _ in range(2)]
        for step, x in enumerate(dit.drifting_input(B, H, W, C, 3)):
            out, slot_of = block.step(x, cond, step == 0)
            want = plain_step(block, x, cond, slot_of, cache, kvs, kv)
            if step:
                assert int((slot_of >= 0).sum()) == B * (block.per - block.n_reuse) < block.n
            for got, ref in ((out, want), (block.cache[0], cache[0]), (block.cache[1], cache[1])):
                err = (got.float() - ref.float()).norm() / ref.float().norm()
                assert err <= allowed, f"step {step}: {err}"
        assert ctx.device_status() == oc.OK
        launched = ctx.launches()
        assert launched["kv_put"] == 3 and launched["attention"] == 3
