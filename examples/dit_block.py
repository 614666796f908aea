"""One transformer block under Token Cache, with everything around its attention on this library's kernels.

    python examples/dit_block.py [--steps 4] [--kv i8]      (on a B200)

An SD3-shaped block (adaptive norms, attention, feed-forward) is run for a few denoising steps.  The first step computes
every token and fills the caches; each later step matches and selects on the block's input, computes the kept tokens
only and takes the others from the step before:

    modulation  linear_int8(silu(condition))                       shift, scale and gate of both halves
    select      match, select                                       slot_of, kept_idx
    norm        block_norm(x) -> 8-bit rows of the kept tokens       gather and quantisation on the way
    attention   linear_int8 -> rope(q, k at the kept tokens' positions) -> attention -> quantize_rows -> linear_int8
    between     block_norm: restore from cache, gate, residual, next norm, 8-bit rows of the kept tokens
    feed-fwd    linear_int8 -> gelu -> quantize_rows -> linear_int8
    after       block_norm: restore from cache, gate, residual

Attention is the wrapped layer's own (torch here), among the kept tokens alone, or with --kv over a cache of all tokens'
keys and values, in which those of the reused tokens are still there from the steps before:

    attention  rope -> kv_put (the kept tokens' keys and values to their pages) -> attention (kept queries, all keys)

The gelu is torch's.  Weights are random: this shows the calls, not a model.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch
import torch.nn.functional as F

if __package__ in (None, ""):
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_23844_b200 import omnicache as oc  # noqa: E402

EPS = 1e-6
BF16 = torch.bfloat16


class Int8Linear:
    """A weight matrix in 8 bits with a scale per output channel, and its bias."""

    def __init__(self, ctx: oc.Context, weight: torch.Tensor, bias: torch.Tensor):
        self.N, self.K = weight.shape
        self.w = torch.empty(self.N, self.K, dtype=torch.int8, device="cuda")
        self.scale = torch.empty(self.N, device="cuda")
        ctx.quantize_rows(weight, oc.DTYPE_F32, self.N, self.K, self.w, self.scale)
        self.bias = bias

    def __call__(self, ctx: oc.Context, q: torch.Tensor, q_scale: torch.Tensor) -> torch.Tensor:
        out = torch.empty(q.shape[0], self.N, dtype=BF16, device="cuda")
        ctx.linear_int8(q, q_scale, q.shape[0], self.K, self.w, self.scale, self.N, out, oc.DTYPE_BF16, bias=self.bias)
        return out


def to_int8(ctx: oc.Context, x: torch.Tensor):
    q = torch.empty(x.shape, dtype=torch.int8, device="cuda")
    scale = torch.empty(x.shape[0], device="cuda")
    ctx.quantize_rows(x, oc.DTYPE_BF16, x.shape[0], x.shape[1], q, scale)
    return q, scale


class Block:
    """The block's weights, its two caches (the outputs of attention and feed-forward) and one step of it."""

    def __init__(self, ctx: oc.Context, B: int, H: int, W: int, heads: int, head_dim: int, reuse: float, seed: int = 0,
                 kv: str | None = None):
        self.ctx, self.B, self.H, self.W, self.heads, self.D = ctx, B, H, W, heads, head_dim
        C = self.C = heads * head_dim
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def rand(*shape, std):
            return torch.randn(shape, generator=gen, device="cuda") * std
        self.weights = {n: (rand(o, i, std=i ** -0.5), rand(o, std=0.1))
                        for n, o, i in (("mod", 6 * C, C), ("qkv", 3 * C, C), ("proj", C, C), ("up", 4 * C, C), ("down", C, 4 * C))}
        self.lin = {n: Int8Linear(ctx, w, b) for n, (w, b) in self.weights.items()}
        self.q_w, self.k_w = 1 + rand(head_dim, std=0.1), 1 + rand(head_dim, std=0.1)
        self.layout = oc.Layout(oc.KIND_TOKEN, oc.DTYPE_BF16, B, 1, H, W, C)
        groups, self.per, reps = self.layout.counts()
        self.n = groups * self.per
        self.n_reuse = int(reuse * (self.per - reps))
        self.cache = [torch.empty(self.n, C, dtype=BF16, device="cuda") for _ in range(2)]
        self.axes = (0, head_dim // 2, head_dim - head_dim // 2)
        table_desc = oc.rope_desc(1, oc.DTYPE_BF16, head_dim, self.axes, (1, H, W), heads)
        self.table = oc.rope_table(table_desc).cuda()
        self.kv = None
        if kv is not None:                                                    # a sequence for each image, keys and values of every token
            kind = {"bf16": oc.DTYPE_BF16, "i8": oc.DTYPE_I8, "i4": oc.DTYPE_I4}[kv]
            self.kv = oc.kv_desc(kind, heads, head_dim, B, self.per, page_rows=64)
            (self.k_pool, self.k_scale), (self.v_pool, self.v_scale) = oc.kv_pools(self.kv), oc.kv_pools(self.kv)

    def select(self, x: torch.Tensor):
        """(slot_of, kept_idx, kept tokens per batch element) of this step's input."""
        keep, n = self.per - self.n_reuse, self.n
        sim, idx = torch.empty(n, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
        kept = torch.empty(self.B * keep, dtype=torch.int32, device="cuda")
        count = torch.empty(self.B, dtype=torch.int32, device="cuda")
        match_map, slot_of = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
        self.ctx.match(self.layout, x, sim, idx)
        self.ctx.select(self.layout, sim, idx, oc.SELECT_COUNT, 0.0, self.n_reuse, keep, kept, count, match_map, slot_of)
        return slot_of, kept, keep

    def attend(self, q, k, v, kept, dense: int) -> torch.Tensor:
        """The kept tokens' keys and values into the cache, their queries over all of it: [dense, C]."""
        ctx, kv = self.ctx, self.kv
        ctx.kv_put(kv, oc.kv_rows(kv, dense, oc.DTYPE_BF16, k=k, v=v), k, self.k_pool, v, self.v_pool, k_scale=self.k_scale,
                   v_scale=self.v_scale, idx=kept)
        a = torch.empty(dense, self.heads, self.D, dtype=BF16, device="cuda")
        d = oc.attention_desc(kv, dense, oc.DTYPE_BF16, self.heads, self.D ** -0.5, q=q, out=a)
        ctx.attention(kv, d, q, self.k_pool, self.v_pool, a, k_scale=self.k_scale, v_scale=self.v_scale, idx=kept)
        return a.view(dense, self.C)

    def step(self, x: torch.Tensor, condition: torch.Tensor, first: bool):
        """x [n, C] bf16, condition [B, C] bf16 -> (the block's output, this step's slot_of or None)."""
        ctx, C, n, D = self.ctx, self.C, self.n, self.D
        mod = self.lin["mod"](ctx, *to_int8(ctx, F.silu(condition)))          # [B, 6C]
        shift1, scale1, gate1, shift2, scale2, gate2 = (mod[:, i * C:(i + 1) * C] for i in range(6))
        slot_of, kept, keep = (None, None, self.per) if first else self.select(x)
        dense = self.B * keep
        common = dict(rows_per_group=self.per, mod_stride=6 * C, dense_rows=dense, post_eps=EPS, pre_eps=EPS)

        # norm and modulation, gather and quantisation in one pass
        h, h_scale = torch.empty(dense, C, dtype=torch.int8, device="cuda"), torch.empty(dense, device="cuda")
        d = oc.block_norm_desc(n, C, oc.DTYPE_BF16, oc.DTYPE_I8, oc.DTYPE_BF16, pre_norm=oc.NORM_LAYER, **common)
        ctx.block_norm(d, x, slot_of=slot_of, scale=scale1, shift=shift1, h=h, h_scale=h_scale)

        qkv = self.lin["qkv"](ctx, h, h_scale).view(dense, 3, self.heads, D)
        q, k, v = qkv[:, 0], qkv[:, 1], qkv[:, 2]
        qo, ko = (torch.empty(self.B, self.heads, keep, D, dtype=BF16, device="cuda") for _ in range(2))
        d = oc.rope_desc(dense, oc.DTYPE_BF16, D, self.axes, (1, self.H, self.W), self.heads, self.heads, rows_per_batch=keep,
                         eps=EPS, q=q, q_out=qo, k=k, k_out=ko)
        ctx.rope(d, self.table, q, qo, k=k, k_out=ko, idx=kept, q_w=self.q_w, k_w=self.k_w)
        if self.kv is None:
            a = F.scaled_dot_product_attention(qo, ko, v.view(self.B, keep, self.heads, D).transpose(1, 2))
            a = a.transpose(1, 2).reshape(dense, C)
        else:
            a = self.attend(qo, ko, v, kept, dense)
        z = self.lin["proj"](ctx, *to_int8(ctx, a))

        # restore, gate, residual, the next norm and its 8-bit rows in one pass
        mid = torch.empty_like(x)
        d = oc.block_norm_desc(n, C, oc.DTYPE_BF16, oc.DTYPE_I8, oc.DTYPE_BF16, pre_norm=oc.NORM_LAYER, **common)
        ctx.block_norm(d, x, z=z, slot_of=slot_of, cache=None if first else self.cache[0], cache_out=self.cache[0], out=mid,
                       gate=gate1, scale=scale2, shift=shift2, h=h, h_scale=h_scale)

        u = F.gelu(self.lin["up"](ctx, h, h_scale), approximate="tanh")
        z = self.lin["down"](ctx, *to_int8(ctx, u))
        out = torch.empty_like(x)
        d = oc.block_norm_desc(n, C, oc.DTYPE_BF16, oc.DTYPE_BF16, oc.DTYPE_BF16, **common)
        ctx.block_norm(d, mid, z=z, slot_of=slot_of, cache=None if first else self.cache[1], cache_out=self.cache[1], out=out, gate=gate2)
        return out, slot_of


def drifting_input(B: int, H: int, W: int, C: int, steps: int, seed: int = 1):
    """Smooth features that drift a little from step to step."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = F.interpolate(torch.randn(B, C, max(H // 4, 1), max(W // 4, 1), generator=gen, device="cuda"), size=(H, W), mode="bilinear")
    x = x.permute(0, 2, 3, 1).reshape(B * H * W, C) + 0.1 * torch.randn(B * H * W, C, generator=gen, device="cuda")
    for _ in range(steps):
        yield x.to(BF16).contiguous()
        x = x + 0.02 * torch.randn(x.shape, generator=gen, device="cuda")


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--kv", choices=["bf16", "i8", "i4"], help="attend over a cache of all tokens' keys and values, of this type")
    a = ap.parse_args()
    B, H, W, heads, D = 2, 64, 64, 24, 64
    layout = oc.Layout(oc.KIND_TOKEN, oc.DTYPE_BF16, B, 1, H, W, heads * D)
    with oc.Context(0, oc.match_workspace_bytes(layout)) as ctx:
        block = Block(ctx, B, H, W, heads, D, reuse=0.5, kv=a.kv)
        condition = torch.randn(B, heads * D, device="cuda").to(BF16)
        for step, x in enumerate(drifting_input(B, H, W, heads * D, a.steps)):
            for _ in range(3):
                block.step(x, condition, step == 0)
            start, end = torch.cuda.Event(True), torch.cuda.Event(True)
            start.record()
            out, slot_of = block.step(x, condition, step == 0)
            end.record()
            torch.cuda.synchronize()
            computed = block.n if slot_of is None else int((slot_of >= 0).sum())
            print(f"step {step}: {computed} of {block.n} tokens computed, {start.elapsed_time(end) * 1e3:.0f} us, rms {out.float().pow(2).mean().sqrt():.3f}")
        assert ctx.device_status() == oc.OK
        print({k: v for k, v in ctx.launches().items() if v})


if __name__ == "__main__":
    main()
