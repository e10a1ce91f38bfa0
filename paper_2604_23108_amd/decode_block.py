"""One decoder block for decoding, put together from the library's calls: norm, projections with 4-bit weights, a paged cache and
attention over it, norm, MoHGE layer.

    python -m paper_2604_23108_amd.decode_block --seqs 32 --steps 20

runs such a block with random weights, over a cache filled with random rows, and prints the time of a step.  Position embeddings and sampling are the
caller's; several blocks are stacked by handing `forward`'s two results to the next one.
"""
from __future__ import annotations

import argparse
from typing import Optional, Sequence

import torch

from .binding import BF16, Config, MohgeError, MoHGELayer, SELECT_GLOBAL
from .block_binding import E4M3, CacheConfig, KVCache, NormConfig, ProjConfig, ProjW4, ResidualNorm


class DecodeBlock:
    """A pre-norm block for one new token of each of `seqs` sequences (at most 32, the decode layer's limit):

        s = x + residual,  a = W_o attention(W_qkv norm(s)),  s' = s + a,  y = MoHGE(norm(s'));  returns (y, s').

    The rows that go into the query, key and value projection are bf16, or with `norm_8bit` 8-bit codes with a scale per row (which that
    product turns into bf16 again: 73.0 us a step instead of 72.2, for 32 sequences of 1000 positions).  All buffers are made here; `forward` allocates nothing unless a sequence needs a new page.
    """

    def __init__(self, layer: MoHGELayer, attention_norm: torch.Tensor, qkv: tuple, out: tuple, layer_norm: torch.Tensor,
                 cache: CacheConfig, group: int = 128, eps: float = 1e-6, norm_8bit: bool = False):
        """qkv and out: (codes, scales, zeros or None) of `quantize_w4`: rows for queries, keys and values one after the other, and the
        projection back; attention_norm and layer_norm: fp32 weights [d]."""
        c, T, d = cache, layer.cfg.T, layer.cfg.d
        if c.n_seqs != T or layer.cfg.dtype != BF16 or c.dtype != BF16:
            raise MohgeError("a decode block takes a bf16 layer and cache, one token for each sequence")
        self.q_size, self.kv_size = c.n_heads * c.head_size, c.n_kv_heads * c.head_size
        self.layer, self.cache = layer, KVCache(c, device=attention_norm.device)
        x_dtype = E4M3 if norm_8bit else BF16
        self.attention_norm = ResidualNorm(NormConfig(T, d, y_dtype=x_dtype, eps=eps), attention_norm)
        self.qkv = ProjW4(ProjConfig(T, d, self.q_size + 2 * self.kv_size, group=group, x_dtype=x_dtype), *qkv)
        self.out = ProjW4(ProjConfig(T, self.q_size, d, group=group), *out)
        self.layer_norm = ResidualNorm(NormConfig(T, d, eps=eps), layer_norm)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None, active: Optional[Sequence[bool]] = None):
        """x [seqs, d]: the output of the block before (with the residual stream that came with it) or the embeddings.
        `active` says which sequences have a new token (all unless given).  The cache of the others stays as it is (a finished one's
        pages are given back by `cache.free`); their rows of x hold any finite numbers, their rows of the results mean nothing."""
        n = self.cache.cfg.n_seqs
        self.cache.grow([1] * n if active is None else [int(bool(a)) for a in active])
        return self.step(x, residual)

    def step(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None):
        """`forward` after the cache has grown: kernels only (this part can be recorded into a graph)."""
        c, T = self.cache.cfg, x.shape[0]
        h = self.attention_norm.forward(x, residual)
        stream = x if residual is None else self.attention_norm.sum
        qkv = self.qkv.forward(h, self.attention_norm.y_scale)
        q = qkv[:, :self.q_size].view(T, c.n_heads, c.head_size)
        k = qkv[:, self.q_size:self.q_size + self.kv_size].view(T, c.n_kv_heads, c.head_size)
        v = qkv[:, self.q_size + self.kv_size:].view(T, c.n_kv_heads, c.head_size)
        self.cache.append(k, v)
        a = self.out.forward(self.cache.attend(q).view(T, self.q_size))
        y = self.layer.forward(self.layer_norm.forward(a, stream))
        return y, self.layer_norm.sum


def random_block(seqs: int, d: int = 1024, heads: int = 16, kv_heads: int = 4, head_size: int = 64, page_size: int = 64,
                 longest: int = 4096, cache_dtype: int = BF16, norm_8bit: bool = False, seed: int = 0, device="cuda") -> DecodeBlock:
    """A block with random weights around a layer of 8 groups of 4 experts."""
    from .weights import quantize_w4
    gen = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen, device=device)  # noqa: E731
    widths = (256, 320, 384, 512, 640, 768, 832, 896)
    cfg = Config(T=seqs, d=d, n_groups=8, experts_per_group=4, d_ff=widths, k_groups=3, k_experts=6, select_mode=SELECT_GLOBAL)
    w13 = [(normal(4, 2 * f, d) * 0.02).bfloat16() for f in widths]
    w2 = [(normal(4, d, f) * 0.02).bfloat16() for f in widths]
    layer = MoHGELayer(cfg, normal(8, d) * 0.02, normal(32, d) * 0.02, w13, w2, device=device)
    columns = -(-longest // page_size)
    cache = CacheConfig(seqs, heads, kv_heads, head_size, page_size, seqs * columns, columns, cache_dtype=cache_dtype)
    qkv = quantize_w4(normal((heads + 2 * kv_heads) * head_size, d) * 0.02)
    out = quantize_w4(normal(d, heads * head_size) * 0.02)
    return DecodeBlock(layer, 1 + 0.1 * normal(d), qkv, out, 1 + 0.1 * normal(d), cache, norm_8bit=norm_8bit)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--seqs", type=int, default=32)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--prompt", type=int, default=1000, help="positions in the cache before the first step")
    ap.add_argument("--d", type=int, default=1024)
    ap.add_argument("--cache-8bit", action="store_true")
    ap.add_argument("--norm-8bit", action="store_true")
    a = ap.parse_args(argv)
    block = random_block(a.seqs, d=a.d, longest=a.prompt + a.steps + 8, cache_dtype=E4M3 if a.cache_8bit else BF16,
                         norm_8bit=a.norm_8bit)
    c = block.cache.cfg
    if a.prompt:
        block.cache.grow([a.prompt] * a.seqs)
        rows = torch.randn((a.seqs * a.prompt, 2, c.n_kv_heads, c.head_size), device="cuda").bfloat16()
        block.cache.append(rows[:, 0], rows[:, 1], torch.arange(0, a.seqs * a.prompt + 1, a.prompt, dtype=torch.int32, device="cuda"))
    x = torch.randn((a.seqs, a.d), device="cuda").bfloat16()
    for _ in range(3):
        block.forward(x)
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(a.steps):
        y, stream = block.forward(x)
    stop.record()
    stop.synchronize()
    us = start.elapsed_time(stop) / a.steps * 1e3
    print(f"decode block: {a.seqs} sequences of {block.cache.lengths[0]} positions, d = {a.d}: {us:.1f} us a step, "
          f"|y| {float(y.float().norm()):.3f}, |stream| {float(stream.float().norm()):.3f}")


if __name__ == "__main__":
    main()
