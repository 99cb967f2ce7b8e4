"""A stack of attention blocks serving a few token streams that fork.

Each block is a pre-norm with its residual sum, a projection to queries, keys and
values, rotary positions, attention over a window of a cache in 4 bits, and a
projection back; all blocks share one set of pages.  Prompts of unequal lengths go in
as one call, then one stream goes on as two, drafted tokens are partly taken back, and
the streams advance token by token; at the end the same tokens as clips give the same
outputs (Definition 1).  Random weights, synthetic tokens.

    python examples/stream_attention.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2204_03418_amd import coinf  # noqa: E402

DEV, DTYPE = "cuda", torch.bfloat16


class Block:
    def __init__(self, gen, pages, layer, dim, heads, window):
        def randn(*shape, scale):
            return torch.randn(shape, generator=gen, device=DEV) * scale

        D, K = pages.head_dim, pages.kv_heads
        self.split = (heads, K, K)
        self.w_in = randn(dim, (heads + 2 * K) * D, scale=dim ** -0.5).to(DTYPE)
        self.w_out = randn(heads * D, dim, scale=(heads * D) ** -0.5).to(DTYPE)
        self.norm = coinf.CoNorm(torch.ones(dim, device=DEV), residual="before")
        self.attention = coinf.CoAttention(pages, layer, heads=heads, window=window, dtype=DTYPE)

    def __call__(self, rotary, mode, x, residual, positions, lengths):
        """(x, residual) -> the block's output and the residual before it."""
        x, residual = self.norm.forward(x, residual=residual)
        qkv = (x @ self.w_in).unflatten(-1, (sum(self.split), -1))
        q, k, v = qkv.split(self.split, -2)
        turn = rotary.forward_step if mode == "forward_step" else rotary.forward
        q, k = turn(q, k, positions=positions, lengths=lengths)
        run = getattr(self.attention, mode)
        y = run(q, k, v, lengths) if mode == "forward" else run(q, k, v)
        return y.flatten(-2) @ self.w_out, residual


class Model:
    def __init__(self, batch, dim=256, layers=3, heads=8, kv_heads=2, head_dim=64, window=128,
                 seed=0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.window = window
        self.pages = coinf.CoPages(batch=batch, pages=16 * batch, stream_pages=16, page_tokens=32,
                                   layers=layers, kv_heads=kv_heads, head_dim=head_dim, device=DEV)
        self.rotary = coinf.CoRotary(head_dim, device=DEV)
        self.blocks = [Block(gen, self.pages, i, dim, heads, window) for i in range(layers)]
        self.last = coinf.CoNorm(torch.ones(dim, device=DEV), residual="before")

    def __call__(self, mode, x, lengths=None):
        positions = None  # a clip's are 0, 1, ...
        if mode != "forward":
            T = 1 if mode == "forward_step" else x.shape[1]
            lengths = self.pages.reserve(T, lengths, keep=self.window)
            positions = self.pages.base
        residual = torch.zeros(x.shape, dtype=torch.float32, device=DEV)
        for block in self.blocks:
            x, residual = block(self.rotary, mode, x, residual, positions, lengths)
        return self.last.forward(x, residual=residual)[0]


def main(batch=4, longest=200, drafted=5, tokens=20, dim=256):
    gen = torch.Generator(device=DEV).manual_seed(1)
    n = torch.tensor([longest, longest // 3, 1, 70][:batch], dtype=torch.int32, device=DEV)
    x = torch.randn(batch, longest + tokens, dim, generator=gen, device=DEV).to(DTYPE)
    model = Model(batch, dim=dim)
    pages = model.pages
    model("forward_steps", x[:, :longest].contiguous(), n)
    # the last stream becomes a copy of the first, and goes on with its own tokens
    source = torch.arange(batch, dtype=torch.int32, device=DEV)
    source[-1] = 0
    pages.select(source)
    seen = [x[int(s), :int(n[int(s)])] for s in source]
    # drafted tokens, of which each stream keeps two
    own = torch.randn(batch, drafted + tokens, dim, generator=gen, device=DEV).to(DTYPE)
    model("forward_steps", own[:, :drafted].contiguous())
    pages.truncate(pages.base + 2)
    steps = [model("forward_step", own[:, drafted + i].contiguous()) for i in range(tokens)]
    worst = 0.0
    for i in range(batch):
        clip = torch.cat((seen[i], own[i, :2], own[i, drafted:]))
        whole = model("forward", clip.expand(batch, -1, -1).contiguous())[0, -tokens:].float()
        got = torch.stack([s[i] for s in steps]).float()
        off = float((got - whole).norm() / whole.norm())
        print(f"stream {i}: {len(clip)} tokens, steps against clip: {off:.1e}", flush=True)
        worst = max(worst, off)
    print(f"{int((pages.refs > 0).sum())} pages in use, {int(pages.refused.sum())} tokens refused")
    return worst


if __name__ == "__main__":
    # single tokens and clips take the sums in another order; a key or value that this moves over
    # the border of two codes is a step off
    sys.exit(0 if main() < 0.05 else 1)
