"""One attention layer with shared key heads and rotary positions: a training
step, and the same weights serving a prompt and then one token at a time from a
paged cache.

    python examples/gqa_layer.py

The layer is y = Wo attention(norm and rotation of the rows of Wqkv x).  Both
ways compute the same attention, so the served rows are checked against the
training forward's.
"""
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2402_07901_amd import fastmax as fm  # noqa: E402


class Rows(torch.autograd.Function):
    """A projection's rows [B, N, Hq + 2 Hkv, D] as the attention's q, k, v."""

    @staticmethod
    def forward(ctx, rows, wq, wk, pos, cos, sin, heads):
        ctx.save_for_backward(rows, wq, wk, pos, cos, sin)
        ctx.heads = heads
        return fm.fastmax_rope_fwd(*rows.split(heads, dim=2), pos, cos, sin, wq, wk)

    @staticmethod
    def backward(ctx, gq, gk, gv):
        rows, wq, wk, pos, cos, sin = ctx.saved_tensors
        q, k, _ = rows.split(ctx.heads, dim=2)
        grad = torch.empty_like(rows)
        *_, dwq, dwk = fm.fastmax_rope_bwd(q, k, gq.contiguous(), gk.contiguous(),
                                           gv.contiguous(), pos, cos, sin, wq, wk,
                                           out=grad.split(ctx.heads, dim=2))
        return grad, dwq, dwk, None, None, None, None


class Attention(torch.autograd.Function):
    """Causal Fastmax attention, p = 2."""

    @staticmethod
    def forward(ctx, q, k, v):
        o, g = fm.fastmax_fwd(q, k, v, p=2, causal=True)
        ctx.save_for_backward(q, k, v, o, g)
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, g = ctx.saved_tensors
        return fm.fastmax_bwd(q, k, v, o, do.contiguous(), g, p=2, causal=True)


class Layer:
    def __init__(self, width, Hq, Hkv, D, dtype=torch.bfloat16, positions=4096, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def weight(n, m):
            w = torch.randn((n, m), generator=gen, device="cuda") / m ** 0.5
            return w.to(dtype).requires_grad_()

        self.Hq, self.Hkv, self.D, self.dtype = Hq, Hkv, D, dtype
        self.heads = [Hq, Hkv, Hkv]
        self.qkv, self.out = weight(sum(self.heads) * D, width), weight(width, Hq * D)
        self.wq, self.wk = (torch.ones(D, device="cuda").requires_grad_() for _ in range(2))
        angle = (torch.arange(positions, device="cuda", dtype=torch.float64)[:, None]
                 * 10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D))
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    def parameters(self):
        return [self.qkv, self.out, self.wq, self.wk]

    def train(self, x):
        """x [B, N, width] -> y [B, N, width], differentiable."""
        B, N, _ = x.shape
        pos = torch.arange(N, dtype=torch.int32, device="cuda").expand(B, N).contiguous()
        rows = (x @ self.qkv.t()).unflatten(-1, (sum(self.heads), self.D))
        q, k, v = Rows.apply(rows, self.wq, self.wk, pos, self.cos, self.sin, self.heads)
        o = Attention.apply(q, k, v)
        return o.transpose(1, 2).flatten(2) @ self.out.t()

    @torch.no_grad()
    def serve(self, x, cache, pos, slots, lens, q_start=None, max_q=1):
        """New tokens x [T, width] of several sequences through the cache."""
        k_cache, v_cache, table = cache
        rows = (x @ self.qkv.t()).unflatten(-1, (sum(self.heads), self.D))
        q = fm.fastmax_cache_append(*rows.split(self.heads, dim=1), k_cache, v_cache, slots, pos,
                                    self.cos, self.sin, self.wq, self.wk)
        o = fm.fastmax_paged_fwd(q, k_cache, v_cache, table, lens, q_start=q_start, max_q=max_q)
        return o.flatten(1) @ self.out.t()


def prompts_then_tokens(layer, x, prompt, page=64):
    """x [B, N, width] served as prompts of ``prompt`` tokens and then token by
    token: y [B, N, width], and the seconds of the single-token steps."""
    B, N, _ = x.shape
    cols = -(-N // page)
    kv = torch.zeros((2, B * cols, layer.Hkv, page, layer.D), dtype=layer.dtype, device="cuda")
    table = torch.randperm(B * cols, device="cuda").to(torch.int32).reshape(B, cols)
    cache = (kv[0], kv[1], table)

    def slots(n):                                    # of positions n [B, t]
        return table.long().gather(1, n // page) * page + n % page

    def many(value, size, dtype=torch.int32):
        return torch.full((size,), value, dtype=dtype, device="cuda")

    n = torch.arange(prompt, device="cuda").expand(B, prompt)
    start = torch.arange(B + 1, dtype=torch.int32, device="cuda") * prompt
    y = [layer.serve(x[:, :prompt].flatten(0, 1), cache, n.flatten().int(), slots(n).flatten(),
                     many(prompt, B), start, prompt).unflatten(0, (B, prompt))]
    torch.cuda.synchronize()
    began = time.perf_counter()
    for i in range(prompt, N):
        y.append(layer.serve(x[:, i], cache, many(i, B), slots(many(i, B, torch.int64)[:, None])[:, 0],
                             many(i + 1, B))[:, None])
    torch.cuda.synchronize()
    return torch.cat(y, 1), time.perf_counter() - began


def main(B=4, N=777, prompt=700, width=768, Hq=12, Hkv=4, D=64, dtype=torch.bfloat16):
    layer = Layer(width, Hq, Hkv, D, dtype)
    x = torch.randn((B, N, width), device="cuda").to(dtype)
    y = layer.train(x)
    y.float().square().mean().backward()
    grads = {n: p.grad.float().norm().item()
             for n, p in zip(("qkv", "out", "wq", "wk"), layer.parameters())}
    served, seconds = prompts_then_tokens(layer, x, prompt)
    off = ((served.float() - y.float()).norm() / y.float().norm()).item()
    print(f"gradients {grads}")
    print(f"served against trained: {off:.1e} of the output's size; "
          f"{(N - prompt) * B / seconds:.0f} tokens/s after the prompts")
    return off, grads


if __name__ == "__main__":
    main()
