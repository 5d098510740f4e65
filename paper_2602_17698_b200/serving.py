"""The attention block of a quantised decoder, as a serving program runs it: weights and activations
in a microscaled 4-bit format, keys and values in a paged cache of 8 or 4 bits.

    x -> 4 bits -> QKV product (+ adapters) -> rotary positions -> append to the cache -> attention over the cache
      -> 4 bits -> O product (+ adapters)

Every call only enqueues; requests' lengths, the page table and the tensor scales are read on the
device, so one captured CUDA graph serves a decode batch while its requests grow.

    python -m paper_2602_17698_b200.serving        # a small block: prompts, then decode steps from a graph
    python -m paper_2602_17698_b200.serving --cache 4 --rotary --adapters 3
"""
from __future__ import annotations

import argparse
import sys
from contextlib import contextmanager
from typing import Callable, Optional, Sequence, Union

import torch

from .binding import (SB_KV8_BLOCK, Context, Fp4Matrix, Kv4Cache, Kv8Cache, LoraAdapters, RotaryTable, fp4_scale_bytes,
                      rotary_frequencies)


@contextmanager
def _stream_of(ctx: Context, *inputs: torch.Tensor):
    """Makes the context's stream torch's current one, behind what the current one has enqueued and ahead of what it will."""
    here = torch.cuda.current_stream(ctx.device)
    if here == ctx.stream:
        yield
        return
    ctx.stream.wait_stream(here)
    for t in inputs:
        t.record_stream(ctx.stream)
    with torch.cuda.stream(ctx.stream):
        yield
    here.wait_stream(ctx.stream)


def tensor_scale(x: torch.Tensor) -> torch.Tensor:
    """A tensor scale for the "nv" format, on the device: the smallest power of two under which the
    largest block scale of x still fits e4m3.  (A power of two leaves every quotient exact.)"""
    return torch.exp2(torch.ceil(torch.log2(x.float().abs().amax().clamp_min(2.0 ** -100) / (6 * 448)))).reshape(1)


def quantize_weight(ctx: Context, W: torch.Tensor, fmt: str = "nv") -> Fp4Matrix:
    """A bf16 weight [out][in] in 4 bits, with a tensor scale of its own where the format has one."""
    with _stream_of(ctx, W):
        m = Fp4Matrix.empty(W.shape[0], W.shape[1], fmt, tensor_scale(W) if fmt == "nv" else None, W.device)
        return ctx.fp4_quantize(W, m)


def page_table(lens, page_tokens: int, pages: int, device="cuda") -> torch.Tensor:
    """Pages handed out in order, `lens` tokens (rounded up to pages) for every request: int32 [requests][pages of the longest]."""
    need = [-(-int(n) // page_tokens) for n in lens]
    if sum(need) > pages:
        raise ValueError(f"{sum(need)} pages are needed, the cache has {pages}")
    table = torch.zeros((len(need), max(need)), dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = torch.arange(at, at + n, dtype=torch.int32)
        at += n
    return table.to(device)


class QuantizedAttention:
    """Weights, cache and workspaces of one attention block with `heads` query heads over `kv_heads` heads of `dim`.

    w_qkv: bf16 [(heads + 2 kv_heads) dim][hidden], w_o: bf16 [hidden][heads dim].  x_scale, o_scale:
    tensor scales of the block's input and of the attention's output ("nv" only; None: 1, which suits
    activations of the order of 1).  max_tokens: rows of a call at most.  rotary: turns the projected queries and keys by their
    positions.  qkv_adapters, o_adapters: low-rank adapters of many requests beside the two projections (of the bf16 inputs).  Everything runs on the context's stream; where
    torch's current stream is another, that waits for this one and this one for that."""

    def __init__(self, ctx: Context, w_qkv: torch.Tensor, w_o: torch.Tensor, heads: int, kv_heads: int, dim: int,
                 cache: Union[Kv8Cache, Kv4Cache], max_tokens: int, fmt: str = "nv", x_scale: Optional[torch.Tensor] = None,
                 o_scale: Optional[torch.Tensor] = None, rotary: Optional[RotaryTable] = None, qkv_adapters: Optional[LoraAdapters] = None,
                 o_adapters: Optional[LoraAdapters] = None):
        hidden = w_o.shape[0]
        if w_qkv.shape != ((heads + 2 * kv_heads) * dim, hidden) or w_o.shape[1] != heads * dim:
            raise ValueError("w_qkv: [(heads + 2 kv_heads) dim][hidden], w_o: [hidden][heads dim]")
        for what, adapters, w in (("qkv_adapters", qkv_adapters, w_qkv), ("o_adapters", o_adapters, w_o)):
            if adapters is not None and (adapters.outer, adapters.inner) != tuple(w.shape):
                raise ValueError(f"{what}: adapters of the projection's sizes")
        self.ctx, self.cache, self.fmt, self.heads, self.kv_heads, self.dim = ctx, cache, fmt, heads, kv_heads, dim
        self.w_qkv, self.w_o = quantize_weight(ctx, w_qkv, fmt), quantize_weight(ctx, w_o, fmt)
        self.x_scale, self.o_scale = x_scale, o_scale
        self.rotary, self.qkv_adapters, self.o_adapters = rotary, qkv_adapters, o_adapters
        dev = w_o.device
        with _stream_of(ctx):
            self.qkv = torch.empty((max_tokens, w_qkv.shape[0]), dtype=torch.bfloat16, device=dev)
            self.att = torch.empty((max_tokens, heads, dim), dtype=torch.bfloat16, device=dev)
            self.y = torch.empty((max_tokens, hidden), dtype=torch.bfloat16, device=dev)
            # 4-bit workspaces of max_tokens rows by width; a call's matrix is the first part of both tensors
            self._low = {c: Fp4Matrix.empty(max_tokens, c, fmt, None, dev) for c in (hidden, heads * dim)}
        self._part = {}                                # the last call's matrix by width

    def _in_4_bits(self, x: torch.Tensor, scale) -> Fp4Matrix:
        rows, cols = x.shape
        m = self._part.get(cols)
        if m is None or m.rows != rows:
            whole = self._low[cols]
            m = self._part[cols] = Fp4Matrix(whole.codes[:rows], whole.scales[:fp4_scale_bytes(rows, cols, self.fmt)], rows, cols, self.fmt)
        m.tensor_scale = scale
        return self.ctx.fp4_quantize(x, m)

    def __call__(self, x: torch.Tensor, starts: torch.Tensor, lens: torch.Tensor, max_new: int, max_len: int, window: int = 0,
                 rotate: Optional[Callable] = None, ids: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x: bf16 [tokens][hidden], request b's new tokens in rows starts[b] .. starts[b + 1]; lens: its
        length with them.  rotate(q, k): called on the projected queries and keys, in place, with the
        context's stream as torch's current one.  ids: every request's adapter (int32, -1: none; None: no request has one).  Returns the block's output (a workspace: valid until
        the next call)."""
        t, ctx = x.shape[0], self.ctx
        if not 0 < t <= len(self.y) or x.shape[1] != self.y.shape[1]:
            raise ValueError("x: [tokens][hidden], one token at least and max_tokens at most")
        nq, nk = self.heads * self.dim, self.kv_heads * self.dim
        with _stream_of(ctx, x, starts, lens, *(() if ids is None else (ids,))):
            qkv = ctx.fp4_gemm(self._in_4_bits(x, self.x_scale), self.w_qkv, out=self.qkv[:t])
            if ids is not None and self.qkv_adapters is not None:
                ctx.lora_add(self.qkv_adapters, x, qkv, ids, starts, max_new)
            q = qkv[:, :nq].view(t, self.heads, self.dim)
            k = qkv[:, nq:nq + nk].view(t, self.kv_heads, self.dim)
            v = qkv[:, nq + nk:].view(t, self.kv_heads, self.dim)
            if self.rotary is not None:
                ctx.rotary(self.rotary, q, k, starts, lens, max_new)
            if rotate is not None:
                rotate(q, k)
            append, attention = (ctx.kv4_append, ctx.kv4_attention) if isinstance(self.cache, Kv4Cache) else (ctx.kv8_append, ctx.kv8_attention)
            append(self.cache, k, v, starts, lens, max_new)
            att, _ = attention(self.cache, q, starts, lens, max_new, max_len, window=window, out=self.att[:t])
            att = att.view(t, nq)
            y = ctx.fp4_gemm(self._in_4_bits(att, self.o_scale), self.w_o, out=self.y[:t])
            if ids is not None and self.o_adapters is not None:
                ctx.lora_add(self.o_adapters, att, y, ids, starts, max_new)
            return y


def main(argv: Sequence[str] = ()) -> None:
    """Prompts of different lengths, then decode steps replayed from one graph; prints how far the
    quantised block is from the same block in bf16 weights and an unquantised cache."""
    ap = argparse.ArgumentParser(prog="paper_2602_17698_b200.serving")
    ap.add_argument("--cache", type=int, choices=(8, 4), default=8, help="bits of the key/value cache")
    ap.add_argument("--rotary", action="store_true", help="rotary positions")
    ap.add_argument("--adapters", type=int, default=0, help="low-rank adapters; request i has number i - 1")
    args = ap.parse_args(list(argv))
    torch.manual_seed(0)
    dev, hidden, heads, kv_heads, dim, page = "cuda", 1024, 16, 4, 64, 32
    prompts, steps = [300, 77, 1, 500], 8
    n, most = len(prompts), max(prompts) + steps
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = Context(stream=stream)
        w_qkv = (torch.randn((heads + 2 * kv_heads) * dim, hidden, device=dev) * hidden ** -0.5).bfloat16()
        w_o = (torch.randn(hidden, heads * dim, device=dev) * (heads * dim) ** -0.5).bfloat16()
        table = page_table([p + steps for p in prompts], page, 64, dev)
        cache = (Kv8Cache if args.cache == 8 else Kv4Cache).empty(64, kv_heads, page, dim, table)
        turn = RotaryTable(rotary_frequencies(dim).to(dev)) if args.rotary else None
        beside = [LoraAdapters((torch.randn(args.adapters, 16, w.shape[1], device=dev) * w.shape[1] ** -0.5).bfloat16(),
                               (torch.randn(args.adapters, w.shape[0], 16, device=dev) * 0.1).bfloat16()) if args.adapters else None for w in (w_qkv, w_o)]
        who = [i - 1 if i <= args.adapters else -1 for i in range(n)]
        ids = torch.tensor(who, dtype=torch.int32, device=dev) if args.adapters else None
        block = QuantizedAttention(ctx, w_qkv, w_o, heads, kv_heads, dim, cache, sum(prompts), o_scale=torch.full((1,), 2.0 ** -4, device=dev),
                                   rotary=turn, qkv_adapters=beside[0], o_adapters=beside[1])
        xs = [torch.randn(p + steps, hidden, device=dev).bfloat16() for p in prompts]

        starts = torch.tensor([0] + prompts, dtype=torch.int32).cumsum(0).to(torch.int32).to(dev)
        lens = torch.tensor(prompts, dtype=torch.int32, device=dev)
        ys = [list(y.clone().split(1)) for y in
              block(torch.cat([x[:p] for x, p in zip(xs, prompts)]), starts, lens, max(prompts), max(prompts),
                    ids=ids).split(prompts)]

        # one new token each: a graph whose requests grow
        one, x_in = torch.arange(n + 1, dtype=torch.int32, device=dev), torch.empty(n, hidden, dtype=torch.bfloat16, device=dev)
        x_in.copy_(torch.stack([x[p] for x, p in zip(xs, prompts)]))
        lens += 1
        block(x_in, one, lens, 1, most, ids=ids)                 # workspaces exist before the capture
        ctx.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y_out = block(x_in, one, lens, 1, most, ids=ids)
        for s in range(steps):
            x_in.copy_(torch.stack([x[p + s] for x, p in zip(xs, prompts)]))
            graph.replay()
            for i in range(n):
                ys[i].append(y_out[i:i + 1].clone())
            lens += 1
        ctx.sync()

    def project(i, x, w, adapters):
        y = x @ w.float().t()
        return y + x @ adapters.a[who[i]].float().t() @ adapters.b[who[i]].float().t() if adapters and who[i] >= 0 else y

    def turned(x):
        if turn is None:
            return x
        angle = torch.arange(x.shape[1], device=dev)[:, None] * turn.freq
        a, b = x.chunk(2, -1)
        return torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1)

    for i, (x, y) in enumerate(zip(xs, ys)):
        qkv = project(i, x.float(), w_qkv, beside[0])
        q, k, v = (t.unflatten(1, (-1, dim)).transpose(0, 1) for t in qkv.split((heads * dim, kv_heads * dim, kv_heads * dim), 1))
        k, v = (t.repeat_interleave(heads // kv_heads, 0) for t in (turned(k), v))
        q = turned(q)
        score = (q @ k.transpose(1, 2) * dim ** -0.5).masked_fill(torch.ones(len(x), len(x), device=dev).triu(1).bool(), float("-inf"))
        want = project(i, (score.softmax(-1) @ v).transpose(0, 1).flatten(1), w_o, beside[1])
        got = torch.cat(y).float()
        print(f"request {i}: {prompts[i]} + {steps} tokens, relative difference to the unquantised block "
              f"{float((got - want).norm() / want.norm()):.3f} (cache " +
              (f"blocks of {SB_KV8_BLOCK} tokens)" if args.cache == 8 else "in 4 bits)"))
    del graph
    ctx.close()


if __name__ == "__main__":
    main(sys.argv[1:])
