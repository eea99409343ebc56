"""One attention layer of a tensor-parallel model as its ranks run it, with the quantized all-reduce behind it, on one GPU.

    python -m paper_2412_04964_amd.attention_block [--ranks 4] [--hidden 4096] [--query-heads 32] [--kv-heads 8] [--prompts 4] [--length 512] [--steps 16]

Each rank has its share of the query and key/value heads: its slices of the projections, and its own paged cache of 8-bit keys and
values.  A prompt step turns queries and keys to their positions, attends within the packed prompts and appends them to the
cache; a decode step turns the queries, appends one token a sequence (its keys turned on the way) and attends over the cache.
The ranks' partial outputs, a binary16 tensor each, are summed by fc.allreduce_sim, the arithmetic of the quantized all-reduce.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


class AttentionRank:
    """One rank's part of the layer: weights [hidden, heads * dim] for queries, keys and values side by side, [heads * dim, hidden] behind
    the attention, and the cache.  pages: int32 [sequences, width], the page of every `page` tokens of a sequence."""

    def __init__(self, fc, w_qkv, w_out, heads: int, group: int, dim: int, pages, page: int, quantizer: int):
        import torch
        self.fc, self.w_qkv, self.w_out, self.heads, self.group, self.dim = fc, w_qkv, w_out, heads, group, dim
        self.pages, self.quantizer = pages, quantizer
        shape = (int(pages.max()) + 1, heads, page, dim)
        self.cache = (torch.empty(shape, dtype=torch.uint8, device="cuda"), torch.empty(shape, dtype=torch.uint8, device="cuda"),
                      torch.empty(shape[:2], dtype=torch.float32, device="cuda"), torch.empty(shape[:2], dtype=torch.float32, device="cuda"))

    def _split(self, x):
        qkv = (x @ self.w_qkv).view(x.shape[0], self.heads * (self.group + 2), self.dim)
        queries = self.heads * self.group
        return qkv[:, :queries], qkv[:, queries:queries + self.heads], qkv[:, queries + self.heads:], qkv[:, :queries + self.heads]

    def prompt(self, x, table, positions, offsets, held, longest):
        """x [tokens, hidden], whole prompts of sequences that hold nothing yet -> this rank's partial output"""
        q, k, v, turned = self._split(x)
        self.fc.rotary(turned, table, positions, out=turned)
        o = self.fc.prompt_attention(q, k, v, offsets, longest)
        self.fc.cache_append(k, v, self.cache, self.pages, offsets, held, longest, self.quantizer)
        return o.view(x.shape[0], -1) @ self.w_out

    def decode(self, x, table, offsets, held, longest):
        """x [sequences, hidden], one token each at position held -> this rank's partial output; longest: tokens that a sequence holds, with
        the new one"""
        q, k, v, _ = self._split(x)
        self.fc.rotary(q, table, held, out=q)
        self.fc.cache_append(k, v, self.cache, self.pages, offsets, held, 1, self.quantizer, table)
        o = self.fc.cache_attention(q, self.cache, self.pages, offsets, held, 1, longest, self.quantizer)
        return o.view(x.shape[0], -1) @ self.w_out


def random_layer(hidden, query_heads, kv_heads, dim, ranks, seed=0):
    """w_qkv, w_out of every rank: float16, of a variance that keeps activations at one"""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    heads, group = kv_heads // ranks, query_heads // kv_heads
    make = lambda a, b, n: (torch.randn((a, b), generator=g, device="cuda") * n ** -0.5).half()     # noqa: E731
    return [(make(hidden, heads * (group + 2) * dim, hidden), make(heads * group * dim, hidden, query_heads * dim)) for _ in range(ranks)]


def exact_layer(fc, layer, xs, lengths, table, heads, group, dim):
    """The same layer in float32 without a cache, codes or a quantized sum: every sequence's tokens xs[b] [tokens, hidden] at once"""
    import torch
    out = []
    for x in xs:
        n, total = x.shape[0], 0
        rows = table[:n]
        c, s = rows[:, None, :dim // 2], rows[:, None, dim // 2:]
        for w_qkv, w_out in layer:
            qkv = (x.float() @ w_qkv.float()).view(n, heads * (group + 2), dim)
            turned, v = qkv[:, :heads * (group + 1)], qkv[:, heads * (group + 1):]
            a, b = turned[..., :dim // 2], turned[..., dim // 2:]
            turned = torch.cat([a * c - b * s, b * c + a * s], -1).transpose(0, 1)
            q, k = turned[:heads * group], turned[heads * group:].repeat_interleave(group, 0)
            w = q @ k.transpose(1, 2).contiguous() * dim ** -0.5
            w = torch.softmax(w.masked_fill(~torch.ones((n, n), dtype=torch.bool, device="cuda").tril(), float("-inf")), -1)
            o = (w @ v.transpose(0, 1).repeat_interleave(group, 0)).transpose(0, 1).reshape(n, -1)
            total = total + o @ w_out.float()
        out.append(total)
    return out


def run(ranks=4, hidden=4096, query_heads=32, kv_heads=8, dim=128, prompts=4, length=512, steps=16, page=16, quantizer=None, bits=8, seed=0):
    """Runs prompts of uneven lengths and `steps` decode steps; returns the relative errors (2-norm) of the prompts' outputs and of each step's
    against the layer in float32, and the milliseconds of the prompt step and of a decode step."""
    import torch

    import paper_2412_04964_amd as fc
    if kv_heads % ranks or query_heads % kv_heads:
        raise ValueError("ranks must divide the key/value heads, and those the query heads")
    quantizer = fc.QUANTIZER_SYM if quantizer is None else quantizer
    heads, group = kv_heads // ranks, query_heads // kv_heads
    lengths = [max(1, length - 37 * b) for b in range(prompts)]
    width = -(-(max(lengths) + steps) // page)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    pages = torch.randperm(prompts * width, generator=g, device="cuda").to(torch.int32).view(prompts, width)
    table = fc.rotary_table(width * page, fc.rotary_frequencies(dim))
    layer = random_layer(hidden, query_heads, kv_heads, dim, ranks, seed)
    members = [AttentionRank(fc, *w, heads, group, dim, pages, page, quantizer) for w in layer]
    xs = [torch.randn((n + steps, hidden), generator=g, device="cuda").half() for n in lengths]
    want = exact_layer(fc, layer, xs, lengths, table, heads, group, dim)
    group_size = 128

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def timed(call):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        result = call()
        end.record()
        end.synchronize()
        return result, begin.elapsed_time(end)

    def error(got, wanted):
        return float((got.float() - wanted).norm() / wanted.norm())

    starts = [0]
    for n in lengths:
        starts.append(starts[-1] + n)
    x = torch.cat([t[:n] for t, n in zip(xs, lengths)])
    positions = torch.cat([torch.arange(n, dtype=torch.int32, device="cuda") for n in lengths])
    offsets, held = ints(starts), ints([0] * prompts)

    def whole_prompts():
        return fc.allreduce_sim(torch.stack([m.prompt(x, table, positions, offsets, held, max(lengths)) for m in members]), group_size, bits, bits)

    y, prompt_ms = timed(whole_prompts)
    errors = [error(y, torch.cat([w[:n] for w, n in zip(want, lengths)]))]
    offsets, held, step_ms = ints(list(range(prompts + 1))), ints(lengths), []
    for i in range(steps):
        x = torch.stack([t[n + i] for t, n in zip(xs, lengths)])
        y, ms = timed(lambda: fc.allreduce_sim(torch.stack([m.decode(x, table, offsets, held, max(lengths) + i + 1) for m in members]), group_size, bits, bits))
        errors.append(error(y, torch.stack([w[n + i] for w, n in zip(want, lengths)])))
        step_ms.append(ms)
        held += 1
    return errors, prompt_ms, sorted(step_ms)[len(step_ms) // 2] if step_ms else 0.0


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("ranks", 4), ("hidden", 4096), ("query-heads", 32), ("kv-heads", 8), ("prompts", 4), ("length", 512), ("steps", 16)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    import paper_2412_04964_amd as fc
    run(a.ranks, a.hidden, a.query_heads, a.kv_heads, prompts=a.prompts, length=a.length, steps=1)       # libraries and memory
    for name, quantizer in (("INT8", fc.QUANTIZER_SYM), ("E4M3", fc.QUANTIZER_FP8)):
        errors, prompt_ms, step_ms = run(a.ranks, a.hidden, a.query_heads, a.kv_heads, prompts=a.prompts, length=a.length, steps=a.steps, quantizer=quantizer)
        print("%s cache, INT8 all-reduce: prompts %.2f ms, error %.4f; decode step %.3f ms, error %.4f at most"
              % (name, prompt_ms, errors[0], step_ms, max(errors[1:], default=0.0)))


if __name__ == "__main__":
    main()
