"""Attention layers of a tensor-parallel model as its ranks run them, with the quantized all-reduce behind each, on one GPU.

    python -m paper_2412_04964_amd.attention_block [--ranks 4] [--hidden 4096] [--query-heads 32] [--kv-heads 8] [--prompts 4] [--length 512] [--steps 16]
                                                   [--piece 0] [--samples 1] [--layers 1]

Each rank has its share of the query and key/value heads: its slices of the projections, and its own paged cache of 8-bit keys and
values.  A prompt step turns queries and keys to their positions, attends within the packed prompts and appends them to the
cache; a decode step turns the queries, appends one token a sequence (its keys turned on the way) and attends over the cache.
The ranks' partial outputs, a binary16 tensor each, are summed by fc.allreduce_sim, the arithmetic of the quantized all-reduce.

--piece N takes the prompts N tokens of each at a time: a piece attends over what its sequence has in the cache and over itself.
--samples N continues every prompt N times: its continuations share its pages until they write to them.  With either the pages come from
a pool as they are needed, and half way through the decode steps those in use move together.
--layers N: a further layer's input is the norm of the sum of all that is behind it.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


class AttentionRank:
    """One rank's part of the layer: weights [hidden, heads * dim] for queries, keys and values side by side, [heads * dim, hidden] behind
    the attention, and the cache.  pages: int32 [sequences, width], the page of every `page` tokens of a sequence; pool: pages of the cache,
    those that it names unless given."""

    def __init__(self, fc, w_qkv, w_out, heads: int, group: int, dim: int, pages, page: int, quantizer: int, pool: int = 0):
        import torch
        self.fc, self.w_qkv, self.w_out, self.heads, self.group, self.dim = fc, w_qkv, w_out, heads, group, dim
        self.pages, self.quantizer = pages, quantizer
        shape = (pool or int(pages.max()) + 1, heads, page, dim)
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

    def piece(self, x, table, positions, offsets, held, most, longest):
        """x [tokens, hidden], pieces of prompts of at most `most` tokens whose sequences hold what was before them -> this rank's partial output;
        longest: tokens that a sequence holds, with the new ones"""
        q, k, v, turned = self._split(x)
        self.fc.rotary(turned, table, positions, out=turned)
        o = self.fc.chunk_attention(q, k, v, self.cache, self.pages, offsets, held, longest, self.quantizer)
        self.fc.cache_append(k, v, self.cache, self.pages, offsets, held, most, self.quantizer)
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


def exact_stack(fc, layers, norms, xs, lengths, table, heads, group, dim):
    """exact_layer through all layers -> the last one's output"""
    out = exact_layer(fc, layers[0], xs, lengths, table, heads, group, dim)
    before = [x.float() for x in xs]
    for layer, w in zip(layers[1:], norms):
        before = [a + b for a, b in zip(before, out)]
        out = exact_layer(fc, layer, [a * (a.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w.float() for a in before], lengths, table, heads, group, dim)
    return out


def run(ranks=4, hidden=4096, query_heads=32, kv_heads=8, dim=128, prompts=4, length=512, steps=16, page=16, quantizer=None, bits=8, seed=0, piece=0,
        samples=1, layers=1):
    """Runs prompts of uneven lengths and `steps` decode steps; returns the relative errors (2-norm) of the prompts' outputs (of each piece's, where
    they come in pieces) and of each step's against the layers in float32, and the milliseconds of all prompts and of a decode step."""
    import torch

    import paper_2412_04964_amd as fc
    if kv_heads % ranks or query_heads % kv_heads:
        raise ValueError("ranks must divide the key/value heads, and those the query heads")
    if piece < 0 or samples < 1 or layers < 1:
        raise ValueError("a piece has no negative length, and there are one sample and one layer at least")
    quantizer = fc.QUANTIZER_SYM if quantizer is None else quantizer
    heads, group = kv_heads // ranks, query_heads // kv_heads
    lengths = [max(1, length - 37 * b) for b in range(prompts)]
    width = -(-(max(lengths) + steps) // page)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    pages = torch.randperm(prompts * width, generator=g, device="cuda").to(torch.int32).view(prompts, width)
    table = fc.rotary_table(width * page, fc.rotary_frequencies(dim))
    pooled, pool = piece > 0 or samples > 1, 0
    if pooled:
        pool = prompts * samples * width
        pages = torch.full((prompts, width), -1, dtype=torch.int32, device="cuda")
        uses = torch.zeros(pool, dtype=torch.int32, device="cuda")
    weights = [random_layer(hidden, query_heads, kv_heads, dim, ranks, seed + 17 * i) for i in range(layers)]
    stack = [[AttentionRank(fc, *w, heads, group, dim, pages, page, quantizer, pool) for w in layer] for layer in weights]
    xs = [torch.randn((n + steps, hidden), generator=g, device="cuda").half() for n in lengths]
    norms = [(1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).half() for _ in range(layers - 1)]
    # every prompt's samples, which begin with it and go on with tokens of their own
    xs = [x if i == 0 else torch.cat([x[:n], torch.randn((steps, hidden), generator=g, device="cuda").half()]) for x, n in zip(xs, lengths) for i in range(samples)]
    want = exact_stack(fc, weights, norms, xs, lengths, table, heads, group, dim)
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

    def through(x, call):
        """x through all layers; call: what a rank does with it"""
        before = x
        for i, members in enumerate(stack):
            if i:
                x, before = fc.rms_norm(y, norms[i - 1], residual=before)
            y = fc.allreduce_sim(torch.stack([call(m, x) for m in members]), group_size, bits, bits)
        return y

    lacking = []

    def room(offsets, held):
        """pages for the step's tokens, and the copies of those that others go on to read"""
        if not pooled:
            return
        source, target, lack = fc.pages_reserve(pages, held, uses, offsets, page)
        lacking.append(lack)
        copied(source, target)

    def copied(source, target):
        for members in stack:
            for m in members:
                m.pages = pages
                fc.cache_copy(m.cache, source, target)

    def step_of(begins, ends):
        """tokens begins[b]:ends[b] of the prompts: x, positions, offsets, held, and what they should become"""
        starts = [0]
        for b, e in zip(begins, ends):
            starts.append(starts[-1] + e - b)
        positions = torch.cat([torch.arange(b, e, dtype=torch.int32, device="cuda") for b, e in zip(begins, ends)])
        return (torch.cat([t[b:e] for t, b, e in zip(xs[::samples], begins, ends)]), positions, ints(starts), ints(begins),
                torch.cat([w[b:e] for w, b, e in zip(want[::samples], begins, ends)]))

    errors, prompt_ms, begins = [], 0.0, [0] * prompts
    while begins != lengths:
        ends = [min(b + (piece or n), n) for b, n in zip(begins, lengths)]
        x, positions, offsets, held, wanted = step_of(begins, ends)
        most, longest = max(e - b for b, e in zip(begins, ends)), max(ends)

        def taken():
            room(offsets, held)
            if piece:
                return through(x, lambda m, x: m.piece(x, table, positions, offsets, held, most, longest))
            return through(x, lambda m, x: m.prompt(x, table, positions, offsets, held, longest))

        y, ms = timed(taken)
        errors.append(error(y, wanted))
        prompt_ms += ms
        begins = ends
    held = ints(lengths)
    lengths = [n for n in lengths for _ in range(samples)]
    if pooled:
        pages, held = fc.pages_fork(pages, held, uses, ints([b for b in range(prompts) for _ in range(samples)]), page)
    offsets, step_ms = ints(list(range(prompts * samples + 1))), []
    for i in range(steps):
        x = torch.stack([t[n + i] for t, n in zip(xs, lengths)])

        def stepped():
            room(offsets, held)
            return through(x, lambda m, x: m.decode(x, table, offsets, held, max(lengths) + i + 1))

        y, ms = timed(stepped)
        errors.append(error(y, torch.stack([w[n + i] for w, n in zip(want, lengths)])))
        step_ms.append(ms)
        held += 1
        if pooled and i == steps // 2:
            pages, uses, source, target, _ = fc.pages_compact(pages, uses)
            copied(source, target)
    if any(int(lack) for lack in lacking):
        raise RuntimeError("the pool of %d pages was too small" % pool)
    return errors, prompt_ms, sorted(step_ms)[len(step_ms) // 2] if step_ms else 0.0


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("ranks", 4), ("hidden", 4096), ("query-heads", 32), ("kv-heads", 8), ("prompts", 4), ("length", 512), ("steps", 16),
                        ("piece", 0), ("samples", 1), ("layers", 1)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    import paper_2412_04964_amd as fc
    more = dict(prompts=a.prompts, length=a.length, piece=a.piece, samples=a.samples, layers=a.layers)
    run(a.ranks, a.hidden, a.query_heads, a.kv_heads, steps=1, **more)       # libraries and memory
    for name, quantizer in (("INT8", fc.QUANTIZER_SYM), ("E4M3", fc.QUANTIZER_FP8)):
        errors, prompt_ms, step_ms = run(a.ranks, a.hidden, a.query_heads, a.kv_heads, steps=a.steps, quantizer=quantizer, **more)
        print("%s cache, INT8 all-reduce: prompts %.2f ms, error %.4f; decode step %.3f ms, error %.4f at most"
              % (name, prompt_ms, max(errors[:len(errors) - a.steps]), step_ms, max(errors[len(errors) - a.steps:], default=0.0)))


if __name__ == "__main__":
    main()
