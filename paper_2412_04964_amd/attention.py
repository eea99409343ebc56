"""Attention of a tensor-parallel rank: rotary positions, the paged cache of keys and values in 8-bit codes, attention over that
cache and over whole prompts.  The front end of the C entry points of the same names (include/fc.h has the formulas).

Activations are float16 or bfloat16 tensors [tokens, heads, dim] whose last axis is dense; the other two may have any strides that are
multiples of 8 elements, so slices of a joint projection are taken as they are.  A batch's sequences are packed one behind the
other: `offsets` (int32 [sequences + 1]) says where each one's tokens of this call begin, `held` (int32 [sequences]) how many it
held before.  A cache is a tuple (k_cache, v_cache, k_scales, v_scales): codes uint8 [pages, heads, page, dim], float32 [pages, heads];
`pages` (int32 [sequences, width]) names the page of each `page` tokens of a sequence.

Every call is asynchronous on ``torch.cuda.current_stream()``, reads no device value on the host and can be captured into a HIP graph;
with `out` (and `workspace`) given it allocates nothing.  Serving only: no call records a gradient (``rotary(..., inverse=True)`` is
the rotation's), so activations that require one are refused unless gradients are off (``torch.no_grad()``).
"""
from __future__ import annotations

import math

from . import binding
from .binding import QUANTIZER_SYM, FcError, _check, _dev, _meet, _shape, _stream, _torch

_TYPES = None


def _type(t, what):
    global _TYPES
    if _TYPES is None:
        torch = _torch()
        _TYPES = {torch.float16: 0, torch.bfloat16: 1}
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError("%s must be float16 or bfloat16, got %s" % (what, t.dtype))
    return code


def _strides(t):
    """(token stride, head stride) in elements; an axis of one element has none"""
    return (t.stride(0) if t.shape[0] > 1 else 0), (t.stride(1) if t.shape[1] > 1 else 0)


def _rows(t, what, dtype=None, shape=None):
    """a [tokens, heads, dim] activation on the current device, in 128-bit units"""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor; this library has no CPU path" % what)
    if dtype is None:
        _type(t, what)
    elif t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (what, dtype, t.dtype))
    if t.dim() != 3:
        raise ValueError("%s must be [tokens, heads, dim], got shape %s" % (what, tuple(t.shape)))
    if shape is not None:
        _shape(t, shape, what)
    if t.device.index != torch.cuda.current_device():
        raise ValueError("%s lives on %s but the current device is cuda:%d; the C ABI works on the current device"
                         % (what, t.device, torch.cuda.current_device()))
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError("%s requires a gradient, which no attention call records: call it under torch.no_grad(), or on %s.detach()" % (what, what))
    if t.numel() and (t.stride(2) != 1 or any(s % 8 for s in _strides(t)) or t.data_ptr() % 16):
        raise ValueError("%s must have a dense last axis, other strides that are multiples of 8 elements and a 16-byte aligned "
                         "start, got strides %s" % (what, tuple(t.stride())))
    return t


def _out_rows(out, like, shape, what="out"):
    torch = _torch()
    if out is None:
        return torch.empty(shape, dtype=like.dtype, device=like.device)
    _rows(out, what, like.dtype, shape)
    (small, n), (large, _) = _axes(out)
    if out.numel() and (small < out.shape[2] or large < small * (n - 1) + out.shape[2]):
        raise ValueError("%s must not overlap itself, got strides %s" % (what, tuple(out.stride())))
    return out


def _axes(t):
    """((smaller stride, its length), (larger stride, its length)) of the first two axes; one element: no stride to speak of"""
    far = 1 << 62
    return sorted((t.stride(i) if t.shape[i] > 1 else far, t.shape[i]) for i in (0, 1))


def _index(t, what, shape):
    return _shape(_dev(t, _torch().int32, what), shape, what)


def _step(offsets, held=None):
    """the number of sequences of a call's index arrays"""
    _dev(offsets, _torch().int32, "offsets")
    if offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("offsets must be int32 [sequences + 1], got shape %s" % (tuple(offsets.shape),))
    n = offsets.shape[0] - 1
    if held is not None:
        _index(held, "held", (n,))
    return n


def _cache(cache, pages=None, sequences=0):
    """(heads, page, dim, number of pages) of a checked cache, and the width of its page table if there is one"""
    torch = _torch()
    if len(cache) != 4:
        raise ValueError("cache must hold k_cache, v_cache, k_scales and v_scales")
    k, v, ks, vs = cache
    _dev(k, torch.uint8, "k_cache")
    if k.dim() != 4:
        raise ValueError("k_cache must be [pages, heads, page, dim], got shape %s" % (tuple(k.shape),))
    _shape(_dev(v, torch.uint8, "v_cache"), k.shape, "v_cache")
    _shape(_dev(ks, torch.float32, "k_scales"), k.shape[:2], "k_scales")
    _shape(_dev(vs, torch.float32, "v_scales"), k.shape[:2], "v_scales")
    if pages is None:
        return k.shape[1], k.shape[2], k.shape[3], k.shape[0]
    _dev(pages, torch.int32, "pages")
    if pages.dim() != 2:
        raise ValueError("pages must be int32 [sequences, width], got shape %s" % (tuple(pages.shape),))
    _shape(pages, (sequences, pages.shape[1]), "pages")
    return k.shape[1], k.shape[2], k.shape[3], k.shape[0], pages.shape[1]


def rotary_frequencies(rotary: int, base: float = 10000.0, method: str = "none", factor: float = 1.0, original: int = 0,
                       low: float = 1.0, high: float = 4.0):
    """float64 [rotary / 2] on the host: the angles by which a pair turns per position, base^(-2 i / rotary), for contexts `factor`
    times as long as trained:
      "linear"  every frequency divided by factor (position interpolation: Chen et al. 2023, arXiv 2306.15595)
      "base"    base times factor^(rotary / (rotary - 2)): the slowest pair gets factor, the fastest none (NTK-aware scaling, as
                described by Peng et al. 2023, arXiv 2309.00071)
      "bands"   pairs with at most `low` turns in the `original` context divided by factor, those with `high` and more unchanged,
                in between by a mix that is linear in the number of turns (NTK-by-parts, the same paper)
      "ramp"    the same with a mix that is linear in the pair's index, between the indices where a pair has `high` and `low` turns
                (rounded outwards, as published models compute it); goes with a magnitude of 0.1 ln(factor) + 1 (YaRN, the same paper)
    Checked against these formulas, not against another implementation's output."""
    torch = _torch()
    if rotary < 2 or rotary % 2 or factor <= 0 or base <= 1:
        raise ValueError("rotary must be even and positive, factor positive and base above 1")
    if method == "base":
        if rotary == 2:
            raise ValueError("the base of a single pair has no effect")
        base = base * factor ** (rotary / (rotary - 2))
    f = base ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)
    if method in ("none", "base"):
        return f
    if method == "linear":
        return f / factor
    if method not in ("bands", "ramp"):
        raise ValueError("method must be none, linear, base, bands or ramp, got %r" % (method,))
    if original < 1 or not 0 < low < high:
        raise ValueError("%s needs the original context and 0 < low < high" % method)
    if method == "bands":
        keep = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
    else:
        def index(turns):
            return rotary * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        first, last = max(math.floor(index(high)), 0), min(math.ceil(index(low)), rotary - 1)
        keep = 1 - ((torch.arange(rotary // 2, dtype=torch.float64) - first) / max(last - first, 1e-3)).clamp(0, 1)
    return f * keep + f / factor * (1 - keep)


def rotary_table(rows: int, frequencies, magnitude: float = 1.0, out=None):
    """fc_rotary_table -> float32 [rows, rotary]: cosines of every pair's angle, then sines, times magnitude.  frequencies:
    float64 [rotary / 2] (rotary_frequencies), on either side."""
    torch = _torch()
    if not isinstance(frequencies, torch.Tensor) or frequencies.dtype != torch.float64 or frequencies.dim() != 1:
        raise TypeError("frequencies must be a float64 tensor [rotary / 2]")
    f = _dev(frequencies.to(device="cuda" if not frequencies.is_cuda else None).contiguous(), torch.float64, "frequencies")
    rotary = 2 * f.shape[0]
    if rows < 0 or rotary == 0:
        raise FcError(-4, "fc_rotary_table")
    if out is None:
        out = torch.empty((rows, rotary), dtype=torch.float32, device=f.device)
    _shape(_dev(out, torch.float32, "table (out)"), (rows, rotary), "table (out)")
    _check(binding.lib().fc_rotary_table(f.data_ptr(), rows, rotary, magnitude, out.data_ptr(), _stream()), "fc_rotary_table")
    return out


def _table(table):
    """(address, rows, rotary) of a rotation table"""
    _dev(table, _torch().float32, "table")
    if table.dim() != 2:
        raise ValueError("table must be float32 [rows, rotary], got shape %s" % (tuple(table.shape),))
    return table.data_ptr(), table.shape[0], table.shape[1]


def rotary(x, table, positions, interleaved: bool = False, inverse: bool = False, out=None):
    """fc_rotary.  x [tokens, heads, dim] with the first table.shape[1] elements of each head turned to positions (int32 [tokens]);
    out=x turns in place."""
    done = (binding._native or binding._calls()).rotary(x, table, positions, interleaved, inverse, out)
    if done is not None:
        return done
    _rows(x, "x")
    address, rows, turned = _table(table)
    tokens, heads, dim = x.shape
    _index(positions, "positions", (tokens,))
    y = _out_rows(out, x, tuple(x.shape))
    _check(binding.lib().fc_rotary(x.data_ptr(), *_strides(x), address, rows, positions.data_ptr(), tokens, heads, dim, turned,
                                   int(interleaved), int(inverse), _type(x, "x"), y.data_ptr(), *_strides(y), _stream()), "fc_rotary")
    return y


def cache_append(k, v, cache, pages, offsets, held, longest: int, quantizer: int = QUANTIZER_SYM, table=None,
                 interleaved: bool = False):
    """fc_cache_append: puts k, v [tokens, heads, dim] behind the tokens that each sequence holds, keys turned to their positions on
    the way if a rotation table is given.  longest: no sequence gets more tokens.  Returns the cache."""
    done = (binding._native or binding._calls()).cache_append(k, v, cache, pages, offsets, held, longest, quantizer, table, interleaved)
    if done is not None:
        return done
    _rows(k, "k")
    _rows(v, "v", k.dtype, tuple(k.shape))
    sequences = _step(offsets, held)
    heads, page, dim, count, width = _cache(cache, pages, sequences)
    tokens = k.shape[0]
    _shape(k, (tokens, heads, dim), "k")
    address, rows, turned = _table(table) if table is not None else (None, 0, 0)
    _check(binding.lib().fc_cache_append(
        k.data_ptr(), *_strides(k), v.data_ptr(), *_strides(v), tokens, heads, dim, _type(k, "k"), address, rows, turned,
        int(interleaved), quantizer, cache[0].data_ptr(), cache[1].data_ptr(), cache[2].data_ptr(), cache[3].data_ptr(), count, page,
        pages.data_ptr(), width, offsets.data_ptr(), held.data_ptr(), sequences, longest, _stream()), "fc_cache_append")
    return cache


def cache_attention_workspace_bytes(tokens: int, sequences: int, heads: int, group: int, dim: int, queries: int, longest: int) -> int:
    return int(binding.lib().fc_cache_attention_workspace_bytes(tokens, sequences, heads, group, dim, queries, longest))


def _group(q, heads, what):
    if heads < 1 or q.shape[1] < 1 or q.shape[1] % heads:
        raise ValueError("q has %d heads, which %s's %d key/value heads do not divide" % (q.shape[1], what, heads))
    return q.shape[1] // heads


def cache_attention(q, cache, pages, offsets, held, queries: int, longest: int, quantizer: int = QUANTIZER_SYM, scale=None,
                    out=None, workspace=None):
    """fc_cache_attention: q [tokens, query heads, dim] over the cache that cache_append has put the same step's tokens into; query i
    of a sequence sees its first held + i + 1 tokens.  queries and longest: the most new tokens, and the most in all, that a
    sequence has.  scale: dim^-0.5 unless given."""
    done = (binding._native or binding._calls()).cache_attention(q, cache, pages, offsets, held, queries, longest, quantizer, scale, out, workspace)
    if done is not None:
        return done
    torch = _torch()
    _rows(q, "q")
    sequences = _step(offsets, held)
    heads, page, dim, count, width = _cache(cache, pages, sequences)
    tokens = q.shape[0]
    _shape(q, (tokens, q.shape[1], dim), "q")
    group = _group(q, heads, "cache")
    y = _out_rows(out, q, tuple(q.shape))
    need = cache_attention_workspace_bytes(tokens, sequences, heads, group, dim, queries, longest)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    _dev(workspace, torch.uint8, "workspace")
    if workspace.numel() < need:
        raise FcError(-6, "fc_cache_attention")
    _check(binding.lib().fc_cache_attention(
        q.data_ptr(), *_strides(q), tokens, heads, group, dim, _type(q, "q"), quantizer, cache[0].data_ptr(), cache[1].data_ptr(),
        cache[2].data_ptr(), cache[3].data_ptr(), count, page, pages.data_ptr(), width, offsets.data_ptr(), held.data_ptr(), sequences,
        queries, longest, dim ** -0.5 if scale is None else scale, y.data_ptr(), *_strides(y), workspace.data_ptr(), workspace.numel(),
        _stream()), "fc_cache_attention")
    return y


def prompt_attention(q, k, v, offsets, longest: int, causal: bool = True, scale=None, out=None):
    """fc_prompt_attention: every sequence of the packed q [tokens, query heads, dim], k, v [tokens, heads, dim] attends to itself.
    longest: no sequence has more tokens.  scale: dim^-0.5 unless given."""
    done = (binding._native or binding._calls()).prompt_attention(q, k, v, offsets, longest, causal, scale, out)
    if done is not None:
        return done
    _rows(q, "q")
    _rows(k, "k", q.dtype)
    _rows(v, "v", q.dtype, tuple(k.shape))
    sequences = _step(offsets)
    tokens, heads, dim = k.shape
    _shape(q, (tokens, q.shape[1], dim), "q")
    group = _group(q, heads, "k")
    y = _out_rows(out, q, tuple(q.shape))
    _check(binding.lib().fc_prompt_attention(
        q.data_ptr(), *_strides(q), k.data_ptr(), *_strides(k), v.data_ptr(), *_strides(v), tokens, heads, group, dim, _type(q, "q"),
        offsets.data_ptr(), sequences, longest, int(causal), dim ** -0.5 if scale is None else scale, y.data_ptr(), *_strides(y),
        _stream()), "fc_prompt_attention")
    return y


def chunk_attention_workspace_bytes(tokens: int, sequences: int, heads: int, group: int, dim: int, longest: int) -> int:
    return int(binding.lib().fc_chunk_attention_workspace_bytes(tokens, sequences, heads, group, dim, longest))


def chunk_attention(q, k, v, cache, pages, offsets, held, longest: int, quantizer: int = QUANTIZER_SYM, scale=None, out=None, workspace=None):
    """fc_chunk_attention: a prompt that is taken in pieces.  q [tokens, query heads, dim] over the held tokens of every sequence in the cache and
    over the new ones up to itself, whose k, v [tokens, heads, dim] (keys turned) need not be in the cache.  longest: the most tokens,
    held and new, that a sequence has.  scale: dim^-0.5 unless given.  out may be q, row for row; what overlaps otherwise is refused."""
    done = (binding._native or binding._calls()).chunk_attention(q, k, v, cache, pages, offsets, held, longest, quantizer, scale, out, workspace)
    if done is not None:
        return done
    torch = _torch()
    _rows(q, "q")
    _rows(k, "k", q.dtype)
    _rows(v, "v", q.dtype, tuple(k.shape))
    sequences = _step(offsets, held)
    heads, page, dim, count, width = _cache(cache, pages, sequences)
    tokens = q.shape[0]
    _shape(q, (tokens, q.shape[1], dim), "q")
    _shape(k, (tokens, heads, dim), "k")
    group = _group(q, heads, "cache")
    y = _out_rows(out, q, tuple(q.shape))
    need = chunk_attention_workspace_bytes(tokens, sequences, heads, group, dim, longest)
    dense = zip(("k_cache", "v_cache", "k_scales", "v_scales", "pages", "offsets", "held"), (*cache, pages, offsets, held))
    read = [("q", q), ("k", k), ("v", v)] + [(name, t.view(-1)) for name, t in dense]
    for name, t in read if out is not None else ():
        if _meet(y, t) and not (name == "q" and y.data_ptr() == q.data_ptr() and _strides(y) == _strides(q)):
            raise ValueError("out must not overlap %s%s" % (name, ", unless it has the same rows" if name == "q" else ""))
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    elif _dev(workspace, torch.uint8, "workspace").numel() < need:
        raise FcError(-6, "fc_chunk_attention")
    else:
        for name, t in read + [("out", y)]:
            if _meet(workspace.view(-1), t):
                raise ValueError("workspace must not overlap %s" % name)
    _check(binding.lib().fc_chunk_attention(
        q.data_ptr(), *_strides(q), k.data_ptr(), *_strides(k), v.data_ptr(), *_strides(v), tokens, heads, group, dim, _type(q, "q"), quantizer,
        cache[0].data_ptr(), cache[1].data_ptr(), cache[2].data_ptr(), cache[3].data_ptr(), count, page, pages.data_ptr(), width,
        offsets.data_ptr(), held.data_ptr(), sequences, longest, dim ** -0.5 if scale is None else scale, y.data_ptr(), *_strides(y),
        workspace.data_ptr(), workspace.numel(), _stream()), "fc_chunk_attention")
    return y
