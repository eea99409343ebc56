"""The pages of the paged cache when sequences fork, grow, end and move together.  The front end of the C entry points of the same names
(include/fc.h says exactly what they do).

`pages` (int32 [sequences, width]) is the page table of attention.py, -1 where there is no page, `held` (int32 [sequences]) the tokens of each
sequence, `uses` (int32 [number of pages]) in how many rows a page is named; 0 is a free page.  Table and counts are common to all layers;
each layer's cache is copied by a cache_copy of its own.  One step of a server:

    pages, held = pages_fork(pages, held, uses, parents, page)               # beams choose their parents, finished sequences go (-1)
    source, target, lacking = pages_reserve(pages, held, uses, offsets, page)    # room for the step's tokens; shared pages part
    for cache in layers: cache_copy(cache, source, target)

Nothing is read on the host: every call is asynchronous on ``torch.cuda.current_stream()``, and with `out` and `workspace` given it
allocates nothing and can be captured into a HIP graph.
"""
from __future__ import annotations

from . import binding
from .attention import _cache, _index
from .binding import FcError, _check, _dev, _meet, _stream, _torch


def _table(pages, what="pages"):
    _dev(pages, _torch().int32, what)
    if pages.dim() != 2 or pages.shape[1] < 1:
        raise ValueError("%s must be int32 [sequences, width], got shape %s" % (what, tuple(pages.shape)))
    return pages.shape


def _count(uses, what="uses"):
    _dev(uses, _torch().int32, what)
    if uses.dim() != 1 or uses.shape[0] < 1:
        raise ValueError("%s must be int32 [pages], got shape %s" % (what, tuple(uses.shape)))
    return uses.shape[0]


def _results(out, shapes, like):
    """int32 tensors of these shapes: new ones, or the caller's"""
    torch = _torch()
    if out is None:
        return tuple(torch.empty(shape, dtype=torch.int32, device=like.device) for _, shape in shapes)
    out = tuple(out)
    if len(out) != len(shapes):
        raise ValueError("out must hold %s" % ", ".join(name for name, _ in shapes))
    return tuple(_index(t, name + " (out)", shape) for t, (name, shape) in zip(out, shapes))


def _apart(written, read=()):
    """no two (name, tensor) of `written` have a byte in common, and none has with one of `read`"""
    for i, (name, t) in enumerate(written):
        for other, u in (*written[:i], *read):
            if _meet(t.view(-1), u.view(-1)):
                raise ValueError("%s and %s must not overlap" % (name, other))


def _space(workspace, need, like, what):
    torch = _torch()
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=like.device)
    if _dev(workspace, torch.uint8, "workspace").numel() < need:
        raise FcError(-6, what)
    return workspace


def pages_fork(pages, held, uses, parents, page: int, out=None):
    """fc_pages_fork -> (pages, held) of the next step: row b is what row parents[b] (int32 [rows]; -1: an empty one) holds, pages reserved beyond
    that given back.  uses is brought up to date.  out: a table [rows, width] and held [rows] other than the old ones."""
    done = (binding._native or binding._calls()).pages_fork(pages, held, uses, parents, page, out)
    if done is not None:
        return done
    sequences, width = _table(pages)
    _index(held, "held", (sequences,))
    count = _count(uses)
    _dev(parents, _torch().int32, "parents")
    if parents.dim() != 1:
        raise ValueError("parents must be int32 [rows], got shape %s" % (tuple(parents.shape),))
    rows = parents.shape[0]
    table, now = _results(out, [("pages", (rows, width)), ("held", (rows,))], pages)
    if out is not None:
        _apart([("uses", uses), ("the new table", table), ("the new held", now)], [("pages", pages), ("held", held), ("parents", parents)])
    _check(binding.lib().fc_pages_fork(pages.data_ptr(), held.data_ptr(), sequences, width, page, uses.data_ptr(), count, parents.data_ptr(), rows,
                                       table.data_ptr(), now.data_ptr(), _stream()), "fc_pages_fork")
    return table, now


def pages_reserve(pages, held, uses, offsets, page: int, out=None, workspace=None):
    """fc_pages_reserve: pages for the step's tokens (offsets, held as cache_append takes them behind it), in place in pages and uses ->
    (source, target [sequences], lacking [1]): the copies that are to be made (-1: none), and how many free pages are missing, in
    which case nothing has changed."""
    done = (binding._native or binding._calls()).pages_reserve(pages, held, uses, offsets, page, out, workspace)
    if done is not None:
        return done
    sequences, width = _table(pages)
    _index(held, "held", (sequences,))
    _index(offsets, "offsets", (sequences + 1,))
    count = _count(uses)
    source, target, lacking = _results(out, [("source", (sequences,)), ("target", (sequences,)), ("lacking", (1,))], pages)
    L = binding.lib()
    given = out is not None or workspace is not None
    workspace = _space(workspace, int(L.fc_pages_reserve_workspace_bytes(count)), pages, "fc_pages_reserve")
    if given:
        _apart([("pages", pages), ("uses", uses), ("source", source), ("target", target), ("lacking", lacking), ("workspace", workspace)],
               [("held", held), ("offsets", offsets)])
    _check(L.fc_pages_reserve(pages.data_ptr(), held.data_ptr(), offsets.data_ptr(), sequences, width, page, uses.data_ptr(), count, source.data_ptr(),
                              target.data_ptr(), lacking.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream()), "fc_pages_reserve")
    return source, target, lacking


def pages_compact(pages, uses, out=None, workspace=None):
    """fc_pages_compact -> (pages, uses, source, target, used): table and counts after the pages in use have been given the lowest numbers, the
    moves for cache_copy (int32 [number of pages // 2], -1 behind the last), and how many pages are in use (int32 [1]).  out: these five;
    the table may be the old one."""
    done = (binding._native or binding._calls()).pages_compact(pages, uses, out, workspace)
    if done is not None:
        return done
    sequences, width = _table(pages)
    count = _count(uses)
    results = _results(out, [("pages", (sequences, width)), ("uses", (count,)), ("source", (count // 2,)), ("target", (count // 2,)), ("used", (1,))], pages)
    L = binding.lib()
    given = out is not None or workspace is not None
    workspace = _space(workspace, int(L.fc_pages_compact_workspace_bytes(count)), pages, "fc_pages_compact")
    if given:
        written = [*zip(("the new table", "the new counts", "source", "target", "used"), results), ("workspace", workspace)]
        _apart(written, [("uses", uses)] + ([("pages", pages)] if results[0].data_ptr() != pages.data_ptr() else []))
    _check(L.fc_pages_compact(pages.data_ptr(), sequences, width, uses.data_ptr(), count, *[t.data_ptr() for t in results], workspace.data_ptr(),
                              workspace.numel(), _stream()), "fc_pages_compact")
    return results


def cache_copy(cache, source, target):
    """fc_cache_copy: page target[i] of the cache becomes page source[i] (int32 [pairs]; -1: nothing).  No page is a target twice, or a target and a
    source.  Returns the cache."""
    done = (binding._native or binding._calls()).cache_copy(cache, source, target)
    if done is not None:
        return done
    _dev(source, _torch().int32, "source")
    if source.dim() != 1:
        raise ValueError("source must be int32 [pairs], got shape %s" % (tuple(source.shape),))
    pairs = source.shape[0]
    _index(target, "target", (pairs,))
    heads, page, dim, count = _cache(cache)
    _check(binding.lib().fc_cache_copy(cache[0].data_ptr(), cache[1].data_ptr(), cache[2].data_ptr(), cache[3].data_ptr(), count, heads, page, dim,
                                       source.data_ptr(), target.data_ptr(), pairs, _stream()), "fc_cache_copy")
    return cache
