"""More operators of one rank of a tensor-parallel model that serves requests: attention of a chunk of new tokens over the paged
8-bit cache, the cache's pages when sequences fork, grow and end, and the norm behind an all-reduce.

`run` is the plain form (elementary torch operations in 32 bits, the norm's sums in 64) or, where `own` is true, the framework's
kernels.  Head counts and hidden sizes are those of perf/operators.py: heads of 128, 32 query and 8 key/value heads for hidden 4096,
64 and 8 for 8192, 40 and 40 for 5120, alone or over 4 ranks.
"""
import math
import random

import torch

own = False

FLT_MIN = 1.1754943508222875e-38
LARGEST = {"int8": 127.0, "fp8": 448.0}
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5


# ---- cases ----

def listed():
    return [
        # a short turn of a chat whose earlier turns are cached: a rank of hidden 4096 over 4, latency
        dict(name="chunk turn", op="chunk", sequences=1, tokens=17, kv_heads=2, group=4, dim=128, page=16, context=129, code="int8", type="f16", ragged=1),
        # the usual step of a prompt that is taken in pieces: 512 tokens behind 8191, rank of hidden 8192 over 4
        dict(name="chunk usual", op="chunk", sequences=1, tokens=512, kv_heads=2, group=8, dim=128, page=16, context=8191, code="fp8", type="bf16", ragged=2),
        # prompts of several requests that continue, of uneven lengths, some without a cache; all heads of hidden 4096
        dict(name="chunk batch", op="chunk", sequences=9, tokens=4099, kv_heads=8, group=4, dim=128, page=64, context=4000, code="int8", type="f16", ragged=3),
        # a piece of a long document behind much of it, rank of hidden 8192 over 4
        dict(name="chunk long document", op="chunk", sequences=1, tokens=2048, kv_heads=2, group=8, dim=128, page=32, context=65531, code="fp8", type="bf16", ragged=4),
        # one decode step of a few beams: they choose their parents, get pages for a token, copy the pages that they share
        dict(name="fork few beams", op="fork", groups=1, beams=4, kv_heads=2, dim=128, page=16, context=300, new=1, code="int8", ragged=5),
        # the same for many requests with several drafted tokens, all heads of hidden 4096
        dict(name="fork many beams", op="fork", groups=60, beams=4, kv_heads=8, dim=128, page=32, context=4095, new=5, code="fp8", ragged=6),
        # a small pool after most sequences have ended
        dict(name="compact small pool", op="compact", pages=257, sequences=4, kv_heads=2, dim=128, page=16, used=0.4, code="int8", ragged=7),
        # a large pool, half of it in use, all heads of hidden 4096
        dict(name="compact large pool", op="compact", pages=20011, sequences=61, kv_heads=8, dim=128, page=16, used=0.5, code="fp8", ragged=8),
        # behind the all-reduce of a decode step of 8 requests, hidden 8192
        dict(name="norm decode", op="norm", tokens=8, hidden=8192, group=0, residual=True, code="", type="bf16"),
        # the same for one request, hidden 4096, with codes of 128 values for what follows
        dict(name="norm decode codes", op="norm", tokens=1, hidden=4096, group=128, residual=True, code="int8", type="f16"),
        # behind the all-reduce of prompts, hidden 8192
        dict(name="norm prompt", op="norm", tokens=8192, hidden=8192, group=0, residual=True, code="", type="f16"),
        # prompts of hidden 5120, odd number of tokens, one scale a token
        dict(name="norm prompt codes", op="norm", tokens=16383, hidden=5120, group=5120, residual=True, code="fp8", type="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["chunk", "chunk", "fork", "compact", "norm"])
    ragged = rng.randrange(1000, 1000000)
    if op == "chunk":
        heads, group = rng.choice([(1, 8), (2, 4), (2, 8), (8, 4), (8, 8), (10, 1), (40, 1), (1, 5), (2, 16)])
        tokens = _log(rng, 2, 4099)
        most = min(65531, 2048 * 65531 * 16 // (tokens * heads * group))
        return dict(op=op, sequences=_log(rng, 1, min(16, tokens)), tokens=tokens, kv_heads=heads, group=group, dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64]),
                    context=_log(rng, 1, most), code=rng.choice(["int8", "fp8"]), type=rng.choice(["f16", "bf16"]), ragged=ragged)
    if op == "fork":
        groups, beams = _log(rng, 1, 60), rng.choice([1, 2, 3, 4, 8])
        heads = rng.choice([1, 2, 8, 10])
        context = _log(rng, 3, max(3, min(4095, 60 * 4 * 4095 * 8 // (groups * beams * heads))))
        return dict(op=op, groups=groups, beams=beams, kv_heads=heads, dim=rng.choice([64, 128, 256]), page=rng.choice([16, 32, 64]), context=context,
                    new=rng.choice([1, 1, 2, 5, 37]), code=rng.choice(["int8", "fp8"]), ragged=ragged)
    if op == "compact":
        heads, page, dim = rng.choice([1, 2, 8, 10]), rng.choice([16, 32, 64]), rng.choice([64, 128, 256])
        pages = _log(rng, 8, max(8, min(100000, 20011 * 8 * 16 * 128 // (heads * page * dim))))
        return dict(op=op, pages=pages, sequences=_log(rng, 1, min(61, pages // 4 + 1)), kv_heads=heads, dim=dim, page=page, used=rng.choice([0.1, 0.4, 0.5, 0.9]),
                    code=rng.choice(["int8", "fp8"]), ragged=ragged)
    hidden = rng.choice([512, 1024, 2048, 4096, 5120, 8192, 16384])
    code = rng.choice(["", "int8", "fp8"])
    group = rng.choice([32, 64, 128, 256, 512, hidden]) if code else 0
    return dict(op=op, tokens=_log(rng, 1, min(32768, 8192 * 8192 // hidden)), hidden=hidden, group=group, residual=rng.random() < 0.75, code=code,
                type=rng.choice(["f16", "bf16"]))


def _split(total, parts, seed):
    """`total` into `parts` uneven whole numbers of at least 1."""
    rng = random.Random(seed)
    weights = [rng.uniform(0.1, 1.0) for _ in range(parts)]
    scale = (total - parts) / sum(weights)
    got = [1 + int(w * scale) for w in weights]
    for i in range(total - sum(got)):
        got[i % parts] += 1
    return got


def _steps(case):
    """(new tokens, tokens held before) of each sequence of a chunk case: the first one holds `context`, others from half of it on, every
    third one nothing."""
    rng = random.Random(case["ragged"])
    n = case["context"]
    held = [n if b == 0 else 0 if b % 3 == 2 else rng.randint((n + 1) // 2, n) for b in range(case["sequences"])]
    return _split(case["tokens"], case["sequences"], case["ragged"]), held


def _beams(case):
    """A fork case's table before the step, as lists of pages, what each row holds, and the parents.  A group's beams share the full pages
    of a prompt, and have their own tails; some groups are finished, and one row is new."""
    rng = random.Random(case["ragged"])
    page, beams = case["page"], case["beams"]
    rows, held, parents, at = [], [], [], 0
    for g in range(case["groups"]):
        n = case["context"] if g == 0 else rng.randint((case["context"] + 1) // 2, case["context"])
        shared = n // page // 2
        common = list(range(at, at + shared))
        at += shared
        for b in range(beams):
            own_pages = -(-n // page) - shared
            rows.append(common + list(range(at, at + own_pages)))
            at += own_pages
            held.append(n)
            parents.append(-1 if g % 7 == 6 else g * beams + rng.randrange(beams))
    parents.append(-1)
    return rows, held, parents, at


def _pool(case):
    """The pages that a compact case's sequences have: a list for each, shared ones among them."""
    rng = random.Random(case["ragged"])
    order = list(range(case["pages"]))
    rng.shuffle(order)
    used = order[:max(1, int(case["used"] * case["pages"]))]
    lengths = _split(max(len(used), case["sequences"]), case["sequences"], case["ragged"])
    rows, at = [], 0
    for n in lengths:
        rows.append(used[at:at + n])
        at += n
    for b in range(1, len(rows), 3):                       # sequences that share the beginning of another
        if rows[b]:
            rows[b] = rows[b - 1][:len(rows[b - 1]) // 2] + rows[b]
    return rows


# ---- inputs ----

def _values(shape, gen, dtype, outliers=False):
    """Activations: normal, some channels much larger than the others where `outliers`."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    if outliers:
        gain = torch.ones(shape[-1], device="cuda")
        gain[torch.randperm(shape[-1], generator=gen, device="cuda")[:max(1, shape[-1] // 64)]] = 6.0
        x = x * gain
    return x.to(dtype)


def _codes(shape, gen, code):
    x = torch.empty(shape, dtype=torch.uint8, device="cuda")
    flat = x.view(-1)
    for at in range(0, flat.numel(), 1 << 28):
        part = flat[at:at + (1 << 28)]
        v = torch.randn(part.numel(), generator=gen, device="cuda", dtype=torch.float32)
        if code == "int8":
            part.copy_((v * 36).round().clamp(-127, 127).to(torch.int8).view(torch.uint8))
        else:
            part.copy_((v * 120).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    return x


def _cache(case, pages, gen):
    heads, code = case["kv_heads"], case["code"]
    shape = (pages, heads, case["page"], case["dim"])
    top = 36.0 if code == "int8" else 120.0
    scales = [(0.6 + 0.8 * torch.rand((pages, heads), generator=gen, device="cuda")) / top for _ in range(2)]
    return dict(k_cache=_codes(shape, gen, code), v_cache=_codes(shape, gen, code), k_scales=scales[0], v_scales=scales[1])


def _table(rows, width, pages, gen):
    """Rows of page numbers, which a permutation of the pool names anew, and how many rows use each page."""
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32).cpu().tolist() if gen is not None else list(range(pages))
    table, uses = [[-1] * width for _ in rows], [0] * pages
    for b, row in enumerate(rows):
        for i, p in enumerate(row):
            table[b][i] = order[p]
            uses[order[p]] += 1
    return table, uses


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lengths):
    got = [0]
    for n in lengths:
        got.append(got[-1] + n)
    return got


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    op = case["op"]
    if op == "norm":
        dtype, shape = TYPES[case["type"]], (case["tokens"], case["hidden"])
        s["x"] = _values(shape, gen, dtype, outliers=True)
        s["r"] = _values(shape, gen, dtype, outliers=True) if case["residual"] else None
        s["weight"] = (0.5 + torch.rand(case["hidden"], generator=gen, device="cuda")).to(dtype)
        return s
    if op == "chunk":
        new, held = _steps(case)
        need = [-(-(h + n) // case["page"]) for n, h in zip(new, held)]
        pages, at, rows = sum(need) + 3, 0, []
        for n in need:
            rows.append(list(range(at, at + n)))
            at += n
        table, _ = _table(rows, max(need), pages, gen)
        s.update(_cache(case, pages, gen))
        s.update(pages=_ints(table), offsets=_ints(_offsets(new)), held=_ints(held), new_host=new, held_host=held, longest=max(h + n for n, h in zip(new, held)))
        heads, group = case["kv_heads"], case["group"]
        qkv = _values((case["tokens"], heads * (group + 2), case["dim"]), gen, TYPES[case["type"]])
        s.update(q=qkv[:, :heads * group], k=qkv[:, heads * group:heads * (group + 1)], v=qkv[:, heads * (group + 1):])
        return s
    if op == "fork":
        rows, held, parents, used = _beams(case)
        page = case["page"]
        width = -(-(case["context"] + case["new"]) // page) + 1
        # room for every row's copy and new tokens
        pages = used + (len(parents) + 1) * (2 + -(-case["new"] // page))
        table, uses = _table(rows, width, pages, gen)
        s.update(_cache(case, pages, gen))
        s.update(pages=_ints(table), uses=_ints(uses), held=_ints(held), parents=_ints(parents), offsets=_ints([case["new"] * b for b in range(len(parents) + 1)]))
        return s
    rows = _pool(case)
    table, uses = _table(rows, max(len(r) for r in rows), case["pages"], gen)
    s.update(_cache(case, case["pages"], gen))
    s.update(pages=_ints(table), uses=_ints(uses))
    return s


# ---- the operators in their plain form ----

def _to_codes(x, code):
    if code == "int8":
        return x.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def _numbers(c, code):
    return c.view(torch.int8 if code == "int8" else torch.float8_e4m3fn)


def _held(s):
    """The cache's codes as the numbers that they are, and their scales."""
    return _numbers(s["k_cache"], s["code"]), _numbers(s["v_cache"], s["code"]), s["k_scales"], s["v_scales"]


def _softmax(scores, seen):
    """Over the last axis, where `seen`; a row that sees nothing is all zeros."""
    scores = torch.where(seen, scores, torch.full((), -math.inf, device=scores.device))
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total)


def _chunk(s):
    heads, group, dim, page, code = s["kv_heads"], s["group"], s["dim"], s["page"], s["code"]
    out, at = torch.empty_like(s["q"], memory_format=torch.contiguous_format), 0
    for b, (n, have) in enumerate(zip(s["new_host"], s["held_host"])):
        mine = s["pages"][b, :-(-have // page)].long()

        def rows(cache, scales, new):
            x = (_numbers(cache[mine], code).float() * scales[mine][..., None, None]).transpose(0, 1).reshape(heads, -1, dim)[:, :have]
            return torch.cat([x, new[at:at + n].float().transpose(0, 1)], 1)

        q = s["q"][at:at + n].float().view(n, heads, group, dim).permute(1, 2, 0, 3).reshape(heads, group * n, dim)
        scores = (torch.bmm(q, rows(s["k_cache"], s["k_scales"], s["k"]).transpose(1, 2).contiguous()) / math.sqrt(dim)).view(heads, group, n, have + n)
        seen = torch.arange(have + n, device="cuda")[None, :] <= have + torch.arange(n, device="cuda")[:, None]
        weights = _softmax(scores, seen).view(heads, group * n, have + n)
        o = torch.bmm(weights, rows(s["v_cache"], s["v_scales"], s["v"])).view(heads, group, n, dim)
        out[at:at + n] = o.permute(2, 0, 1, 3).reshape(n, heads * group, dim).to(out.dtype)
        at += n
    return out


def _copy(s, source, target):
    there = (source >= 0).nonzero()[:, 0]
    a, b = source[there].long(), target[there].long()
    for name in ("k_cache", "v_cache", "k_scales", "v_scales"):
        s[name][b] = s[name][a]


def _fork(s):
    page, parents = s["page"], s["parents"].long()
    table, width = s["pages"], s["pages"].shape[1]
    uses = s["uses"].clone()
    slot = torch.arange(width, device="cuda")
    kept = torch.where(slot < ((s["held"] + page - 1) // page)[:, None], table, torch.full_like(table, -1))
    chosen = parents >= 0
    got = torch.where(chosen[:, None], kept[parents.clamp(min=0)], torch.full((), -1, dtype=torch.int32, device="cuda"))
    held = torch.where(chosen, s["held"][parents.clamp(min=0)], torch.zeros((), dtype=torch.int32, device="cuda"))
    for t, change in ((table, -1), (got, 1)):
        there = t >= 0
        uses.index_add_(0, t.clamp(min=0).long().flatten(), (there.int() * change).flatten())
    source, target, lacking = _reserve(got, held, uses, s["offsets"], page)
    _copy(s, source, target)
    return got, held, uses, source, target, lacking


def _reserve(table, held, uses, offsets, page):
    sequences, width = table.shape
    none = torch.full((), -1, dtype=torch.int32, device="cuda")
    new = offsets[1:] - offsets[:-1]
    begin, end = held.clamp(min=0), held + new
    first, last = begin // page, (end + page - 1) // page - 1
    slot = torch.arange(width, device="cuda")
    written = (slot >= first[:, None]) & (slot <= last[:, None]) & (end > begin)[:, None]
    # a page that holds tokens and is written: which rows do that, and who keeps it
    mine = table.gather(1, first.clamp(max=width - 1).long()[:, None])[:, 0]
    writes = (begin % page != 0) & (end > begin) & (first < width) & (mine >= 0)
    same = (mine[:, None] == mine[None, :]) & writes[:, None] & writes[None, :]
    later = torch.triu(same, 1).any(1)
    users = uses[mine.clamp(min=0).long()]
    copies = writes & (users > 1) & (later | (same.sum(1) < users))
    wants = written & ((table < 0) | (copies[:, None] & (slot == first[:, None])))
    rank = wants.flatten().cumsum(0) - 1
    needed = int(wants.sum())
    free = (uses == 0).nonzero()[:, 0]
    if needed > free.shape[0]:
        nothing = torch.full((sequences,), -1, dtype=torch.int32, device="cuda")
        return nothing, nothing.clone(), _ints([needed - free.shape[0]])
    if needed == 0:
        nothing = torch.full((sequences,), -1, dtype=torch.int32, device="cuda")
        return nothing, nothing.clone(), _ints([0])
    fresh = free[rank.clamp(min=0, max=needed - 1)].view(sequences, width).int()
    source = torch.where(copies, mine, none)
    target = torch.where(copies, fresh.gather(1, first.clamp(max=width - 1).long()[:, None])[:, 0], none)
    uses.index_add_(0, mine.clamp(min=0).long(), -copies.int())
    uses[free[:needed]] = 1
    table.copy_(torch.where(wants, fresh, table))
    return source, target, _ints([0])


def _compact(s):
    uses, table = s["uses"], s["pages"]
    pages = uses.shape[0]
    number = torch.arange(pages, device="cuda")
    used = int((uses > 0).sum())
    holes = ((uses <= 0) & (number < used)).nonzero()[:, 0]
    movers = ((uses > 0) & (number >= used)).nonzero()[:, 0]
    place = number.clone()
    place[movers] = holes
    now = uses.clone()
    now[holes] = uses[movers]
    now[used:] = 0
    got = torch.where(table >= 0, place[table.clamp(min=0).long()].int(), table)
    source, target = (torch.full((pages // 2,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    source[:movers.shape[0]] = movers.int()
    target[:holes.shape[0]] = holes.int()
    _copy(s, source, target)
    return got, now, source, target, _ints([used])


def _norm(s):
    h = s["x"].float()
    if s["r"] is not None:
        h = h + s["r"].float()
    # the sum of squares in 64 bits: codes are next to borders, so it has to be the same in every order
    d = (1 / torch.sqrt(h.double().square().sum(-1, keepdim=True) / s["hidden"] + EPS)).float()
    y = (h * d) * s["weight"].float()
    total = (h.to(s["x"].dtype),) if s["r"] is not None else ()
    if not s["code"]:
        return (y.to(s["x"].dtype), *total)
    g = y.view(s["tokens"], -1, s["group"])
    scale = g.abs().amax(-1) / torch.full((), LARGEST[s["code"]], device="cuda")
    scale = torch.where(scale >= FLT_MIN, scale, torch.ones_like(scale))
    codes = _to_codes(g * (torch.ones_like(scale) / scale)[..., None], s["code"]).view(s["tokens"], -1)
    return (_numbers(codes, s["code"]), scale, *total)


# ---- one pass ----

def run(state):
    s = state
    if not own:
        if s["op"] in ("fork", "compact"):
            return (*(_fork if s["op"] == "fork" else _compact)(s), *_held(s))
        return (_chunk if s["op"] == "chunk" else _norm)(s)
    import paper_2412_04964_amd as fc
    if s["op"] == "norm":
        if s["code"]:
            quantizer = fc.QUANTIZER_SYM if s["code"] == "int8" else fc.QUANTIZER_FP8
            codes, *rest = fc.rms_norm_quantize(s["x"], s["weight"], EPS, s["group"], quantizer, residual=s["r"])
            return (_numbers(codes, s["code"]), *rest)
        y = fc.rms_norm(s["x"], s["weight"], EPS, residual=s["r"])
        return y if s["r"] is not None else (y,)
    cache = (s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"])
    if s["op"] == "chunk":
        quantizer = fc.QUANTIZER_SYM if s["code"] == "int8" else fc.QUANTIZER_FP8
        return fc.chunk_attention(s["q"], s["k"], s["v"], cache, s["pages"], s["offsets"], s["held"], s["longest"], quantizer)
    if s["op"] == "fork":
        uses = s["uses"].clone()
        table, held = fc.pages_fork(s["pages"], s["held"], uses, s["parents"], s["page"])
        source, target, lacking = fc.pages_reserve(table, held, uses, s["offsets"], s["page"])
        fc.cache_copy(cache, source, target)
        return (table, held, uses, source, target, lacking, *_held(s))
    table, uses, source, target, used = fc.pages_compact(s["pages"], s["uses"])
    fc.cache_copy(cache, source, target)
    return (table, uses, source, target, used, *_held(s))


def work(case):
    op = case["op"]
    if op == "norm":
        n = case["tokens"] * case["hidden"]
        out = 1 + 4 / case["group"] if case["code"] else 2
        return {"bytes": int(n * (2 + (4 if case["residual"] else 0) + out)) + 2 * case["hidden"], "flops": 5 * n}
    dim, page, heads = case["dim"], case["page"], case["kv_heads"]
    if op == "chunk":
        new, held = _steps(case)
        queries = heads * case["group"]
        pages = sum(-(-h // page) for h in held)
        seen = sum(n * h + n * (n + 1) // 2 for n, h in zip(new, held))
        return {"bytes": sum(held) * heads * 2 * dim + pages * (8 * heads + 4) + 4 * sum(new) * dim * (heads + queries), "flops": 4 * dim * queries * seen}
    one = 2 * (2 * page * dim + 8) * heads                  # a page copied: read and written
    if op == "fork":
        rows, held, parents, used = _beams(case)
        # what a step copies: a page for each row whose parent's last page is not full, but for those that stay the only users
        chosen = [p for p in parents if p >= 0 and held[p] % page]
        copied = len(chosen) - len(set(chosen))
        table = sum(len(rows[p]) for p in parents if p >= 0)
        return {"bytes": copied * one + 4 * (3 * table + 2 * used + 3 * len(parents)), "flops": table}
    rows = _pool(case)
    in_use = {p for r in rows for p in r}
    _, uses = _table(rows, max(len(r) for r in rows), case["pages"], None)
    # pages in use have random numbers: so many of them are expected beyond their count
    moved = len(in_use) * (case["pages"] - len(in_use)) // case["pages"]
    return {"bytes": moved * one + 8 * (sum(uses) + case["pages"]), "flops": case["pages"]}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        h = s["x"].double() + (s["r"].double() if s["r"] is not None else 0)
        y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS) * s["weight"].double()
        total = (h,) if s["r"] is not None else ()
        if not case["code"]:
            return (y, *total)
        scale = y.view(case["tokens"], -1, case["group"]).abs().amax(-1) / LARGEST[case["code"]]
        if case["code"] == "int8":                         # whole numbers have to be equal; E4M3 numbers are compared as numbers
            return (None, scale, *total)
        x = y / scale.repeat_interleave(case["group"], -1)
        step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -30))).clamp(min=-6) - 3)
        return ((x / step).round() * step, scale, *total)
    if op == "chunk":
        heads, group, dim, page = case["kv_heads"], case["group"], case["dim"], case["page"]
        number = torch.int8 if case["code"] == "int8" else torch.float8_e4m3fn
        out, at = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), 0
        for b, (n, have) in enumerate(zip(s["new_host"], s["held_host"])):
            pages = s["pages"][b, :-(-have // page)].long()
            hidden = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
            for h in range(heads):
                k, v = (torch.cat([(c[pages, h].view(number).double() * w[pages, h].double()[:, None, None]).reshape(-1, dim)[:have], x[at:at + n, h].double()])
                        for c, w, x in ((s["k_cache"], s["k_scales"], s["k"]), (s["v_cache"], s["v_scales"], s["v"])))
                for g in range(group):
                    score = s["q"][at:at + n, h * group + g].double() @ k.t() * dim ** -0.5
                    score[:, have:].masked_fill_(hidden, -math.inf)
                    out[at:at + n, h * group + g] = torch.softmax(score, -1) @ v
            at += n
        return out
    return None                                            # pages are numbered and copied: nothing is computed in floating point
