"""Attention operators of one rank of a tensor-parallel model that serves requests: rotary positions, the paged 8-bit
cache of keys and values, attention over that cache, and attention over whole packed prompts.

`run` is the plain form (elementary torch operations in 32 bits) or, where `own` is true, the framework's kernels.
Head counts are those of one rank of the models whose hidden sizes the benchmark uses (heads of 128: 32 query and 8
key/value heads for hidden 4096, 64 and 8 for 8192, 40 and 40 for 5120), alone or over 4 or 8 ranks.
"""
import math
import random

import torch

own = False

FLT_MIN = 1.1754943508222875e-38
LARGEST = {"int8": 127.0, "fp8": 448.0}
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


# ---- cases ----

def listed():
    return [
        # one decode step of 8 requests, query and key heads of a rank of hidden 8192 over 4: latency
        dict(name="rotary decode", op="rotary", tokens=8, heads=18, values=2, dim=128, rotary=128, interleaved=False, type="bf16", context=8192),
        # prompts of hidden 5120 on one rank, odd number of tokens, half of each head turned in neighbouring pairs
        dict(name="rotary prompt", op="rotary", tokens=16383, heads=80, values=40, dim=128, rotary=64, interleaved=True, type="f16", context=16384),
        # one decode step of 8 requests on a rank of hidden 8192 over 4: one new token each, small pages
        dict(name="append decode", op="append", sequences=8, tokens=8, kv_heads=2, dim=128, page=16, context=1500, rotary=128, interleaved=False, code="int8", type="bf16", ragged=1),
        # packed prompts and continued ones of uneven lengths, all heads of hidden 4096 on one rank
        dict(name="append prompts", op="append", sequences=9, tokens=32771, kv_heads=8, dim=128, page=64, context=700, rotary=128, interleaved=False, code="fp8", type="f16", ragged=2),
        # a large decode batch, keys and values of hidden 5120, rotation done before
        dict(name="append batch", op="append", sequences=256, tokens=256, kv_heads=40, dim=128, page=32, context=300, rotary=0, interleaved=False, code="int8", type="f16", ragged=3),
        # the first tokens of one chat: a single request with a short cache
        dict(name="cache one request", op="cache", sequences=1, queries=1, kv_heads=2, group=4, dim=128, page=16, context=129, code="int8", type="f16", ragged=4),
        # the usual decode step: 8 requests of about a thousand tokens, rank of hidden 8192 over 4
        dict(name="cache decode", op="cache", sequences=8, queries=1, kv_heads=2, group=8, dim=128, page=16, context=1536, code="fp8", type="bf16", ragged=5),
        # a large batch with long contexts, all heads of hidden 4096
        dict(name="cache batch", op="cache", sequences=64, queries=1, kv_heads=8, group=4, dim=128, page=64, context=8192, code="int8", type="bf16", ragged=6),
        # one request with a very long document; several drafted tokens are verified at once
        dict(name="cache long document", op="cache", sequences=1, queries=5, kv_heads=8, group=8, dim=128, page=32, context=131071, code="fp8", type="f16", ragged=7),
        # one prompt of 1024 tokens, rank of hidden 4096 over 4
        dict(name="prompt 1024", op="prompt", sequences=1, tokens=1024, kv_heads=2, group=4, dim=128, causal=True, type="bf16", ragged=8),
        # packed prompts of uneven lengths, every query head with a key/value head of its own (hidden 5120)
        dict(name="prompt packed", op="prompt", sequences=11, tokens=8191, kv_heads=40, group=1, dim=128, causal=True, type="f16", ragged=9),
        # one long document, rank of hidden 8192 over 4
        dict(name="prompt long document", op="prompt", sequences=1, tokens=16384, kv_heads=2, group=8, dim=128, causal=True, type="bf16", ragged=10),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "append", "cache", "prompt"])
    dim = rng.choice([64, 128, 128, 128])
    case = dict(op=op, dim=dim, type=rng.choice(["f16", "bf16"]))
    ragged = rng.randrange(1000, 1000000)
    if op == "rotary":
        tokens, heads = _log(rng, 1, 16383), _log(rng, 1, 80)
        case.update(tokens=tokens, heads=heads, values=_log(rng, 1, 40), rotary=rng.choice([dim, dim, dim // 2]), interleaved=rng.random() < 0.5, context=rng.randrange(16384, 32769))
    elif op == "append":
        heads = rng.choice([1, 2, 4, 8, 10, 40])
        sequences = _log(rng, 1, 256)
        tokens = sequences if rng.random() < 0.5 else max(sequences, _log(rng, 16, 32771 * 8 // max(8, heads)))
        # the whole cache is an output: kept to a size like the listed ones'
        context = _log(rng, 1, max(2, min(2000, 500000 // (sequences * max(1, heads // 8)))))
        case.update(sequences=sequences, tokens=tokens, kv_heads=heads, page=rng.choice([16, 32, 64]), context=context, rotary=rng.choice([0, dim, dim, dim // 2]), interleaved=rng.random() < 0.3, code=rng.choice(["int8", "fp8"]), ragged=ragged)
    elif op == "cache":
        sequences = _log(rng, 1, 64)
        heads = rng.choice([1, 2, 4, 8, 10])
        context = _log(rng, 1, min(131071, 64 * 8192 * 8 // (sequences * heads)))
        group = rng.choice([1, 2, 4, 5, 8]) if heads < 10 else 1
        queries = rng.choice([1, 1, 1, 2, 4, 5]) if context >= 8 else 1
        if sequences * context * heads * group * queries > 131071 * 8 * 40:
            queries = 1
        case.update(sequences=sequences, queries=queries, kv_heads=heads, group=group, page=rng.choice([16, 32, 64]), context=context, code=rng.choice(["int8", "fp8"]), ragged=ragged)
    else:
        heads, group = rng.choice([(1, 8), (2, 4), (2, 8), (8, 4), (8, 8), (10, 1), (40, 1), (1, 5)])
        tokens = _log(rng, 1, int(16384 * math.sqrt(min(1.0, 16 / (heads * group)))))
        case.update(sequences=_log(rng, 1, min(16, tokens)), tokens=tokens, kv_heads=heads, group=group, causal=rng.random() < 0.75, ragged=ragged)
    return case


def _split(total, parts, seed):
    """`total` into `parts` uneven whole numbers of at least 1."""
    rng = random.Random(seed)
    weights = [rng.uniform(0.1, 1.0) for _ in range(parts)]
    scale = (total - parts) / sum(weights)
    got = [1 + int(w * scale) for w in weights]
    for i in range(total - sum(got)):
        got[i % parts] += 1
    return got


def _contexts(case):
    """Tokens each sequence holds: the first one `context`, others from half of it on (none for some where prompts are appended)."""
    rng = random.Random(case["ragged"])
    n = case["context"]
    got = [n if b == 0 else rng.randint((n + 1) // 2, n) for b in range(case["sequences"])]
    if case["op"] == "append" and case["tokens"] > case["sequences"]:
        got = [0 if b % 3 == 1 else g for b, g in enumerate(got)]
    return got


def _steps(case):
    """(new tokens, tokens held before) of each sequence."""
    held = _contexts(case)
    if case["op"] == "append":
        return _split(case["tokens"], case["sequences"], case["ragged"]), held
    new = [case["queries"]] * case["sequences"]
    return new, [max(0, h - n) for h, n in zip(held, new)]


# ---- inputs ----

def _values(shape, gen, dtype, outliers=True):
    """Activations: normal, some channels of a head much larger than the others."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    if outliers:
        gain = torch.ones(shape[-1], device="cuda")
        gain[torch.randperm(shape[-1], generator=gen, device="cuda")[:max(1, shape[-1] // 64)]] = 6.0
        x = x * gain
    return x.to(dtype)


def _rotation_table(rows, rotary):
    """[rows, rotary]: the cosines of a position's rotary / 2 angles, then their sines."""
    f = 10000.0 ** (-torch.arange(0, rotary, 2, device="cuda", dtype=torch.float64) / rotary)
    angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * f
    return torch.cat([angle.cos(), angle.sin()], 1).float()


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


def _cache(case, new, held, gen):
    page, heads, dim, code = case["page"], case["kv_heads"], case["dim"], case["code"]
    need = [-(-(h + n) // page) for n, h in zip(new, held)]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(new), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    top = 36.0 if code == "int8" else 120.0
    scales = [(0.6 + 0.8 * torch.rand((pages, heads), generator=gen, device="cuda")) / top for _ in range(2)]
    return dict(k_cache=_codes((pages, heads, page, dim), gen, code), v_cache=_codes((pages, heads, page, dim), gen, code), k_scales=scales[0], v_scales=scales[1], pages=table)


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
    dtype, op = TYPES[case["type"]], case["op"]
    if op == "rotary":
        # the joint projection of queries, keys and values, whose query and key heads are turned
        qkv = _values((case["tokens"], case["heads"] + case["values"], case["dim"]), gen, dtype)
        s["x"] = qkv[:, :case["heads"]]
        s["table"] = _rotation_table(case["context"], case["rotary"])
        if case["tokens"] <= 64:
            s["positions"] = torch.randint(0, case["context"], (case["tokens"],), generator=gen, device="cuda").to(torch.int32)
        else:
            first = int(torch.randint(0, case["context"] - case["tokens"] + 1, (1,), generator=gen, device="cuda"))
            s["positions"] = torch.arange(first, first + case["tokens"], device="cuda", dtype=torch.int32)
        return s
    if op == "prompt":
        heads, group = case["kv_heads"], case["group"]
        lengths = _split(case["tokens"], case["sequences"], case["ragged"])
        qkv = _values((case["tokens"], heads * (group + 2), case["dim"]), gen, dtype, outliers=False)
        s.update(q=qkv[:, :heads * group], k=qkv[:, heads * group:heads * (group + 1)], v=qkv[:, heads * (group + 1):])
        s.update(offsets=_ints(_offsets(lengths)), lengths=lengths, longest=max(lengths))
        return s
    new, held = _steps(case)
    s.update(_cache(case, new, held, gen))
    s.update(offsets=_ints(_offsets(new)), held=_ints(held), new_host=new, held_host=held, longest=max(h + n for n, h in zip(new, held)))
    total = sum(new)
    if op == "append":
        s["longest"] = max(new)
        kv = _values((total, 2 * case["kv_heads"], case["dim"]), gen, dtype)
        s.update(k=kv[:, :case["kv_heads"]], v=kv[:, case["kv_heads"]:])
        s["table"] = _rotation_table(max(h + n for n, h in zip(new, held)), case["rotary"]) if case["rotary"] else None
    else:
        s["q"] = _values((total, case["kv_heads"] * case["group"], case["dim"]), gen, dtype, outliers=False)
    return s


# ---- the operators in their plain form ----

def _turn(x, table, positions, interleaved):
    """x: float32 [tokens, heads, dim], the first table.shape[1] of each head turned by its position's angles"""
    rotary = table.shape[1]
    rows = table[positions.long()]
    c, s = rows[:, None, :rotary // 2], rows[:, None, rotary // 2:]
    part = x[..., :rotary]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :rotary // 2], part[..., rotary // 2:])
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rotary:]], -1)


def _rotary(s):
    return _turn(s["x"].float(), s["table"], s["positions"], s["interleaved"]).to(s["x"].dtype)


def _to_codes(x, code):
    if code == "int8":
        return x.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def _from_codes(c, code):
    return c.view(torch.int8 if code == "int8" else torch.float8_e4m3fn).float()


def _append_one(x, cache, scales, s, sequence, position):
    code, page = s["code"], s["page"]
    top = torch.full((), LARGEST[code], device=x.device)
    # the page each sequence goes on with: its scale counts where it holds tokens already
    held = s["held"].long()
    last = (held // page).clamp(max=s["pages"].shape[1] - 1)
    first_page = s["pages"].long().gather(1, last[:, None])[:, 0].clamp(min=0)
    filled = torch.where(s["offsets"][1:] > s["offsets"][:-1], held % page, torch.zeros_like(held))
    before = torch.zeros_like(scales)
    before[first_page] = torch.where((filled > 0)[:, None], scales[first_page], torch.zeros_like(scales[first_page]))
    # the largest magnitude that comes to each page, and the page's new scale
    target = s["pages"].long()[sequence, position // page]
    most = torch.zeros_like(scales).index_reduce_(0, target, x.abs().amax(-1), "amax")
    now = torch.maximum(torch.maximum(most / top, torch.full_like(most, FLT_MIN)), before)
    touched = torch.zeros(scales.shape[0], dtype=torch.bool, device=x.device).index_fill_(0, target, True)
    # what the page holds, in the new scale
    old = cache[first_page]
    ratio = scales[first_page] / now[first_page]
    keep = torch.arange(page, device=x.device)[None, :] < filled[:, None]
    again = _to_codes(_from_codes(old, code) * ratio[:, :, None, None], code)
    grown = keep[:, None, :, None] & (now[first_page] > scales[first_page])[:, :, None, None]
    cache[first_page] = torch.where(grown, again, old)
    scales.copy_(torch.where(touched[:, None], now, scales))
    inverse = torch.ones_like(now) / now
    cache[target, :, position % page] = _to_codes(x * inverse[target][:, :, None], code)


def _append(s):
    tokens = torch.arange(s["k"].shape[0], device="cuda")
    sequence = torch.searchsorted(s["offsets"].long(), tokens, right=True) - 1
    position = s["held"].long()[sequence] + tokens - s["offsets"].long()[sequence]
    k, v = s["k"].float(), s["v"].float()
    if s["table"] is not None:
        k = _turn(k, s["table"], position, s["interleaved"])
    _append_one(k, s["k_cache"], s["k_scales"], s, sequence, position)
    _append_one(v, s["v_cache"], s["v_scales"], s, sequence, position)
    return _held(s)


def _held(s):
    """The cache's codes as the numbers that they are, and their scales."""
    number = torch.int8 if s["code"] == "int8" else torch.float8_e4m3fn
    return s["k_cache"].view(number), s["v_cache"].view(number), s["k_scales"], s["v_scales"]


def _softmax(scores, seen):
    """Over the last axis, where `seen`; a row that sees nothing is all zeros."""
    scores = torch.where(seen, scores, torch.full((), -math.inf, device=scores.device))
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total)


def _cache_attention(s):
    heads, group, dim, code = s["kv_heads"], s["group"], s["dim"], s["code"]
    table = s["pages"].long().clamp(min=0)
    sequences, n = table.shape[0], s["queries"]

    def rows(cache, scales):
        x = _from_codes(cache[table], code) * scales[table][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(sequences * heads, -1, dim)

    q = s["q"].float().view(sequences, n, heads, group, dim).permute(0, 2, 1, 3, 4).reshape(sequences * heads, n * group, dim)
    scores = torch.bmm(q, rows(s["k_cache"], s["k_scales"]).transpose(1, 2).contiguous()) / math.sqrt(dim)
    at = torch.arange(scores.shape[-1], device="cuda")
    sees = s["held"].long()[:, None] + torch.arange(n, device="cuda") + 1
    seen = (at < sees[:, :, None])[:, None, :, None, :].expand(sequences, heads, n, group, -1).reshape(scores.shape)
    out = torch.bmm(_softmax(scores, seen), rows(s["v_cache"], s["v_scales"]))
    return out.view(sequences, heads, n, group, dim).permute(0, 2, 1, 3, 4).reshape(sequences * n, heads * group, dim).to(s["q"].dtype)


def _prompt_attention(s):
    heads, group, dim, tokens = s["kv_heads"], s["group"], s["dim"], s["q"].shape[0]
    q = s["q"].float().transpose(0, 1).reshape(heads, group * tokens, dim)
    k = s["k"].float().permute(1, 2, 0).contiguous()
    v = s["v"].float().transpose(0, 1).contiguous()
    scores = (torch.bmm(q, k) / math.sqrt(dim)).view(heads, group, tokens, tokens)
    at = torch.arange(tokens, device="cuda")
    sequence = torch.searchsorted(s["offsets"].long(), at, right=True)
    seen = sequence[:, None] == sequence[None, :]
    if s["causal"]:
        seen = seen & (at[None, :] <= at[:, None])
    weights = _softmax(scores, seen).view(heads, group * tokens, tokens)
    return torch.bmm(weights, v).view(heads * group, tokens, dim).transpose(0, 1).to(s["q"].dtype).contiguous()


# ---- one pass ----

def run(state):
    s = state
    if not own:
        return {"rotary": _rotary, "append": _append, "cache": _cache_attention, "prompt": _prompt_attention}[s["op"]](s)
    import paper_2412_04964_amd as fc
    if s["op"] == "rotary":
        return fc.rotary(s["x"], s["table"], s["positions"], s["interleaved"])
    if s["op"] == "prompt":
        return fc.prompt_attention(s["q"], s["k"], s["v"], s["offsets"], s["longest"], s["causal"])
    quantizer = fc.QUANTIZER_SYM if s["code"] == "int8" else fc.QUANTIZER_FP8
    cache = (s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"])
    if s["op"] == "append":
        fc.cache_append(s["k"], s["v"], cache, s["pages"], s["offsets"], s["held"], s["longest"], quantizer, s["table"], s["interleaved"])
        return _held(s)
    return fc.cache_attention(s["q"], cache, s["pages"], s["offsets"], s["held"], s["queries"], s["longest"], quantizer)


def work(case):
    dim, op = case["dim"], case["op"]
    if op == "rotary":
        n = case["tokens"] * case["heads"]
        return {"bytes": 4 * n * dim + case["tokens"] * (4 * case["rotary"] + 4), "flops": 3 * n * case["rotary"]}
    if op == "prompt":
        lengths = _split(case["tokens"], case["sequences"], case["ragged"])
        heads, queries = case["kv_heads"], case["kv_heads"] * case["group"]
        pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lengths)
        return {"bytes": 2 * case["tokens"] * dim * 2 * (heads + queries), "flops": 4 * dim * queries * pairs}
    new, held = _steps(case)
    heads = case["kv_heads"]
    if op == "append":
        total = sum(new)
        pages = sum(-(-(h + n) // case["page"]) - h // case["page"] for n, h in zip(new, held))
        return {"bytes": 2 * total * heads * dim * 3 + 4 * total * case["rotary"] + 2 * pages * heads * 8, "flops": total * heads * (4 * dim + 3 * case["rotary"])}
    reads = sum(h + n for n, h in zip(new, held))
    pages = sum(-(-(h + n) // case["page"]) for n, h in zip(new, held))
    queries = heads * case["group"]
    seen = sum(n * h + n * (n + 1) // 2 for n, h in zip(new, held))
    return {"bytes": reads * heads * 2 * dim + 2 * pages * heads * 4 + 4 * pages + sum(new) * queries * dim * 4, "flops": 4 * dim * queries * seen}


# ---- the definitions in 64 bits ----

def _turn64(x, table, position, interleaved):
    y = x.clone()
    half = table.shape[1] // 2
    for i in range(half):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = table[position, i].double()[:, None], table[position, half + i].double()[:, None]
        y[:, :, p] = x[:, :, p] * c - x[:, :, q] * s
        y[:, :, q] = x[:, :, q] * c + x[:, :, p] * s
    return y


def _nearest(x, code):
    """The number that a code holds for x, ties to even."""
    if code == "int8":
        return x.round().clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -30))).clamp(min=-6) - 3)
    return ((x / step).round() * step).clamp(-448, 448)


def _append64(s, values, codes, scales, table):
    held = codes.view(torch.int8 if s["code"] == "int8" else torch.float8_e4m3fn).double()
    scales = scales.double()
    at = 0
    for b, (n, have) in enumerate(zip(s["new_host"], s["held_host"])):
        x = values[at:at + n]
        if table is not None:
            x = _turn64(x, table, torch.arange(have, have + n, device="cuda"), s["interleaved"])
        done = 0
        while done < n:
            page, slot = divmod(have + done, s["page"])
            take = min(s["page"] - slot, n - done)
            p = int(s["pages"][b, page])
            part = x[done:done + take].transpose(0, 1)
            now = (part.abs().amax((1, 2)) / LARGEST[s["code"]]).clamp(min=FLT_MIN)
            if slot:
                now = torch.maximum(now, scales[p])
                grown = now > scales[p]
                again = _nearest(held[p, :, :slot] * (scales[p] / now)[:, None, None], s["code"])
                held[p, :, :slot] = torch.where(grown[:, None, None], again, held[p, :, :slot])
            scales[p] = now
            held[p, :, slot:slot + take] = _nearest(part / now[:, None, None], s["code"])
            done += take
        at += n
    return held, scales


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rotary":
        return _turn64(s["x"].double(), s["table"], s["positions"].long(), s["interleaved"])
    if op == "append":
        if case["kv_heads"] * case["dim"] * s["k_cache"].shape[0] * case["page"] > 1 << 30:
            return None
        k = _append64(s, s["k"].double(), s["k_cache"], s["k_scales"], s["table"])
        v = _append64(s, s["v"].double(), s["v_cache"], s["v_scales"], None)
        whole = case["code"] == "int8"         # whole numbers have to be equal; E4M3 numbers are compared as numbers
        return (None if whole else k[0]), (None if whole else v[0]), k[1], v[1]
    heads, group, dim = case["kv_heads"], case["group"], case["dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    if op == "prompt":
        at = 0
        for n in s["lengths"]:
            below = torch.ones((n, n), dtype=torch.bool, device="cuda").tril() if case["causal"] else None
            for h in range(heads * group):
                score = s["q"][at:at + n, h].double() @ s["k"][at:at + n, h // group].double().t() / math.sqrt(dim)
                if below is not None:
                    score = score.masked_fill(~below, -math.inf)
                out[at:at + n, h] = torch.softmax(score, -1) @ s["v"][at:at + n, h // group].double()
            at += n
        return out
    number = torch.int8 if case["code"] == "int8" else torch.float8_e4m3fn
    at = 0
    for b, (n, have) in enumerate(zip(s["new_host"], s["held_host"])):
        total = have + n
        pages = s["pages"][b, :-(-total // case["page"])].long()
        sees = torch.arange(total, device="cuda")[None, :] <= have + torch.arange(n, device="cuda")[:, None]
        for h in range(heads):
            k, v = ((c[pages, h].view(number).double() * w[pages, h].double()[:, None, None]).reshape(-1, dim)[:total]
                    for c, w in ((s["k_cache"], s["k_scales"]), (s["v_cache"], s["v_scales"])))
            for g in range(group):
                score = s["q"][at:at + n, h * group + g].double() @ k.t() / math.sqrt(dim)
                out[at:at + n, h * group + g] = torch.softmax(score.masked_fill(~sees, -math.inf), -1) @ v
        at += n
    return out
