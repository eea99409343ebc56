"""The attention operators on the GPU: rotation and append bit for bit against the formulas of include/fc.h in fp32 on the CPU,
attention against its definition in 64 bits.

Tolerances of attention, per element, from the roundings the kernels make (u = 2^-11 for float16, 2^-9 for bfloat16, half a unit in
the last place): one of the result, u |o|; and of each weight, relatively, one to the weights' type, and less than 2^-12 from the
fp32 score (dims of 256 at most, |score| < 64) and from the sums.  With E = sum_t w_t |v_t| the error is below
(u_w + 2^-11) E + u |o|, which the tests allow twice, plus the smallest subnormal numbers."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F16, BF16 = torch.float16, torch.bfloat16
FLT_MIN = 1.1754943508222875e-38
SYM, FP8 = 1, 2
TOP = {SYM: 127.0, FP8: 448.0}


@pytest.fixture(scope="module")
def fc():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests selected but no GPU is visible")
    import paper_2412_04964_amd as m
    m.lib()
    return m


def gen(seed):
    return torch.Generator().manual_seed(seed)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def offsets_of(lengths):
    return ints([0] + list(np.cumsum(lengths)))


def bits(t):
    return t.cpu().contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


def same(a, b):
    """equal bits, any NaN equal to any other"""
    a, b = a.cpu(), b.cpu()
    nan = torch.isnan(a) & torch.isnan(b)
    return bool(((bits(a) == bits(b)) | nan).all())


def fused(tokens, counts, dim, dtype, seed, spread=1.0):
    """slices of one joint projection [tokens, sum of counts, dim], on the GPU"""
    x = (torch.randn((tokens, sum(counts), dim), generator=gen(seed)) * spread).to(dtype).cuda()
    return x.split(list(counts), dim=1)


# ---- rotation ----

def turned(x, table, positions, interleaved, inverse=False):
    """x float32 [tokens, heads, dim]; each operation rounded to fp32"""
    rotary = table.shape[1]
    half = rotary // 2
    y = x.clone()
    ok = (positions >= 0) & (positions < table.shape[0])
    row = table[positions.clamp(0, table.shape[0] - 1).long()]
    row = torch.where(ok[:, None], row, torch.full_like(row, math.nan))
    c, s = row[:, None, :half], row[:, None, half:]
    if inverse:
        s = -s
    lo, hi = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, half), slice(half, rotary))
    a, b = x[..., lo], x[..., hi]
    y[..., lo] = a * c - b * s
    y[..., hi] = b * c + a * s
    return y


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rotary", [(128, 128), (64, 32), (80, 80), (96, 24), (128, 2), (8, 6), (256, 144)])
def test_rotary_matches_the_formula_bit_for_bit(fc, dtype, interleaved, dim, rotary):
    for tokens, heads in ((1, 1), (3, 5), (67, 9)):
        print("rotary", dtype, interleaved, dim, rotary, tokens, heads, flush=True)
        x, _ = fused(tokens, (heads, 2), dim, dtype, tokens + dim)
        table = fc.rotary_table(301, fc.rotary_frequencies(rotary))
        positions = torch.randint(0, 301, (tokens,), generator=gen(tokens)).to(torch.int32)
        positions[0] = 300
        if tokens > 3:
            positions[1], positions[2] = -1, 301                     # no such rows
        for inverse in (False, True):
            y = fc.rotary(x, table, positions.cuda(), interleaved, inverse)
            assert same(y, turned(x.float().cpu(), table.cpu(), positions, interleaved, inverse).to(dtype))


def test_rotary_in_place_and_its_inverse(fc):
    q, rest = fused(33, (6, 3), 128, BF16, 1)
    table = fc.rotary_table(64, fc.rotary_frequencies(128))
    positions = torch.arange(33, dtype=torch.int32, device="cuda")
    before, beside = q.clone(), rest.clone()
    want = fc.rotary(q, table, positions)
    assert fc.rotary(q, table, positions, out=q) is q
    assert same(q, want) and same(rest, beside)
    back = fc.rotary(q, table, positions, inverse=True)
    assert (back.float() - before.float()).abs().max() <= 2 * 2.0 ** -8 * before.float().abs().max()


def test_inverse_rotation_is_the_gradient(fc):
    # the rotation is linear: <R x, g> = <x, R' g>, and differences of a linear map are exact up to the two roundings
    x, g = fused(7, (4, 4), 64, F16, 2)
    table = fc.rotary_table(16, fc.rotary_frequencies(48))
    p = torch.arange(7, dtype=torch.int32, device="cuda")
    for interleaved in (False, True):
        y, gx = fc.rotary(x, table, p, interleaved), fc.rotary(g, table, p, interleaved, inverse=True)
        left, right = (y.double() * g.double()).sum(), (x.double() * gx.double()).sum()
        bound = 2.0 ** -10 * ((y.double() * g.double()).abs().sum() + (x.double() * gx.double()).abs().sum())
        assert abs(left - right) <= bound


def test_rotary_table_has_the_angles_of_64_bits(fc):
    for method in ("none", "linear", "base", "bands", "ramp"):
        f = fc.rotary_frequencies(64, method=method, factor=4.0, original=2048, low=1.0, high=32.0 if method == "ramp" else 4.0)
        table = fc.rotary_table(100001, f, 1.25).cpu()
        angle = torch.arange(100001, dtype=torch.float64)[:, None] * f
        want = torch.cat([angle.cos(), angle.sin()], 1) * 1.25
        assert (table.double() - want).abs().max() <= 2.0 ** -24 * 1.25 * 2


# ---- the cache ----

def codes_of(x, quantizer):
    """fp32 -> codes, nearest even"""
    if quantizer == SYM:
        return x.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def values_of(codes, quantizer, dtype=torch.float32):
    return codes.view(torch.int8 if quantizer == SYM else torch.float8_e4m3fn).to(dtype)


def append_one(codes, scales, table, offsets, held, x, quantizer, limit):
    """the header's formulas, page by page and token by token; x float32 [tokens, heads, dim], all on the CPU"""
    page = codes.shape[2]
    top = torch.tensor(TOP[quantizer])
    for b in range(len(held)):
        first = offsets[b]
        places = [(held[b] + i, first + i) for i in range(offsets[b + 1] - first)]
        places = [(p, t) for p, t in places if 0 <= p < min(limit, table.shape[1] * page)]
        for index in sorted({p // page for p, _ in places}):
            mine = [(p % page, t) for p, t in places if p // page == index]
            id = int(table[b, index])
            if not 0 <= id < codes.shape[0]:
                continue
            filled = mine[0][0]
            most = torch.stack([x[t] for _, t in mine]).abs().amax((0, 2))
            now = torch.maximum(most / top, torch.full_like(most, FLT_MIN))
            if filled:
                before = scales[id].clone()
                now = torch.fmax(now, before)                                    # a NaN scale says nothing
                for h in range(codes.shape[1]):
                    if now[h] > before[h]:
                        codes[id, h, :filled] = codes_of(values_of(codes[id, h, :filled], quantizer) * (before[h] / now[h]), quantizer)
            inverse = torch.ones_like(now) / now
            scales[id] = now
            for slot, t in mine:
                codes[id, :, slot] = codes_of(x[t] * inverse[:, None], quantizer)


def new_cache(pages, heads, page, dim, seed=0, fill=None):
    """junk: whatever a page held before, NaN codes among it"""
    c = [torch.randint(0, 256, (pages, heads, page, dim), generator=gen(seed + i), dtype=torch.uint8) if fill is None else
         torch.full((pages, heads, page, dim), fill, dtype=torch.uint8) for i in range(2)]
    s = [torch.full((pages, heads), math.nan) for _ in range(2)]
    return tuple(t.cuda() for t in (*c, *s))


def page_table(sequences, width, pages, seed):
    order = torch.randperm(pages, generator=gen(seed))[:sequences * width]
    return order.view(sequences, width).to(torch.int32)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("quantizer", [SYM, FP8])
@pytest.mark.parametrize("page,dim,rotary,interleaved", [(16, 128, 128, False), (32, 64, 32, True), (64, 128, 0, False), (16, 256, 18, False),
                                                         (64, 256, 256, True), (16, 64, 12, True)])
def test_append_matches_the_formula_bit_for_bit(fc, dtype, quantizer, page, dim, rotary, interleaved):
    heads = 3
    # steps of one cache: prompts (one of them empty), single tokens, uneven ones; the last one finds a full page, an absent slot
    steps = [[5, 0, page + 1, 2 * page], [1, 1, 1, 1], [1, 2, page, 1], [1, 1, 1, 1], [page - 7, 1, 3, page]]
    width = 5
    table = page_table(4, width, 4 * width + 2, 3)
    cache = new_cache(4 * width + 2, heads, page, dim)
    want = [t.cpu().clone() for t in cache]
    angles = fc.rotary_table(width * page, fc.rotary_frequencies(rotary)) if rotary else None
    held = [0, 0, 0, 0]
    for n, new in enumerate(steps):
        print("append", dtype, quantizer, page, dim, rotary, interleaved, "step", n, flush=True)
        k, v = fused(sum(new), (heads, heads), dim, dtype, n, 1.0 + 2 * n)       # larger every step: scales grow
        k[:, 1] *= 0                                                                # a head of zeros
        offsets = [0] + [int(i) for i in np.cumsum(new)]
        got = fc.cache_append(k, v, cache, table.cuda(), ints(offsets), ints(held), max(new), quantizer, angles, interleaved)
        assert got is cache
        positions = torch.cat([torch.arange(h, h + c) for h, c in zip(held, new)])
        turned_k = turned(k.float().cpu(), angles.cpu(), positions, interleaved) if rotary else k.float().cpu()
        append_one(want[0], want[2], table, offsets, held, turned_k, quantizer, width * page)
        append_one(want[1], want[3], table, offsets, held, v.float().cpu(), quantizer, width * page)
        for name, a, b in zip(("k", "v"), cache[:2], want[:2]):
            assert torch.equal(a.cpu(), b), name
        for a, b in zip(cache[2:], want[2:]):
            assert same(a, b)
        held = [h + c for h, c in zip(held, new)]


def test_append_leaves_out_what_has_no_place(fc):
    page, heads, dim, quantizer = 16, 2, 64, SYM
    table = torch.tensor([[0, 1], [2, -1], [9, 4], [5, 6], [7, 8]], dtype=torch.int32)      # no page, a page that is not there
    new, held = [3, 20, 2, 40, 4], [-2, 0, 0, 10, 30]
    offsets = [0] + [int(i) for i in np.cumsum(new)]
    for rows in (32, 13):                                                        # page table, then rotation table ends first
        cache = new_cache(9, heads, page, dim)
        want = [t.cpu().clone() for t in cache]
        k, v = fused(sum(new), (heads, heads), dim, BF16, rows)
        angles = fc.rotary_table(rows, fc.rotary_frequencies(dim))
        fc.cache_append(k, v, cache, table.cuda(), ints(offsets), ints(held), 40, quantizer, angles)
        positions = torch.cat([torch.arange(h, h + c) for h, c in zip(held, new)])
        append_one(want[0], want[2], table, offsets, held, turned(k.float().cpu(), angles.cpu(), positions, False), quantizer, min(rows, 32))
        append_one(want[1], want[3], table, offsets, held, v.float().cpu(), quantizer, min(rows, 32))
        for a, b in zip(cache, want):
            assert torch.equal(a.cpu().view(torch.uint8), b.view(torch.uint8))


def check(got, want, weight, dtype, bf16_weights):
    """want, weight = sum w |v|: float64"""
    u = 2.0 ** -9 if dtype == BF16 else 2.0 ** -11
    uw = 2.0 ** -9 if bf16_weights else 2.0 ** -11
    bound = 2 * ((uw + 2.0 ** -11) * weight + u * want.abs()) + (0.0 if dtype == BF16 else 2.0 ** -23)
    got = got.double().cpu()
    assert bool(torch.isfinite(got).all())
    worst = ((got - want).abs() / bound.clamp(min=1e-30)).max().item() if got.numel() else 0.0
    assert bool(((got - want).abs() <= bound).all()), worst


def cache_reference(q, cache, table, offsets, held, quantizer, scale):
    """64 bits; returns the outputs and sum w |v|"""
    q = q.double().cpu()
    codes, scales = [t.cpu() for t in cache[:2]], [t.cpu().double() for t in cache[2:]]
    heads, page, dim = codes[0].shape[1:]
    group = q.shape[1] // heads
    out, weight = torch.zeros_like(q), torch.zeros_like(q)
    for b in range(len(held)):
        n = offsets[b + 1] - offsets[b]
        total = min(held[b] + n, table.shape[1] * page)
        if total <= 0:
            continue
        ids = table[b, :-(-total // page)].long()
        k, v = (((values_of(c[ids], quantizer, torch.float64) * s[ids][..., None, None]).transpose(0, 1).reshape(heads, -1, dim))[:, :total]
                for c, s in zip(codes, scales))
        for i in range(n):
            sees = min(held[b] + i + 1, total)
            if sees <= 0:
                continue
            x = q[offsets[b] + i].view(heads, group, dim)
            w = torch.softmax(x @ k[:, :sees].transpose(1, 2) * scale, -1)
            out[offsets[b] + i] = (w @ v[:, :sees]).reshape(-1, dim)
            weight[offsets[b] + i] = (w @ v[:, :sees].abs()).reshape(-1, dim)
    return out, weight


def filled_cache(pages, heads, page, dim, quantizer, held, new, table, seed):
    """codes and scales of the tokens there are; beyond them NaN bytes (E4M3), -128 and NaN scales"""
    cache = [t.cpu() for t in new_cache(pages, heads, page, dim, fill=0xFF if quantizer == FP8 else 0x80)]
    g = gen(seed)
    for b in range(len(held)):
        total = min(held[b] + new[b], table.shape[1] * page)
        for index in range(-(-max(total, 0) // page)):
            id, n = int(table[b, index]), min(page, total - index * page)
            for i in range(2):
                x = torch.randn((heads, n, dim), generator=g) * (36 if quantizer == SYM else 120)
                cache[i][id, :, :n] = codes_of(x.clamp(-TOP[quantizer], TOP[quantizer]), quantizer)
                cache[2 + i][id] = (0.2 + 1.5 * torch.rand(heads, generator=g)) / (36 if quantizer == SYM else 120)
    return tuple(t.cuda() for t in cache)


CACHES = [
    # heads, group, dim, page, held, new, hints (queries, longest) or None
    (1, 1, 64, 16, [0], [1], None),
    (2, 4, 128, 16, [128], [1], None),
    (2, 8, 128, 64, [1499, 0, 63, 64, 300], [1, 1, 1, 1, 1], None),
    (1, 5, 128, 32, [7, 700, 31], [3, 5, 1], None),
    (2, 8, 64, 16, [33, 0, 16], [5, 40, 0], None),                    # several row blocks; a prompt; nothing new
    (3, 2, 256, 32, [259, 5], [1, 2], None),
    (1, 4, 128, 16, [-1, 200, -3, 0], [1, 1, 2, 1], None),            # empty slots of a padded batch
    (1, 3, 128, 64, [5000, 17], [2, 2], None),
    (1, 8, 128, 16, [900, 40], [9, 2], (1, 50)),                      # more queries and tokens than announced
    (2, 1, 64, 64, [20000], [1], None),
    (1, 5, 256, 64, [3000, 900], [1, 4], None),
    # contexts shared out evenly, cut anywhere; some of them empty, short, or with several queries
    (8, 2, 64, 64, [25000, 3, 24000, -1, 700, 8, 15999], [1, 1, 1, 1, 2, 0, 3], None),
    (8, 5, 128, 32, [24000, 21007, 22000, 0], [8, 1, 9, 20], None),   # three tiles of rows at a time
    (2, 4, 256, 16, [131070, 130000], [1, 1], None),
]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("quantizer", [SYM, FP8])
@pytest.mark.parametrize("case", range(len(CACHES)))
def test_cache_attention_matches_its_definition(fc, dtype, quantizer, case):
    heads, group, dim, page, held, new, hints = CACHES[case]
    print("cache attention", dtype, quantizer, CACHES[case], flush=True)
    width = max(1, max(-(-(h + n) // page) for h, n in zip(held, new)))
    pages = len(held) * width + 1
    table = page_table(len(held), width, pages, case)
    cache = filled_cache(pages, heads, page, dim, quantizer, held, new, table, case)
    offsets = [0] + [int(i) for i in np.cumsum(new)]
    q, _ = fused(sum(new), (heads * group, 1), dim, dtype, 50 + case)
    queries, longest = hints or (max(new), max(1, max(h + n for h, n in zip(held, new))))
    got = fc.cache_attention(q, cache, table.cuda(), ints(offsets), ints(held), queries, longest, quantizer)
    want, weight = cache_reference(q, cache, table, offsets, held, quantizer, dim ** -0.5)
    check(got, want, weight, dtype, False)
    again = fc.cache_attention(q, cache, table.cuda(), ints(offsets), ints(held), queries, longest, quantizer)
    assert same(got, again)


@pytest.mark.parametrize("quantizer", [SYM, FP8])
def test_cache_attention_extremes(fc, quantizer):
    # queries over bfloat16's range (rows that binary16 could not hold), pages of very different scales, another softmax scale
    heads, group, dim, page, held, new = 2, 4, 128, 16, [100, 450], [1, 1]
    table = page_table(2, 29, 60, 1)
    cache = filled_cache(60, heads, page, dim, quantizer, held, new, table, 5)
    cache[2].mul_(torch.logspace(-6, 0, 60, device="cuda")[:, None])
    cache[3].mul_(torch.logspace(-5, 3, 60, device="cuda")[:, None])
    q, _ = fused(2, (heads * group, 1), dim, BF16, 9)
    q = (q.float() * torch.logspace(-30, 8, 8, device="cuda")[None, :, None]).to(BF16)
    scale = 1e-8
    got = fc.cache_attention(q, cache, table.cuda(), ints([0, 1, 2]), ints(held), 1, 451, quantizer, scale=scale)
    want, weight = cache_reference(q, cache, table, [0, 1, 2], held, quantizer, scale)
    check(got, want, weight, BF16, False)


@pytest.mark.parametrize("quantizer", [SYM, FP8])
@pytest.mark.parametrize("heads,group,dim,page,held,new", [(2, 4, 128, 16, [100, 450], [1, 1]), (1, 5, 64, 32, [3000], [3]),
                                                           (8, 2, 256, 64, [30000, 5], [1, 2])])
def test_cache_attention_over_the_range_of_bfloat16(fc, quantizer, heads, group, dim, page, held, new):
    # page scales up to where sums of that many tokens still fit fp32, down to the least one, and pages of both in one context
    width = max(-(-(h + n) // page) for h, n in zip(held, new))
    pages = len(held) * width + 1
    table = page_table(len(held), width, pages, 1)
    q, _ = fused(sum(new), (heads * group, 1), dim, BF16, 9)
    offsets = [0] + [int(i) for i in np.cumsum(new)]
    for name, scales in (("1e9", [1e9]), ("1e12", [1e12]), ("1e30", [1e30]), ("1e-30", [1e-30]), ("least", [FLT_MIN]), ("least, 1e30", [FLT_MIN, 1e30]),
                         ("1, 1e20", [1.0, 1.0, 1e20]), ("many", [10.0 ** i for i in range(-37, 31)])):
        cache = filled_cache(pages, heads, page, dim, quantizer, held, new, table, 5)
        cache[3].copy_(torch.tensor([scales[i % len(scales)] for i in range(pages)], device="cuda")[:, None].expand(-1, heads))
        print("cache attention", quantizer, heads, group, dim, page, held, new, name, flush=True)
        got = fc.cache_attention(q, cache, table.cuda(), ints(offsets), ints(held), max(new), max(h + n for h, n in zip(held, new)), quantizer)
        want, weight = cache_reference(q, cache, table, offsets, held, quantizer, dim ** -0.5)
        check(got, want, weight, BF16, False)


def peaked_cache(heads, dim, page, quantizer, held, table, seed):
    """the first token of each sequence has the largest key code everywhere and a value of 0 in every other element; all other keys are 0"""
    cache = filled_cache(int(table.max()) + 2, heads, page, dim, quantizer, held, [1] * len(held), table, seed)
    for t in cache[2:]:
        t.fill_(2.0 ** -7)
    for b, n in enumerate(held):
        for index in range(-(-(n + 1) // page)):
            cache[0][int(table[b, index])] = 0
    first = table[:, 0].long()
    cache[0][first, :, 0] = codes_of(torch.tensor([TOP[quantizer]]), quantizer).cuda()
    cache[1][first, :, 0, ::2] = 0
    return cache


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("quantizer", [SYM, FP8])
@pytest.mark.parametrize("heads,group,dim,held", [(1, 1, 128, [1000]), (2, 4, 64, [3000, 40]), (1, 3, 256, [300]), (8, 2, 128, [30000, 17, 29000])])
def test_cache_attention_of_one_token_far_above_the_rest(fc, dtype, quantizer, heads, group, dim, held):
    # what the elements have in which the first token is 0 comes from weights far below its own
    page = 64
    width = max(held) // page + 1
    table = page_table(len(held), width, len(held) * width + 1, 2)
    cache = peaked_cache(heads, dim, page, quantizer, held, table, 3)
    q = torch.ones((len(held), heads * group, dim), dtype=dtype, device="cuda")
    offsets = list(range(len(held) + 1))
    for above in (0.0, 9.4, 14.7, 17.6, 20.35, 21.3, 23.7, 25.6):                   # powers of two
        scale = above * math.log(2) / (dim * TOP[quantizer] * 2.0 ** -7) if above else dim ** -0.5 * 1e-3
        got = fc.cache_attention(q, cache, table.cuda(), ints(offsets), ints(held), 1, max(held) + 1, quantizer, scale=scale)
        print("cache attention", dtype, quantizer, heads, group, dim, held, above, flush=True)
        want, weight = cache_reference(q, cache, table, offsets, held, quantizer, scale)
        check(got, want, weight, dtype, False)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("quantizer", [SYM, FP8])
@pytest.mark.parametrize("heads,group,dim", [(2, 3, 64), (2, 8, 128), (2, 1, 256)])
@pytest.mark.parametrize("longest", [205, 6000, 1 << 20])                           # one workgroup a context, pieces, ranges
def test_cache_attention_sees_nothing_of_later_tokens(fc, dtype, quantizer, heads, group, dim, longest):
    # of several new tokens: later queries, and infinities and NaN among later keys, values and scales, change no bit of earlier rows
    page, held, new = 16, [62, 200], [5, 4]                                          # the third and no one's tokens begin a page
    table = page_table(2, 13, 27, 1)
    cache = filled_cache(27, heads, page, dim, quantizer, held, new, table, 4)
    q, _ = fused(9, (heads * group, 1), dim, dtype, 3)

    def attend(q, cache):
        return fc.cache_attention(q, cache, table.cuda(), ints([0, 5, 9]), ints(held), 5, longest, quantizer)

    clean = attend(q, cache)
    print("cache attention", dtype, quantizer, heads, group, dim, longest, flush=True)
    loud = q.clone()
    loud[2:5] *= 40                                                                  # raises maxima of the rows beside
    loud[7] = math.nan
    got = attend(loud, cache)
    assert same(got[:2], clean[:2]) and same(got[5:7], clean[5:7]) and same(got[8], clean[8]) and bool(torch.isnan(got[7]).all())
    last = int(table[0, 4])                                                          # page of the first sequence's tokens from 64 on
    for which, value in ((2, math.inf), (2, math.nan), (3, math.inf), (3, math.nan), (3, 1e30)):
        broken = tuple(t.clone() for t in cache)
        broken[which][last] = value
        got = attend(q, broken)
        assert same(got[:2], clean[:2]) and same(got[5:], clean[5:]), (which, value)
        if value != 1e30 and (which, value) != (2, math.inf):                        # (scores of minus infinity weigh nothing)
            assert not bool(torch.isfinite(got[2:5]).all(-1).any())
    if quantizer == FP8:
        broken = tuple(t.clone() for t in cache)
        broken[0][last, 0, 1, 3] = 0x7F                                              # token 65: key of one head, value of the other
        broken[1][last, 1, 1, dim - 2] = 0xFF
        got = attend(q, broken)
        assert same(got[:3], clean[:3]) and same(got[5:], clean[5:])
        assert bool(torch.isnan(got[3:5, :group]).all()) and bool(torch.isnan(got[3:5, group:, dim - 2]).all())


def test_cache_attention_beyond_32_bit_offsets(fc):
    heads, dim, page = 8, 128, 64
    pages = (1 << 32) // (heads * dim * page) + 40
    k = torch.empty((pages, heads, page, dim), dtype=torch.uint8, device="cuda")
    v = torch.empty_like(k)
    scales = [torch.full((pages, heads), 0.01, device="cuda") for _ in range(2)]
    table = torch.tensor([[pages - 1, 0, pages - 33], [pages - 2, 5, pages // 2 + 3]], dtype=torch.int32)
    kv = fused(2 * 150, (heads, heads), dim, F16, 4)
    cache = (k, v, *scales)
    fc.cache_append(kv[0], kv[1], cache, table.cuda(), ints([0, 150, 300]), ints([0, 0]), 150)
    q, _ = fused(2, (16, 1), dim, F16, 6)
    got = fc.cache_attention(q, cache, table.cuda(), ints([0, 1, 2]), ints([149, 149]), 1, 150)
    ids = table.flatten().long().cuda()
    small = tuple(t[ids].contiguous() for t in cache)
    renamed = torch.arange(6, dtype=torch.int32).view(2, 3)
    want, weight = cache_reference(q, small, renamed, [0, 1, 2], [149, 149], SYM, dim ** -0.5)
    check(got, want, weight, F16, False)


@pytest.mark.parametrize("form", ["whole", "pieces", "ranges"])
def test_cache_attention_stays_in_its_tensors(fc, form):
    # whatever offsets, lengths and page table are, only rows of q's tokens are written.  Ranges: sequences that overlap, with more
    # pairs of query and context together than 32 bits count
    heads, group, dim, page, tokens, guard = 1, 8, 64, 64, 4096, 100
    width = (1 << 20) // page
    cache = new_cache(3, heads, page, dim, fill=1)
    for s in cache[2:]:
        s.fill_(0.01)
    q, _ = fused(tokens, (heads * group, 1), dim, F16, 3)
    overlapping = [0, 4096] * 128 + [1000, 4096] * 128 + [1000]
    few = [[0, 5, 9000, -1, 4096], [4096, 0, 7, 3, 2 ** 31 - 1], [-2 ** 31, 3, 4097, 2, 1]]
    for offsets in [overlapping] if form == "ranges" else few:
        sequences = len(offsets) - 1
        held = [2 ** 31 - 1] * sequences if form == "ranges" else [500, 2 ** 31 - 1, -2 ** 31, 100]
        queries, longest = (tokens, 1 << 20) if form == "ranges" else (8, 300 if form == "whole" else 6000)
        table = torch.randint(-1, 4, (sequences, width if form == "ranges" else 10), generator=gen(1)).to(torch.int32)
        need = fc.cache_attention_workspace_bytes(tokens, sequences, heads, group, dim, queries, longest)
        assert (need == 0) == (form == "whole")
        print("cache attention", form, sequences, offsets[:5], need, flush=True)
        big = torch.full((guard + tokens + guard, heads * group, dim), 7.0, dtype=F16, device="cuda")
        space = torch.full((guard * 16 + need + guard * 16,), 7, dtype=torch.uint8, device="cuda")
        fc.cache_attention(q, cache, table.cuda(), ints(offsets), ints(held), queries, longest, out=big[guard:guard + tokens],
                           workspace=space[guard * 16:guard * 16 + need])
        assert bool((big[:guard] == 7).all()) and bool((big[guard + tokens:] == 7).all())
        assert bool((space[:guard * 16] == 7).all()) and bool((space[guard * 16 + need:] == 7).all())


# ---- prompts ----

def prompt_reference(q, k, v, lengths, causal, scale):
    q, k, v = (t.double().cpu() for t in (q, k, v))
    group = q.shape[1] // k.shape[1]
    out, weight = torch.zeros_like(q), torch.zeros_like(q)
    at = 0
    for n in lengths:
        part = slice(at, at + n)
        kk, vv = (t[part].transpose(0, 1).repeat_interleave(group, 0) for t in (k, v))
        s = q[part].transpose(0, 1) @ kk.transpose(1, 2) * scale
        if causal:
            s = s.masked_fill(~torch.ones((n, n), dtype=torch.bool).tril(), -math.inf)
        w = torch.softmax(s, -1)
        out[part], weight[part] = (w @ vv).transpose(0, 1), (w @ vv.abs()).transpose(0, 1)
        at += n
    return out, weight


PROMPTS = [
    # heads, group, dim, lengths
    (1, 1, 64, [1]),
    (1, 2, 128, [2, 1, 0, 33]),
    (2, 4, 128, [130]),
    (1, 8, 64, [31, 32, 33, 127, 128, 129]),
    (3, 1, 128, [257, 64, 5, 600]),
    (2, 5, 64, [191, 0, 0, 320]),
    (1, 1, 128, [1537]),
    # more rows than fit the chip once, and than fit it twice
    (8, 4, 128, [400, 397, 700, 1, 502]),
    (8, 4, 64, [400, 397, 700, 1, 502]),
    (16, 4, 128, [300, 321, 330, 64, 500, 129, 31, 640, 444, 441]),
]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", range(len(PROMPTS)))
def test_prompt_attention_matches_its_definition(fc, dtype, causal, case):
    heads, group, dim, lengths = PROMPTS[case]
    print("prompt attention", dtype, causal, PROMPTS[case], flush=True)
    q, k, v = fused(sum(lengths), (heads * group, heads, heads), dim, dtype, case)
    got = fc.prompt_attention(q, k, v, offsets_of(lengths), max(lengths), causal)
    want, weight = prompt_reference(q, k, v, lengths, causal, dim ** -0.5)
    check(got, want, weight, dtype, dtype == BF16)
    assert same(got, fc.prompt_attention(q, k, v, offsets_of(lengths), max(lengths), causal))


def test_prompt_attention_keeps_sequences_apart(fc):
    # infinities and NaN of one request change no bit of another's rows
    lengths = [40, 100, 64, 7]
    q, k, v = fused(sum(lengths), (4, 2, 2), 128, F16, 3)
    q, k, v = q.clone(), k.clone(), v.clone()
    clean = fc.prompt_attention(q, k, v, offsets_of(lengths), 100)
    for t in (q, k, v):
        t[40:140:3] = math.nan
        t[41:140:3] = math.inf
    got = fc.prompt_attention(q, k, v, offsets_of(lengths), 100)
    assert same(got[:40], clean[:40]) and same(got[140:], clean[140:])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dim,lengths", [(128, [70, 300]), (64, [513])])
def test_prompt_attention_sees_nothing_of_later_tokens(fc, dtype, dim, lengths):
    # infinities and NaN among later tokens, in the same tile and in others: rows before them are what they would be without
    tokens, heads, group = sum(lengths), 2, 2
    q, k, v = (t.clone() for t in fused(tokens, (heads * group, heads, heads), dim, dtype, 7))
    bad = 50                                                      # in the first sequence; 45 and 200 in the second
    places = [bad] if len(lengths) == 1 else [bad, lengths[0] + 45, lengths[0] + 200]
    want, weight = prompt_reference(q, k, v, lengths, True, dim ** -0.5)
    for i, p in enumerate(places):
        v[p, 0, 3 + i] = (math.nan, math.inf, -math.inf)[i]
        k[p, 1, 5] = math.nan
    got = fc.prompt_attention(q, k, v, offsets_of(lengths), max(lengths))
    at = 0
    for n in lengths:
        first = min(p for p in places if at <= p < at + n)
        check(got[at:first], want[at:first], weight[at:first], dtype, dtype == BF16)
        assert not bool(torch.isfinite(got[first:at + n, :group, 3:6]).all(-1).any())     # heads of the first key/value head
        assert bool(torch.isnan(got[first:at + n, group:]).all())
        clean = got[first:at + n, :group, 8:].double().cpu()
        assert bool(((clean - want[first:at + n, :group, 8:]).abs() <= 2.0 ** -6 * weight[first:at + n, :group, 8:] + 2.0 ** -6 * clean.abs()).all())
        at += n


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group,dim,n,first", [(1, 1, 128, 3000, 0), (2, 1, 64, 700, 0), (16, 4, 128, 1100, 0), (8, 8, 64, 1000, 0), (2, 4, 128, 20000, 0),
                                                     (2, 2, 128, 5000, 3333), (8, 8, 128, 1200, 700)])
def test_prompt_attention_of_one_token_far_above_the_rest(fc, dtype, causal, heads, group, dim, n, first):
    # Token `first` has a score of `above` powers of two over all others, which are alike, and a value of 0 in every other element: what
    # those elements have comes from weights far below its own.  The definition in 64 bits is then a quotient of running sums.
    v = torch.randn((n, heads, dim), generator=gen(n + dim)).to(dtype)
    v[first, :, ::2] = 0
    k = torch.zeros((n, heads, dim), dtype=dtype)
    k[first] = 1
    q = torch.ones((n, heads * group, dim), dtype=dtype, device="cuda")
    on_card = k.cuda(), v.cuda()
    for above in (9.4, 14.7, 17.6, 20.35, 21.3, 23.7, 25.6, 31.3, 38.5, 59.0):
        w = torch.ones(n, dtype=torch.float64)
        w[first] = 2.0 ** above
        sums = [((w[:, None, None] * x).cumsum(0) if causal else (w[:, None, None] * x).sum(0, keepdim=True).expand(n, -1, -1)) for x in (v.double(), v.double().abs())]
        total = w.cumsum(0)[:, None, None] if causal else w.sum()
        want, weight = ((x / total).repeat_interleave(group, 1) for x in sums)
        print("prompt attention", dtype, causal, heads, group, dim, n, first, above, flush=True)
        got = fc.prompt_attention(q, *on_card, ints([0, n]), n, causal, scale=above * math.log(2) / dim)
        check(got, want, weight, dtype, dtype == BF16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group,dim,lengths", [(1, 1, 128, [600, 37]), (1, 2, 64, [129, 900]), (16, 4, 64, [500, 470]), (16, 4, 128, [520, 480])])
def test_prompt_attention_with_peaks(fc, dtype, causal, heads, group, dim, lengths):
    # scores of tens: the running maximum rises by more than any slack, early and late, and falls far behind
    q, k, v = (t.clone() for t in fused(sum(lengths), (heads * group, heads, heads), dim, dtype, 21))
    q *= 8
    for n, loud in enumerate((3.0, 0.05, 1.5)):
        kk = k.clone()
        kk[n * 61:n * 61 + 200] *= loud                                              # stretches of loud and quiet keys
        kk[-150:] /= loud
        scale = dim ** -0.5 / max(1.0, loud)                                         # |score| < 64
        print("prompt attention", dtype, causal, heads, group, dim, lengths, loud, flush=True)
        got = fc.prompt_attention(q, kk, v, offsets_of(lengths), max(lengths), causal, scale=scale)
        want, weight = prompt_reference(q, kk, v, lengths, causal, scale)
        check(got, want, weight, dtype, dtype == BF16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads,group,dim,lengths", [(1, 2, 64, [70, 300]), (2, 1, 128, [65, 410]), (8, 8, 64, [130, 900]), (4, 8, 128, [64, 1700]), (16, 4, 128, [90, 3100])])
def test_no_bit_of_a_causal_row_depends_on_later_tokens(fc, dtype, heads, group, dim, lengths):
    # by 8 and 4 wavefronts, tiles of 32 and 64 tokens: louder queries, keys and values, infinities and NaN from token p of the last sequence on
    q, k, v = (t.clone() for t in fused(sum(lengths), (heads * group, heads, heads), dim, dtype, 30))
    offsets, at = offsets_of(lengths), lengths[0]
    clean = fc.prompt_attention(q, k, v, offsets, max(lengths))
    for p in (1, 17, 32, 47, 63, lengths[1] - 3):
        for what in ("loud", "inf", "nan", "mixed"):
            qq, kk, vv = q.clone(), k.clone(), v.clone()
            if what == "loud":
                for t in (qq, kk, vv):
                    t[at + p:at + p + 20] *= 30
            elif what == "mixed":
                qq[at + p], kk[at + p + 1, :, 3], vv[at + p, :, 1], vv[at + p, :, 2] = math.nan, -math.inf, math.inf, math.nan
                vv[at + p + 2, :, 1] = -math.inf
            else:
                vv[at + p, :, dim - 1] = math.inf if what == "inf" else math.nan
            got = fc.prompt_attention(qq, kk, vv, offsets, max(lengths))
            print("prompt attention", dtype, heads, group, dim, lengths, p, what, flush=True)
            assert same(got[:at + p], clean[:at + p]), (p, what)
            if what in ("inf", "nan"):
                assert same(got[..., :dim - 1], clean[..., :dim - 1])
                rest = got[at + p:, :, dim - 1]
                assert bool((rest == math.inf if what == "inf" else torch.isnan(rest)).all()), (p, what)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group,dim", [(1, 2, 64), (16, 4, 128)])         # tokens split over wavefronts, and not
def test_prompt_attention_stays_in_its_tensors(fc, causal, heads, group, dim):
    # whatever the offsets are, only rows of q's tokens are written; tokens of no sequence are left alone
    tokens, guard = 2000, 200
    q, k, v = fused(tokens, (heads * group, heads, heads), dim, F16, 8)
    for offsets in ([0, 1000, 1200, -100000, 2000], [2000, 0, 2000, 0], [-5, 300, 3000, 2000], [700, 650, 1999, 100, 2 ** 31 - 1],
                    [1900, 2000, 5, -2 ** 31], [2001, 2002]):
        print("prompt attention", causal, heads, group, dim, offsets, flush=True)
        big = torch.full((guard + tokens + guard, heads * group, dim), 7.0, dtype=F16, device="cuda")
        fc.prompt_attention(q, k, v, ints(offsets), 1000, causal, out=big[guard:guard + tokens])
        assert bool((big[:guard] == 7).all()) and bool((big[guard + tokens:] == 7).all())
    lengths = [40, 333]
    big = torch.full((tokens, heads * group, dim), 7.0, dtype=F16, device="cuda")
    fc.prompt_attention(q, k, v, ints([900, 940, 1273]), 333, causal, out=big)
    assert bool((big[:900] == 7).all()) and bool((big[1273:] == 7).all())
    want, weight = prompt_reference(q[900:1273], k[900:1273], v[900:1273], lengths, causal, dim ** -0.5)
    check(big[900:1273], want, weight, F16, False)


# ---- calls ----

def test_strided_operands_and_results(fc):
    # heads outside tokens, gaps between both, results into a slice of a larger tensor
    tokens, heads, dim = 50, 2, 64
    q = torch.randn((8, tokens, dim), generator=gen(1)).to(F16).cuda().transpose(0, 1)
    k = torch.randn((tokens, 3, heads, dim + 8), generator=gen(2)).to(F16).cuda()[:, 1, :, :dim]
    v = torch.randn((tokens, heads, dim), generator=gen(3)).to(F16).cuda()
    big = torch.full((tokens, 12, dim), 5.0, dtype=F16, device="cuda")
    out = big[:, 2:10]
    assert fc.prompt_attention(q, k, v, ints([0, tokens]), tokens, out=out) is out
    want, weight = prompt_reference(q, k, v, [tokens], True, dim ** -0.5)
    check(out, want, weight, F16, False)
    assert bool((big[:, :2] == 5).all()) and bool((big[:, 10:] == 5).all())
    table = fc.rotary_table(64, fc.rotary_frequencies(dim))
    p = torch.arange(tokens, dtype=torch.int32, device="cuda")
    assert same(fc.rotary(q, table, p), fc.rotary(q.contiguous(), table, p))
    assert same(fc.rotary(k, table, p, out=out[:, :heads]), fc.rotary(k.contiguous(), table, p))
    cache, twin = new_cache(4, heads, 16, dim, 1), new_cache(4, heads, 16, dim, 1)
    pages = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    for c, kk in ((cache, k), (twin, k.contiguous())):
        fc.cache_append(kk, v, c, pages, ints([0, tokens]), ints([0]), tokens, table=table)
    for a, b in zip(cache, twin):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    y = fc.cache_attention(q[-3:], cache, pages, ints([0, 3]), ints([47]), 3, 50, out=big[:3, 2:10])
    assert same(y, fc.cache_attention(q[-3:].contiguous(), cache, pages, ints([0, 3]), ints([47]), 3, 50))


def test_a_step_on_another_stream_and_from_a_graph(fc):
    heads, group, dim, page, width = 2, 4, 128, 16, 40
    table = page_table(3, width, 3 * width, 0).cuda()
    angles = fc.rotary_table(width * page, fc.rotary_frequencies(dim))
    held, offsets = ints([500, 0, 77]), ints([0, 1, 2, 3])
    qkv = torch.randn((3, heads * (group + 2), dim), generator=gen(0)).to(BF16).cuda()
    q, k, v = qkv.split([heads * group, heads, heads], 1)
    start = filled_cache(3 * width, heads, page, dim, SYM, [500, 0, 77], [0, 0, 0], table.cpu(), 1)
    cache = tuple(t.clone() for t in start)
    turned_q, out = torch.empty_like(q.contiguous()), torch.empty_like(q.contiguous())
    space = torch.empty(max(16, fc.cache_attention_workspace_bytes(3, 3, heads, group, dim, 1, 501)), dtype=torch.uint8, device="cuda")

    def step():
        fc.rotary(q, angles, held, out=turned_q)
        fc.cache_append(k, v, cache, table, offsets, held, 1, SYM, angles)
        fc.cache_attention(turned_q, cache, table, offsets, held, 1, 501, SYM, out=out, workspace=space)

    def fresh(seed):
        qkv.copy_(torch.randn(qkv.shape, generator=gen(seed)))
        for a, b in zip(cache, start):
            a.copy_(b)
        out.fill_(7.0)

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        fresh(0)
        step()
    side.synchronize()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step()
    for seed in (0, 1, 2, 0, 3):
        fresh(seed)
        step()
        torch.cuda.synchronize()
        want, kept = out.clone(), [t.clone() for t in cache]
        fresh(seed)
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, want)
        for a, b in zip(cache, kept):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        if seed == 0:
            assert same(out, first)


def test_empty_calls(fc):
    q, k, v = fused(0, (4, 2, 2), 64, F16, 0)
    table = fc.rotary_table(4, fc.rotary_frequencies(64))
    assert fc.rotary(q, table, ints([])).shape == q.shape
    cache = new_cache(2, 2, 16, 64)
    before = [t.clone() for t in cache]
    pages = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    fc.cache_append(k, v, cache, pages, ints([0, 0]), ints([3]), 1)
    assert fc.cache_attention(q, cache, pages, ints([0, 0]), ints([3]), 1, 4).shape == q.shape
    assert fc.prompt_attention(q, k, v, ints([0, 0]), 1).shape == q.shape
    torch.cuda.synchronize()
    for a, b in zip(cache, before):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_refusals(fc):
    q, k, v = fused(8, (4, 2, 2), 64, F16, 0)
    o, held, pages = ints([0, 8]), ints([0]), torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    cache = new_cache(2, 2, 16, 64)
    table = fc.rotary_table(16, fc.rotary_frequencies(64))
    p = torch.arange(8, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        fc.rotary(q.float(), table, p)
    with pytest.raises(TypeError):
        fc.rotary(q, table, p.long())
    with pytest.raises(TypeError):
        fc.rotary(q.cpu(), table, p)
    with pytest.raises(ValueError):
        fc.rotary(q, table, p[:5])
    with pytest.raises(fc.FcError):
        fc.rotary(q[..., :48], table, p)                                          # more turned than there is
    with pytest.raises(ValueError):
        fc.rotary(q[..., 1:57], table[:, :32].contiguous(), p)                    # not aligned
    with pytest.raises(ValueError):
        fc.rotary(q, table, p, out=torch.empty((1, 4, 64), dtype=F16, device="cuda").expand(8, 4, 64))
    with pytest.raises(TypeError):
        fc.prompt_attention(q, k.bfloat16(), v.bfloat16(), o, 8)
    with pytest.raises(ValueError):
        fc.prompt_attention(q[:, :3], k, v, o, 8)                                 # 3 heads over 2
    with pytest.raises(ValueError):
        fc.prompt_attention(q, k[:7], v, o, 8)
    with pytest.raises(fc.FcError):
        fc.prompt_attention(q[..., :32], k[..., :32], v[..., :32], o, 8)          # head size
    with pytest.raises(ValueError):
        fc.cache_append(k, v, cache[:3], pages, o, held, 8)
    with pytest.raises(ValueError):
        fc.cache_append(k, v, cache, pages, o, ints([0, 0]), 8)
    with pytest.raises(ValueError):
        fc.cache_append(q, q, cache, pages, o, held, 8)                           # 4 heads into a cache of 2
    with pytest.raises(fc.FcError) as e:
        fc.cache_append(k, v, cache, pages, o, held, 8, fc.QUANTIZER_ASYM)
    assert e.value.code == -8
    with pytest.raises(fc.FcError):
        fc.cache_append(k, v, new_cache(2, 2, 8, 64), pages, o, held, 8)          # page of 8
    with pytest.raises(fc.FcError):
        fc.cache_attention(q, cache, pages, o, held, 0, 8)
    for scale in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(fc.FcError):
            fc.cache_attention(q, cache, pages, o, held, 8, 8, scale=scale)
        with pytest.raises(fc.FcError):
            fc.prompt_attention(q, k, v, o, 8, scale=scale)
    far = torch.empty(((1 << 26) + 128,), dtype=F16, device="cuda").as_strided((2, 2, 64), (1 << 26, 64, 1))
    with pytest.raises(fc.FcError):
        fc.prompt_attention(q[:2], far, far, ints([0, 2]), 2)            # token stride
    with pytest.raises(fc.FcError) as e:
        long = ints([30000])
        fc.cache_attention(q[:1], cache, pages, ints([0, 1]), long, 1, 30001, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -6
    torch.cuda.synchronize()


def test_calls_that_a_gradient_would_have_to_pass_are_refused(fc):
    q, k, v = (t.clone() for t in fused(8, (4, 2, 2), 64, BF16, 0))
    o, held, pages, p = ints([0, 8]), ints([0]), torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.arange(8, dtype=torch.int32, device="cuda")
    cache, table = new_cache(1, 2, 16, 64), fc.rotary_table(16, fc.rotary_frequencies(64))
    calls = {"rotary": lambda q, k, v: fc.rotary(q, table, p), "append": lambda q, k, v: fc.cache_append(k, v, cache, pages, o, held, 8)[0],
             "cache": lambda q, k, v: fc.cache_attention(q, cache, pages, o, held, 8, 8), "prompt": lambda q, k, v: fc.prompt_attention(q, k, v, o, 8)}
    uses = {"rotary": (0,), "append": (1, 2), "cache": (0,), "prompt": (0, 1, 2)}
    for name, call in calls.items():
        want = call(q, k, v).clone()
        for i in uses[name]:
            args = [q, k, v]
            args[i] = args[i].clone().requires_grad_()
            with pytest.raises(ValueError, match="gradient"):
                call(*args)
            args[i] = args[i] * 1                                                # not a leaf
            with pytest.raises(ValueError, match="gradient"):
                call(*args)
            with torch.no_grad():
                assert torch.equal(call(*args), want)
            assert torch.equal(call(*(t.detach() for t in args)), want)
    with pytest.raises(ValueError, match="gradient"):
        fc.rotary(q, table, p, out=torch.empty_like(q).requires_grad_())


def test_ordinary_calls_are_native(fc):
    # what the module does not take it returns as None, and the checked path makes the same call
    native = fc.binding._calls()
    qkv = fused(20, (4, 2, 2), 64, F16, 0)
    q, k, v = qkv
    table, p = fc.rotary_table(32, fc.rotary_frequencies(64)), torch.arange(20, dtype=torch.int32, device="cuda")
    o, held, pages = ints([0, 20]), ints([0]), torch.arange(2, dtype=torch.int32, device="cuda")[None]
    cache, twin = new_cache(2, 2, 16, 64), new_cache(2, 2, 16, 64)
    got = [native.rotary(q, table, p, False, False, None), native.cache_append(k, v, cache, pages, o, held, 20, SYM, table, False),
           native.cache_attention(q, cache, pages, o, held, 20, 20, SYM, None, None, None), native.prompt_attention(q, k, v, o, 20, True, None, None)]
    assert all(g is not None for g in got) and got[1] is cache
    assert native.rotary(q, table, p, 0, False, None) is None and native.prompt_attention(q, k, v, o, 20.0, True, None, None) is None
    binding, module = fc.binding, fc.binding._native
    binding._native = binding._NoNativeCalls()
    try:
        again = [fc.rotary(q, table, p), fc.cache_append(k, v, twin, pages, o, held, 20, SYM, table), fc.cache_attention(q, twin, pages, o, held, 20, 20),
                 fc.prompt_attention(q, k, v, o, 20)]
    finally:
        binding._native = module
    for i in (0, 2, 3):
        assert same(got[i], again[i])
    for a, b in zip(cache, twin):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_large_calls_equal_their_parts(fc):
    # inputs beyond the memory-side cache are read in another way
    tokens, heads, dim = 8200, 66, 128
    x = (torch.rand((tokens, heads, dim), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) - 0.5).half()
    assert x.numel() * 2 > 128 << 20
    table = fc.rotary_table(tokens, fc.rotary_frequencies(dim))
    positions = torch.arange(tokens, dtype=torch.int32, device="cuda")
    for interleaved in (False, True):
        whole = fc.rotary(x, table, positions, interleaved)
        for part in (slice(0, 3000), slice(3000, tokens)):
            assert torch.equal(whole[part], fc.rotary(x[part], table, positions[part], interleaved))
    kv_heads, page, lengths = 33, 32, [4100, 100, 4000]
    width = -(-max(lengths) // page)
    pages = torch.randperm(3 * width, generator=gen(1)).view(3, width).to(torch.int32)
    whole, parts = new_cache(3 * width, kv_heads, page, dim, fill=1), new_cache(3 * width, kv_heads, page, dim, fill=1)
    k, v = x[:, :kv_heads], x[:, kv_heads:]
    fc.cache_append(k, v, whole, pages.cuda(), offsets_of(lengths), ints([0, 0, 0]), max(lengths), FP8, table)
    at = 0
    for b, n in enumerate(lengths):
        fc.cache_append(k[at:at + n], v[at:at + n], parts, pages[b:b + 1].cuda(), ints([0, n]), ints([0]), n, FP8, table)
        at += n
    for a, b in zip(whole, parts):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_rotary_of_more_than_32_bits_of_elements(fc):
    # 2^32 elements and more: the last tokens of a call equal a call of them alone
    tokens, heads, dim = (1 << 20) + 5, 64, 64
    x = torch.empty((tokens, heads, dim), dtype=F16, device="cuda")
    x[-64:] = torch.randn((64, heads, dim), generator=gen(1)).to(F16).cuda()
    x[:64] = x[-64:]
    for turned_part, interleaved in ((64, False), (12, True)):
        table = fc.rotary_table(100, fc.rotary_frequencies(turned_part))
        positions = (torch.arange(tokens, device="cuda") % 100).to(torch.int32)
        y = fc.rotary(x, table, positions, interleaved)
        for part in (slice(0, 64), slice(tokens - 64, tokens)):
            assert same(y[part], fc.rotary(x[part], table, positions[part], interleaved))
        del y


# ---- the layer ----

@pytest.mark.parametrize("quantizer,bound", [(SYM, 0.06), (FP8, 0.09)])
def test_attention_layer_of_four_ranks(fc, quantizer, bound):
    # Prompts see no cache: binary16 activations and one INT8 all-reduce, whose groups of 128 span about six standard deviations in 255 steps,
    # twice: 6 / 255 / 12^0.5 * 2^0.5 = 0.010.  A decode step's keys and values are codes: signed ones have steps of 4.5 deviations / 127
    # (0.010 of each value, and the all-reduce's again; a page's growing scale rounds its first codes a few times more), E4M3 has 3
    # fraction bits (0.026).  The scores' errors move the weights by about as much again.  Together below 0.03 and 0.06; allowed 1.5 times.
    from paper_2412_04964_amd import attention_block
    errors, _, _ = attention_block.run(ranks=4, hidden=1024, query_heads=16, kv_heads=4, dim=64, prompts=3, length=150, steps=20, quantizer=quantizer)
    assert errors[0] < 0.02
    assert max(errors[1:]) < bound, errors
