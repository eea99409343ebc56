"""Attention of a chunk of new tokens over the paged cache and over itself, on the GPU, against its definition in 64 bits.

Tolerances, per element.  Half a step of a rounding: 2^-11 of the value in float16, 2^-8 in bfloat16 (u).  A weight is rounded once, u; the
fp32 score it comes from, below 2^6 in powers of two and added up from 128 products at most, is off by less than 2^-12, as are the exponential, the
logarithm of a page's scale and the sums together.  With E = sum_t w_t |v_t| that is (u + 2 * 2^-12) E, and the result's own rounding u |o|.  Float16
weights more than 2^8 below the largest of their 64 tokens have an absolute error instead, 2^-25 where the largest is at 2^-6 or more: 2^-19 of
that weight, so with F = sum over tiles of (largest w) * sum |v| another 2^-19 F.  Results below float16's normal numbers: 2^-25."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F16, BF16 = torch.float16, torch.bfloat16
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


def same(a, b):
    a, b = a.cpu().contiguous(), b.cpu().contiguous()
    return bool(((a.view(torch.int16) == b.view(torch.int16)) | (torch.isnan(a) & torch.isnan(b))).all())


def codes_of(x, quantizer):
    return x.round().clamp(-127, 127).to(torch.int8).view(torch.uint8) if quantizer == SYM else x.to(torch.float8_e4m3fn).view(torch.uint8)


def values_of(codes, quantizer):
    return codes.view(torch.int8 if quantizer == SYM else torch.float8_e4m3fn).double()


class Step:
    """a cache that holds `held` tokens of every sequence (what its pages have beyond them is NaN or -128, under scales of NaN), and `new` ones"""

    def __init__(self, heads, group, dim, page, held, new, dtype, quantizer, seed, room=0, spread=1.0, pad=3):
        g = gen(seed)
        self.heads, self.group, self.dim, self.page, self.held, self.new, self.quantizer = heads, group, dim, page, held, new, quantizer
        self.width = max(1, max(-(-max(h, 0) // page) for h in held)) + room
        pages = sum(-(-max(h, 0) // page) for h in held) + pad
        order = torch.randperm(pages, generator=g).tolist()
        self.table = torch.full((len(held), self.width), -1, dtype=torch.int32)
        cache = [torch.full((pages, heads, page, dim), 0x80 if quantizer == SYM else 0xFF, dtype=torch.uint8) for _ in range(2)]
        cache += [torch.full((pages, heads), float("nan")) for _ in range(2)]
        for b, h in enumerate(held):
            for i in range(-(-max(h, 0) // page)):
                id, n = order.pop(), min(page, h - i * page)
                self.table[b, i] = id
                for c in range(2):
                    x = torch.randn((heads, n, dim), generator=g) * TOP[quantizer] / 3.6
                    cache[c][id, :, :n] = codes_of(x.clamp(-TOP[quantizer], TOP[quantizer]), quantizer)
                    cache[2 + c][id] = (0.2 + 1.5 * torch.rand(heads, generator=g)) * 3.6 / TOP[quantizer]
        self.cache = tuple(t.cuda() for t in cache)
        qkv = (torch.randn((sum(new), heads * (group + 2), dim), generator=g) * spread).to(dtype).cuda()
        self.q, self.k, self.v = qkv[:, :heads * group], qkv[:, heads * group:heads * (group + 1)], qkv[:, heads * (group + 1):]
        self.longest = max(1, max(max(h, 0) + n for h, n in zip(held, new)))

    def call(self, fc, **more):
        more = {"longest": self.longest, **more}
        longest = more.pop("longest")
        return fc.chunk_attention(self.q, self.k, self.v, self.cache, self.table.cuda(), offsets_of(self.new), ints(self.held), longest, self.quantizer, **more)

    def exact(self, scale=None):
        """outputs, E and F of the docstring, in 64 bits"""
        scale = self.dim ** -0.5 if scale is None else scale
        out = torch.zeros(self.q.shape, dtype=torch.float64, device="cuda")
        weight, tiles = torch.zeros_like(out), torch.zeros_like(out)
        at = 0
        for b, (h, n) in enumerate(zip(self.held, self.new)):
            skip, have = max(0, -h), max(0, min(h, self.width * self.page))
            ids = self.table[b, :-(-have // self.page)].long().cuda()
            for head in range(self.heads):
                k, v = (torch.cat([(values_of(c[ids, head], self.quantizer) * s[ids, head].double()[:, None, None]).reshape(-1, self.dim)[:have], x[at:at + n, head].double()])
                        for c, s, x in ((self.cache[0], self.cache[2], self.k), (self.cache[1], self.cache[3], self.v)))
                i = torch.arange(n, device="cuda")
                seen = torch.cat([torch.ones((n, have), dtype=torch.bool, device="cuda") & (i[:, None] >= skip), (i[None] <= i[:, None]) & (i[None] >= skip)], 1)
                for g in range(self.group):
                    score = (self.q[at:at + n, head * self.group + g].double() @ k.t() * scale).masked_fill(~seen, float("-inf"))
                    w = torch.softmax(score, -1).nan_to_num(0.0)
                    q = head * self.group + g
                    out[at:at + n, q] = w @ v
                    weight[at:at + n, q] = w @ v.abs()
                    for t in range(0, have + n, 64):
                        tiles[at:at + n, q] += w[:, t:t + 64].amax(-1, keepdim=True) * v[t:t + 64].abs().sum(0)
            at += n
        return out, weight, tiles


def check(got, want, weight, tiles):
    u = torch.finfo(got.dtype).eps / 2
    bound = (u + 2.0 ** -11) * weight + u * want.abs()
    if got.dtype == F16:
        bound += 2.0 ** -19 * tiles + 2.0 ** -25
    assert bool(torch.isfinite(got).all())
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (off / bound.clamp(min=1e-300)).max().item()


STEPS = [
    # heads, group, dim, page, held, new, announced longest or None
    (1, 1, 64, 16, [0], [1], None),
    (1, 1, 128, 16, [1], [1], None),
    (2, 4, 128, 16, [129], [17], None),
    (2, 8, 128, 16, [1023], [64], None),
    (1, 5, 128, 32, [64, 65, 63], [65, 1, 0], None),                  # whole tiles, one more and one less; nothing new
    (2, 8, 64, 64, [700, 0, 16, 300], [130, 257, 5, 31], None),       # one without a cache
    (3, 2, 64, 32, [2049], [129], None),
    (1, 4, 128, 16, [-1, 200, -3, 0, -5], [1, 1, 2, 1, 70], None),    # padded slots; tokens without a place before those that have one
    (8, 4, 128, 64, [4000, 0, 17, 1500], [100, 700, 33, 512], None),
    (1, 16, 128, 16, [900], [40], 10),                                # more than announced
    (2, 1, 128, 16, [5000, 1], [3, 1000], None),
    (5, 3, 64, 16, [511, 1025, 0], [127, 3, 400], 1),
    (1, 200, 64, 16, [100], [9], None),                               # more query heads than a workgroup has rows
    (2, 2, 64, 16, [40] * 150, [1 + b % 3 for b in range(150)], None),         # more sequences than lanes
    (1, 8, 128, 16, [30000], [7], None),                              # few rows over a long context
    (8, 8, 64, 16, [100, 0, 333, 64, 1, 500], [200, 150, 33, 257, 1, 259], None),        # many items
    (8, 8, 128, 32, [0, 70, 333, 64, 1, 500], [200, 150, 33, 257, 1, 259], None),
]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("quantizer", [SYM, FP8])
@pytest.mark.parametrize("case", range(len(STEPS)))
def test_chunk_attention_matches_its_definition(fc, dtype, quantizer, case):
    *shape, longest = STEPS[case]
    print("chunk", dtype, quantizer, STEPS[case][:6], flush=True)
    s = Step(*shape, dtype, quantizer, case)
    want = s.exact()
    for announced in (s.longest, 3000, 1 << 20, 1) if longest is None else (longest,):        # items cut or not, workgroups of four or eight wavefronts
        got = s.call(fc, longest=announced)
        check(got, *want)
        assert same(got, s.call(fc, longest=announced))
    if case in (2, 7):                                   # another softmax scale
        check(s.call(fc, scale=0.5), *s.exact(0.5))


@pytest.mark.parametrize("announced", [None, 1 << 20])                 # workgroups of four wavefronts, and of eight
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("quantizer", [SYM, FP8])
def test_pages_of_very_different_scales(fc, announced, dtype, quantizer):
    # key scales change what is seen, value scales what it counts for; a page of zeros under the least scale counts in the sum of weights
    s = Step(2, 4, 128, 16, [600, 1200], [40, 70], dtype, quantizer, 3)
    g = gen(9)
    ks, vs = s.cache[2], s.cache[3]
    ks *= torch.exp2(torch.randint(-6, 2, ks.shape, generator=g).float()).cuda()
    vs *= torch.exp2(torch.randint(-9, 9, vs.shape, generator=g).float()).cuda()
    for i in (3, 17):
        id = int(s.table[1, i])
        s.cache[0][id] = 0
        s.cache[1][id] = 0
        ks[id] = vs[id] = torch.finfo(torch.float32).tiny
    check(s.call(fc, longest=announced or s.longest), *s.exact())
    # values far below and far above: float32 has the range for their sums (float16 results have not)
    if dtype == BF16:
        for factor in (2.0 ** -60, 2.0 ** 60):
            t = Step(1, 2, 64, 16, [500], [30], dtype, quantizer, 4)
            t.cache[3].mul_(factor)
            t.v.mul_(factor)
            check(t.call(fc, longest=announced or t.longest), *t.exact())


@pytest.mark.parametrize("announced", [None, 1 << 20])                 # workgroups of four wavefronts, and of eight
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads,group,dim,held,new", [(1, 4, 128, [700], [100]), (2, 1, 64, [0, 5000], [200, 3])])
def test_one_token_far_above_the_rest(fc, announced, dtype, heads, group, dim, held, new):
    # a peak in the cache or among the new tokens; the weights beside it, 2^-20 of it and less, have to be right where the peak's value is zero
    for place in ("cached", "new"):
        s = Step(heads, group, dim, 16, held, new, dtype, SYM, 5)
        b = len(held) - 1 if place == "cached" else 0
        off = sum(new[:b])
        s.q[off:off + new[b]].abs_()
        if place == "cached":
            id = int(s.table[b, held[b] // 32])
            s.cache[0][id, :, 5] = 127
            s.cache[1][id, :, 5] = 0
            s.cache[2][id] = 40 / 127 / dim ** 0.5
        else:
            s.k[off + 1] = 40 / dim ** 0.5
            s.v[off + 1] = 0
        want, weight, tiles = s.exact()
        check(s.call(fc, longest=announced or s.longest), want, weight, tiles)


@pytest.mark.parametrize("announced", [None, 1 << 20])                 # workgroups of four wavefronts, and of eight
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads,group,dim,held,new", [(2, 4, 128, [100, 0], [70, 200]), (1, 1, 64, [0], [300]), (1, 8, 128, [-3, 1000], [60, 17])])
def test_no_bit_of_a_row_depends_on_later_tokens(fc, announced, dtype, heads, group, dim, held, new):
    s = Step(heads, group, dim, 16, held, new, dtype, FP8, 6)
    plain = s.call(fc, longest=announced or s.longest)
    check(plain, *s.exact())
    off = 0
    for b, n in enumerate(new):
        first = max(0, -held[b])
        for at, value in ((n - 1, float("nan")), (n // 2, float("inf")), (n // 2, -60000.0), (first, float("nan"))):
            k, v = s.k.clone(), s.v.clone()
            s.k[off + at:off + n], s.v[off + at:off + n] = value, value
            got = s.call(fc, longest=announced or s.longest)
            rows = list(range(off, off + at)) + list(range(0, off)) + list(range(off + n, sum(new)))
            assert same(got[rows], plain[rows]), (b, at, value)
            if value == float("inf"):                    # a weight above zero of an infinity, and scores of either sign
                assert not torch.isfinite(got[off + at:off + n]).any()
            s.k.copy_(k)
            s.v.copy_(v)
        # tokens without a place
        k, v = s.k.clone(), s.v.clone()
        s.k[off:off + first], s.v[off:off + first] = float("nan"), float("-inf")
        assert same(s.call(fc, longest=announced or s.longest), plain) and not plain[off:off + first].any()
        s.k.copy_(k)
        s.v.copy_(v)
        off += n
    # values alone: the weights are finite, so an infinity is the result of all that see it, and only theirs
    v = s.v.clone()
    s.v[new[0] // 2, 0, 3] = float("inf")
    got = s.call(fc, longest=announced or s.longest)
    want = plain.clone()
    want[new[0] // 2:new[0], :group, 3] = float("inf")
    assert same(got, want)
    s.v.copy_(v)


@pytest.mark.parametrize("announced", [None, 1 << 20])                 # workgroups of four wavefronts, and of eight
def test_nan_in_the_cache_is_seen_by_its_own_rows_only(fc, announced):
    s = Step(2, 4, 128, 16, [100, 200], [30, 40], F16, FP8, 7)
    plain = s.call(fc, longest=announced or s.longest)
    s.cache[1][int(s.table[1, 3]), 1, 4, 9] = 0x7F
    got = s.call(fc, longest=announced or s.longest)
    assert torch.isnan(got[30:, 4:, 9]).all()
    got[30:, 4:, 9] = plain[30:, 4:, 9]
    assert same(got, plain)


@pytest.mark.parametrize("announced", [None, 1 << 20])                 # workgroups of four wavefronts, and of eight
def test_weights_of_a_flat_tail(fc, announced):
    # a cached peak of weight ~1 whose value is zero, and thousands of equal tokens 2^-14 below it, whose values add up to what counts
    s = Step(1, 1, 128, 64, [40000], [3], F16, SYM, 8)
    s.cache[0].zero_()
    s.cache[2].fill_(1.0)
    s.cache[3].fill_(1.0)
    s.cache[1].fill_(1)
    s.q.fill_(1.0)
    s.k.zero_()
    s.v.zero_()
    s.k[:] = 14 * 0.6931471805599453 / 128 ** 0.5
    check(s.call(fc, longest=announced or s.longest), *s.exact())


def test_strides_results_and_guards(fc):
    s = Step(2, 3, 128, 32, [77, 0, 500], [20, 0, 140], BF16, SYM, 9)
    want = s.call(fc)
    big = torch.full((162, 8, 128), 5.0, dtype=BF16, device="cuda")
    out = big[1:161, 1:7]
    assert s.call(fc, out=out) is out and same(out, want)
    assert bool((big[[0, 161]] == 5).all()) and bool((big[:, [0, 7]] == 5).all())
    # heads before tokens in memory
    flip = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)      # noqa: E731
    table, offsets, held = s.table.cuda(), offsets_of(s.new), ints(s.held)
    got = fc.chunk_attention(flip(s.q), flip(s.k), flip(s.v), s.cache, table, offsets, held, s.longest, SYM, out=flip(torch.zeros_like(want)))
    assert same(got, want)
    # rows behind the last sequence and before the first stay as they were
    q, k, v = (torch.cat([t[:2], t, t[:5]]) for t in (s.q, s.k, s.v))
    got = torch.full(q.shape, 7.0, dtype=BF16, device="cuda")
    fc.chunk_attention(q, k, v, s.cache, table, offsets + 2, held, s.longest, SYM, out=got)
    assert same(got[2:162], want) and bool((got[:2] == 7).all()) and bool((got[162:] == 7).all())
    # a workspace of exactly the bytes that are asked for, and nothing written behind it
    for longest in (s.longest, 5000):
        need = fc.chunk_attention_workspace_bytes(160, 3, 2, 3, 128, longest)
        space = torch.full((need + 64,), 99, dtype=torch.uint8, device="cuda")
        got = s.call(fc, longest=longest)
        check(got, *s.exact())
        assert same(s.call(fc, longest=longest, workspace=space[:need]), got) and bool((space[need:] == 99).all())


def test_index_arrays_that_make_no_sense_touch_nothing_else(fc):
    s = Step(1, 4, 64, 16, [300, 40], [50, 60], F16, SYM, 10)
    table = s.table.cuda()
    big = torch.full((130, 4, 64), 3.0, dtype=F16, device="cuda")
    for offsets, held, pages in (([0, 60, 50], s.held, table), ([0, 50, 111], s.held, table), ([-5, 50, 110], s.held, table), ([0, 1 << 30, 110], s.held, table),
                                 ([0, 50, 110], [1 << 30, 2147483647], table), ([0, 50, 110], [-2147483648, -1], table), ([0, 50, 110], s.held, table * 0 + 99999),
                                 ([0, 50, 110], s.held, table * 0 - 99999), ([0, 0, 110], [5, 40], table)):
        for longest in (400, 1 << 20):
            print("indexes", offsets, held, longest, flush=True)
            fc.chunk_attention(s.q, s.k, s.v, s.cache, pages, ints(offsets), ints(held), longest, SYM, out=big[10:120])
            torch.cuda.synchronize()
        assert bool((big[:10] == 3).all()) and bool((big[120:] == 3).all())
    assert same(s.call(fc), s.call(fc))


def test_held_beyond_the_table_ends_with_it(fc):
    s = Step(2, 2, 128, 16, [160, 32], [9, 20], F16, SYM, 11)
    want = s.call(fc)
    s.held = [5000, 32]                                  # 160 tokens have a place in its 10 pages
    assert same(s.call(fc), want)


def test_beyond_32_bit_offsets(fc):
    heads, page, dim = 8, 64, 128
    pages = (1 << 31) // (heads * page * dim) + 40       # 65536 bytes a page
    s = Step(heads, 2, dim, page, [150], [70], BF16, FP8, 12)
    want = s.call(fc)
    cache = (*[torch.empty((pages, heads, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2)], *[torch.empty((pages, heads), device="cuda") for _ in range(2)])
    for i in range(3):
        for big, small in zip(cache, s.cache):
            big[pages - 1 - i] = small[int(s.table[0, i])]
        s.table[0, i] = pages - 1 - i
    s.cache = cache
    assert same(s.call(fc), want)


def test_large_tokens_beyond_32_bit_offsets(fc):
    # q, k, v and the result as views of one tensor of 4.3 GB: token stride 2^15 elements, 66000 tokens
    tokens, heads, dim = 66000, 1, 64
    base = torch.zeros((tokens, 1 << 15), dtype=F16, device="cuda")
    view = base.view(tokens, 512, 64)
    s = Step(heads, 1, dim, 16, [50, 40], [tokens - 90, 90], F16, SYM, 13)
    view[:, :1], view[:, 1:2], view[:, 2:3] = s.q, s.k, s.v
    want = s.call(fc)
    s.q, s.k, s.v = view[:, :1], view[:, 1:2], view[:, 2:3]
    got = s.call(fc, out=view[:, 9:10])
    assert same(got, want)


def test_a_prompt_without_a_cache_is_prompt_attention(fc):
    for dtype in (F16, BF16):
        s = Step(2, 4, 128, 16, [0, 0, 0], [300, 1, 90], dtype, SYM, 14)
        want, weight, tiles = s.exact()
        check(s.call(fc), want, weight, tiles)
        other = fc.prompt_attention(s.q, s.k, s.v, offsets_of(s.new), 300)
        u = torch.finfo(dtype).eps / 2                   # both within the bound
        assert bool(((s.call(fc).double() - other.double()).abs() <= 2 * ((u + 2.0 ** -11) * weight + u * want.abs() + 2.0 ** -19 * tiles + 2.0 ** -25)).all())


def test_graphs_streams_and_the_native_call(fc):
    s = Step(2, 4, 128, 16, [500, 70], [33, 100], BF16, FP8, 15)
    want = s.call(fc)
    table, offsets, held = s.table.cuda(), offsets_of(s.new), ints(s.held)
    args = (s.q, s.k, s.v, s.cache, table, offsets, held, 5000, FP8)          # (announced as long enough to be cut)
    want = s.call(fc, longest=5000)
    native = fc.binding._calls()
    assert native.chunk_attention(*args, None, None, None) is not None
    fc.binding._native = fc.binding._NoNativeCalls()
    try:
        assert same(fc.chunk_attention(*args), want)
    finally:
        fc.binding._native = native
    need = fc.chunk_attention_workspace_bytes(133, 2, 2, 4, 128, 5000)
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], [torch.empty_like(want) for _ in range(2)]
    with torch.cuda.stream(side):
        assert same(fc.chunk_attention(*args), want)
        for out in outs:                                 # two graphs that share a workspace, replayed one after the other
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                fc.chunk_attention(*args, out=out, workspace=space)
            graphs.append(graph)
    torch.cuda.synchronize()
    for seed in range(3):
        fresh = Step(2, 4, 128, 16, [500, 70], [33, 100], BF16, FP8, 30 + seed)
        for a, b in ((s.q, fresh.q), (s.k, fresh.k), (s.v, fresh.v)):
            a.copy_(b)
        held.copy_(ints([500 - 100 * seed, 70 - seed]))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = fc.chunk_attention(*args)
        assert same(outs[0], want) and same(outs[1], want)


def test_empty_calls_and_refusals(fc):
    s = Step(2, 2, 64, 16, [20], [8], F16, SYM, 16)
    table, offsets, held = s.table.cuda(), offsets_of(s.new), ints(s.held)
    args = [s.q, s.k, s.v, s.cache, table, offsets, held, 28]
    assert fc.chunk_attention(s.q[:0], s.k[:0], s.v[:0], s.cache, table, ints([0, 0]), held, 28).shape == (0, 4, 64)
    with pytest.raises(TypeError):
        fc.chunk_attention(s.q.float(), *args[1:])
    with pytest.raises(TypeError):
        fc.chunk_attention(s.q, s.k.to(BF16), *args[2:])
    with pytest.raises(TypeError):
        fc.chunk_attention(*args[:5], offsets.long(), held, 28)
    for at, bad in ((1, s.k[:-1]), (2, s.v[:, :1]), (0, s.q[:, :3]), (0, s.q[..., :32]), (4, table[:0]), (6, held[:0]), (3, s.cache[:3])):
        with pytest.raises((ValueError, fc.FcError)):
            fc.chunk_attention(*args[:at], bad, *args[at + 1:])
    for more in (dict(quantizer=0), dict(quantizer=3), dict(scale=0.0), dict(scale=float("inf"))):
        with pytest.raises(fc.FcError):
            fc.chunk_attention(*args, **more)
    with pytest.raises(fc.FcError):
        fc.chunk_attention(*args[:7], 100000, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(fc.FcError):
        fc.chunk_attention(*args[:7], 0)
    with pytest.raises(ValueError):
        fc.chunk_attention(*args, out=s.q[:1].expand(8, 4, 64))
    q = s.q.clone().requires_grad_()
    with pytest.raises(ValueError):
        fc.chunk_attention(q, *args[1:])
    with torch.no_grad():
        assert same(fc.chunk_attention(q, *args[1:]), fc.chunk_attention(*args))
