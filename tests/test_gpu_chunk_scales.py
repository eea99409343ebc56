"""Attention of a chunk of new tokens where the pages' value scales lie far apart, against its definition in 64 bits.

Tolerances as in test_gpu_chunk.py.  A page that has no weight is there with a value scale of its own, or with 0 where the definition is evaluated: its scores
are 160 and more below those of other tokens (in natural logarithms), so with values of at most 2^109 it adds less than 2^-120 to any sum."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_chunk import BF16, F16, FP8, SYM, TOP, Step, check, codes_of, fc, gen  # noqa: E402,F401

CASES = [(1, 4, 128, 16, [3000], [70]), (2, 2, 64, 32, [1500, 0, 2100], [40, 10, 300]), (1, 8, 128, 64, [1030], [300])]


def set_keys(s, b, page, value):
    """all keys of a page of sequence b, every element of them: value"""
    id, n = int(s.table[b, page]), min(s.page, s.held[b] - page * s.page)
    s.cache[0][id, :, :n] = codes_of(torch.tensor(TOP[s.quantizer] if value > 0 else -TOP[s.quantizer]), s.quantizer).cuda()
    s.cache[2][id] = abs(value) / TOP[s.quantizer]
    return id


@pytest.mark.parametrize("announced", [None, 1 << 20])                 # workgroups of four wavefronts, and of eight
@pytest.mark.parametrize("dtype,factor", [(BF16, 2.0 ** 70), (BF16, 2.0 ** 100), (F16, 2.0 ** 40), (F16, 2.0 ** 46)])
@pytest.mark.parametrize("quantizer", [SYM, FP8])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_a_page_of_a_large_scale_and_no_weight(fc, announced, dtype, factor, quantizer, case):
    heads, group, dim, page, held, new = CASES[case]
    b = len(held) - 1
    last = -(-held[b] // page) - 1
    # beside ordinary pages, in the 1024 tokens before others, right before the new tokens
    for places in ([2], [last], [1, last // 2, last - 1], [1000 // page, 1024 // page]):
        s = Step(heads, group, dim, page, held, new, dtype, quantizer, 20 + case)
        s.q.abs_()                                       # (sums of |q| are 0.8 dim and little off it, so these scores are -45 * 0.8 * dim^0.5)
        ids = [set_keys(s, b, min(p, last), -45.0) for p in places]
        for id in ids:
            s.cache[3][id] = 0.0
        want = s.exact()
        for id in ids:
            s.cache[3][id] = factor
        print("scale", dtype, factor, quantizer, CASES[case], places, announced, flush=True)
        check(s.call(fc, longest=announced or s.longest), *want)


@pytest.mark.parametrize("announced", [None, 1 << 20])
@pytest.mark.parametrize("dtype,factor", [(BF16, 2.0 ** -70), (BF16, 2.0 ** -110), (F16, 2.0 ** -40)])
@pytest.mark.parametrize("quantizer", [SYM, FP8])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_a_page_of_a_small_scale_and_nearly_all_weight(fc, announced, dtype, factor, quantizer, case):
    # what it counts for is the sum of weights; the values that are left come from others, of weights 2^-20 and less
    heads, group, dim, page, held, new = CASES[case]
    b = len(held) - 1
    for place in (2, -(-held[b] // page) - 1):
        s = Step(heads, group, dim, page, held, new, dtype, quantizer, 30 + case)
        s.q.abs_()
        s.cache[3][set_keys(s, b, place, 1.7)] = factor
        print("scale", dtype, factor, quantizer, CASES[case], place, announced, flush=True)
        check(s.call(fc, longest=announced or s.longest), *s.exact())


@pytest.mark.parametrize("announced", [None, 1 << 20])
@pytest.mark.parametrize("quantizer", [SYM, FP8])
@pytest.mark.parametrize("direction", [-1, 0, 1])
def test_scales_over_the_whole_range_of_bfloat16(fc, announced, quantizer, direction):
    # falling and rising along the sequence, and at random: each of 190 binary orders counts where it is the largest that a row sees
    s = Step(2, 2, 128, 16, [3000], [130], BF16, quantizer, 40)
    ids = s.table[0, :188].long().cuda()
    power = torch.arange(188) - 94.0 if direction else torch.randint(-94, 94, (188,), generator=gen(41)).float()
    s.cache[3][ids] *= torch.exp2(power * (direction or 1)).cuda()[:, None]
    check(s.call(fc, longest=announced or s.longest), *s.exact())
    # every second page seen by nobody: the sums have to be right where a scale 2^94 above was met and where it was not
    s.q.abs_()
    far = [set_keys(s, 0, i, -45.0) for i in range(187) if s.cache[3][int(s.table[0, i]), 0] > 1.0]
    keep = s.cache[3][far].clone()
    s.cache[3][far] = 0.0
    want = s.exact()
    s.cache[3][far] = keep
    check(s.call(fc, longest=announced or s.longest), *want)
