"""The norm behind an all-reduce on the GPU: bit for bit against the formulas of include/fc.h, with the sum of squares in 64 bits on the CPU.

The formula leaves two results open where the 64-bit sums of two orders fall on different sides of a border between fp32 numbers: d then
differs by one step, 2^-23 relative.  Inputs here have few significant bits (float16 and bfloat16 values, sums of two of them), so their squares add
up exactly in 64 bits as long as their exponents are within 2^20 or so of each other, and equality is asserted; the wide-range test allows
the one step."""
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


def same(a, b):
    a, b = a.cpu().contiguous(), b.cpu().contiguous()
    assert a.dtype == b.dtype and a.shape == b.shape
    if a.is_floating_point():
        kind = torch.int16 if a.element_size() == 2 else torch.int32
        return bool(((a.view(kind) == b.view(kind)) | (torch.isnan(a) & torch.isnan(b))).all())
    return torch.equal(a, b)


def normed(x, weight, eps, residual=None):
    """(y in fp32, sum in fp32) of CPU tensors"""
    h = x.float()
    if residual is not None:
        h = h + residual.float()
    d = (1.0 / torch.sqrt(h.double().square().sum(-1, keepdim=True) / x.shape[1] + eps)).float()
    return (h * d) * weight.float(), h


def coded(y, group, quantizer):
    """(codes uint8, scales) of fp32 rows"""
    g = y.reshape(y.shape[0], -1, group)
    s = g.abs().amax(-1) / torch.tensor(TOP[quantizer])
    s = torch.where(s >= FLT_MIN, s, torch.ones_like(s))
    v = g * (torch.ones_like(s) / s)[..., None]
    codes = v.round().clamp(-127, 127).to(torch.int8).view(torch.uint8) if quantizer == SYM else v.to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.reshape(y.shape), s


def inputs(tokens, hidden, dtype, seed, spread=1.0):
    x = (torch.randn((tokens, hidden), generator=gen(seed)) * spread).to(dtype)
    r = (torch.randn((tokens, hidden), generator=gen(seed + 1)) * 3 * spread).to(dtype)
    return x, r, 0.5 + torch.rand(hidden, generator=gen(seed + 2))


ROWS = [(1, 8), (3, 40), (1, 512), (2, 520), (5, 1024), (1, 4096), (7, 5120), (65, 2048), (2, 8192), (3, 8200), (1, 16384), (2, 24576), (3, 32768)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("tokens,hidden", ROWS)
def test_norm_matches_the_formula_bit_for_bit(fc, dtype, tokens, hidden):
    print("norm", dtype, tokens, hidden, flush=True)
    x, r, w = inputs(tokens, hidden, dtype, hidden)
    for weight in (w, w.to(dtype)):
        y, _ = normed(x, weight, 1e-5)
        assert same(fc.rms_norm(x.cuda(), weight.cuda()), y.to(dtype))
        y, h = normed(x, weight, 1e-6, r)
        got, total = fc.rms_norm(x.cuda(), weight.cuda(), 1e-6, residual=r.cuda())
        assert same(got, y.to(dtype)) and same(total, h.to(dtype))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("quantizer", [SYM, FP8])
@pytest.mark.parametrize("tokens,hidden,group", [(1, 8, 8), (3, 40, 40), (2, 512, 32), (3, 4096, 128), (1, 4096, 4096), (5, 5120, 1024), (4, 5120, 5120), (2, 8192, 512), (1, 8192, 8192),
                                                 (3, 16384, 2048), (2, 16384, 16384), (2, 32768, 16384), (1, 32768, 32768), (2, 32768, 64), (1, 24584, 24584), (33, 1024, 256)])
def test_codes_match_the_formula_bit_for_bit(fc, dtype, quantizer, tokens, hidden, group):
    print("norm codes", dtype, quantizer, tokens, hidden, group, flush=True)
    x, r, w = inputs(tokens, hidden, dtype, hidden + group)
    x[0, :8] = 0                                         # (hidden 8: a row of zeros without the residual)
    codes, scales = coded(normed(x, w, 1e-5)[0], group, quantizer)
    got = fc.rms_norm_quantize(x.cuda(), w.cuda(), 1e-5, group, quantizer)
    assert same(got[0], codes) and same(got[1], scales)
    y, h = normed(x, w, 1e-5, r)
    codes, scales = coded(y, group, quantizer)
    got = fc.rms_norm_quantize(x.cuda(), w.cuda(), 1e-5, group, quantizer, residual=r.cuda())
    assert same(got[0], codes) and same(got[1], scales) and same(got[2], h.to(dtype))


def test_codes_are_the_librarys(fc):
    # dequantize_sym and dequantize_fp8 read them: half a step of the code, and half a step of float16
    x, _, w = inputs(9, 4096, F16, 5)
    y = normed(x, w, 1e-5)[0].double()
    for quantizer, read, step in ((SYM, fc.dequantize_sym, None), (FP8, fc.dequantize_fp8, 2.0 ** -4)):
        codes, scales = fc.rms_norm_quantize(x.cuda(), w.cuda(), 1e-5, 128, quantizer)
        got = (read(codes, scales, 4096, 128, 8) if quantizer == SYM else read(codes, scales, 4096, 128)).cpu().double()
        s = scales.cpu().double().repeat_interleave(128, 1)
        off = 0.5 * s if step is None else torch.maximum(step * y.abs(), 2.0 ** -10 * s)
        assert bool(((got - y).abs() <= off * (1 + 1e-5) + 2.0 ** -11 * y.abs() + 2.0 ** -25).all())


def test_zeros_tiny_and_huge_rows(fc):
    w = torch.ones(1024)
    x = torch.zeros((6, 1024), dtype=BF16)
    x[1, 5] = 2.0 ** -126
    x[2] = 2.0 ** -60
    x[3] = 2.0 ** 100                                   # squares beyond fp32
    x[4, ::2] = -2.0 ** 127
    x[5, 7] = 2.0 ** -133
    for eps in (1e-5, 1e-30):
        y, _ = normed(x, w, eps)
        assert same(fc.rms_norm(x.cuda(), w.cuda(), eps), y.to(BF16)) and torch.isfinite(y).all()
        for quantizer in (SYM, FP8):
            codes, scales = fc.rms_norm_quantize(x.cuda(), w.cuda(), eps, 32, quantizer)
            want = coded(y, 32, quantizer)
            assert same(codes, want[0]) and same(scales, want[1])


def test_exponents_far_apart(fc):
    # a row whose squares do not add up exactly: d may be one step off, 2^-23, and h d and (h d) w half a step each more than the formula's
    # (2 * 2^-24 on either side).  Then y is rounded to bfloat16: 8 bits, so a step at 1 is 2^-7 and half of one 2^-8 of the value.
    x = (torch.randn((16, 8192), generator=gen(3)) * 2.0 ** torch.randint(-40, 40, (16, 8192), generator=gen(4))).to(BF16)
    r = (torch.randn((16, 8192), generator=gen(5)) * 2.0 ** torch.randint(-40, 40, (16, 8192), generator=gen(6))).to(BF16)
    w = torch.rand(8192, generator=gen(7))
    y, h = normed(x, w, 1e-5, r)
    got, total = fc.rms_norm(x.cuda(), w.cuda(), 1e-5, residual=r.cuda())
    assert same(total, h.to(BF16))
    assert bool(((got.cpu().double() - y.double()).abs() <= (2.0 ** -8 + 2.0 ** -21) * y.double().abs() + 2.0 ** -133).all())


def test_what_is_not_finite_stays_in_its_row(fc):
    x, r, w = inputs(5, 2048, F16, 8)
    x[1, 3], x[3, 2000] = float("inf"), float("nan")
    y, h = normed(x, w, 1e-5, r)
    got, total = fc.rms_norm(x.cuda(), w.cuda(), 1e-5, residual=r.cuda())
    assert same(total, h.to(F16)) and same(got, y.to(F16))
    assert torch.isfinite(got[[0, 2, 4]]).all()
    codes, scales = fc.rms_norm_quantize(x.cuda(), w.cuda(), 1e-5, 64, SYM, residual=r.cuda())[:2]
    want = coded(y, 64, SYM)
    assert same(codes[[0, 2, 4]], want[0][[0, 2, 4]]) and same(scales[[0, 2, 4]], want[1][[0, 2, 4]])


def test_strides_and_guards(fc):
    for dtype, hidden in ((F16, 1032), (BF16, 4096), (F16, 5120)):
        x, r, w = inputs(6, hidden, dtype, 9)
        big = torch.full((3, 8, hidden + 24), 7.0, dtype=dtype, device="cuda")
        a, b, y = (big[i, 1:7, 8:8 + hidden] for i in range(3))
        total = torch.full((6, 2, hidden), 7.0, dtype=dtype, device="cuda")
        a.copy_(x)
        b.copy_(r)
        before = big.clone()
        got = fc.rms_norm(a, w.cuda(), 1e-5, residual=b, out=y, sum_out=total[:, 1])
        assert got[0] is y
        want, h = normed(x, w, 1e-5, r)
        assert same(y, want.to(dtype)) and same(total[:, 1], h.to(dtype)) and bool((total[:, 0] == 7).all())
        before[2, 1:7, 8:8 + hidden] = y
        assert same(big, before)
        # in place: the sum over the residual, the norm over x
        assert fc.rms_norm(a, w.cuda(), 1e-5, residual=b, out=a, sum_out=b)[1] is b
        assert same(a, want.to(dtype)) and same(b, h.to(dtype))
        # row 0 repeated, as an expanded input
        one = fc.rms_norm(x.cuda()[:1].expand(6, hidden), w.cuda(), 1e-5)
        assert same(one, normed(x[:1], w, 1e-5)[0].to(dtype).expand(6, hidden))
    codes, scales = torch.full((8, 4096), 99, dtype=torch.uint8, device="cuda"), torch.full((8, 32), 5.0, device="cuda")
    x, r, w = inputs(6, 4096, F16, 10)
    out = (codes[1:7], scales[1:7])
    assert fc.rms_norm_quantize(x.cuda(), w.cuda(), 1e-5, 128, SYM, out=out) is out
    want = coded(normed(x, w, 1e-5)[0], 128, SYM)
    assert same(codes[1:7], want[0]) and same(scales[1:7], want[1])
    assert bool((codes[[0, 7]] == 99).all()) and bool((scales[[0, 7]] == 5).all())


def test_many_rows_equal_single_ones(fc):
    # the forms of the launch give the same bits
    for hidden, group in ((8192, 128), (5120, 5120), (512, 64), (16384, 4096)):
        x, r, w = (t.cuda() for t in inputs(3000, hidden, BF16, hidden))
        y, total = fc.rms_norm(x, w, 1e-5, residual=r)
        codes, scales, _ = fc.rms_norm_quantize(x, w, 1e-5, group, FP8, residual=r)
        for at in (0, 1, 1499, 2998):
            few, t = fc.rms_norm(x[at:at + 2], w, 1e-5, residual=r[at:at + 2])
            assert same(few, y[at:at + 2]) and same(t, total[at:at + 2])
            c, s, _ = fc.rms_norm_quantize(x[at:at + 2], w, 1e-5, group, FP8, residual=r[at:at + 2])
            assert same(c, codes[at:at + 2]) and same(s, scales[at:at + 2])


def test_streams_graphs_and_the_native_call(fc):
    x, r, w = (t.cuda() for t in inputs(8, 4096, F16, 11))
    want, total = fc.rms_norm(x, w, 1e-5, residual=r)
    codes = fc.rms_norm_quantize(x, w, 1e-5, 128, SYM, residual=r)
    native = fc.binding._calls()
    assert native.rms_norm(x, w, 1e-5, r, None, None) is not None
    assert native.rms_norm_quantize(x, w, 1e-5, 128, SYM, r, None, None) is not None
    fc.binding._native = fc.binding._NoNativeCalls()
    try:
        got = fc.rms_norm(x, w, 1e-5, residual=r)
        coded_too = fc.rms_norm_quantize(x, w, 1e-5, 128, SYM, residual=r)
    finally:
        fc.binding._native = native
    assert same(got[0], want) and same(got[1], total) and all(same(a, b) for a, b in zip(coded_too, codes))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, t = torch.empty_like(x), torch.empty_like(x)
    out = tuple(torch.empty_like(c) for c in codes[:2])
    with torch.cuda.stream(side):
        assert same(fc.rms_norm(x, w, 1e-5, residual=r)[0], want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            fc.rms_norm(x, w, 1e-5, residual=r, out=y, sum_out=t)
            fc.rms_norm_quantize(t, w, 1e-5, 128, SYM, out=out)
    torch.cuda.synchronize()
    for seed in range(3):
        x.copy_(inputs(8, 4096, F16, 20 + seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        want, total = fc.rms_norm(x, w, 1e-5, residual=r)
        codes = fc.rms_norm_quantize(total, w, 1e-5, 128, SYM)
        assert same(y, want) and same(t, total) and same(out[0], codes[0]) and same(out[1], codes[1])


def test_norm_of_more_than_32_bits_of_elements(fc):
    # 2^31 elements and more: the last rows lie beyond 32-bit byte offsets, and beyond 2^31 elements
    tokens, hidden = (1 << 17) + 3, 16384
    x = torch.zeros((tokens, hidden), dtype=F16, device="cuda")
    w = torch.ones(hidden, device="cuda")
    x[-2:].copy_(inputs(2, hidden, F16, 12)[0])
    y = fc.rms_norm(x, w, 1e-5, out=x)
    want = normed(inputs(2, hidden, F16, 12)[0], torch.ones(hidden), 1e-5)[0].to(F16)
    assert same(y[-2:], want) and not y[:-2].any()


def test_empty_calls_and_refusals(fc):
    x, r, w = (t.cuda() for t in inputs(4, 512, F16, 13))
    assert fc.rms_norm(x[:0], w).shape == (0, 512)
    codes, scales, total = fc.rms_norm_quantize(x[:0], w, 1e-5, 64, SYM, residual=r[:0])
    assert codes.shape == (0, 512) and scales.shape == (0, 8) and total.shape == (0, 512)
    for bad in (lambda: fc.rms_norm(x.float(), w), lambda: fc.rms_norm(x, w.to(BF16)), lambda: fc.rms_norm(x, w, residual=r.to(BF16)), lambda: fc.rms_norm(x.cpu(), w)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: fc.rms_norm(x, w[:-8]), lambda: fc.rms_norm(x, w, residual=r[:-1]), lambda: fc.rms_norm(x[:, ::2], w[::2].contiguous()), lambda: fc.rms_norm(x[:, 4:], w[:-4].contiguous()),
                lambda: fc.rms_norm(x, w, out=x[:1].expand(4, 512)), lambda: fc.rms_norm(x, w, sum_out=r), lambda: fc.rms_norm(x, w, residual=r, out=x, sum_out=x),
                lambda: fc.rms_norm(x[0], w), lambda: fc.rms_norm(x, torch.zeros(513, device="cuda")[1:])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: fc.rms_norm(x, w, 0.0), lambda: fc.rms_norm(x, w, float("nan")), lambda: fc.rms_norm_quantize(x, w, 1e-5, 48), lambda: fc.rms_norm_quantize(x, w, 1e-5, 1024),
                lambda: fc.rms_norm_quantize(x, w, 1e-5, 64, 0), lambda: fc.rms_norm(torch.zeros((1, 32776), dtype=F16, device="cuda"), torch.zeros(32776, device="cuda")),
                lambda: fc.rms_norm(x[:, :508], w[:508].contiguous())):
        with pytest.raises(fc.FcError):
            bad()
    # nothing records a gradient
    for which in range(3):
        t = [x.clone(), w.clone(), r.clone()]
        t[which].requires_grad_()
        with pytest.raises(ValueError):
            fc.rms_norm(t[0], t[1], residual=t[2])
        with torch.no_grad():
            assert same(fc.rms_norm(t[0], t[1], residual=t[2])[0], fc.rms_norm(x, w, residual=r)[0])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("wide_weight", [False, True])
@pytest.mark.parametrize("tokens,hidden,groups", [(65543, 512, (64, 512)), (4099, 8192, (128, 8192)), (6561, 5120, (1024, 5120)), (2053, 16384, (64, 16384))])
def test_more_than_the_caches_hold_equals_pieces_of_it(fc, dtype, wide_weight, tokens, hidden, groups):
    """134 MB of rows and more are read and written past the caches, with one, two and four units a lane: the bits are those of 1000 rows at a time,
    and of the formula"""
    assert tokens * hidden * 4 > 1 << 27
    x, r, w = inputs(tokens, hidden, dtype, hidden + 3)
    w = w if wide_weight else w.to(dtype)
    at = [0, 1, tokens // 2, tokens - 1]
    y, h = normed(x[at], w, 1e-5, r[at])
    cx, cr, cw = x.cuda(), r.cuda(), w.cuda()
    print("norm past the caches", dtype, wide_weight, tokens, hidden, flush=True)
    got, total = fc.rms_norm(cx, cw, 1e-5, residual=cr)
    alone = fc.rms_norm(cx, cw, 1e-5)
    assert same(got[at], y.to(dtype)) and same(total[at], h.to(dtype)) and same(alone[at], normed(x[at], w, 1e-5)[0].to(dtype))
    parts = [slice(i, min(i + 1000, tokens)) for i in range(0, tokens, 1000)]
    for p in parts:
        a, b = fc.rms_norm(cx[p], cw, 1e-5, residual=cr[p])
        assert torch.equal(a, got[p]) and torch.equal(b, total[p]) and torch.equal(fc.rms_norm(cx[p], cw, 1e-5), alone[p])
    for quantizer in (SYM, FP8):
        for group in groups:
            codes, scales, sums = fc.rms_norm_quantize(cx, cw, 1e-5, group, quantizer, residual=cr)
            want = coded(y, group, quantizer)
            assert same(codes[at], want[0]) and same(scales[at], want[1]) and torch.equal(sums, total)
            for p in parts:
                a, b, _ = fc.rms_norm_quantize(cx[p], cw, 1e-5, group, quantizer, residual=cr[p])
                assert torch.equal(a, codes[p]) and torch.equal(b, scales[p])
