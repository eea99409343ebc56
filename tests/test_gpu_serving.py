"""The serving operators together, as a server runs them: prompts in pieces, samples that share pages, a pool that is reserved from and compacted,
norms between the layers."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

SYM, FP8 = 1, 2


@pytest.fixture(scope="module")
def fc():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests selected but no GPU is visible")
    import paper_2412_04964_amd as m
    m.lib()
    return m


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("quantizer,bound", [(SYM, 0.06), (FP8, 0.09)])
@pytest.mark.parametrize("piece,samples,layers", [(64, 1, 1), (0, 3, 1), (37, 2, 1), (50, 2, 2), (0, 1, 2)])
def test_layers_of_four_ranks(fc, quantizer, bound, piece, samples, layers):
    # A piece behind the first reads codes as a decode step does, whose bounds are 0.06 and 0.09 with one layer: binary16 activations and an INT8
    # all-reduce of 0.010, keys and values of 0.010 (signed) or 0.026 (E4M3) and about as much again by the weights, 1.5 times.  A second
    # layer's input has the first one's error, at most as large beside the sum as beside its output, and adds its own: 2^0.5 times.
    from paper_2412_04964_amd import attention_block
    errors, _, _ = attention_block.run(ranks=4, hidden=1024, query_heads=16, kv_heads=4, dim=64, prompts=3, length=150, steps=20, quantizer=quantizer,
                                       piece=piece, samples=samples, layers=layers)
    assert max(errors) < bound * layers ** 0.5, errors
    if piece == 0:
        assert errors[0] < 0.02 * layers ** 0.5


def test_the_default_run_takes_prompts_whole(fc):
    from paper_2412_04964_amd import attention_block
    sizes = dict(ranks=2, hidden=512, query_heads=8, kv_heads=2, dim=64, prompts=2, length=70, steps=3)
    assert attention_block.run(**sizes)[0] == attention_block.run(piece=0, samples=1, layers=1, **sizes)[0]
    for bad in (dict(piece=-1), dict(samples=0), dict(layers=0)):
        with pytest.raises(ValueError):
            attention_block.run(**sizes, **bad)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("quantizer,page,group", [(SYM, 16, 4), (FP8, 32, 1), (SYM, 64, 6)])
def test_samples_on_shared_pages_answer_as_samples_with_pages_of_their_own(fc, dtype, quantizer, page, group):
    """Every bit: sharing, copies and moved pages change where codes are, and nothing else."""
    heads, dim, hidden, samples, piece, steps = 2, 128, 1024, 3, 90, 37
    lengths = [200, 1, 64, 150]
    g = torch.Generator(device="cuda").manual_seed(page)
    weight = torch.rand(hidden, generator=g, device="cuda").add_(0.5)
    project = (torch.randn((hidden, heads * (group + 2) * dim), generator=g, device="cuda") * hidden ** -0.5).to(dtype)
    table = fc.rotary_table(512, fc.rotary_frequencies(dim))
    prompts = [torch.randn((n, hidden), generator=g, device="cuda").to(dtype) for n in lengths]
    tokens = torch.randn((steps, len(lengths) * samples, hidden), generator=g, device="cuda").to(dtype)
    width = -(-(max(lengths) + steps) // page)
    rows = len(lengths) * samples

    def qkv(parts):
        # what a projection of 8-bit codes takes, and one of 16-bit rows
        x = torch.cat(parts)
        codes, scales = fc.rms_norm_quantize(x, weight, 1e-5, 128, quantizer)
        y = fc.rms_norm(x, weight, 1e-5)
        decoded = (fc.dequantize_sym(codes, scales, hidden, 128, 8) if quantizer == SYM else fc.dequantize_fp8(codes, scales, hidden, 128)).float()
        # half a step of 1 / 127 or of 4 bits of the largest of a group, and of a value for the norm's rounding and the decoded one's to binary16
        worst = y.float().abs().view(-1, 128).amax(1, keepdim=True) * (0.5 / 127 if quantizer == SYM else 2.0 ** -4) * 1.01 + 1e-6
        assert ((decoded - y.float()).view(-1, 128).abs() <= worst + y.float().view(-1, 128).abs() * (torch.finfo(dtype).eps / 2 + 1.1 * 2.0 ** -11)).all()
        # (a product of its own for each sequence: a library's bits may depend on the number of rows)
        z = torch.cat([p @ project for p in y.split([len(p) for p in parts])]).view(x.shape[0], heads * (group + 2), dim)
        return z[:, :heads * group], z[:, heads * group:heads * (group + 1)], z[:, heads * (group + 1):], z[:, :heads * (group + 1)]

    def serve(shared):
        """outputs of the prompts, and of each step for all samples"""
        pool = rows * width
        shape = (pool, heads, page, dim)
        cache = (torch.full(shape, 0xFF, dtype=torch.uint8, device="cuda"), torch.full(shape, 0xFF, dtype=torch.uint8, device="cuda"),
                 torch.full(shape[:2], float("nan"), device="cuda"), torch.full(shape[:2], float("nan"), device="cuda"))
        uses = torch.zeros(pool, dtype=torch.int32, device="cuda")

        def room(pages, offsets, held):
            source, target, lacking = fc.pages_reserve(pages, held, uses, offsets, page)
            assert int(lacking) == 0
            fc.cache_copy(cache, source, target)

        def take_prompts():
            """(how a step's work is cut depends on all of its sequences: every copy is taken in the same company)"""
            pages = torch.full((len(prompts), width), -1, dtype=torch.int32, device="cuda")
            outputs, begin = [[] for _ in prompts], 0
            while begin < max(lengths):
                parts = [x[begin:begin + piece] for x in prompts]
                offsets = ints([0] + [len(p) for p in parts]).cumsum(0).int()
                held = ints([min(begin, n) for n in lengths])
                positions = torch.cat([torch.arange(len(p), dtype=torch.int32, device="cuda") + begin for p in parts])
                room(pages, offsets, held)
                q, k, v, turned = qkv(parts)
                fc.rotary(turned, table, positions, out=turned)
                o = fc.chunk_attention(q, k, v, cache, pages, offsets, held, max(lengths), quantizer)
                fc.cache_append(k, v, cache, pages, offsets, held, piece, quantizer)
                for out, part in zip(outputs, o.split([len(p) for p in parts])):
                    out.append(part)
                begin += piece
            return pages, [torch.cat(o) for o in outputs]

        if shared:
            pages, outputs = take_prompts()
            outputs = [o for o in outputs for _ in range(samples)]
            parents = ints([b for b in range(len(prompts)) for _ in range(samples)])
            pages, held = fc.pages_fork(pages, ints(lengths), uses, parents, page)
        else:
            taken = [take_prompts() for _ in range(samples)]
            pages = torch.stack([pages for pages, _ in taken], 1).view(rows, width)
            outputs = [outputs[b] for b in range(len(prompts)) for _, outputs in taken]
            held = ints([n for n in lengths for _ in range(samples)])
        offsets, out = ints(list(range(rows + 1))), []
        for i in range(steps):
            if shared and i in (5, 20):
                pages, uses, source, target, used = fc.pages_compact(pages, uses)
                fc.cache_copy(cache, source, target)
                # as many pages as the tokens need: full pages of the prompts are there once, what follows them once a sample
                need = sum(n // page + samples * (-(-(n + i) // page) - n // page) for n in lengths)
                assert int(used) == need and int((uses > 0).sum()) == need and bool((uses[:need] > 0).all())
            room(pages, offsets, held)
            q, k, v, _ = qkv([tokens[i]])
            fc.rotary(q, table, held, out=q)
            fc.cache_append(k, v, cache, pages, offsets, held, 1, quantizer, table)
            out.append(fc.cache_attention(q, cache, pages, offsets, held, 1, max(lengths) + i + 1, quantizer).clone())
            held += 1
        return outputs, out

    (got, steps_got), (want, steps_want) = serve(True), serve(False)
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), "prompt %d" % i
    for i, (a, b) in enumerate(zip(steps_got, steps_want)):
        assert torch.isfinite(a.float()).all() and torch.equal(a, b), "step %d" % i
