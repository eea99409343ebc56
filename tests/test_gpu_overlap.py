"""Results that lie over what a call reads, or over each other, are refused; those in place, and views of one buffer whose rows lie between each other's,
are not."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F16 = torch.float16


@pytest.fixture(scope="module")
def fc():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests selected but no GPU is visible")
    import paper_2412_04964_amd as m
    m.lib()
    return m


@pytest.fixture(params=["native", "python"])
def path(request, fc):
    native = fc.binding._calls()
    fc.binding._native = native if request.param == "native" else fc.binding._NoNativeCalls()
    yield request.param
    fc.binding._native = native


def test_norms(fc, path):
    g = torch.Generator().manual_seed(1)
    buf = torch.randn((3, 12, 1024), generator=g).half().cuda()
    w = (1 + 0.1 * torch.randn(512, generator=g)).half().cuda()
    x, r = buf[0, 1:7, :512], buf[1, 1:7, :512]
    first = fc.rms_norm(x.clone(), w, residual=r.clone())
    coded = fc.rms_norm_quantize(x.clone(), w, 1e-5, 64, fc.QUANTIZER_SYM, residual=r.clone())
    before = buf.clone()
    dense = buf[2].view(-1)
    over = dense[:3072].view(6, 512)
    bad = [
        dict(out=buf[0, 2:8, :512]), dict(out=buf[0, :6, :512]), dict(out=buf[0, 1:7, 8:520]), dict(out=buf[0, 1:7, 256:768]),       # x, some rows or elements on
        dict(sum_out=buf[0, 2:8, :512]), dict(sum_out=buf[1, 2:8, :512]), dict(out=buf[1, 1:7, 504:1016]),
        dict(out=buf[2, 0:6, :512], sum_out=buf[2, 3:9, :512]), dict(out=buf[2, 0:6, :512], sum_out=buf[2, 0:6, :512]),
        dict(out=buf[2, 0:6, :512], sum_out=buf[2, 0:6, 256:768]), dict(out=over, sum_out=buf[2, 0:6, :512]),                       # rows of other strides
        dict(out=buf[0].view(-1)[1024:1024 + 3072].view(6, 512)),                                                                     # x's start, another stride
    ]
    for more in bad:
        with pytest.raises(ValueError):
            fc.rms_norm(x, w, residual=r, **more)
    # the weight
    base = buf[2].view(-1)
    with pytest.raises(ValueError):
        fc.rms_norm(x, base[512:1024], out=buf[2, 0:6, :512].as_strided((6, 512), (512, 1)))
    # codes and scales
    bytes_ = buf.view(torch.uint8).view(-1)
    at = (x.data_ptr() - buf.data_ptr())
    fresh_codes, fresh_scales = torch.empty((6, 512), dtype=torch.uint8, device="cuda"), torch.empty((6, 8), device="cuda")
    mixed = torch.empty(4096, dtype=torch.uint8, device="cuda")
    for out, more in (((bytes_[at:at + 3072].view(6, 512), fresh_scales), {}), ((bytes_[at + 2048:at + 2048 + 3072].view(6, 512), fresh_scales), {}),
                      ((fresh_codes, bytes_[at:at + 192].view(torch.float32).view(6, 8)), {}), ((mixed[:3072].view(6, 512), mixed[3056:3248].view(torch.float32).view(6, 8)), {}),
                      ((bytes_[-3072:].view(6, 512), fresh_scales), dict(sum_out=buf[2, 6:12, 512:]))):
        with pytest.raises(ValueError):
            fc.rms_norm_quantize(x, w, 1e-5, 64, fc.QUANTIZER_SYM, residual=r, out=out, **more)
    assert torch.equal(buf, before)
    # rows between rows, and in place
    got = fc.rms_norm(x, w, residual=r, out=buf[0, 1:7, 512:], sum_out=buf[1, 1:7, 512:])
    assert all(torch.equal(a, b) for a, b in zip(got, first))
    got = fc.rms_norm_quantize(x, w, 1e-5, 64, fc.QUANTIZER_SYM, residual=r, out=(mixed[:3072].view(6, 512), mixed[3072:3264].view(torch.float32).view(6, 8)), sum_out=buf[0, 1:7, 512:])
    assert all(torch.equal(a, b) for a, b in zip((*got[0:2], got[2]), coded))
    assert torch.equal(fc.rms_norm(x[:1], w, out=x[:1]), fc.rms_norm(before[0, 1:2, :512], w))
    x.copy_(before[0, 1:7, :512])
    got = fc.rms_norm(x, w, residual=r, out=x, sum_out=r)
    assert got[0] is x and all(torch.equal(a, b) for a, b in zip(got, first))


def test_chunk_attention(fc, path):
    from test_gpu_chunk import BF16, SYM, Step, ints, offsets_of, same
    for longest in (None, 5000):                         # items whole, and cut into ranges
        s = Step(2, 2, 128, 16, [500, 30], [40, 100], BF16, SYM, 1)
        joint = torch.zeros((145, 12, 128), dtype=BF16, device="cuda")       # queries 4, keys 2, values 2, and room
        q, k, v = joint[2:142, :4], joint[2:142, 4:6], joint[2:142, 6:8]
        q.copy_(s.q), k.copy_(s.k), v.copy_(s.v)
        args = (q, k, v, s.cache, s.table.cuda(), offsets_of(s.new), ints(s.held), longest or s.longest, SYM)
        want = s.call(fc, longest=longest or s.longest)
        need = fc.chunk_attention_workspace_bytes(140, 2, 2, 2, 128, longest or s.longest)
        before = joint.clone()
        codes = s.cache[0].view(-1)
        assert codes.numel() > 140 * 4 * 128 * 2 + 16
        for out in (joint[2:142, 4:8], joint[2:142, 3:7], joint[2:142, 1:5], joint[3:143, :4], joint[1:141, 6:10], joint[2:142, 7:11],
                    joint.view(-1)[8 * 1536:8 * 1536 + 140 * 512].view(140, 4, 128), codes[:140 * 4 * 128 * 2].view(BF16).view(140, 4, 128)):
            with pytest.raises(ValueError):
                fc.chunk_attention(*args, out=out)
        big = torch.zeros(need + (1 << 20), dtype=torch.uint8, device="cuda")
        y = big[:140 * 1024].view(BF16).view(140, 4, 128)
        if need:
            for space, out in ((big, y), (joint.view(-1).view(torch.uint8), None), (codes, None)):
                with pytest.raises((ValueError, fc.FcError)):
                    fc.chunk_attention(*args, out=out, workspace=space)
        assert torch.equal(joint, before)
        assert same(fc.chunk_attention(*args, out=joint[2:142, 8:12]), want)          # beside the others
        assert same(fc.chunk_attention(*args, out=y, workspace=big[1 << 19:]), want)
        assert fc.chunk_attention(*args, out=q) is q and same(q, want)


def test_pages(fc, path):
    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    pages, held, uses, offsets, parents = ints([[0, -1], [1, 2]]), ints([3, 20]), ints([1, 1, 1, 0, 0, 0, 0, 0]), ints([0, 15, 17]), ints([1, 0])
    room = torch.zeros(64, dtype=torch.int32, device="cuda")
    base = [t.clone() for t in (pages, held, uses, offsets, parents)]
    part = lambda at, *shape: room[at:at + (shape[0] * (shape[1] if len(shape) > 1 else 1))].view(shape)      # noqa: E731
    new = (part(0, 2, 2), part(4, 2))
    for out in ((pages, new[1]), (new[0], held), (new[0], parents), (new[0], part(3, 2)), (uses[:4].view(2, 2), new[1])):
        with pytest.raises(ValueError):
            fc.pages_fork(pages, held, uses, parents, 16, out=out)
    s, t, lack, space = part(0, 2), part(2, 2), part(4, 1), room[8:16].view(torch.uint8)
    for out, work in (((s, s, lack), None), ((s, part(1, 2), lack), None), ((s, t, part(3, 1)), None), ((held, t, lack), None), ((s, uses[2:4], lack), None),
                      ((s, t, offsets[:1]), None), ((s, pages[0], lack), None), ((s, t, lack), room[2:16].view(torch.uint8)), (None, uses.view(torch.uint8)),
                      (None, torch.cat([room, room]).view(torch.uint8)[:8])):
        with pytest.raises((ValueError, fc.FcError)):
            fc.pages_reserve(pages, held, uses, offsets, 16, out=out, workspace=work)
    five = (part(0, 2, 2), part(4, 8), part(12, 4), part(16, 4), part(20, 1))
    space = room[24:40].view(torch.uint8)
    for at, bad in ((0, uses[:4].view(2, 2)), (1, uses), (2, five[3]), (3, five[1][4:]), (4, uses[:1]), (2, pages.view(-1)), (4, pages.view(-1)[:1])):
        with pytest.raises(ValueError):
            fc.pages_compact(pages, uses, out=(*five[:at], bad, *five[at + 1:]))
    for work in (room[16:32].view(torch.uint8), pages.view(torch.uint8).view(-1)[:16], uses.view(torch.uint8)):
        with pytest.raises((ValueError, fc.FcError)):
            fc.pages_compact(pages, uses, out=five, workspace=work)
    assert all(torch.equal(a, b) for a, b in zip((pages, held, uses, offsets, parents), base)) and not room.any()
    # what lies side by side passes, and the table of a compaction in place
    fc.pages_fork(pages, held, uses, parents, 16, out=new)
    assert new[0].tolist() == [[1, 2], [0, -1]] and new[1].tolist() == [20, 3] and uses.tolist() == [1, 1, 1, 0, 0, 0, 0, 0]
    fc.pages_reserve(pages, held, uses, offsets, 16, out=(s, t, lack), workspace=space)
    assert pages.tolist() == [[0, 3], [1, 2]] and lack.item() == 0 and uses.tolist() == [1, 1, 1, 1, 0, 0, 0, 0]
    uses[0] = 0
    pages[0, 0] = -1
    got = fc.pages_compact(pages, uses, out=(pages, *five[1:]), workspace=space)
    assert pages.tolist() == [[-1, 0], [1, 2]] and got[4].item() == 3 and got[1].tolist() == [1, 1, 1, 0, 0, 0, 0, 0]
