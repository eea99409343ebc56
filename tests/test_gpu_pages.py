"""The cache's pages on the GPU against a plain model of them in Python lists: whole numbers, which have to be equal."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def fc():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests selected but no GPU is visible")
    import paper_2412_04964_amd as m
    m.lib()
    return m


def ints(values, shape=None):
    t = torch.tensor(values, dtype=torch.int32)
    return (t if shape is None else t.reshape(shape)).cuda()


def filled(held, page):
    return max(0, -(-held // page))


def fork(table, held, uses, parents, page):
    """lists -> (table, held, uses) afterwards"""
    pages, width = len(uses), len(table[0]) if table else 0
    uses = list(uses)
    for row in table:
        for p in row:
            if 0 <= p < pages:
                uses[p] -= 1
    out, now = [], []
    for parent in parents:
        there = 0 <= parent < len(table)
        n = filled(held[parent], page) if there else 0
        out.append([p if i < n and 0 <= p < pages else -1 for i, p in enumerate(table[parent])] if there else [-1] * width)
        now.append(held[parent] if there else 0)
        for p in out[-1]:
            if p >= 0:
                uses[p] += 1
    return out, now, uses


def reserve(table, held, uses, offsets, page):
    """lists -> (table, uses, source, target, lacking)"""
    pages, width, n = len(uses), len(table[0]), len(table)
    slots, writes = [], []
    for b in range(n):
        begin, end = max(held[b], 0), held[b] + offsets[b + 1] - offsets[b]
        mine = [i for i in range(begin // page, (end - 1) // page + 1) if i < width] if end > begin else []
        slots.append(mine)
        p = table[b][mine[0]] if mine and begin % page else -1
        writes.append(p if 0 <= p < pages else -1)
    copies = []
    for b, p in enumerate(writes):
        later = p in writes[b + 1:]
        copies.append(p >= 0 and uses[p] > 1 and (later or writes.count(p) < uses[p]))
    wants = [(b, i) for b in range(n) for i in slots[b] if not 0 <= table[b][i] < pages or (copies[b] and i == slots[b][0])]
    free = [p for p in range(pages) if uses[p] == 0]
    if len(wants) > len(free):
        return table, uses, [-1] * n, [-1] * n, len(wants) - len(free)
    table, uses, source, target = [list(r) for r in table], list(uses), [-1] * n, [-1] * n
    for (b, i), p in zip(wants, free):
        if copies[b] and i == slots[b][0]:
            source[b], target[b] = writes[b], p
            uses[writes[b]] -= 1
        table[b][i] = p
        uses[p] = 1
    return table, uses, source, target, 0


def compact(table, uses):
    pages = len(uses)
    used = sum(u > 0 for u in uses)
    holes = [p for p in range(used) if uses[p] <= 0]
    movers = [p for p in range(used, pages) if uses[p] > 0]
    place = dict(zip(movers, holes))
    now = [uses[p] if uses[p] > 0 and p < used else 0 for p in range(pages)]
    for s, t in place.items():
        now[t] = uses[s]
    rest = [-1] * (pages // 2 - len(movers))
    return [[place.get(p, p) for p in row] for row in table], now, movers + rest, holes + rest, used


def state(sequences, width, pages, page, seed, shared=0.5, reserved=False):
    """a consistent table: rows with pages of their own, some of which begin with another row's pages"""
    rng = random.Random(seed)
    order = list(range(pages))
    rng.shuffle(order)
    table, held = [], []
    for b in range(sequences):
        n = rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, max(0, width - 2) * page)])
        n = min(n, (width - 1) * page)
        k = filled(n, page)
        row = []
        if b and rng.random() < shared:
            row = table[b - 1][:min(k, held[b - 1] // page)]      # full pages of the row before
        if len(order) < k - len(row) + (1 if reserved else 0):
            n = k = 0
            row = []
        row = row + [order.pop() for _ in range(k - len(row))]
        if reserved and rng.random() < 0.5 and order and k < width:
            row.append(order.pop())
        table.append(row + [-1] * (width - len(row)))
        held.append(n)
    uses = [0] * pages
    for row in table:
        for p in row:
            if p >= 0:
                uses[p] += 1
    return table, held, uses


SIZES = [(1, 1, 4, 16), (1, 5, 9, 16), (3, 4, 40, 32), (17, 9, 300, 64), (64, 33, 5000, 16), (300, 70, 9001, 16), (1100, 5, 12345, 32), (5, 1500, 4097, 16)]


@pytest.mark.parametrize("size", SIZES)
def test_fork(fc, size):
    sequences, width, pages, page = size
    for seed in range(3):
        table, held, uses = state(sequences, width, pages, page, seed, reserved=True)
        rng = random.Random(seed)
        rows = rng.choice([sequences, max(1, sequences // 2), 2 * sequences + 1])
        parents = [rng.choice([-1, sequences, rng.randrange(sequences), rng.randrange(sequences)]) for _ in range(rows)]
        if sequences > 1:
            held[1], table[1] = -3, table[1]              # a padded slot
        print("fork", size, seed, rows, flush=True)
        want = fork(table, held, uses, parents, page)
        got_uses = ints(uses)
        got, now = fc.pages_fork(ints(table), ints(held), got_uses, ints(parents), page)
        assert got.tolist() == want[0] and now.tolist() == want[1] and got_uses.tolist() == want[2]


def test_fork_with_entries_that_are_no_pages(fc):
    table, uses = [[5, 99, -7, 2], [1 << 30, 0, 5, -1]], [1, 0, 1, 0, 0, 2, 0]
    want = fork(table, [64, 64], uses, [1, 1, 0], 16)
    got_uses = ints(uses)
    got, now = fc.pages_fork(ints(table), ints([64, 64]), got_uses, ints([1, 1, 0]), 16)
    assert got.tolist() == want[0] and got_uses.tolist() == want[2]
    # all rows go
    got, now = fc.pages_fork(got, now, got_uses, ints([-1]), 16)
    assert got.tolist() == [[-1] * 4] and now.tolist() == [0] and got_uses.tolist() == [0] * 7


@pytest.mark.parametrize("size", SIZES)
def test_reserve(fc, size):
    sequences, width, pages, page = size
    for seed in range(4):
        table, held, uses = state(sequences, width, pages, page, seed, reserved=seed % 2 == 1)
        rng = random.Random(seed)
        if seed > 1:                                     # shared partly filled pages, as a fork leaves them
            parents = [rng.randrange(sequences) for _ in range(sequences)]
            table, held, uses = fork(table, held, uses, parents, page)
        new = [rng.choice([0, 1, 1, 2, page, 3 * page + 1]) for _ in range(sequences)]
        if sequences > 2:
            held[2], new[2] = -1, rng.choice([1, 2])     # a padded slot: its first token has no place
            for i, p in enumerate(table[2]):
                if p >= 0:
                    uses[p] -= 1
                table[2][i] = -1
        offsets = [0]
        for n in new:
            offsets.append(offsets[-1] + n)
        print("reserve", size, seed, flush=True)
        want = reserve(table, held, uses, offsets, page)
        t, u = ints(table), ints(uses)
        source, target, lacking = fc.pages_reserve(t, ints(held), u, ints(offsets), page)
        assert lacking.tolist() == [want[4]]
        assert t.tolist() == want[0] and u.tolist() == want[1] and source.tolist() == want[2] and target.tolist() == want[3]
        # and once more: there is room now, and nobody writes to what others name
        if not want[4]:
            source, target, lacking = fc.pages_reserve(t, ints(held), u, ints(offsets), page)
            assert t.tolist() == want[0] and u.tolist() == want[1] and set(source.tolist()) | set(target.tolist()) <= {-1} and lacking.tolist() == [0]


def test_reserve_of_long_prompts(fc):
    # thousands of slots at once, from one sequence and several, one of them beyond the table
    for new, width in (([40000], 2600), ([1, 9000, 0, 17000], 1000)):
        n, page = len(new), 16
        table = [[-1] * width for _ in new]
        offsets = [sum(new[:i]) for i in range(n + 1)]
        uses = [int(p % 3 == 0) for p in range(6001)]
        want = reserve(table, [0] * n, uses, offsets, page)
        t, u = ints(table), ints(uses)
        _, _, lacking = fc.pages_reserve(t, ints([0] * n), u, ints(offsets), page)
        assert lacking.tolist() == [0] and t.tolist() == want[0] and u.tolist() == want[1]


def test_reserve_all_or_nothing(fc):
    table, uses = [[0, -1], [1, -1], [0, -1]], [2, 1, 0, 0]
    for free, lacking in (([2, 3], 1), ([2], 2), ([], 3)):
        u = [uses[p] if p < 2 or p in free else 1 for p in range(4)]
        t, got = ints(table), ints(u)
        out = fc.pages_reserve(t, ints([5, 16, 16]), got, ints([0, 1, 2, 3]), 16)
        assert [x.tolist() for x in out] == [[-1] * 3, [-1] * 3, [lacking]] and t.tolist() == table and got.tolist() == u
    # offsets that do not ascend take nothing
    t, got = ints(table), ints(uses)
    out = fc.pages_reserve(t, ints([5, 16, 16]), got, ints([5, 3, 2, -100]), 16)
    assert [x.tolist() for x in out] == [[-1] * 3, [-1] * 3, [0]] and t.tolist() == table and got.tolist() == uses


@pytest.mark.parametrize("offsets", [[0, 40, 20, 60], [-1, 5, 6, 7], [0, 1 << 30, 5, 1 << 30], [7, 6, 5, 4], [0, 3, 4, -(1 << 31)]])
def test_offsets_that_do_not_ascend_reserve_nothing(fc, offsets):
    """A row whose own tokens would need pages among them: what all rows need together may be more than 32 bits count"""
    table, held, uses = [[0, 1, -1, -1], [0, 1, -1, -1], [2, -1, -1, -1]], [20, 20, 3], [2, 2, 1, 0, 0, 0, 0, 0]
    t, u = ints(table), ints(uses)
    source, target, lacking = fc.pages_reserve(t, ints(held), u, ints(offsets), 16)
    assert t.tolist() == table and u.tolist() == uses and lacking.tolist() == [0]
    assert source.tolist() == [-1, -1, -1] == target.tolist()


def test_reserve_more_rows_than_lanes_with_offsets_astray(fc):
    rows = 2500
    table = torch.full((rows, 2), -1, dtype=torch.int32, device="cuda")
    offsets = torch.arange(rows + 1, dtype=torch.int32, device="cuda")
    offsets[2400] = 7                                    # (below the one before it)
    uses = torch.zeros(4096, dtype=torch.int32, device="cuda")
    source, target, lacking = fc.pages_reserve(table, torch.zeros(rows, dtype=torch.int32, device="cuda"), uses, offsets, 16)
    assert bool((table == -1).all()) and bool((uses == 0).all()) and bool((source == -1).all()) and bool((target == -1).all()) and int(lacking) == 0


def test_the_last_of_all_writers_keeps_a_page(fc):
    # three users: all write, two of them write, one writes
    for new, copied in (([1, 1, 1], [0, 1]), ([1, 0, 1], [0, 2]), ([0, 1, 0], [1])):
        t, u = ints([[4, -1]] * 3), ints([0, 0, 0, 0, 3, 0])
        offsets = [0, new[0], new[0] + new[1], sum(new)]
        source, target, lacking = fc.pages_reserve(t, ints([7, 7, 7]), u, ints(offsets), 16)
        assert [b for b in range(3) if source[b] >= 0] == copied and lacking.item() == 0
        assert [t[b, 0].item() for b in copied] == list(range(len(copied))) and u[4].item() == 3 - len(copied)


@pytest.mark.parametrize("pages,sequences,width", [(1, 1, 1), (2, 1, 2), (7, 2, 3), (64, 3, 20), (4095, 5, 300), (4096, 9, 300), (4097, 9, 300), (12289, 40, 200), (100003, 50, 1500)])
def test_compact(fc, pages, sequences, width):
    for seed in range(4):
        rng = random.Random(seed)
        table, _, uses = state(sequences, width, pages, 16, seed)
        if seed == 3:                                    # in order already, or nothing in use
            table, uses = ([[-1] * width for _ in range(sequences)], [0] * pages) if rng.random() < 0.5 else compact(table, uses)[:2]
        print("compact", pages, sequences, seed, flush=True)
        want = compact(table, uses)
        t, u = ints(table), ints(uses)
        got = fc.pages_compact(t, u)
        assert got[4].item() == want[4] and got[0].tolist() == want[0] and got[1].tolist() == want[1]
        assert got[2].tolist() == want[2] and got[3].tolist() == want[3]
        assert t.tolist() == table and u.tolist() == uses
        out = (t, *[torch.empty_like(x) for x in got[1:]])                # the table in place
        assert fc.pages_compact(t, u, out=out) is out
        assert all(torch.equal(a, b) for a, b in zip(out, got))


@pytest.mark.parametrize("pages", [5, 4095, 4096, 20011, 32768, 32769, 70001])
def test_compact_pools_of_any_fill(fc, pages):
    for fill in (0.02, 0.5, 0.97, 1.0):
        rng = random.Random(pages)
        uses = [rng.randint(1, 3) if rng.random() < fill else rng.choice([0, 0, -2]) for _ in range(pages)]
        table = [[rng.randrange(-2, pages + 2) for _ in range(37)] for _ in range(11)]
        want = compact([[p if 0 <= p < pages and uses[p] > 0 else -5 for p in row] for row in table], uses)
        got = fc.pages_compact(ints(table), ints(uses))
        assert got[4].item() == want[4] and got[1].tolist() == want[1] and got[2].tolist() == want[2] and got[3].tolist() == want[3]
        for row, mine, old in zip(got[0].tolist(), want[0], table):
            assert row == [m if m != -5 else p for m, p in zip(mine, old)]        # entries that name no page in use stay


def cache_of(pages, heads, page, dim, seed):
    g = torch.Generator().manual_seed(seed)
    codes = [torch.randint(0, 256, (pages, heads, page, dim), dtype=torch.uint8, generator=g).cuda() for _ in range(2)]
    return (*codes, *[torch.rand((pages, heads), generator=g).cuda() for _ in range(2)])


@pytest.mark.parametrize("pages,heads,page,dim", [(3, 1, 16, 64), (9, 2, 64, 128), (30, 5, 32, 256), (50, 40, 16, 128)])
def test_copy(fc, pages, heads, page, dim):
    cache = cache_of(pages, heads, page, dim, pages)
    want = [t.clone() for t in cache]
    half = pages // 2
    source, target = [0] * half, list(range(half + 1, half + 1 + half))        # the same source several times
    for i in range(1, half):
        source[i] = i % half
    source += [-1, 3, pages, 1 << 30, 0, 0]
    target += [0, -1, 0, 0, pages, -(1 << 30)]
    for s, t in zip(source, target):
        if 0 <= s < pages and 0 <= t < pages:
            for c in want:
                c[t] = c[s]
    print("copy", pages, heads, page, dim, flush=True)
    assert fc.cache_copy(cache, ints(source), ints(target)) is cache
    assert all(torch.equal(a, b) for a, b in zip(cache, want))
    fc.cache_copy(cache, ints([]), ints([]))
    fc.cache_copy(cache, ints([2]), ints([2]))
    assert all(torch.equal(a, b) for a, b in zip(cache, want))


def test_copy_beyond_32_bit_offsets(fc):
    pages, heads, page, dim = 8200, 16, 64, 256          # 262144 bytes a page, 2.1 GB a cache
    cache = (*[torch.zeros((pages, heads, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2)], *[torch.zeros((pages, heads), device="cuda") for _ in range(2)])
    one = cache_of(1, heads, page, dim, 4)
    for c, o in zip(cache, one):
        c[8198] = o[0]
    fc.cache_copy(cache, ints([8198, 8198]), ints([8199, 5]))
    for c, o in zip(cache, one):
        assert torch.equal(c[8199], o[0]) and torch.equal(c[5], o[0]) and not c[:5].any() and not c[6:8198].any()


def test_a_step_in_a_graph_and_without_the_native_module(fc):
    page, width, pages = 16, 12, 200
    table, held, uses = state(6, width, pages, page, 1)
    parents, offsets = [1, 1, 0, 5, 5, -1], [0, 1, 2, 3, 4, 5, 9]
    ft, fh, fu = fork(table, held, uses, parents, page)
    want = reserve(ft, fh, fu, offsets, page)
    cache = cache_of(pages, 2, page, 64, 2)
    t, h, u, p, o = ints(table), ints(held), ints(uses), ints(parents), ints(offsets)
    new, now = torch.empty_like(t), torch.empty_like(h)
    out = tuple(torch.empty(n, dtype=torch.int32, device="cuda") for n in (6, 6, 1))
    work = torch.empty(4 * pages, dtype=torch.uint8, device="cuda")

    def step():
        fc.pages_fork(t, h, u, p, page, out=(new, now))
        fc.pages_reserve(new, now, u, o, page, out=out, workspace=work)
        fc.cache_copy(cache, out[0], out[1])

    def check():
        assert new.tolist() == want[0] and now.tolist() == fh and u.tolist() == want[1]
        assert out[0].tolist() == want[2] and out[1].tolist() == want[3] and out[2].item() == 0
        for a, b in zip(want[2], want[3]):
            if a >= 0:
                assert all(torch.equal(c[a], c[b]) for c in cache)

    native = fc.binding._calls()
    assert native.pages_fork(t, h, u.clone(), p, page, None) is not None and native.cache_copy(cache, out[0].fill_(-1), out[1]) is cache
    assert native.pages_reserve(t.clone(), h, u.clone(), o, page, None, None) is not None and native.pages_compact(t, u, None, None) is not None
    step()
    check()
    u.copy_(ints(uses))
    fc.binding._native = fc.binding._NoNativeCalls()
    try:
        step()
        check()
        assert fc.pages_compact(t, ints(uses))[4].item() == sum(x > 0 for x in uses)
    finally:
        fc.binding._native = native
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.synchronize()
    for _ in range(3):
        u.copy_(ints(uses))
        for c in cache:
            c.copy_(torch.rand(c.shape, device="cuda").mul(200).to(c.dtype))
        graph.replay()
        torch.cuda.synchronize()
        check()


def test_refusals(fc):
    t, h, u, p = ints([[0, -1], [1, 2]]), ints([3, 20]), ints([1, 1, 1, 0]), ints([0, 1])
    cache = cache_of(4, 2, 16, 64, 1)
    for bad in (lambda: fc.pages_fork(t.long(), h, u, p, 16), lambda: fc.pages_fork(t.cpu(), h, u, p, 16), lambda: fc.cache_copy(cache, p.long(), p)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: fc.pages_fork(t, h[:1], u, p, 16), lambda: fc.pages_fork(t, h, u, p, 16, out=(t, h.clone())), lambda: fc.pages_fork(t, h, u, p, 16, out=(t.clone(), h)),
                lambda: fc.pages_fork(t, h, u, p, 16, out=(t[:1], h.clone())), lambda: fc.pages_fork(t[0], h, u, p, 16), lambda: fc.pages_reserve(t, h, u, p, 16),
                lambda: fc.pages_compact(t, u, out=(t, u, p, p.clone(), ints([0]))), lambda: fc.pages_compact(t[:, 1:], u), lambda: fc.cache_copy(cache, p, p[:1]),
                lambda: fc.cache_copy(cache[:3], p, p), lambda: fc.cache_copy((cache[0], cache[1][:3], *cache[2:]), p, p)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: fc.pages_fork(t, h, u, p, 48), lambda: fc.pages_reserve(t, h, u, ints([0, 1, 2]), 8), lambda: fc.pages_reserve(t, h, u, ints([0, 1, 2]), 16, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")),
                lambda: fc.cache_copy(cache_of(4, 2, 8, 64, 1), p, p)):
        with pytest.raises(fc.FcError):
            bad()
    assert t.tolist() == [[0, -1], [1, 2]] and u.tolist() == [1, 1, 1, 0]


@pytest.mark.parametrize("needed", [[4096], [4097], [9001], [1, 4094], [1, 4096], [2000, 0, 2096, 1], [3000, 2999, 4000]])
@pytest.mark.parametrize("lack", [0, 1])
def test_reserve_lists_many_pages_in_the_workspace(fc, needed, lack):
    """More fresh pages than are listed in LDS (4096), for one row and for several, the last ones of which also part with a shared page"""
    page, pages, width, n = 16, 20011, max(needed) + 2, len(needed)
    shared = pages - 1                                   # partly filled, of all rows but the first, and of one that is not in this step
    table = [[shared if b else -1] + [-1] * (width - 1) for b in range(n)]
    held = [5 if b else 0 for b in range(n)]
    # a row with a partly filled page copies it: one of the pages that it needs
    new = [(k - 1) * page + 11 if b and k else k * page for b, k in enumerate(needed)]
    offsets = [sum(new[:b]) for b in range(n + 1)]
    total = sum(needed)
    rng = random.Random(total)
    free = set(rng.sample(range(pages - 1), total - lack))
    uses = [0 if p in free else 1 for p in range(pages)]
    uses[shared] = n
    want = reserve(table, held, uses, offsets, page)
    assert want[4] == lack
    need = fc.lib().fc_pages_reserve_workspace_bytes(pages)
    space = torch.full((need + 4096,), 99, dtype=torch.uint8, device="cuda")
    t, u = ints(table), ints(uses)
    print("reserve many", needed, lack, flush=True)
    source, target, lacking = fc.pages_reserve(t, ints(held), u, ints(offsets), page, workspace=space[:need])
    assert lacking.tolist() == [lack] and bool((space[need:] == 99).all())
    assert t.tolist() == want[0] and u.tolist() == want[1] and source.tolist() == want[2] and target.tolist() == want[3]


@pytest.mark.parametrize("heads,page,dim,pages", [(5, 32, 128, 7000), (1, 16, 64, 140000), (8, 16, 128, 9000)])
def test_copy_of_more_than_the_caches_hold(fc, heads, page, dim, pages):
    """134 MB and more are copied past the caches; pages whose last 16 KB are not whole, pages smaller than that, and pairs that name no page"""
    cache = cache_of(pages, heads, page, dim, pages)
    half = pages // 2
    g = torch.Generator().manual_seed(3)
    source, target = torch.randint(0, half, (half,), generator=g), half + torch.randperm(half, generator=g)
    for at, s, t in ((0, -1, half), (half // 2, 3, -1), (half - 1, pages, half + 1), (7, 1, pages)):
        source[at], target[at] = s, t
    assert half * heads * page * dim * 2 > 1 << 27
    there = (source >= 0) & (source < half) & (target >= 0) & (target < pages)
    want = [c.clone() for c in cache]
    for c in want:
        c[target[there].cuda()] = c[source[there].cuda()]
    print("copy", heads, page, dim, pages, flush=True)
    fc.cache_copy(cache, source.to(torch.int32).cuda(), target.to(torch.int32).cuda())
    assert all(torch.equal(a, b) for a, b in zip(cache, want))
