"""Norm and page operators without a GPU: argument checks of the C entry points, and the launches that they make."""
import json
import subprocess
import sys

import pytest

import paper_2412_04964_amd as fc
import launches

P = 0x10000      # a fake, 16-byte aligned, non-NULL device address; never dereferenced


@pytest.fixture(scope="module")
def L():
    return fc.lib()


def norm(L, x=P, xs=512, r=None, rs=0, w=P, wt=0, tokens=4, hidden=512, eps=1e-5, type=0, sum=None, ss=0, y=P, ys=512):
    return L.fc_rms_norm(x, xs, r, rs, w, wt, tokens, hidden, eps, type, sum, ss, y, ys, None)


def coded(L, x=P, xs=512, r=None, rs=0, w=P, wt=2, tokens=4, hidden=512, eps=1e-5, type=1, group=64, quantizer=1, sum=None, codes=P, scales=P):
    return L.fc_rms_norm_quantize(x, xs, r, rs, w, wt, tokens, hidden, eps, type, group, quantizer, sum, 512, codes, scales, None)


def test_norm_argument_checks(L):
    for call in (norm, coded):
        assert call(L, type=2) == call(L, type=-1) == call(L, wt=3) == call(L, type=0, wt=1) == -8
        assert call(L, tokens=-1) == call(L, hidden=0) == call(L, hidden=516) == call(L, hidden=32776) == -4
        assert call(L, eps=0.0) == call(L, eps=-1.0) == call(L, eps=float("nan")) == call(L, eps=float("inf")) == -4
        assert call(L, x=None) == call(L, w=None) == -1
        assert call(L, x=P + 2) == call(L, xs=4) == call(L, r=P + 8) == call(L, r=P, rs=12) == call(L, sum=P + 8) == call(L, w=P + 4) == -5
        assert call(L, tokens=0, x=None, w=None) == 0
    assert norm(L, y=None) == -1 and norm(L, y=P + 2) == norm(L, ys=3) == norm(L, sum=P, ss=4) == -5
    assert coded(L, quantizer=0) == coded(L, quantizer=3) == -8
    assert coded(L, group=0) == coded(L, group=16) == coded(L, group=48) == coded(L, group=1024) == coded(L, hidden=520, group=512) == -3
    assert coded(L, codes=None) == coded(L, scales=None) == -1 and coded(L, codes=P + 8) == -5
    assert coded(L, tokens=0, codes=None, scales=None) == 0


def fork(L, table=P, held=P, sequences=2, width=3, page=16, uses=P, pages=8, parents=P, rows=2, out=P, held_out=P):
    return L.fc_pages_fork(table, held, sequences, width, page, uses, pages, parents, rows, out, held_out, None)


def reserve(L, table=P, held=P, offsets=P, sequences=2, width=3, page=16, uses=P, pages=8, source=P, target=P, lacking=P, ws=P, bytes=32):
    return L.fc_pages_reserve(table, held, offsets, sequences, width, page, uses, pages, source, target, lacking, ws, bytes, None)


def compact(L, table=P, sequences=2, width=3, uses=P, pages=8, out=P, uses_out=P, source=P, target=P, used=P, ws=P, bytes=36):
    return L.fc_pages_compact(table, sequences, width, uses, pages, out, uses_out, source, target, used, ws, bytes, None)


def copy(L, k=P, v=P, ks=P, vs=P, pages=8, heads=2, page=16, dim=64, source=P, target=P, count=3):
    return L.fc_cache_copy(k, v, ks, vs, pages, heads, page, dim, source, target, count, None)


def test_page_argument_checks(L):
    for call in (fork, reserve, compact):
        assert call(L, width=0) == call(L, pages=0) == call(L, pages=1 << 31) == call(L, sequences=-1) == -4
    for call in (fork, reserve, copy):
        assert call(L, page=8) == call(L, page=48) == call(L, page=128) == -4
    assert fork(L, rows=-1) == -4
    for name in ("table", "held", "uses", "parents", "out", "held_out"):
        assert fork(L, **{name: None}) == -1, name
    assert fork(L, sequences=0, rows=0, uses=None) == 0
    for name in ("table", "held", "offsets", "uses", "source", "target", "lacking"):
        assert reserve(L, **{name: None}) == -1, name
    assert L.fc_pages_reserve_workspace_bytes(8) == 32 and L.fc_pages_reserve_workspace_bytes(0) == 0
    assert reserve(L, ws=None) == reserve(L, bytes=31) == -6 and reserve(L, ws=P + 4) == -5
    for name in ("table", "uses", "out", "uses_out", "source", "target", "used"):
        assert compact(L, **{name: None}) == -1, name
    assert L.fc_pages_compact_workspace_bytes(8) == 36 and L.fc_pages_compact_workspace_bytes(-1) == 0
    assert compact(L, ws=None) == compact(L, bytes=35) == -6 and compact(L, ws=P + 4) == -5
    assert copy(L, pages=0) == copy(L, heads=0) == copy(L, dim=32) == copy(L, count=-1) == -4
    for name in ("k", "v", "ks", "vs", "source", "target"):
        assert copy(L, **{name: None}) == -1, name
    assert copy(L, k=P + 8) == copy(L, v=P + 1) == -5
    assert copy(L, count=0, k=None, source=None) == 0


def test_cpu_tensors_are_refused():
    torch = pytest.importorskip("torch")
    i = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: fc.rms_norm(torch.zeros((2, 64), dtype=torch.float16), torch.zeros(64)), lambda: fc.pages_fork(i[:, None], i, i, i, 16),
                 lambda: fc.pages_compact(i[:, None], i), lambda: fc.cache_copy((i, i, i, i), i, i)):
        with pytest.raises(TypeError):
            call()


_CHILD = """
import ctypes, json, sys
ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2])
for name, args in json.load(sys.stdin):
    print("R", getattr(L, name)(*[{float: ctypes.c_double, str: lambda a: ctypes.c_float(float(a)), int: ctypes.c_int64}[type(a)](a) for a in args]), flush=True)
"""


def launched(*calls):
    """(return code, [(kernel, workgroups, lanes), ...]) of each call, where nothing runs and no address is followed (launches.py)"""
    r = subprocess.run([sys.executable, "-c", _CHILD, launches._stand_in(), launches.LIB], input=json.dumps(calls), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out, seen = [], []
    for line in r.stdout.splitlines():
        if line.startswith("L "):
            _, name, grid, block, _ = line.split()
            seen.append((launches._readable(name), int(grid), int(block)))
        else:
            out.append((int(line[2:]), seen))
            seen = []
    return out


def norm_call(tokens, hidden):
    return "fc_rms_norm", [P, hidden, P, hidden, P, 0, tokens, hidden, 1e-5, 0, P, hidden, P, hidden, 0]


def test_calls_are_launched_up_to_what_the_runtime_takes():
    most = (1 << 31) - 1
    fine = [norm_call(1, 8), norm_call(most, 8), norm_call(most, 32768),
            ("fc_pages_fork", [P, P, 1 << 22, 4, 16, P, most, P, 1 << 22, P, P, 0]), ("fc_pages_reserve", [P, P, P, 1 << 22, 4, 16, P, most, P, P, P, P, 1 << 34, 0]),
            ("fc_pages_compact", [P, 1 << 10, 1 << 20, P, 1 << 30, P, P, P, P, P, P, 1 << 34, 0]), ("fc_cache_copy", [P, P, P, P, most, 8, 16, 128, P, P, 1 << 22, 0])]
    for call, (rc, seen) in zip(fine, launched(*fine)):
        assert rc == 0 and seen, (call, rc, seen)
    over = [("fc_pages_fork", [P, P, 1 << 23, 4, 16, P, most, P, 1 << 23, P, P, 0]), ("fc_cache_copy", [P, P, P, P, most, 8, 16, 128, P, P, 1 << 24, 0]),
            ("fc_pages_compact", [P, 1 << 12, 1 << 20, P, 8, P, P, P, P, P, P, 1 << 34, 0])]
    for call, (rc, seen) in zip(over, launched(*over)):
        assert rc == -4 and not seen, (call, rc, seen)


def chunk(L, q=P, k=P, v=P, tokens=4, heads=2, group=2, dim=64, type=0, quantizer=1, cache=P, scales=P, pages=4, page=16, pt=P, width=2, offsets=P, held=P, sequences=1,
          longest=64, scale=0.1, out=P, ws=P, bytes=1 << 40, vt=128):
    return L.fc_chunk_attention(q, 256, 64, k, 128, 64, v, vt, 64, tokens, heads, group, dim, type, quantizer, cache, cache, scales, scales, pages, page, pt, width,
                                offsets, held, sequences, longest, scale, out, 256, 64, ws, bytes, None)


def test_chunk_attention_argument_checks(L):
    assert chunk(L, type=2) == chunk(L, quantizer=0) == chunk(L, quantizer=3) == -8
    assert chunk(L, dim=256) == chunk(L, dim=32) == chunk(L, heads=0) == chunk(L, group=0) == chunk(L, group=40000) == chunk(L, longest=0) == chunk(L, tokens=-1) == -4
    assert chunk(L, page=8) == chunk(L, pages=0) == chunk(L, width=0) == chunk(L, sequences=0) == chunk(L, vt=1 << 25) == chunk(L, tokens=(1 << 31) - 1) == chunk(L, tokens=1 << 30) == -4
    assert chunk(L, scale=0.0) == chunk(L, scale=-1.0) == chunk(L, scale=float("nan")) == -4
    for name in ("q", "k", "v", "cache", "scales", "pt", "offsets", "held", "out"):
        assert chunk(L, **{name: None}) == -1, name
    assert chunk(L, q=P + 2) == chunk(L, vt=12) == chunk(L, cache=P + 8) == -5
    need = L.fc_chunk_attention_workspace_bytes(4, 1, 2, 2, 64, 100000)
    assert need > 0 and need % 4 == 0
    assert chunk(L, longest=100000, bytes=need - 1) == chunk(L, longest=100000, ws=None) == -6 and chunk(L, longest=100000, ws=P + 4) == -5
    assert chunk(L, tokens=0, q=None, k=None, v=None, out=None, cache=None, ws=None) == 0
    for bad in ((4, 1, 2, 2, 256, 64), (4, 1, 0, 2, 64, 64), (-1, 1, 2, 2, 64, 64), (4, 1, 2, 2, 64, 0)):
        assert L.fc_chunk_attention_workspace_bytes(*bad) == 0
    # announced lengths are bounds, up to the largest that their types hold
    for sequences, heads in ((256, 8), (1, 1), (65536, 64)):
        needs = [L.fc_chunk_attention_workspace_bytes(1 << 20, sequences, heads, 8, 128, longest) for longest in (1 << 20, 1 << 26, (1 << 31) - 1)]
        assert needs[0] > 0 and needs == [needs[0]] * 3


def chunk_call(tokens, heads, group, dim, sequences, longest, ws=1 << 40, scale="0.125"):
    row = heads * group * dim
    return "fc_chunk_attention", [P, row, dim, P, heads * dim, dim, P, heads * dim, dim, tokens, heads, group, dim, 0, 1, P, P, P, P, 1 << 20, 16, P, 1 << 20, P, P,
                                  sequences, longest, scale, P, row, dim, P, ws, 0]


def test_chunk_attention_launches(L):
    """One kernel where no sequence is long, and the join behind it where items may be cut; workgroups of 4 wavefronts where there is little to do"""
    calls = [chunk_call(4, 2, 4, 64, 2, 60), chunk_call(400, 2, 4, 64, 2, 600), chunk_call(1200, 8, 4, 64, 6, 300), chunk_call(4, 2, 4, 64, 2, 6000),
             chunk_call(4000, 8, 4, 128, 2, 600000),
             chunk_call((1 << 31) - 1025, 1, 1, 128, 1, (1 << 31) - 1025), chunk_call(1, 32, 1, 64, 1 << 20, 64), chunk_call(1, 1, 1, 64, 1, 1 << 30)]
    # (kernels, lanes): short contexts with few and with many items; ranges with little and with much work; the longest; too many workgroups for one an item
    want = [(1, 256), (2, 256), (1, 512), (2, 256), (2, 512), (2, 512), (2, 512), (2, 512)]
    names = []
    for call, (rc, seen), (kernels, block) in zip(calls, launched(*calls), want):
        assert rc == 0 and len(seen) == kernels and seen[0][2] == block, (call, rc, seen)
        names.append([k for k, _, _ in seen])
        assert all(grid * lanes < 1 << 32 for _, grid, lanes in seen), seen
    assert all("k_chunk_attention" in n[0] for n in names) and all("k_chunk_join" in n[1] for n in names if len(n) == 2)
    # what a plan needs is what the entry point asks for
    for call in calls:
        a = call[1]
        need = L.fc_chunk_attention_workspace_bytes(a[9], a[25], a[10], a[11], a[12], a[26])
        less = list(a)
        less[32] = need - 1
        enough = list(a)
        enough[32] = need
        results = launched(*([(call[0], less)] if need else []), (call[0], enough))
        assert [rc for rc, _ in results] == ([-6] if need else []) + [0], (a, need, results)
